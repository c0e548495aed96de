"""The paged KV cache through the C ABI: append with rotation, attention over the pages and reading back, against the float64
oracle, in both builds.  Unless a test says otherwise, cache memory that no position owns holds NaN."""
import numpy as np
import pytest

from oracle import paged as P
from tests import _util as U

pytestmark = pytest.mark.gpu

# Relative rounding errors: half a step of the type a value is rounded to.
HALF_BF16, HALF_E4M3, HALF_F32 = 2.0 ** -8, 2.0 ** -4, 2.0 ** -24
E4M3_TINY = 2.0 ** -10           # half the smallest e4m3 step

BUILDS = pytest.mark.parametrize("fp32", [False, True], ids=["bf16", "fp32dbg"])
CACHES = pytest.mark.parametrize("e4m3", [False, True], ids=["act", "e4m3"])


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


class World:
    """A pool of pages in no order, a table, sequences with (new tokens, cached positions), and what all of it holds in
    float64."""

    def __init__(self, torch, seqs, Hq, Hkv, d, page, *, fp32=False, e4m3=False, seed=0, amplitude=1.0, rope=True, slots=None,
                 absent=(), scales=(0.02, 0.03), pad=0, extra_rows=0):
        import paper_2412_17246_amd as lib
        self.torch, self.lib, self.fp32, self.e4m3 = torch, lib, fp32, e4m3
        self.Hq, self.Hkv, self.d, self.page, self.seqs = Hq, Hkv, d, page, seqs
        rng = np.random.default_rng([11, seed])
        self.piece = 16 if e4m3 else 8
        self.scales = scales if e4m3 else (1.0, 1.0)
        self.act = torch.float32 if fp32 else torch.bfloat16
        self.kind = torch.float8_e4m3fn if e4m3 else self.act
        self.slots = list(range(len(seqs))) if slots is None else slots
        per = [-(-(n + b) // page) for n, b in seqs]
        rows, width = max(self.slots) + 1, max(max(per), 1)
        pool = sum(per) + 2
        order = rng.permutation(pool)
        self.table = np.full((rows, width), -1, dtype=np.int32)
        at = 0
        for s, slot in enumerate(self.slots):
            self.table[slot, :per[s]] = order[at:at + per[s]]
            at += per[s]
        for s, i in absent:
            self.table[self.slots[s], i] = -1
        shape = (pool, Hkv, page * d)
        self.hk, self.hv = np.full(shape, np.nan), np.full(shape, np.nan)     # numbers as the cache holds them
        self.old = []
        for s, (n, b) in enumerate(seqs):
            there = self.present(s, b)
            pos = np.arange(b)[there]
            k, v = (self.rounded(rng.standard_normal((len(pos), Hkv, d)) * amplitude / sc) for sc in self.scales)
            if len(pos):
                kp, vp = P.places(self.table[self.slots[s]], pos, Hkv, page, d, self.piece)
                self.hk[kp], self.hv[vp] = k, v
        T = sum(n for n, _ in seqs)
        self.T = T
        self.q_start = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.row = (Hq + 2 * Hkv) * d + pad
        bits = U.W.bf16_bits_from_f32((rng.standard_normal((T + extra_rows, self.row)) * amplitude).astype(np.float32))
        self.qkv64 = U.f64(bits)
        self.qkv = U.to_device(bits, fp32)
        self.q, self.k, self.v = (self.qkv[:, a * d:b * d] for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        self.rope64 = lib.rope_table(width * page, d, 10000.0) if rope else None
        self.rope = torch.from_numpy(self.rope64).cuda() if rope else None
        self.dk, self.dv = self.upload(self.hk), self.upload(self.hv)
        self.dtable = torch.from_numpy(self.table).cuda()
        self.kv = lib.PagedKv(page, Hkv, d, k=self.dk, v=self.dv, page_table=self.dtable, k_scale=self.scales[0],
                              v_scale=self.scales[1], fp32_debug=fp32)
        self.batch = lib.Batch(lib.load_library(fp32), self.q_start, self.slots, [b for _, b in seqs])
        torch.cuda.synchronize()

    def rounded(self, x):
        """x as the cache's type holds it."""
        t = self.torch.from_numpy(np.asarray(x, dtype=np.float32))
        if self.e4m3:
            t = t.clamp(-448, 448)
        elif not self.fp32:
            t = t.bfloat16()
        return t.to(self.kind).float().numpy().astype(np.float64)

    def upload(self, x):
        return self.torch.from_numpy(x.astype(np.float32)).to(self.kind).cuda().contiguous()

    def download(self, t):
        self.torch.cuda.synchronize()
        return t.cpu().float().numpy().astype(np.float64)

    def present(self, s, m):
        """Which of positions 0..m-1 of sequence s are on a page that is there."""
        return self.table[self.slots[s]][np.arange(m) // self.page] >= 0

    def new_rows(self, s):
        """k (rotated) and v of the sequence's new tokens in float64, before they are rounded."""
        a, b = self.q_start[s], self.q_start[s + 1]
        n, before = self.seqs[s]
        x = self.qkv64[a:b, :(self.Hq + 2 * self.Hkv) * self.d].reshape(n, self.Hq + 2 * self.Hkv, self.d)
        pos = before + np.arange(n)
        k, v = x[:, self.Hq:self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:]
        return (P.rotate(k, pos, self.rope64) if self.rope64 is not None else k), v

    def write_new(self):
        """Puts the new tokens into the pages from the host, rounded as the append rounds them."""
        for s, (n, before) in enumerate(self.seqs):
            k, v = self.new_rows(s)
            pos = before + np.arange(n)
            there = self.table[self.slots[s]][pos // self.page] >= 0
            if there.any():
                kp, vp = P.places(self.table[self.slots[s]], pos[there], self.Hkv, self.page, self.d, self.piece)
                self.hk[kp], self.hv[vp] = self.rounded(k[there] / self.scales[0]), self.rounded(v[there] / self.scales[1])
        self.dk.copy_(self.upload(self.hk))
        self.dv.copy_(self.upload(self.hv))

    def sequence(self, s):
        """k and v [m, Hkv, d] of sequence s as the pages hold them, scales applied, and which positions are there."""
        m = sum(self.seqs[s])
        there = self.present(s, m)
        k, v = np.zeros((m, self.Hkv, self.d)), np.zeros((m, self.Hkv, self.d))
        if there.any():
            kp, vp = P.places(self.table[self.slots[s]], np.arange(m)[there], self.Hkv, self.page, self.d, self.piece)
            k[there], v[there] = self.hk[kp] * self.scales[0], self.hv[vp] * self.scales[1]
        return k, v, there

    def append(self, **kw):
        self.lib.op_paged_append(self.batch, self.kv, self.k, self.v, rope=self.rope, **kw)

    def workspace(self, window=0):
        n = self.lib.op_paged_attention_workspace_bytes(self.batch, self.kv, self.Hq, window=window)
        return self.torch.full((max(n, 16),), 0xff, dtype=self.torch.uint8, device="cuda")     # NaN everywhere

    def attend(self, window=0, scale=0.0, out=None, workspace=None, **kw):
        if out is None:
            out = self.torch.full((self.T, self.Hq * self.d), 7.0, dtype=self.act, device="cuda")
        self.lib.op_paged_attention(self.batch, self.kv, self.q, out, window=window, scale=scale, rope=self.rope,
                                    workspace=self.workspace(window) if workspace is None else workspace, **kw)
        return out

    def check(self, got, window=0, scale=0.0, only=None):
        """The derived bound, element by element, and the rms of all errors.  q is rounded to the activation type after its
        rotation, a weight to bf16, the output to the activation type; sums are fp32: of d products in a score, of m weights and
        products behind it (fp32 build: these alone)."""
        got = self.download(got).reshape(self.T, self.Hq, self.d)
        err, ref = [], []
        for s in range(len(self.seqs)) if only is None else only:
            n, before = self.seqs[s]
            if n == 0:
                continue
            a, b = self.q_start[s], self.q_start[s + 1]
            pos = before + np.arange(n)
            q = self.qkv64[a:b, :self.Hq * self.d].reshape(n, self.Hq, self.d)
            if self.rope64 is not None:
                q = P.rotate(q, pos, self.rope64)
            k, v, there = self.sequence(s)
            want, moved = P.attention(q, k, v, pos, there, scale or self.d ** -0.5, window)
            half = HALF_F32 if self.fp32 else HALF_BF16
            sums = (len(there) + self.d) * HALF_F32 * 2
            tol = half * np.abs(want) + moved(half + sums, (0 if self.fp32 else HALF_BF16) + sums) * (1 + 2 ** -4) + 1e-30
            assert np.all(np.isfinite(got[a:b])), "non-finite output of sequence %d" % s
            worst = np.max(np.abs(got[a:b] - want) / tol)
            assert worst <= 1, (s, self.seqs[s], worst)
            err.append((got[a:b] - want).ravel())
            ref.append(want.ravel())
        err, ref = np.concatenate(err), np.concatenate(ref)
        # three independent roundings (q, weights, output) of at most half a step each, evenly spread: rms half / sqrt(3) each
        rms = float(np.sqrt(np.mean(err ** 2)) / max(np.sqrt(np.mean(ref ** 2)), 1e-30))
        assert rms <= (1e-5 if self.fp32 else HALF_BF16 * 1.5), rms
        return rms


def check_append(w, before_k, before_v):
    """Every element: appended ones within the rounding of their type, all others untouched, bit for bit."""
    bits = w.torch.uint8 if w.e4m3 else w.torch.int32 if w.fp32 else w.torch.int16
    raw = lambda t: t.view(bits).cpu().numpy()  # noqa: E731
    got_k, got_v = w.download(w.dk), w.download(w.dv)
    touched = np.zeros(w.hk.shape, dtype=bool), np.zeros(w.hk.shape, dtype=bool)
    for s, (n, before) in enumerate(w.seqs):
        if n == 0:
            continue
        k, v = w.new_rows(s)
        pos = before + np.arange(n)
        there = w.table[w.slots[s]][pos // w.page] >= 0
        if not there.any():
            continue
        kp, vp = P.places(w.table[w.slots[s]], pos[there], w.Hkv, w.page, w.d, w.piece)
        for got, at, want, sc, mark in ((got_k, kp, k[there], w.scales[0], touched[0]), (got_v, vp, v[there], w.scales[1], touched[1])):
            mark[at] = True
            want = want / sc
            half = HALF_E4M3 if w.e4m3 else HALF_F32 if w.fp32 else HALF_BF16
            want = np.clip(want, -448, 448) if w.e4m3 else want
            # products and their difference in fp32: each term is at most the pair's length sqrt(2) * max
            slack = 4 * HALF_F32 * np.max(np.abs(want), axis=-1, keepdims=True)
            tol = half * np.abs(want) + slack + (E4M3_TINY if w.e4m3 else 0)
            worst = np.max(np.abs(got[at] - want) / tol)
            assert worst <= 1, (s, worst)
        if not w.e4m3:
            assert np.array_equal(got_v[vp], v[there])
    for now, was, mark in ((raw(w.dk), before_k, touched[0]), (raw(w.dv), before_v, touched[1])):
        assert np.array_equal(now[~mark], was[~mark])


SEQS = {
    "one": [(1, 0)],
    "ones": [(1, 5), (1, 31), (1, 32), (1, 255), (1, 256), (1, 600)],
    "prompts": [(33, 0), (2, 0), (130, 7), (64, 64), (1, 40)],
    "ragged": [(0, 10), (3, 61), (1, 0), (29, 35), (0, 0), (5, 300)],
}
HEADS = [(4, 4, 64), (8, 2, 128), (7, 1, 128), (6, 2, 64)]


@BUILDS
@CACHES
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("seqs", list(SEQS))
def test_append(torch, fp32, e4m3, heads, seqs):
    w = World(torch, SEQS[seqs], *heads, 32 if heads[2] == 64 else 64, fp32=fp32, e4m3=e4m3, slots=[2 * i + 1 for i in range(len(SEQS[seqs]))])
    bits = torch.uint8 if e4m3 else torch.int32 if fp32 else torch.int16
    was = w.dk.view(bits).cpu().numpy(), w.dv.view(bits).cpu().numpy()
    w.append()
    check_append(w, *was)


@CACHES
def test_append_without_rotation_keeps_the_bits_and_spares_absent_pages(torch, e4m3):
    w = World(torch, [(70, 20), (1, 64), (40, 90)], 4, 2, 128, 32, e4m3=e4m3, rope=False, absent=[(0, 1), (1, 2), (2, 3)], pad=24)
    bits = torch.uint8 if e4m3 else torch.int16
    was = w.dk.view(bits).cpu().numpy(), w.dv.view(bits).cpu().numpy()
    w.append()
    check_append(w, *was)


@BUILDS
def test_e4m3_saturates_and_keeps_nan(torch, fp32):
    w = World(torch, [(1, 3), (9, 0)], 2, 2, 64, 32, fp32=fp32, e4m3=True, rope=False, scales=(2.0, 0.5))
    w.k[:, :4] = torch.tensor([1e30, -1e30, float("inf"), float("nan")])
    w.v[:, :4] = torch.tensor([224.0, -225.0, -float("inf"), float("nan")])
    w.append()
    for s, (n, before) in enumerate(w.seqs):
        kp, vp = P.places(w.table[s], before + np.arange(n), 2, 32, 64, 16)
        assert np.array_equal(w.download(w.dk)[kp][:, 0, :4], [[448, -448, 448, np.nan]] * n, equal_nan=True)
        assert np.array_equal(w.download(w.dv)[vp][:, 0, :4], [[448, -448, -448, np.nan]] * n, equal_nan=True)


@BUILDS
@CACHES
@pytest.mark.parametrize("heads", HEADS + [(40, 1, 64), (5, 5, 128)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("seqs", list(SEQS))
def test_attention(torch, fp32, e4m3, heads, seqs):
    w = World(torch, SEQS[seqs], *heads, 64 if heads[2] == 64 else 32, fp32=fp32, e4m3=e4m3, slots=list(range(len(SEQS[seqs])))[::-1])
    w.write_new()
    w.check(w.attend())


@CACHES
@pytest.mark.parametrize("window", [1, 31, 64, 100, 5000])
@pytest.mark.parametrize("page", [32, 256])
def test_attention_window(torch, e4m3, window, page):
    w = World(torch, [(1, 700), (150, 333), (6, 257), (1, 0), (3, 31), (1, 63)], 8, 2, 128, page, e4m3=e4m3)
    w.write_new()
    w.check(w.attend(window=window), window=window)


@BUILDS
@CACHES
def test_attention_with_absent_pages(torch, fp32, e4m3):
    """Pages in the middle, at the start and at the end are not there; one sequence has none at all, and one chunk's first tokens
    see nothing."""
    seqs = [(1, 500), (40, 200), (5, 100), (1, 40), (37, 64), (1, 64)]
    absent = [(0, 3), (0, 4), (0, 0), (1, 2), (1, 5), (2, 3), (3, 0), (3, 1), (4, 0), (4, 1), (5, 2)]
    w = World(torch, seqs, 8, 2, 64, 32, fp32=fp32, e4m3=e4m3, absent=absent)
    w.write_new()
    out = w.attend()
    w.check(out)
    assert torch.all(out[w.q_start[3]:w.q_start[4]] == 0)
    w.check(w.attend(window=70), window=70)


def test_attention_of_freed_windows(torch):
    """Pages that have left every window are given back: the result is that of the whole table, bit for bit."""
    seqs, window = [(1, 900), (20, 700), (200, 640)], 256
    w = World(torch, seqs, 8, 8, 128, 64, seed=4)
    w.write_new()
    whole = w.attend(window=window)
    for s, (n, b) in enumerate(seqs):
        w.dtable[s, :(b + 1 - window) // 64] = -1
    freed = w.attend(window=window)
    w.check(whole, window=window)
    assert torch.equal(whole, freed)


@CACHES
def test_attention_scale_and_strides(torch, e4m3):
    """A scale of the caller's, rows further apart than their heads, rows of the output behind the last sequence."""
    w = World(torch, [(1, 77), (65, 30), (4, 200)], 6, 3, 128, 64, e4m3=e4m3, pad=40, extra_rows=3)
    w.write_new()
    wide = torch.full((w.T + 3, w.Hq * w.d + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, 8:8 + w.Hq * w.d]
    w.attend(scale=0.31, out=out)
    w.check(out[:w.T], scale=0.31)
    assert torch.all(wide[w.T:] == 7) and torch.all(wide[:, :8] == 7) and torch.all(wide[:, 8 + w.Hq * w.d:] == 7)


@CACHES
def test_attention_of_large_scores(torch, e4m3):
    """Scores of several hundred: the maximum has to be taken out before the exponential."""
    w = World(torch, [(1, 300), (40, 90), (3, 515)], 4, 2, 64, 32, e4m3=e4m3, amplitude=16.0, scales=(0.3, 0.3), seed=5)
    w.write_new()
    # scores are off by up to eps_q * sum |q k| / 8, tens of units: compare against the oracle's own rounding of q
    for s, (n, before) in enumerate(w.seqs):
        a, b = w.q_start[s], w.q_start[s + 1]
        x = w.qkv64[a:b, :w.Hq * w.d].reshape(n, w.Hq, w.d)
        w.qkv64[a:b, :w.Hq * w.d] = w_rounded(torch, P.rotate(x, before + np.arange(n), w.rope64)).reshape(n, -1)
    w.qkv = U.to_device(U.W.bf16_bits_from_f32(w.qkv64.astype(np.float32)), False)
    w.q = w.qkv[:, :w.Hq * w.d]
    w.rope = w.rope64 = None                                 # rotated already, exactly
    got = w.download(w.attend()).reshape(w.T, w.Hq, w.d)
    for s, (n, before) in enumerate(w.seqs):
        a, b = w.q_start[s], w.q_start[s + 1]
        k, v, there = w.sequence(s)
        want, moved = P.attention(w.qkv64[a:b, :w.Hq * w.d].reshape(n, w.Hq, w.d), k, v, before + np.arange(n), there, 0.125)
        tol = HALF_BF16 * np.abs(want) + moved(2 * (64 + 515) * HALF_F32, HALF_BF16 + 2 * 579 * HALF_F32) * (1 + 2 ** -4)
        assert np.max(np.abs(got[a:b] - want) / tol) <= 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rope", [True, False], ids=["rope", "plain"])
@pytest.mark.parametrize("power", [0, 45, -60, 100])
def test_e4m3_attention_of_any_query_size(torch, d, rope, power):
    """Queries far from one, keys as far the other way, so that scores are ordinary; every third token's queries 2^-30 of the
    others' and every third's with one pair 2^12 above the rest; a token of zeros."""
    w = World(torch, [(1, 300), (90, 700), (3, 515), (300, 40)], 8, 2, d, 64, e4m3=True, rope=rope, seed=7, scales=(0.02, 0.03))
    f = 2.0 ** power
    q, k = w.qkv64[:, :8 * d], w.qkv64[:, 8 * d:10 * d]
    q *= f
    q[1::3] *= 2.0 ** -30
    big = q.reshape(w.T, 8, d)[2::3]                         # a view
    big *= 2.0 ** -12
    big[..., 5] *= 2.0 ** 12
    q[7] = 0
    k /= f
    w.qkv = U.to_device(U.W.bf16_bits_from_f32(w.qkv64.astype(np.float32)), False)
    assert np.array_equal(U.f64(U.W.bf16_bits_from_f32(w.qkv64.astype(np.float32))), w.qkv64)
    w.q, w.k, w.v = (w.qkv[:, a * d:b * d] for a, b in ((0, 8), (8, 10), (10, 12)))
    w.scales = (float(np.float32(0.02)) / f, 0.03)
    w.kv = w.lib.PagedKv(64, 2, d, k=w.dk, v=w.dv, page_table=w.dtable, k_scale=w.scales[0], v_scale=0.03)
    w.write_new()
    w.check(w.attend())


def w_rounded(torch, x):
    return torch.from_numpy(x.astype(np.float32)).bfloat16().float().numpy().astype(np.float64)


@CACHES
def test_shared_pages(torch, e4m3):
    """Two sequences whose rows name the same pages for their common prefix."""
    w = World(torch, [(1, 200), (9, 192)], 8, 2, 128, 64, e4m3=e4m3, seed=3)
    w.table[1, :3] = w.table[0, :3]
    w.dtable.copy_(torch.from_numpy(w.table))
    w.write_new()
    w.check(w.attend())


@BUILDS
@CACHES
@pytest.mark.parametrize("pos0,n", [(0, 1), (3, 90), (32, 64), (95, 7), (0, 160), (17, 0)])
def test_read(torch, fp32, e4m3, pos0, n):
    w = World(torch, [(10, 150), (1, 40)], 4, 3, 64, 32, fp32=fp32, e4m3=e4m3, absent=[(0, 3)])
    w.write_new()
    out = torch.full((2, n + 2, 3, 64), 7.0, dtype=w.act, device="cuda")
    w.lib.op_paged_read(w.kv, 0, pos0, n, out[0], out[1])
    k, v, _ = w.sequence(0)
    got = w.download(out)
    # e4m3 times the scale, rounded to the activation type (and the product to fp32 before)
    half = (HALF_F32 if fp32 else HALF_BF16) + HALF_F32 if e4m3 else 0.0
    for g, want in ((got[0], k), (got[1], v)):
        want = want[pos0:pos0 + n]
        assert np.all(np.abs(g[:n] - want) <= half * np.abs(want))
        assert np.all(g[n:] == 7)


@BUILDS
@CACHES
def test_a_step_and_the_next(torch, fp32, e4m3):
    """Append, attention, the next token's append and attention, and the way out, as a layer of a serving loop uses them."""
    seqs = [(1, 62), (70, 0), (4, 250)]
    w = World(torch, seqs + [(0, 0)], 8, 4, 64, 64, fp32=fp32, e4m3=e4m3)
    ahead = World(torch, [(1, a + b) for a, b in seqs], 8, 4, 64, 64, fp32=fp32, e4m3=e4m3, seed=8)
    bits = torch.uint8 if e4m3 else torch.int32 if fp32 else torch.int16
    was = w.dk.view(bits).cpu().numpy(), w.dv.view(bits).cpu().numpy()
    w.append()
    out = w.attend()
    check_append(w, *was)
    w.hk, w.hv = w.download(w.dk), w.download(w.dv)          # what the attention has read
    w.check(out)
    # one more token each; every row has room for it in its last page
    nxt = ahead
    nxt.table = np.concatenate([w.table[:3], np.full((3, 1), -1, dtype=np.int32)], axis=1)
    nxt.table = nxt.table[:, :w.table.shape[1]]
    nxt.page, nxt.dk, nxt.dv, nxt.hk, nxt.hv = w.page, w.dk, w.dv, w.hk, w.hv
    nxt.dtable = torch.from_numpy(np.ascontiguousarray(nxt.table)).cuda()
    nxt.kv = w.lib.PagedKv(64, 4, 64, k=w.dk, v=w.dv, page_table=nxt.dtable, k_scale=w.scales[0], v_scale=w.scales[1], fp32_debug=fp32)
    nxt.rope64 = w.lib.rope_table(nxt.table.shape[1] * 64, 64, 10000.0)
    nxt.rope = torch.from_numpy(nxt.rope64).cuda()
    nxt.append()
    out = nxt.attend()
    nxt.hk, nxt.hv = nxt.download(nxt.dk), nxt.download(nxt.dv)
    nxt.check(out)
    k = torch.empty(255, 4, 64, dtype=w.act, device="cuda")
    v = torch.empty_like(k)
    w.lib.op_paged_read(nxt.kv, 2, 0, 255, k, v)
    want = nxt.sequence(2)
    half = (HALF_F32 if fp32 else HALF_BF16) + HALF_F32 if e4m3 else 0.0
    assert np.all(np.abs(nxt.download(k) - want[0]) <= half * np.abs(want[0]))
    assert np.all(np.abs(nxt.download(v) - want[1]) <= half * np.abs(want[1]))
