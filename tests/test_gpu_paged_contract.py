"""What the paged KV cache's operations promise beside their results: when a batch may go, what is refused before a launch, how far a
value that is not finite reaches, how precise queries and sums are."""
import numpy as np
import pytest

from oracle import paged as P
from tests import _util as U
from tests.test_gpu_paged import BUILDS, CACHES, HALF_BF16, HALF_F32, World

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


def test_destroy_while_a_stream_that_ran_the_batch_is_captured(torch):
    """Refused, and the capture goes on; the batch stays usable and goes afterwards."""
    import paper_2412_17246_amd as lib
    L = lib.load_library()
    w = World(torch, [(1, 100)], 4, 2, 64, 32, seed=81)
    w.write_new()
    bytes_ = int(L.bz_batch_storage_bytes(1, 1, 256))
    storage = (torch.empty(bytes_, dtype=torch.uint8, device="cuda"), torch.empty(2 * bytes_, dtype=torch.uint8, pin_memory=True),
               torch.cuda.Stream())
    w.batch = batch = lib.Batch(L, [0, 1], [0], [100], storage=storage)
    out, space = torch.zeros(1, w.Hq * w.d, dtype=torch.bfloat16, device="cuda"), w.workspace()
    torch.cuda.synchronize()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    w.attend(out=out, workspace=space, stream=st)
    torch.cuda.synchronize()
    want = out.clone()
    x = torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st, capture_error_mode="relaxed"):
        x += 1
        with pytest.raises(lib.BzError) as e:
            batch.close()
        assert e.value.name == "BZ_ESTATE" and L.bz_batch_tokens(batch.handle) == 1
    graph.replay()
    torch.cuda.synchronize()
    w.attend(out=out, workspace=space, stream=st)
    torch.cuda.synchronize()
    assert torch.all(x == 1) and torch.equal(out, want) and torch.any(want != 0)
    batch.close()
    assert batch.handle is None


def as_e4m3(x):
    """The e4m3 number next to each of x (float64), ties to the even one, beyond the largest that."""
    x = np.clip(x, -448, 448)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(x))), -6)
        step = 2.0 ** (e - 3)
        return np.where(x == 0, 0.0, np.round(x / step) * step)      # numpy rounds halves to even


@BUILDS
@pytest.mark.parametrize("prompt", [False, True], ids=["single", "prompt"])
@pytest.mark.parametrize("scale", [7.0, 0.875, 0.0137, 0.1, 3.0, 2.0 ** -20, 1e30])
def test_e4m3_append_rounds_the_quotient_once(torch, fp32, prompt, scale):
    """Every bf16 number over a scale: the e4m3 number next to the exact quotient.  A tie is one only if the division says so: times
    the scale's reciprocal, 87.5 / 7 is more than 12.5 and would go up."""
    n = 128
    seqs = [(n, 0)] if prompt else [(1, 31 + i % 3) for i in range(n)]
    w = World(torch, seqs, 8, 8, 64, 64, fp32=fp32, e4m3=True, rope=False, scales=(scale, scale), seed=84)
    bits = np.arange(65536, dtype=np.uint32).reshape(n, 512)
    x = (bits << 16).view(np.float32)
    dev = torch.from_numpy(x.copy()).cuda().to(w.act)
    w.k, w.v = dev, dev.clone()
    w.append()
    with np.errstate(all="ignore"):
        want = as_e4m3(x.astype(np.float64) / np.float64(np.float32(scale))).reshape(n, 8, 64)
    got_k, got_v = w.download(w.dk), w.download(w.dv)
    for i, (s, pos) in enumerate([(0, p) for p in range(n)] if prompt else [(s, b) for s, (_, b) in enumerate(seqs)]):
        kp, vp = P.places(w.table[s], [pos], 8, 64, 64, 16)
        assert np.array_equal(got_k[kp][0], want[i], equal_nan=True) and np.array_equal(got_v[vp][0], want[i], equal_nan=True), i


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs", [[(1, 1 + i % 6) for i in range(64)], [(1, 520), (1, 1), (1, 300), (1, 2)], [(4, i % 5) for i in range(24)],
                                  [(5, 300), (3, 600), (2, 0)], [(20, 0), (33, 1), (150, 4)]], ids=["single", "chunks", "drafts", "draft_chunks", "wide"])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (16, 2)], ids=lambda h: "x".join(map(str, h)))
def test_weights_are_summed_as_they_are_multiplied(torch, d, seqs, heads):
    """Values that are the same at every position come back as they are, whatever the weights are rounded to: numerator and denominator
    hold the same weights."""
    v_scale = 0.0121
    w = World(torch, seqs, *heads, d, 64, e4m3=True, scales=(0.02, v_scale), seed=85)
    w.write_new()
    # per head dim one e4m3 number whose product with the scale is far from the middle between two bf16 numbers: nearer to it than
    # that come only sums of 600 positions in fp32, twice, and three roundings more, 1203 * 2^-24 < 2^-13
    c = np.array([m * 2.0 ** e for e in (-3, 0, 4) for m in range(8, 16)]) * np.float64(np.float32(v_scale))
    near = U.f64(U.W.bf16_bits_from_f32(c.astype(np.float32)))
    step = 2.0 ** (np.floor(np.log2(c)) - 7)
    ok = np.abs(np.abs(c - near) - step / 2) > 2.0 ** -13 * c
    per_dim = np.resize((c / np.float64(np.float32(v_scale)))[ok], d)
    want = np.resize(near[ok], d)
    for s, (n, before) in enumerate(w.seqs):
        _, vp = P.places(w.table[s], np.arange(n + before), heads[1], 64, d, 16)
        w.hv[vp] = np.round(per_dim * 2 ** 10) / 2 ** 10
    w.dv.copy_(w.upload(w.hv))
    got = w.download(w.attend()).reshape(w.T, heads[0], d)
    assert np.array_equal(got, np.broadcast_to(want, got.shape)), np.max(np.abs(got / want - 1))


@CACHES
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (8, 1)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("seqs", [[(1, 90), (1, 300), (1, 31), (1, 700)], [(4, 200), (3, 40), (2, 513)], [(64, 130), (150, 0)]],
                         ids=["single", "draft", "wide"])
def test_rotated_queries_keep_their_bits(torch, e4m3, d, heads, seqs):
    """Scores so large that the queries' rounding decides: rotated queries are two bf16 whose sum is off by 2^-16, in the wide
    kernel over e4m3 fp16, off by 2^-11, with weights as precise.  Queries of one bf16 would not pass: two parts by the bound of the
    worst element, fp16 by the rms of all of them."""
    wide = seqs[0][0] > 32
    w = World(torch, seqs, *heads, d, 64, e4m3=e4m3, amplitude=3.0, scales=(0.05, 0.05), seed=86)
    w.write_new()
    got = w.download(w.attend()).reshape(w.T, heads[0], d)
    half = 2.0 ** -11 if wide and e4m3 else HALF_BF16
    worst = worst_of_one = 0.0
    squares = np.zeros(4)                                    # of the error, of the error with queries of one bf16, of output and values
    for s, (n, before) in enumerate(seqs):
        a, b = w.q_start[s], w.q_start[s + 1]
        pos = before + np.arange(n)
        x = w.qkv64[a:b, :heads[0] * d].reshape(n, heads[0], d)
        q = P.rotate(x, pos, w.rope64)
        k, v, there = w.sequence(s)
        want, moved = P.attention(q, k, v, pos, there, d ** -0.5)
        sums = (len(there) + d) * HALF_F32 * 2
        # three fp32 roundings in a rotated element, of terms up to its pair's length: 2^-21 of the pair's two
        eps_q = (2.0 ** -11 if wide and e4m3 else HALF_BF16 ** 2) + 2.0 ** -21 + sums
        # fp16 weights below 2^-20 of the largest are off by up to 2^-31 of it each
        thin = len(there) * 2.0 ** -31 * np.max(np.abs(v)) if wide and e4m3 else 0.0
        # weights in numerator and denominator move the output by half * sum w |v - out|, at most half * (sum w |v| + |out|)
        tol = (HALF_BF16 + half) * np.abs(want) + moved(eps_q, half + sums) * (1 + 2 ** -4) + thin
        worst = max(worst, np.max(np.abs(got[a:b] - want) / tol))
        one = U.f64(U.W.bf16_bits_from_f32(q.astype(np.float32)))
        off = P.attention(one, k, v, pos, there, d ** -0.5)[0] - want
        worst_of_one = max(worst_of_one, np.max(np.abs(off) / tol))
        squares += [want.size * np.mean(x ** 2) for x in (got[a:b] - want, off, want, v)]
    assert worst <= 1, worst
    if not (wide and e4m3):
        assert worst_of_one > 1, worst_of_one                # the test can tell
        return
    # an eighth of the error of one bf16, the output's rounding and twice the weights', evenly spread: half / sqrt(3) each
    rms, rms_of_one, rms_out, rms_v = np.sqrt(squares / (w.T * heads[0] * d))
    bound = rms_of_one / 8 + (HALF_BF16 * rms_out + 2 * half * rms_v) / np.sqrt(3)
    assert rms <= bound and bound < rms_of_one, (rms, bound, rms_of_one)


@CACHES
@pytest.mark.parametrize("heads", [(4, 4), (8, 2)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("n", [3, 90, 300], ids=["draft", "wide", "tiles"])
def test_a_value_that_is_not_finite_under_a_window(torch, e4m3, heads, n):
    """Every query that sees it shows it; other sequences do not, nor do queries once the window of every query of the call has
    left it; what other queries of its sequence and call show is left open."""
    window, d = 64, 128
    seqs = [(1, 200), (n, 100), (1, 90), (2, 130)]
    w = World(torch, seqs, *heads, d, 32, e4m3=e4m3, seed=87)
    w.write_new()
    want = w.attend(window=window)
    a, b, pos = w.q_start[1], w.q_start[2], 100 + np.arange(n)

    def with_nan_at(at):
        place = P.places(w.table[1], [at], heads[1], 32, d, w.piece)[1]
        was, w.hv[place] = w.hv[place], np.nan               # which e4m3 has, too
        w.dv.copy_(w.upload(w.hv))
        w.hv[place] = was
        return w.attend(window=window)

    got = with_nan_at(70)
    same = torch.eq(got.view(torch.int16), want.view(torch.int16)).all(dim=1)
    assert torch.all(same[:a]) and torch.all(same[b:])
    sees = torch.from_numpy((pos >= 70) & (pos - window < 70)).cuda()
    assert sees.any() and torch.isnan(got[a:b][sees]).all()
    assert torch.equal(with_nan_at(20), want)                # before the first query's window
    w.dv.copy_(w.upload(w.hv))
    place = P.places(w.table[1], [70], heads[1], 32, d, w.piece)[0]
    w.hk[place] = np.nan
    w.dk.copy_(w.upload(w.hk))
    got = w.attend(window=window)                            # a key reaches those that see it alone
    same = torch.eq(got.view(torch.int16), want.view(torch.int16)).all(dim=1)
    assert torch.all(same[:a]) and torch.all(same[b:]) and torch.equal(same[a:b], ~sees) and torch.isnan(got[a:b][sees]).all()


def of_bits(x, bits):
    """x rounded to so many significant bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.round(m * 2.0 ** bits), e - bits)


@CACHES
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (16, 2), (16, 1)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("seqs", [[(1, 90), (1, 300), (1, 31), (1, 700)] * 4, [(2, 200), (2, 40), (2, 513)] * 3], ids=["single", "draft"])
def test_weights_of_short_sequences_keep_their_bits(torch, e4m3, d, heads, seqs):
    """Weights of 15 bits, over e4m3 with more than eight rows of 11, and an output rounded to bf16: the rms of all errors is that of
    an oracle with just these roundings, nearer to it than to one whose weights are bf16."""
    w = World(torch, seqs, *heads, d, 64, e4m3=e4m3, seed=88)
    w.write_new()
    got = w.download(w.attend()).reshape(w.T, heads[0], d)
    G = heads[0] // heads[1]
    bits = 11 if e4m3 and max(n for n, _ in seqs) * G > 8 else 15
    err, as_stated, as_bf16 = [], [], []
    for s, (n, before) in enumerate(seqs):
        a, b = w.q_start[s], w.q_start[s + 1]
        pos = before + np.arange(n)
        q = P.rotate(w.qkv64[a:b, :heads[0] * d].reshape(n, heads[0], d), pos, w.rope64)
        k, v, _ = w.sequence(s)
        for h in range(heads[0]):
            score = np.where(np.arange(n + before) <= pos[:, None], q[:, h] @ k[:, h // G].T * d ** -0.5, -np.inf)
            weight = np.exp(score - score.max(axis=1, keepdims=True))
            out = lambda x: x @ v[:, h // G] / x.sum(axis=1, keepdims=True)  # noqa: E731
            stored = lambda x: U.f64(U.W.bf16_bits_from_f32(x.astype(np.float32)))  # noqa: E731
            want = out(weight)
            err.append(got[a:b, h] - want)
            as_stated.append(stored(out(of_bits(weight, bits))) - want)
            as_bf16.append(stored(out(of_bits(weight, 8))) - want)
    rms, stated, bf16 = (np.sqrt(np.mean(np.concatenate(x) ** 2)) for x in (err, as_stated, as_bf16))
    assert stated * 1.1 < bf16                               # the test can tell
    assert rms <= (stated + bf16) / 2, (rms, stated, bf16)


def test_changes_on_the_stream_that_ran_the_batch_and_on_another(torch):
    """Operations and a rebuild on one stream, a rebuild on another, results in between, and the end: no event of the first stream's
    operations was ever recorded."""
    import paper_2412_17246_amd as lib
    L = lib.load_library()
    w = World(torch, [(1, 100)], 4, 2, 64, 32, seed=89)
    w.write_new()
    want = w.attend()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    bytes_ = int(L.bz_batch_storage_bytes(1, 1, 256))
    storage = (torch.empty(bytes_, dtype=torch.uint8, device="cuda"), torch.empty(2 * bytes_, dtype=torch.uint8, pin_memory=True), a)
    outs, space = [torch.zeros_like(want) for _ in range(3)], w.workspace()
    torch.cuda.synchronize()
    w.batch = batch = lib.Batch(L, [0, 1], [0], [100], storage=storage)
    w.attend(out=outs[0], workspace=space, stream=a)
    batch.rebuild([0, 1], [0], [100], stream=a)
    batch.rebuild([0, 1], [0], [100], stream=b)
    w.attend(out=outs[1], workspace=space, stream=b)
    batch.rebuild([0, 1], [0], [100], stream=b)
    w.attend(out=outs[2], workspace=space, stream=b)
    batch.close()                                            # waits
    for out in outs:
        assert torch.equal(out, want)
