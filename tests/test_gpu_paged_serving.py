"""The paged KV cache's operations as a serving program calls them: long key ranges cut into several workgroups, many sequences,
batches that are rebuilt and advanced, several streams, graphs, large pools, refusals."""
import ctypes as C

import numpy as np
import pytest

from tests.test_gpu_paged import CACHES, World, check_append

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


CUT = {
    # wide rows over several key ranges; lengths that end in every part of a tile
    "chunks": [(40, 2000), (17, 700), (300, 513), (1, 900)],
    # a chunk of which some rows' windows and ranges lie before others'
    "long_chunk": [(530, 1500)],
    # one tile of rows, one key more than a multiple of the tile
    "drafts": [(9, 1016), (16, 1009), (3, 4000), (2, 254)],
}


@CACHES
@pytest.mark.parametrize("heads", [(8, 2, 128), (3, 3, 64), (64, 1, 128), (10, 2, 64)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("seqs", list(CUT))
def test_key_ranges(torch, e4m3, heads, seqs):
    w = World(torch, CUT[seqs], *heads, 128, e4m3=e4m3, seed=21)
    w.write_new()
    out = w.attend()
    w.check(out)
    assert torch.equal(out, w.attend())                     # the same call, the same bits
    w.check(w.attend(window=333), window=333)


@CACHES
def test_key_ranges_with_absent_pages(torch, e4m3):
    w = World(torch, [(60, 3000), (1, 3000), (5, 2500)], 8, 2, 128, 32, e4m3=e4m3, seed=22,
              absent=[(s, i) for s in range(3) for i in list(range(3, 40)) + [60, 61, 70]])
    w.write_new()
    w.check(w.attend())


@CACHES
@pytest.mark.parametrize("page", [32, 64, 128, 256, 512, 1024])
def test_page_sizes(torch, e4m3, page):
    w = World(torch, [(1, 1100), (200, 901), (6, 1023)], 4, 2, 64, page, e4m3=e4m3, seed=23)
    bits = torch.uint8 if e4m3 else torch.int16
    was = w.dk.view(bits).cpu().numpy(), w.dv.view(bits).cpu().numpy()
    w.append()
    check_append(w, *was)
    w.write_new()
    w.check(w.attend())


@CACHES
@pytest.mark.parametrize("window", [0, 200])
def test_many_sequences(torch, e4m3, window):
    """Odd and even numbers of chunks, one chunk among them, ends on either side of a chunk's."""
    rng = np.random.default_rng(24)
    seqs = [(1, int(n)) for n in rng.integers(0, 1300, 90)] + [(2, 511), (3, 513), (1, 255), (1, 256), (1, 511), (1, 512)]
    w = World(torch, seqs, 8, 8, 64, 64, e4m3=e4m3, seed=24)
    w.write_new()
    w.check(w.attend(window=window), window=window)


@CACHES
def test_decode_steps_of_an_advanced_batch(torch, e4m3):
    """A batch of single tokens advanced on the device: its chunks and lengths grow, pages fill."""
    from paper_2412_17246_amd import Instance
    import workloads as W
    steps, rng = 6, np.random.default_rng(25)
    lens = [int(n) for n in rng.integers(0, 600, 60)] + [255 - 2, 256 - 2, 511 - 2, 512 - 3, 30, 31]
    worlds = [World(torch, [(1, n + i) for n in lens], 8, 8, 64, 1024, e4m3=e4m3, seed=25 + i) for i in range(steps)]
    first = worlds[0]
    inst = Instance(W.CONFIGS["tiny"], max_seqs=1, max_seq_len=64, max_tokens=1, kv_tokens=32, compute_stream=torch.cuda.current_stream())
    for i, w in enumerate(worlds):                          # the later steps' tokens into the first world's pages
        w.table, w.dtable, w.dk, w.dv, w.kv, w.batch = first.table, first.dtable, first.dk, first.dv, first.kv, first.batch
        if i:
            inst.batch_advance(first.batch)
        w.append()
        out = w.attend()
        w.hk, w.hv = w.download(w.dk), w.download(w.dv)
        w.check(out)
    inst.close()


def test_rebuilt_batches_on_two_streams(torch):
    """A batch in lent memory, rebuilt on one stream while another runs operations on it: the library orders the two on the
    device.  Nothing waits on the host until the end."""
    import paper_2412_17246_amd as lib
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    shapes = [[(1, 700), (5, 300)], [(40, 100)], [(1, 30), (1, 900), (3, 3)], [(64, 64), (1, 1)]]
    worlds = [World(torch, s, 8, 2, 128, 64, seed=30 + i) for i, s in enumerate(shapes)]
    for w in worlds:
        w.write_new()
    bytes_ = int(lib.load_library().bz_batch_storage_bytes(4, 128, 1024))
    dev = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
    pinned = torch.empty(2 * bytes_, dtype=torch.uint8, pin_memory=True)
    spaces = [w.workspace() for w in worlds]
    outs = [torch.full((w.T, w.Hq * w.d), 7.0, dtype=torch.bfloat16, device="cuda") for w in worlds]
    torch.cuda.synchronize()
    batch, others = None, []
    for turn in range(3):
        for w, ws, out in zip(worlds, spaces, outs):
            args = w.q_start, w.slots, [n for _, n in w.seqs]
            if batch is None:
                batch = lib.Batch(lib.load_library(), *args, storage=(dev, pinned, a))
            else:
                batch.rebuild(*args, stream=a if turn < 2 else b)
            others.append(torch.empty_like(out))
            out_b = out if turn == 2 else others[-1]
            lib.op_paged_append(batch, w.kv, w.k, w.v, rope=w.rope, stream=b)
            lib.op_paged_attention(batch, w.kv, w.q, out_b, rope=w.rope, workspace=ws, stream=b)
    torch.cuda.synchronize()
    for w, out in zip(worlds, outs):
        w.hk, w.hv = w.download(w.dk), w.download(w.dv)
        w.check(out)
    batch.close()


@CACHES
def test_output_in_place_of_the_queries(torch, e4m3):
    w = World(torch, [(1, 700), (200, 150), (4, 600), (33, 2000), (1, 20)], 8, 2, 128, 64, e4m3=e4m3, seed=43)
    w.write_new()
    w.q = w.q.contiguous()
    want = w.attend()
    assert torch.equal(w.attend(out=w.q), want)


def test_two_streams_at_once(torch):
    """Two calls in flight, with a workspace each; a batch of its own each, and one for both."""
    import paper_2412_17246_amd as lib
    w = World(torch, [(1, 2000), (30, 1500), (4, 800)], 8, 2, 128, 64, seed=41)
    w.write_new()
    want = w.attend()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(want) for _ in range(2)]
    spaces = [w.workspace() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, out, ws in zip(streams, outs, spaces):
            lib.op_paged_attention(w.batch, w.kv, w.q, out, rope=w.rope, workspace=ws, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@CACHES
def test_captured_step(torch, e4m3):
    """Append and attention in a graph: replayed on other inputs and other pages, with eager calls in between."""
    import paper_2412_17246_amd as lib
    w = World(torch, [(1, 400), (1, 40), (1, 1023)], 8, 2, 128, 64, e4m3=e4m3, seed=51)
    other = World(torch, [(1, 400), (1, 40), (1, 1023)], 8, 2, 128, 64, e4m3=e4m3, seed=52)
    out, ws = torch.empty(w.T, w.Hq * w.d, dtype=torch.bfloat16, device="cuda"), w.workspace()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        lib.op_paged_append(w.batch, w.kv, w.k, w.v, rope=w.rope, stream=st)
        lib.op_paged_attention(w.batch, w.kv, w.q, out, rope=w.rope, workspace=ws, stream=st)
    for turn in range(4):
        if turn % 2:                                        # other inputs in the same memory, other pages for them
            w.qkv.copy_(other.qkv)
            w.dtable.copy_(torch.where(w.dtable >= 0, w.dk.shape[0] - 1 - w.dtable, w.dtable))
        graph.replay()
        torch.cuda.synchronize()
        got, k, v = out.clone(), w.dk.clone(), w.dv.clone()
        w.append()
        eager = w.attend()
        torch.cuda.synchronize()
        raw = torch.uint8 if e4m3 else torch.int16            # bits: the other pages hold NaN, too
        assert torch.equal(got.view(torch.int16), eager.view(torch.int16)) and torch.equal(k.view(raw), w.dk.view(raw)) and torch.equal(v.view(raw), w.dv.view(raw))


def test_capture_of_a_batch_changed_elsewhere_is_refused(torch):
    import paper_2412_17246_amd as lib
    w = World(torch, [(1, 100)], 4, 2, 64, 32, seed=53)
    bytes_ = int(lib.load_library().bz_batch_storage_bytes(1, 1, 256))
    storage = (torch.empty(bytes_, dtype=torch.uint8, device="cuda"), torch.empty(2 * bytes_, dtype=torch.uint8, pin_memory=True),
               torch.cuda.Stream())
    batch = lib.Batch(lib.load_library(), [0, 1], [0], [100], storage=storage)
    torch.cuda.synchronize()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    x = torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph, stream=st):
        x += 1
        with pytest.raises(lib.BzError) as e:
            lib.op_paged_append(batch, w.kv, w.k, w.v, rope=w.rope, stream=st)
        assert e.value.name == "BZ_ESTATE"
    graph.replay()                                          # the capture went on without it
    torch.cuda.synchronize()
    assert torch.all(x == 1)
    batch.close()


def test_batch_in_tight_storage(torch):
    """Lent memory with no room for the list of short sequences: they take the other kernel."""
    import paper_2412_17246_amd as lib
    w = World(torch, [(2, 90), (5, 700), (3, 0)], 4, 2, 128, 64, seed=54)
    w.write_new()
    words = (3 + 1) + 3 + 3 + w.T + 2 * 3
    size = (words * 4 + 31) // 32 * 32 + 64
    for bytes_ in (max(size, 128), 4096):
        dev = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
        pinned = torch.empty(2 * bytes_, dtype=torch.uint8, pin_memory=True)
        w.batch = lib.Batch(lib.load_library(), w.q_start, w.slots, [b for _, b in w.seqs], storage=(dev, pinned, None))
        w.check(w.attend())
        w.batch.close()


@CACHES
def test_pool_beyond_32_bits(torch, e4m3):
    """A pool of more than 2^32 bytes, and for e4m3 elements, the sequence's pages at its end."""
    import paper_2412_17246_amd as lib
    w = World(torch, [(1, 130), (70, 60)], 8, 8, 128, 256, e4m3=e4m3, seed=55)
    w.write_new()
    want, pool, page = w.attend(), w.dk.shape[0], 8 * 256 * 128
    n = (1 << 32) // page + 40
    k, v = (torch.empty(n, 8, 256 * 128, dtype=w.kind, device="cuda") for _ in range(2))
    raw = torch.uint8 if e4m3 else torch.int16
    k.view(raw)[n - pool:].copy_(w.dk.view(raw))
    v.view(raw)[n - pool:].copy_(w.dv.view(raw))
    table = torch.where(w.dtable >= 0, w.dtable + (n - pool), w.dtable)
    w.kv = lib.PagedKv(256, 8, 128, k=k, v=v, page_table=table, k_scale=w.scales[0], v_scale=w.scales[1])
    assert torch.equal(w.attend(), want)
    w.append()
    old = lib.PagedKv(256, 8, 128, k=w.dk, v=w.dv, page_table=w.dtable, k_scale=w.scales[0], v_scale=w.scales[1])
    lib.op_paged_append(w.batch, old, w.k, w.v, rope=w.rope)
    torch.cuda.synchronize()
    assert torch.equal(k.view(raw)[n - pool:], w.dk.view(raw)) and torch.equal(v.view(raw)[n - pool:], w.dv.view(raw))
    a, b = (torch.empty(2, 130, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.op_paged_read(w.kv, 1, 0, 130, a[0], a[1])
    lib.op_paged_read(old, 1, 0, 130, b[0], b[1])
    assert torch.equal(a, b)


def test_a_value_that_is_not_finite_stays_in_its_sequence(torch):
    w = World(torch, [(1, 200), (33, 64), (1, 90)], 4, 2, 128, 32, seed=56)
    w.write_new()
    want = w.attend()
    w.hv[w.table[1, 0]] = np.inf
    w.dv.copy_(w.upload(w.hv))
    got = w.attend()
    assert torch.equal(got[0], want[0]) and torch.equal(got[34], want[34]) and not torch.any(torch.isfinite(got[1:34]))


def test_refusals(torch):
    import paper_2412_17246_amd as lib
    L = lib.load_library()
    w = World(torch, [(1, 63), (5, 30)], 4, 2, 64, 32, seed=57)
    before = w.dk.view(torch.int16).clone(), w.dv.view(torch.int16).clone()
    out = torch.full((w.T, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    kv, b = w.kv._ref, w.batch.handle
    row, rope, npos = w.row, w.rope.data_ptr(), w.rope.shape[0]
    k, v, q, o = w.k.data_ptr(), w.v.data_ptr(), w.q.data_ptr(), out.data_ptr()

    def append(k=k, ks=row, v=v, vs=row, rope=rope, npos=npos, kv=kv):
        return L.bz_op_paged_append(b, kv, k, ks, v, vs, rope, npos, None)

    def attend(q=q, qs=row, o=o, os=256, hq=4, scale=0.0, window=0, rope=rope, npos=npos, ws=ws.data_ptr(), wsb=ws.numel(), kv=kv, b=b):
        return L.bz_op_paged_attention(b, kv, q, qs, o, os, hq, scale, window, rope, npos, ws, wsb, None)

    EINVAL, ENOMEM, ECAPACITY = -1, -2, -7
    for bad in (dict(k=0), dict(v=0), dict(k=k + 8), dict(ks=row + 4), dict(ks=120), dict(vs=-row), dict(rope=rope + 4), dict(npos=0)):
        assert append(**bad) == EINVAL, bad
    for bad in (dict(q=0), dict(o=0), dict(q=q + 2), dict(o=o + 8), dict(qs=row + 1), dict(qs=248), dict(os=252), dict(hq=0), dict(hq=3),
                dict(hq=2048), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1),
                dict(ws=ws.data_ptr() + 8), dict(rope=rope + 8), dict(npos=-5)):
        assert attend(**bad) == EINVAL, bad
    assert append(npos=63) == ECAPACITY and attend(npos=63) == ECAPACITY
    short = w.kv.desc.__class__.from_buffer_copy(w.kv.desc)
    short.pages_per_row = 1                                 # 32 positions
    assert append(kv=C.byref(short)) == ECAPACITY and attend(kv=C.byref(short)) == ECAPACITY
    few = w.kv.desc.__class__.from_buffer_copy(w.kv.desc)
    few.n_rows = 1
    assert append(kv=C.byref(few)) == EINVAL and attend(kv=C.byref(few)) == EINVAL
    big = World(torch, [(1, 600), (5, 700)], 4, 2, 64, 32, seed=58)
    need = lib.op_paged_attention_workspace_bytes(big.batch, big.kv, 4)
    assert need > 0
    for m in (dict(ws=None), dict(wsb=need - 1), dict(ws=None, wsb=0)):
        assert attend(b=big.batch.handle, kv=big.kv._ref, q=big.q.data_ptr(), qs=big.row, rope=big.rope.data_ptr(), npos=big.rope.shape[0], **m) == ENOMEM
    for n, window in ((0, 0), (3, 0), (4, -1), (2048, 0)):
        assert L.bz_op_paged_attention_workspace_bytes(big.batch.handle, big.kv._ref, n, window) == 0
    torch.cuda.synchronize()
    assert torch.all(out == 7) and torch.equal(w.dk.view(torch.int16), before[0]) and torch.equal(w.dv.view(torch.int16), before[1])

    for bad in (lambda: lib.op_paged_append(w.batch, w.kv, w.k.float(), w.v), lambda: lib.op_paged_append(w.batch, w.kv, w.k[:3], w.v),
                lambda: lib.op_paged_append(w.batch, w.kv, w.k[:, :64], w.v), lambda: lib.op_paged_append(w.batch, w.kv, w.k.cpu(), w.v),
                lambda: lib.op_paged_append(w.batch, w.kv, w.k, w.v, rope=w.rope[:, :16]),
                lambda: lib.op_paged_attention(w.batch, w.kv, w.q, out[:, :64]), lambda: lib.op_paged_attention(w.batch, w.kv, w.q.t(), out),
                lambda: lib.op_paged_read(w.kv, 0, 0, 9, out[:1], out), lambda: lib.PagedKv(32, 2, 64, k=w.dk, v=w.dv[:-1], page_table=w.dtable),
                lambda: lib.PagedKv(32, 2, 64, k=w.dk, v=w.dv, page_table=w.dtable.long()),
                lambda: lib.PagedKv(32, 2, 64, k=w.dk.float(), v=w.dv.float(), page_table=w.dtable)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(lib.BzError):
        lib.PagedKv(16, 2, 128, k=w.dk, v=w.dv, page_table=w.dtable)


def test_a_layer_by_single_operations_agrees_with_run_layers(torch):
    """Two steps of one decoder layer, a prompt with a chunk beside it and then a token each: norm, projections and SwiGLU by the single
    operations around the paged cache, against the oracle and beside bz_run_layers on its own cache."""
    import paper_2412_17246_amd as lib
    import workloads as W
    from oracle import decoder as O
    from tests import _util as U
    s = W.CONFIGS["tiny"]
    bits = W.layer_weights_bits(s, 0)
    inst = U.make_instance(s, max_seqs=2, max_seq_len=256, max_tokens=128, kv_tokens=512)
    pinned = inst.pinned_blob(inst.pack_layer(bits))
    inst.load_layer(0, pinned)
    for slot in range(2):
        inst.kv_reserve(slot, 256)
    blob = pinned.cuda()
    at = lambda name, rows, cols: blob[getattr(inst.layout, name):][:rows * cols * 2].view(torch.bfloat16)  # noqa: E731
    Hq, Hkv, d, H, F = s.Hq, s.Hkv, s.d, s.H, s.F
    nqkv = (Hq + 2 * Hkv) * d
    table = torch.tensor([[3, 0, 5, 1], [2, 4, 7, 6]], dtype=torch.int32, device="cuda")
    k, v = (torch.full((8, Hkv, 64 * d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv = lib.PagedKv(64, Hkv, d, k=k, v=v, page_table=table)
    rope = torch.from_numpy(lib.rope_table(256, d, s.rope_base)).cuda()
    osh, wts, okv = U.oracle_shape(s), {0: U.oracle_weights(bits)}, O.OracleKV()
    for step, (q_start, before) in enumerate([([0, 70, 90], [0, 0]), ([0, 1, 2], [70, 20])]):
        T = q_start[-1]
        xbits = W.bf16_bits_from_f32((np.random.default_rng([61, step]).standard_normal((T, H)) / 16).astype(np.float32))
        x = U.to_device(xbits, False)
        y = x.clone()
        batch = lib.Batch(lib.load_library(), q_start, [0, 1], before)
        normed, qkv = torch.empty_like(x), torch.empty(T, nqkv, dtype=torch.bfloat16, device="cuda")
        attn, act = (torch.empty(T, n, dtype=torch.bfloat16, device="cuda") for n in (Hq * d, F))
        ws = torch.empty(max(16, lib.op_paged_attention_workspace_bytes(batch, kv, Hq)), dtype=torch.uint8, device="cuda")
        lib.op_rmsnorm(x, at("g1", 1, H), normed, s.eps)
        lib.op_gemm(0, normed, at("wq", nqkv, H), None, qkv, T, nqkv, H)
        lib.op_paged_append(batch, kv, qkv[:, Hq * d:(Hq + Hkv) * d], qkv[:, (Hq + Hkv) * d:], rope=rope)
        lib.op_paged_attention(batch, kv, qkv[:, :Hq * d], attn, rope=rope, workspace=ws)
        lib.op_gemm(1, attn, at("wo", H, Hq * d), x, x, T, H, Hq * d)
        lib.op_rmsnorm(x, at("g2", 1, H), normed, s.eps)
        lib.op_gemm(2, normed, at("wg", 2 * F, H), None, act, T, F, H)
        lib.op_gemm(1, act, at("wd", H, F), x, x, T, H, F)
        inst.run_layers(0, 1, batch, y)
        inst.sync()
        want = O.run_layers(osh, wts, 0, 1, U.f64(xbits), O.OracleBatch(q_start, [0, 1], before), okv)
        for got in (x, y):
            assert U.rel_err(U.from_device(got), want) <= U.BF16_TOL
            U.assert_rms(U.from_device(got), want, U.RMS_BF16)
    inst.close()


def test_scales_that_vanish_or_overflow_are_refused(torch):
    """scale times k_scale has to be a normal float: at 0 a masked score, minus infinity, would become a NaN."""
    w = World(torch, [(1, 63), (50, 30)], 4, 2, 64, 32, e4m3=True, seed=71, scales=(2.0 ** -100, 0.03))
    w.write_new()
    assert torch.isfinite(w.attend(scale=2.0 ** -20).float()).all()
    for scale in (2.0 ** -30, 1e-45):
        with pytest.raises(w.lib.BzError):
            w.attend(scale=scale)
    w.kv = w.lib.PagedKv(32, 2, 64, k=w.dk, v=w.dv, page_table=w.dtable, k_scale=2.0 ** 100, v_scale=0.03)
    with pytest.raises(w.lib.BzError):
        w.attend(scale=2.0 ** 28)


def test_rebuild_while_a_stream_that_ran_the_batch_is_captured(torch):
    """The rebuild has to follow the attention on the other stream, which cannot be asked for its end under capture: refused, and
    the capture goes on; afterwards it succeeds."""
    import paper_2412_17246_amd as lib
    L = lib.load_library()
    w = World(torch, [(1, 100)], 4, 2, 64, 32, seed=72)
    w.write_new()
    bytes_ = int(L.bz_batch_storage_bytes(1, 1, 256))
    storage = (torch.empty(bytes_, dtype=torch.uint8, device="cuda"), torch.empty(2 * bytes_, dtype=torch.uint8, pin_memory=True),
               torch.cuda.Stream())
    w.batch = batch = lib.Batch(L, [0, 1], [0], [100], storage=storage)
    torch.cuda.synchronize()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    space = w.workspace()

    def attend():
        out = torch.zeros(1, w.Hq * w.d, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        w.attend(out=out, workspace=space, stream=st)
        return out

    want = attend()
    torch.cuda.synchronize()
    x = torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph, stream=st, capture_error_mode="relaxed"):
        x += 1
        with pytest.raises(lib.BzError) as e:
            batch.rebuild([0, 1], [0], [64])
        assert e.value.name == "BZ_ESTATE"
    graph.replay()
    again = attend()
    torch.cuda.synchronize()
    assert torch.all(x == 1) and torch.equal(again, want)
    batch.rebuild([0, 1], [0], [100])
    again = attend()
    torch.cuda.synchronize()
    assert torch.equal(again, want) and torch.any(want != 0)
    batch.close()


def test_output_over_the_queries_with_another_pitch_is_refused(torch):
    """In place means row by row: with another pitch the first rows would overwrite queries that are still to be read."""
    w = World(torch, [(1, 63), (50, 30)], 4, 2, 64, 32, seed=73)
    w.write_new()
    L, ws = w.lib.load_library(), w.workspace()
    before = w.qkv.clone()
    call = lambda pitch: L.bz_op_paged_attention(w.batch.handle, w.kv._ref, w.q.data_ptr(), w.row, w.q.data_ptr(), pitch, 4, 0.0, 0,  # noqa: E731
                                                 w.rope.data_ptr(), w.rope.shape[0], ws.data_ptr(), ws.numel(), None)
    assert call(w.row - 8) == -1 and call(256) == -1
    torch.cuda.synchronize()
    assert torch.equal(w.qkv, before)
    want = w.attend()
    assert call(w.row) == 0
    torch.cuda.synchronize()
    assert torch.equal(w.q, want)
