"""How a batch is ordered between streams, and what is refused, with a stand-in for the HIP runtime (c_abi/hip_standin.c) that keeps
the books: no GPU, kernels are counted and not run.  Each test is a process of its own, in which the stand-in is loaded first."""
import inspect
import os
import subprocess
import sys
import textwrap

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PRELUDE = """
import ctypes as C, sys
from types import SimpleNamespace
sys.path.insert(0, %r)
hip = C.CDLL(%r, mode=C.RTLD_GLOBAL)
from paper_2412_17246_amd import binding as B
L = B.load_library(%r)
A, S, T = 0x1000, 0x2000, 0x3000                             # streams
stream = lambda h: SimpleNamespace(cuda_stream=h)
for f, ret, args in (("capture", None, [C.c_void_p, C.c_ulonglong]), ("release", None, [C.c_void_p]), ("dead_uses", C.c_int, []),
                     ("forbidden", C.c_int, []), ("pending", C.c_long, [C.c_void_p]), ("unordered", C.c_long, [C.c_void_p, C.c_void_p]),
                     ("work", None, [C.c_void_p]), ("launches", C.c_long, []), ("grid", None, [C.c_void_p])):
    fn = getattr(hip, "standin_" + f)
    fn.restype, fn.argtypes = ret, args
class Lent:
    def __init__(self, n):
        self.raw = C.create_string_buffer(n + 64)
        self.n, self.at = n, (C.addressof(self.raw) + 63) // 64 * 64
    def data_ptr(self): return self.at
    def numel(self): return self.n
def lent(st, q_start=(0, 1), slots=(0,), before=(100,), size=1 << 15):
    return B.Batch(L, q_start, slots, before, storage=(Lent(size), Lent(2 * size), stream(st)))
KV = B.bz_paged_kv(4096, 8192, 256, 64, 64, 16, 16, 2, 64, B.BZ_KV_ACT, 1.0, 1.0)
def append(batch, st, kv=KV):
    width = kv.n_kv_heads * kv.head_dim
    return L.bz_op_paged_append(batch.handle, C.byref(kv), 4096, width, 8192, width, None, 0, st)
def rebuild(batch, st):
    try:
        batch.rebuild([0, 1], [0], [64], stream=stream(st))
    except B.BzError as e:
        return e.status
    return 0
EINVAL, ENOMEM, EHIP, ECAPACITY, ESTATE = -1, -2, -6, -7, -8
"""


@pytest.fixture(scope="module")
def standin(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("standin") / "libstandin.so")
    subprocess.run(["gcc", "-std=c11", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-Werror",
                    os.path.join(ROOT, "tests", "c_abi", "hip_standin.c"), "-o", so], check=True)
    return so


def run(standin, scenario, fp32=False):
    """The body of `scenario`, a function without arguments, in a process of its own."""
    body = textwrap.dedent(inspect.getsource(scenario).split("():\n", 1)[1])
    code = PRELUDE % (ROOT, standin, fp32) + body + '\nprint("scenario done")\n'
    res = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0 and "scenario done" in res.stdout, res.stdout + res.stderr


BUILDS = pytest.mark.parametrize("fp32", [False, True], ids=["bf16", "fp32dbg"])


@BUILDS
def test_destroy_while_a_stream_that_ran_the_batch_is_captured(standin, fp32):
    """Kernels that were enqueued before the capture may still read the batch, and the stream cannot be asked for their end: refused,
    and the batch stays as it was."""
    def scenario():
        b = lent(A)
        assert append(b, S) == 0 and append(b, T) == 0
        hip.standin_capture(S, 7)
        assert L.bz_batch_destroy(b.handle) == ESTATE and hip.standin_pending(S) > 0
        assert L.bz_batch_tokens(b.handle) == 1 and append(b, T) == 0
        hip.standin_capture(S, 0)
        assert L.bz_batch_destroy(b.handle) == 0 and hip.standin_pending(S) == 0 and hip.standin_pending(T) == 0
        b.handle = None
        assert hip.standin_forbidden() == 0 and hip.standin_dead_uses() == 0

    run(standin, scenario, fp32)


@BUILDS
def test_destroy_when_a_stream_cannot_be_asked(standin, fp32):
    def scenario():
        b = lent(A)
        assert append(b, S) == 0
        hip.standin_release(S)                                   # too early
        assert L.bz_batch_destroy(b.handle) == EHIP and L.bz_batch_tokens(b.handle) == 1
        b.handle = None

    run(standin, scenario, fp32)


@BUILDS
def test_a_refused_close_can_be_repeated(standin, fp32):
    def scenario():
        b = lent(A)
        assert append(b, S) == 0
        hip.standin_capture(S, 7)
        try:
            b.close()
            raise SystemExit("closed")
        except B.BzError as e:
            assert e.status == ESTATE and b.handle
        hip.standin_capture(S, 0)
        b.close()
        assert b.handle is None and hip.standin_pending(S) == 0
        b.close()

    run(standin, scenario, fp32)


@BUILDS
def test_a_batch_collected_during_a_capture_is_destroyed_later(standin, fp32):
    """With its storage kept until then: the next batch that is made or closed tries again."""
    def scenario():
        import gc, weakref
        b = lent(A)
        memory = weakref.ref(b._storage[0])
        assert append(b, S) == 0
        hip.standin_capture(S, 7)
        del b
        gc.collect()
        other = lent(A)
        assert hip.standin_pending(S) > 0 and memory() is not None
        hip.standin_capture(S, 0)
        other.close()
        gc.collect()
        assert hip.standin_pending(S) == 0 and memory() is None

    run(standin, scenario, fp32)


@BUILDS
def test_a_stream_is_not_asked_again_after_a_change_on_it(standin, fp32):
    """Operations on S, a rebuild on S, S released: what follows is ordered by the rebuild's event."""
    def scenario():
        b = lent(A)
        for turn in range(2):
            assert append(b, S) == 0
        assert rebuild(b, S) == 0
        hip.standin_release(S)
        assert rebuild(b, T) == 0 and hip.standin_unordered(T, S) == 0
        assert append(b, T) == 0 and rebuild(b, A) == 0 and hip.standin_unordered(A, T) == 0
        b.close()
        assert hip.standin_dead_uses() == 0 and hip.standin_pending(S) == 0 and hip.standin_pending(T) == 0

    run(standin, scenario, fp32)


@BUILDS
def test_an_instance_that_advanced_the_batch_may_go(standin, fp32):
    def scenario():
        import workloads as W
        cfg = B.make_config(W.CONFIGS["tiny"], max_seqs=1, max_seq_len=64, max_tokens=1, kv_tokens=64)
        cfg.compute_stream, cfg.copy_stream = S, A
        inst = C.c_void_p()
        assert L.bz_create(C.byref(cfg), C.byref(inst)) == 0
        b = B.Batch(L, [0, 1], [0], [5])
        assert append(b, S) == 0 and L.bz_batch_advance(inst, b.handle) == 0 and append(b, T) == 0
        assert hip.standin_unordered(T, S) == 0
        assert L.bz_destroy(inst) == 0
        hip.standin_release(S)
        b.close()
        assert hip.standin_dead_uses() == 0 and hip.standin_pending(T) == 0

    run(standin, scenario, fp32)


@BUILDS
def test_a_change_on_another_stream_still_asks(standin, fp32):
    """The event of operations on S is recorded for a change on T, and again after more of them; S's own change in between does not
    stand for what S did later."""
    def scenario():
        b = lent(A)
        assert append(b, S) == 0 and rebuild(b, T) == 0 and hip.standin_unordered(T, S) == 0
        assert append(b, S) == 0 and rebuild(b, S) == 0 and append(b, S) == 0
        assert rebuild(b, T) == 0 and hip.standin_unordered(T, S) == 0
        assert append(b, S) == 0
        b.close()
        assert hip.standin_pending(S) == 0 and hip.standin_dead_uses() == 0 and hip.standin_forbidden() == 0

    run(standin, scenario, fp32)


@BUILDS
def test_a_graph_over_two_streams_orders_a_batch_within_itself(standin, fp32):
    """Steps of a split pair captured into one graph: each half on its own stream, the batch advanced in between."""
    def scenario():
        import workloads as W
        s = W.CONFIGS["tiny"]
        pair = []
        for st in (S, T):
            cfg = B.make_config(s, max_seqs=1, max_seq_len=64, max_tokens=1, kv_tokens=64)
            cfg.compute_stream, cfg.copy_stream = st, A
            inst, sizes = C.c_void_p(), B.bz_sizes()
            assert L.bz_create(C.byref(cfg), C.byref(inst)) == 0 and L.bz_query_sizes(C.byref(cfg), C.byref(sizes)) == 0
            blob = C.create_string_buffer(sizes.layer_bytes)
            for l in range(s.L):
                assert L.bz_load_layer(inst, l, blob, sizes.layer_bytes) == 0
            assert L.bz_kv_reserve(inst, 0, 64) == 0 and L.bz_frontier(inst) == s.L
            pair.append(inst)
        b, hidden = B.Batch(L, [0, 1], [0], [5]), C.create_string_buffer(4 * s.H)
        hip.standin_capture(S, 7)
        for step in range(3):
            assert L.bz_run_layers(pair[0], 0, 1, b.handle, hidden, 0) == 0
            assert L.bz_signal_stream(pair[0], T) == 0           # the hidden states
            hip.standin_work(S)
            assert L.bz_run_layers(pair[1], 1, 2, b.handle, hidden, 0) == 0
            assert hip.standin_unordered(S, T) > 0
            assert L.bz_batch_advance(pair[0], b.handle) == 0
            assert hip.standin_unordered(S, T) == 0
        assert hip.standin_forbidden() == 0
        hip.standin_capture(S, 0); hip.standin_capture(T, 0)

    run(standin, scenario, fp32)


@BUILDS
def test_a_graph_of_single_operations_orders_a_batch_within_itself(standin, fp32):
    """Operations on S, the batch advanced on A, one graph; a second graph knows nothing of the first."""
    def scenario():
        import workloads as W
        cfg = B.make_config(W.CONFIGS["tiny"], max_seqs=1, max_seq_len=64, max_tokens=1, kv_tokens=64)
        cfg.compute_stream, cfg.copy_stream = A, T
        inst = C.c_void_p()
        assert L.bz_create(C.byref(cfg), C.byref(inst)) == 0
        b = lent(A)
        hip.standin_capture(A, 7); hip.standin_capture(S, 7)
        assert append(b, S) == ESTATE                            # the last change was no part of the graph
        assert L.bz_batch_advance(inst, b.handle) == 0
        for turn in range(3):
            assert append(b, S) == 0 and hip.standin_unordered(S, A) == 0 and hip.standin_unordered(A, S) > 0
            assert L.bz_batch_advance(inst, b.handle) == 0 and hip.standin_unordered(A, S) == 0
        hip.standin_capture(A, 0); hip.standin_capture(S, 8)
        assert append(b, S) == ESTATE
        hip.standin_capture(S, 0)
        assert hip.standin_forbidden() == 0

    run(standin, scenario, fp32)


@BUILDS
def test_a_change_outside_a_graph_that_is_being_captured(standin, fp32):
    """Operations on S were captured and S still is: a change or the end of the batch would have to follow what never ran."""
    def scenario():
        b = lent(S)
        hip.standin_capture(S, 7)
        assert append(b, S) == 0 and rebuild(b, T) == ESTATE
        try:
            b.close()
            raise SystemExit("closed")
        except B.BzError as e:
            assert e.status == ESTATE
        hip.standin_capture(S, 0)
        assert rebuild(b, T) == 0                                # replays are the caller's to order
        hip.standin_release(S)
        assert append(b, T) == 0 and rebuild(b, A) == 0
        b.close()
        assert hip.standin_dead_uses() == 0 and hip.standin_forbidden() == 0

    run(standin, scenario, fp32)


@BUILDS
def test_grids_that_a_launch_cannot_have_are_refused(standin, fp32):
    """The runtime counts a grid's threads in 32 bits; a number of workgroups beyond that wrapped round and left sequences out."""
    def scenario():
        import numpy as np
        fp32 = bool(L.bz_build_info())
        top = (1 << 32) // 256 - 1
        def grid():
            out = (C.c_uint32 * 3)()
            hip.standin_grid(out)
            return out[0], out[1], out[2]
        def attend(b, kv, heads=2, window=0):
            width = heads * kv.head_dim
            return L.bz_op_paged_attention(b.handle, C.byref(kv), 4096, width, 8192, width, heads, 0.0, window, None, 0, 4096, 1 << 62, S)
        def batch(n, q, before):
            n_seqs = len(before)
            return B.Batch(L, np.arange(n_seqs + 1) * q, np.arange(n_seqs), before)
        def cache(rows, heads=2):
            return B.bz_paged_kv(4096, 8192, 256, 64, 1024, rows, 1 << 19, heads, 64, B.BZ_KV_ACT, 1.0, 1.0)
        # drafts beside one of 2^29 positions: sequences times the longest's chunks times kv heads
        for n, rc in ((1001, ECAPACITY), (4, ECAPACITY), (3, 0)):  # 2^21 chunks and 2 heads: four are one workgroup too many
            b = batch(n, 2, [(1 << 29) - 2] + [7] * (n - 1))
            launches = hip.standin_launches()
            got = attend(b, cache(n))
            assert got == (0 if fp32 else rc), (n, got)          # the plain kernel has a workgroup per token and head
            assert hip.standin_launches() - launches == (1 if fp32 else 0 if rc else 2)
            assert attend(b, cache(n), window=100) == 0
            b.close()
        # 70000 sequences of two tokens, 32 rows each, on 1024 kv heads
        b = batch(70000, 2, [0] * 70000)
        assert append(b, S, cache(70000, 1024)) == (0 if fp32 else ECAPACITY)
        assert append(b, S, cache(70000, 64)) == 0 and grid()[0] <= top
        assert attend(b, cache(70000, 1024), 1024) == (0 if fp32 else ECAPACITY)
        assert attend(b, cache(70000, 64), 64) == 0
        b.close()
        far = cache(1, 1024)
        launches = hip.standin_launches()
        far.pages_per_row = 1 << 20
        assert L.bz_op_paged_read(C.byref(far), 0, 0, 1 << 30, 4096, 4096, S) == ECAPACITY
        assert hip.standin_launches() == launches
        assert L.bz_op_paged_read(C.byref(far), 0, 0, 1 << 20, 4096, 4096, S) == 0

    run(standin, scenario, fp32)


@BUILDS
def test_a_graph_of_a_batch_that_ran_before(standin, fp32):
    """The same behind eager runs on both streams: what is outside the graph is the caller's to order."""
    def scenario():
        import workloads as W
        s = W.CONFIGS["tiny"]
        pair = []
        for st in (S, T):
            cfg = B.make_config(s, max_seqs=1, max_seq_len=64, max_tokens=1, kv_tokens=64)
            cfg.compute_stream, cfg.copy_stream = st, A
            inst, sizes = C.c_void_p(), B.bz_sizes()
            assert L.bz_create(C.byref(cfg), C.byref(inst)) == 0 and L.bz_query_sizes(C.byref(cfg), C.byref(sizes)) == 0
            blob = C.create_string_buffer(sizes.layer_bytes)
            for l in range(s.L):
                assert L.bz_load_layer(inst, l, blob, sizes.layer_bytes) == 0
            assert L.bz_kv_reserve(inst, 0, 64) == 0 and L.bz_frontier(inst) == s.L
            pair.append(inst)
        b, hidden = B.Batch(L, [0, 1], [0], [5]), C.create_string_buffer(4 * s.H)
        for inst in pair:
            assert L.bz_run_layers(inst, 0, 1, b.handle, hidden, 0) == 0
        hip.standin_capture(S, 7)
        for step in range(3):
            assert L.bz_run_layers(pair[0], 0, 1, b.handle, hidden, 0) == 0
            assert L.bz_signal_stream(pair[0], T) == 0           # the hidden states
            hip.standin_work(S)
            assert L.bz_run_layers(pair[1], 1, 2, b.handle, hidden, 0) == 0
            assert hip.standin_unordered(S, T) > 0
            assert L.bz_batch_advance(pair[0], b.handle) == 0
            assert hip.standin_unordered(S, T) == 0
        assert hip.standin_forbidden() == 0
        hip.standin_capture(S, 0); hip.standin_capture(T, 0)

    run(standin, scenario, fp32)


@BUILDS
def test_the_end_of_a_batch_waits_for_changes_before_a_captured_one(standin, fp32):
    """Eager operations and an eager advance on S, then one more that is captured: its event says nothing of what was eager."""
    def scenario():
        import workloads as W
        cfg = B.make_config(W.CONFIGS["tiny"], max_seqs=1, max_seq_len=64, max_tokens=1, kv_tokens=64)
        cfg.compute_stream, cfg.copy_stream = S, A
        inst = C.c_void_p()
        assert L.bz_create(C.byref(cfg), C.byref(inst)) == 0
        b = B.Batch(L, [0, 1], [0], [5])
        assert append(b, S) == 0 and L.bz_batch_advance(inst, b.handle) == 0
        eager = hip.standin_pending(S)
        hip.standin_capture(S, 7)
        assert append(b, S) == 0 and L.bz_batch_advance(inst, b.handle) == 0
        hip.standin_capture(S, 0)
        both = hip.standin_pending(S)
        assert eager > 0 and both > eager
        b.close()
        assert hip.standin_pending(S) == both - eager and hip.standin_forbidden() == 0

    run(standin, scenario, fp32)
