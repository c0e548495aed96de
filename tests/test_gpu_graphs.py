"""Decode steps of a split pair, on two streams, captured into one graph."""
import pytest

import workloads as W
from tests import _util as U
from tests.test_gpu_serving import SHAPE, _fresh

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


def test_a_graph_of_a_split_pair_that_advances_its_batch(torch):
    """The library orders the advance on one half's stream behind the other half's run, and the next runs behind it, inside the
    graph: the same bits as eager steps."""
    s, lens, steps = SHAPE, [5, 255, 256, 700], 3
    B = len(lens)
    st_t, st_s = torch.cuda.Stream(), torch.cuda.Stream()
    whole = _fresh(torch, s, lens, steps)
    tgt = _fresh(torch, s, lens, steps, layers=[0], stream=st_t)
    src = _fresh(torch, s, lens, steps, layers=[1], stream=st_s)
    xs = [U.to_device(W.hidden_bits(s, B, step=60 + i, scale=1.0 / 16), False) for i in range(steps)]
    want, got = [x.clone() for x in xs], [x.clone() for x in xs]
    torch.cuda.synchronize()
    bw = whole.batch(list(range(B + 1)), list(range(B)), lens)
    for i in range(steps):
        whole.run_layers(0, s.L, bw, want[i])
        whole.batch_advance(bw)
    whole.sync()
    assert tgt.frontier() == 1 and src.layer_ready(1)
    shared = tgt.batch(list(range(B + 1)), list(range(B)), lens)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st_t, capture_error_mode="relaxed"):
        for i in range(steps):
            tgt.run_layers(0, 1, shared, got[i], after_current_stream=False)
            src.wait_stream(st_t)
            src.run_layers(1, 2, shared, got[i], after_current_stream=False)
            tgt.batch_advance(shared)
        tgt.wait_stream(st_s)
    torch.cuda.synchronize()
    for i in range(steps):
        assert torch.equal(got[i], xs[i])                    # captured, not run
    graph.replay()
    torch.cuda.synchronize()
    for i in range(steps):
        assert torch.equal(want[i].view(torch.int16), got[i].view(torch.int16)), i
    shared.close()
    whole.close(); tgt.close(); src.close()
