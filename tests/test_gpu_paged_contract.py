"""What the paged KV cache's operations promise beside their results: when a batch may go, what is refused before a launch, how far a
value that is not finite reaches, how precise queries and sums are."""
import pytest

from tests.test_gpu_paged import World

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
