"""What the binding of the paged operations refuses before the library sees it: tensors of the host in place of the GPU's, and a library
that must not be reached."""
from types import SimpleNamespace

import pytest
import torch

from paper_2412_17246_amd import binding as B


@pytest.fixture
def call(monkeypatch):
    """An attention over a cache "on" the host, with arguments replaced; its calls of the library are counted."""
    monkeypatch.setattr(B, "_on_device", lambda kv: None)
    reached = []

    def attention(*a):
        reached.append(a)
        return 0

    kv = SimpleNamespace(_act=torch.bfloat16, _device=torch.device("cpu"), head_dim=64, n_kv_heads=2, _ref=None,
                         lib=SimpleNamespace(bz_op_paged_attention=attention))
    batch = SimpleNamespace(T=3, handle=None)
    good = dict(q=torch.zeros(3, 256, dtype=torch.bfloat16), out=torch.zeros(3, 256, dtype=torch.bfloat16),
                rope=torch.zeros(8, 32, 2), workspace=torch.zeros(1024, dtype=torch.uint8))

    def attend(**more):
        args = dict(good, **more)
        B.op_paged_attention(batch, kv, args.pop("q"), args.pop("out"), **args)

    return attend, reached


def test_workspaces_that_are_not_memory_on_the_device(call):
    attend, reached = call
    attend()
    attend(workspace=None)
    attend(workspace=torch.zeros(16, 16))                    # any type and shape, side by side
    assert len(reached) == 3 and reached[0][-2] == 1024 and reached[2][-2] == 1024
    space = torch.zeros(64, 64, dtype=torch.uint8)
    for bad in (space.to("meta"), torch.zeros(1, dtype=torch.uint8).expand(1 << 20), space[:, ::2], space.t()):
        with pytest.raises(ValueError):
            attend(workspace=bad)
    assert len(reached) == 3


def test_rotary_tables_of_another_type(call):
    attend, reached = call
    attend(rope=torch.zeros(8, 32, 2))
    for bad in (torch.zeros(8, 32, 2, dtype=torch.int32), torch.zeros(8, 32, 2, dtype=torch.float64), torch.zeros(8, 32, 2).to("meta"),
                torch.zeros(2, 8, 32).permute(1, 2, 0), torch.zeros(8, 64)):
        with pytest.raises(ValueError):
            attend(rope=bad)
    assert len(reached) == 1


class OnGpu:
    """What PagedKv asks of a tensor."""

    def __init__(self, shape, dtype):
        self.t = torch.empty(shape, dtype=dtype, device="meta")
        self.dtype, self.shape, self.is_cuda, self.device = dtype, self.t.shape, True, torch.device("cuda", 0)
        for f in ("dim", "is_contiguous", "numel", "element_size"):
            setattr(self, f, getattr(self.t, f))

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("fp32", [False, True], ids=["bf16", "fp32dbg"])
def test_a_cache_of_no_pages(fp32):
    act = torch.float32 if fp32 else torch.bfloat16
    table = OnGpu((2, 3), torch.int32)
    make = lambda n, table=table: B.PagedKv(32, 2, 64, k=OnGpu((n, 2, 32 * 64), act), v=OnGpu((n, 2, 32 * 64), act),  # noqa: E731
                                            page_table=table, fp32_debug=fp32)
    assert make(1).desc.n_pages == 1
    with pytest.raises(ValueError):
        make(0)
    for shape in ((0, 3), (2, 0)):                           # and of no rows, or none in a row
        with pytest.raises(B.BzError):
            make(1, OnGpu(shape, torch.int32))
