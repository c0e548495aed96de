"""The paged KV cache's argument checks and host helpers, as far as they go without a GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2412_17246_amd import binding as B


@pytest.fixture(scope="module", params=[False, True], ids=["bf16", "fp32dbg"])
def lib(request):
    return B.load_library(fp32_debug=request.param)


def cache(**more):
    d = B.bz_paged_kv(4096, 8192, 256, 10, 64, 4, 16, 8, 128, B.BZ_KV_ACT, 1.0, 1.0)
    for k, v in more.items():
        setattr(d, k, v)
    return d


GOOD = [dict(), dict(page_size=32), dict(page_size=1024), dict(head_dim=64), dict(dtype=1, k_scale=0.01, v_scale=7.0),
        dict(n_pages=1, n_rows=1, pages_per_row=1, n_kv_heads=1)]
BAD = [dict(n_pages=0), dict(n_rows=0), dict(pages_per_row=0), dict(n_kv_heads=0), dict(n_kv_heads=2000), dict(page_size=16),
       dict(page_size=96), dict(page_size=2048), dict(head_dim=96), dict(head_dim=0), dict(dtype=2), dict(dtype=-1),
       dict(k_scale=0.5), dict(v_scale=float("nan")), dict(dtype=1, k_scale=0.0), dict(dtype=1, v_scale=-1.0),
       dict(dtype=1, k_scale=float("inf")), dict(dtype=1, v_scale=1e-45), dict(pages_per_row=1 << 26),
       dict(n_pages=1 << 30)]


@pytest.mark.parametrize("more", GOOD)
def test_cache_bytes(lib, more):
    d = cache(**more)
    item = 1 if d.dtype == 1 else 4 if lib.bz_build_info() else 2
    assert lib.bz_paged_kv_bytes(C.byref(d)) == d.n_pages * d.n_kv_heads * d.page_size * d.head_dim * item


@pytest.mark.parametrize("more", BAD)
def test_bad_caches_are_refused(lib, more):
    d = cache(**more)
    assert lib.bz_paged_kv_bytes(C.byref(d)) == 0
    assert lib.bz_op_paged_read(C.byref(d), 0, 0, 1, 4096, 8192, None) == -1


def test_read_refusals(lib):
    ref = lambda **m: C.byref(cache(**m))  # noqa: E731
    read = lib.bz_op_paged_read
    assert lib.bz_paged_kv_bytes(None) == 0 and read(None, 0, 0, 1, 4096, 8192, None) == -1
    for bad in (dict(k=0), dict(v=0), dict(k=4100), dict(v=8), dict(page_table=0), dict(page_table=258)):
        assert read(ref(**bad), 0, 0, 1, 4096, 8192, None) == -1
    assert read(ref(), 4, 0, 1, 4096, 8192, None) == -1 and read(ref(), -1, 0, 1, 4096, 8192, None) == -1
    assert read(ref(), 0, -1, 1, 4096, 8192, None) == -1 and read(ref(), 0, 0, -1, 4096, 8192, None) == -1
    assert read(ref(), 0, 0, 1, 0, 8192, None) == -1 and read(ref(), 0, 0, 1, 4104, 8192, None) == -1
    assert read(ref(), 0, 1000, 25, 4096, 8192, None) == -7 and read(ref(), 0, 0x7fffffff, 0x7fffffff, 4096, 8192, None) == -7
    assert read(ref(), 0, 1024, 0, 0, 0, None) == 0             # nothing asked for, nothing touched


def test_operations_without_a_batch_are_refused(lib):
    d = cache()
    assert lib.bz_op_paged_append(None, C.byref(d), 4096, 1024, 4096, 1024, None, 0, None) == -1
    assert lib.bz_op_paged_attention(None, C.byref(d), 4096, 1024, 4096, 1024, 8, 0.0, 0, None, 0, None, 0, None) == -1
    assert lib.bz_op_paged_attention_workspace_bytes(None, C.byref(d), 8, 0) == 0


@pytest.mark.parametrize("positions,d,base", [(1, 64, 10000.0), (300, 128, 500000.0), (7, 2, 10.0)])
def test_rope_table(positions, d, base):
    got = B.rope_table(positions, d, base)
    angle = np.arange(positions)[:, None] * np.float64(np.float32(base)) ** (-2.0 * np.arange(d // 2) / d)
    want = np.stack([np.cos(angle), np.sin(angle)], axis=-1)
    # one rounding to float32 of values up to 1, and the last bit of a power in float64 times the position
    assert got.shape == want.shape and np.max(np.abs(got - want)) <= 2.0 ** -25 + positions * 2.0 ** -51


@pytest.mark.parametrize("positions,d,base", [(0, 64, 1e4), (-1, 64, 1e4), (4, 0, 1e4), (4, 63, 1e4), (4, 64, 1.0), (4, 64, float("nan"))])
def test_rope_table_refusals(positions, d, base):
    with pytest.raises(B.BzError):
        B.rope_table(positions, d, base)


def test_rows_of_more_positions_than_kernels_count_are_refused(lib):
    """A tile that ends behind the last position still has to have a 32-bit number."""
    assert lib.bz_paged_kv_bytes(C.byref(cache(page_size=64, pages_per_row=1 << 24))) > 0
    for bad in (dict(page_size=64, pages_per_row=(1 << 24) + 1), dict(page_size=32, pages_per_row=(1 << 26) - 1),
                dict(page_size=1024, pages_per_row=(1 << 21) - 1)):
        assert lib.bz_paged_kv_bytes(C.byref(cache(**bad))) == 0
