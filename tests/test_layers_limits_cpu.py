"""Sizes at the end of what the kernels' 32-bit arithmetic holds, and results that would cross their inputs, are refused before any GPU work."""
import ctypes

import pytest

from test_layers_cpu import P, cache, conv, lib, scan  # noqa: F401


@pytest.mark.parametrize("rows", [(1 << 31) - 1, (1 << 31) - 31, (1 << 31) - 63])
def test_rows(lib, rows):  # noqa: F811
    """A block of 32 rows more than the longest request would pass 2^31."""
    # (without requests nothing is launched whatever the answer)
    assert conv(lib, total_tokens=rows, num_seqs=0) == -1 and scan(lib, total_tokens=rows, num_seqs=0) == -1
    assert conv(lib, total_tokens=(1 << 31) - 64, num_seqs=0) == 0 and scan(lib, total_tokens=(1 << 31) - 64, num_seqs=0) == 0


@pytest.mark.parametrize("pages", [(1 << 31) - 1, (1 << 31) - 100, (1 << 30) + 1])
def test_pages(lib, pages):  # noqa: F811
    """The planning kernels step over the counts by 512, in shares that are rounded up."""
    d = cache(num_pages=pages, workspace_bytes=1 << 40)
    r = ctypes.byref(d)
    # (tables that are not there: refused whatever the answer on the pages)
    assert lib.gdn_cache_fork(r, P, P + 2, P, P, P, 1) == -2
    assert lib.gdn_cache_compact(r, P, P + 2, P, P, P, P) == -2
    d = cache(num_pages=1 << 30, workspace_bytes=1 << 40)
    r = ctypes.byref(d)
    assert lib.gdn_cache_fork(r, P, P + 2, P, P, P, 1) == -1 and lib.gdn_cache_compact(r, P, P + 2, P, P, P, P) == -1


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("name", ["x", "dt", "z"])
def test_results_in_place_at_another_stride(lib, step, name):  # noqa: F811
    """Row 1's result would lie in another row's input, which another part of the call may not have read yet."""
    ptrs = {k: P + 8192 for k in ("x", "dt", "z")}
    ptrs[name] = P
    # (out lies at P; 12 states are refused in any case, with another answer)
    wide = dict(states=12, b_stride=256, c_stride=256)
    assert scan(lib, step, ptrs=ptrs, out_stride=32, **wide) == -1
    assert scan(lib, step, ptrs=ptrs, **{name + "_stride": 32}, **wide) == -1
    assert scan(lib, step, ptrs=ptrs, **wide) == -2
    assert scan(lib, step, ptrs=ptrs, **{name + "_stride": 32}, num_seqs=1, total_tokens=1, **wide) == -2


def test_a_steps_convolution_in_place_at_another_stride(lib):  # noqa: F811
    for kw in (dict(out_stride=32), dict(x_stride=32)):
        assert conv(lib, True, ptrs=dict(out=P), width=5, **kw) == -1
        assert conv(lib, True, ptrs=dict(out=P), width=5, num_seqs=1, **kw) == -2
    assert conv(lib, True, ptrs=dict(out=P), width=5) == -2
