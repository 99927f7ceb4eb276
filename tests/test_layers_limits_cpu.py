"""Sizes at the end of what the kernels' 32-bit arithmetic holds are refused before any GPU work."""
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
