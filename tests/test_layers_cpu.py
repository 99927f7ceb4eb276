"""Refusals of the recurrent layers' operators and of the cache's pages: everything that the host can see is answered before any GPU
work (through the C ABI with memory that is never dereferenced, and through the binding with tensors that are not on the device)."""
import ctypes
import os
import re
import subprocess
import sys

import numpy as np
import pytest

import paper_2608_30310_b200 as gdn
from paper_2608_30310_b200 import _binding as B
from paper_2608_30310_b200 import _layers as L
from paper_2608_30310_b200.build import build_library

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MEM = np.zeros(1 << 16, dtype=np.uint8)
P = MEM.ctypes.data + (-MEM.ctypes.data) % 256


@pytest.fixture(scope="module")
def lib():
    build_library()
    return gdn.load_library()


def test_struct_sizes_match_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "gdn_tail_replay.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu %zu", sizeof(gdn_conv_desc), '
                   'sizeof(gdn_scan_desc), sizeof(gdn_cache_desc), sizeof(gdn_pool), offsetof(gdn_conv_desc, init_slots), '
                   'offsetof(gdn_scan_desc, num_init_states), offsetof(gdn_cache_desc, workspace)); return 0; }\n')
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    got = [int(x) for x in subprocess.check_output([exe]).split()]
    assert got == [ctypes.sizeof(L.ConvDesc), ctypes.sizeof(L.ScanDesc), ctypes.sizeof(L.CacheDesc), ctypes.sizeof(L.Pool),
                   L.ConvDesc.init_slots.offset, L.ScanDesc.num_init_states.offset, L.CacheDesc.workspace.offset]


def test_the_native_path_takes_every_entry_of_the_library(lib):
    text = open(os.path.join(ROOT, "paper_2608_30310_b200", "csrc", "native.cpp")).read()
    names = re.findall(r"\(\*(\w+)\)", text[text.index("struct Library {"):text.index("Library g_lib")])
    assert len(names) == len(L.ENTRIES)
    assert all(hasattr(lib, n) for n in L.ENTRIES)


def conv(lib, step=False, ptrs=None, **kw):
    d = L.ConvDesc()
    d.channels, d.width, d.io_dtype, d.num_seqs, d.total_tokens, d.x_stride, d.out_stride, d.silu = 16, 4, B.GDN_BF16, 2, 8, 16, 16, 1
    d.num_init_states = d.num_out_states = 2
    p = dict(x=P, weight=P, bias=P, cu=P, state_in=P, out=P + 4096, state_out=P)
    p.update(ptrs or {})
    for k, v in kw.items():
        setattr(d, k, v)
    if step:
        return lib.gdn_short_conv_step(ctypes.byref(d), p["x"], p["weight"], p["bias"], p["state_in"], p["out"], p["state_out"])
    return lib.gdn_short_conv(ctypes.byref(d), p["x"], p["weight"], p["bias"], p["cu"], p["state_in"], p["out"], p["state_out"])


def scan(lib, step=False, ptrs=None, **kw):
    d = L.ScanDesc()
    d.channels, d.states, d.groups, d.io_dtype, d.num_seqs, d.softplus, d.total_tokens = 16, 16, 2, B.GDN_F32, 2, 1, 8
    d.x_stride = d.dt_stride = d.z_stride = d.out_stride = 16
    d.b_stride = d.c_stride = 32
    d.num_init_states = d.num_out_states = 2
    p = dict(x=P, dt=P, a=P, b=P, c=P, d=P, z=P, dt_bias=P, cu=P, state_in=P, out=P, state_out=P)
    p.update(ptrs or {})
    for k, v in kw.items():
        setattr(d, k, v)
    head = (ctypes.byref(d), p["x"], p["dt"], p["a"], p["b"], p["c"], p["d"], p["z"], p["dt_bias"])
    if step:
        return lib.gdn_selective_scan_step(*head, p["state_in"], p["out"], p["state_out"])
    return lib.gdn_selective_scan(*head, p["cu"], p["state_in"], p["out"], p["state_out"])


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw", [dict(channels=0), dict(channels=-8), dict(io_dtype=2), dict(num_seqs=-1), dict(x_stride=15), dict(out_stride=0),
                                dict(silu=2), dict(num_init_states=-1), dict(num_out_states=1), dict(num_init_states=1),
                                dict(ptrs=dict(x=0)), dict(ptrs=dict(weight=0)), dict(ptrs=dict(out=0)), dict(ptrs=dict(x=P + 1)),
                                dict(ptrs=dict(state_in=P + 8)), dict(ptrs=dict(state_out=P + 8)), dict(init_slots=P + 2), dict(status_word=P + 1)])
def test_convolution_refuses(lib, step, kw):
    assert conv(lib, step, **kw) == -1
    assert gdn.last_launch_count() == 0


def test_convolution_refuses_more(lib):
    assert lib.gdn_short_conv(None, P, P, P, P, P, P, P) == -1 and lib.gdn_short_conv_step(None, P, P, P, P, P, P) == -1
    assert conv(lib, width=1) == -2 and conv(lib, width=5) == -2 and conv(lib, True, width=5) == -2
    assert conv(lib, ptrs=dict(out=P)) == -1                               # in place
    assert conv(lib, ptrs=dict(cu=0)) == -1 and conv(lib, total_tokens=-1) == -1 and conv(lib, total_tokens=1 << 31) == -1
    assert conv(lib, True, ptrs=dict(state_in=0)) == -1 and conv(lib, True, ptrs=dict(state_out=0)) == -1
    assert conv(lib, num_seqs=0) == 0 and conv(lib, True, num_seqs=0) == 0
    # a pool that names no slot list has to hold every request; with a list it may hold any number
    assert conv(lib, num_seqs=3) == -1 and conv(lib, num_seqs=3, init_slots=P) == -1


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw", [dict(channels=0), dict(groups=0), dict(groups=3), dict(states=0), dict(io_dtype=5), dict(num_seqs=-1), dict(softplus=2),
                                dict(x_stride=8), dict(dt_stride=8), dict(z_stride=8), dict(out_stride=8), dict(b_stride=31), dict(c_stride=16),
                                dict(ptrs=dict(x=0)), dict(ptrs=dict(dt=0)), dict(ptrs=dict(a=0)), dict(ptrs=dict(a=P + 4)), dict(ptrs=dict(b=0)),
                                dict(ptrs=dict(c=P + 2)), dict(ptrs=dict(out=0)), dict(ptrs=dict(d=P + 2)), dict(ptrs=dict(state_out=P + 4)),
                                dict(num_out_states=1), dict(out_slots=P + 1)])
def test_scan_refuses(lib, step, kw):
    assert scan(lib, step, **kw) == -1
    assert gdn.last_launch_count() == 0


def test_scan_refuses_more(lib):
    assert lib.gdn_selective_scan(None, *[P] * 12) == -1 and lib.gdn_selective_scan_step(None, *[P] * 11) == -1
    for states in (4, 12, 24, 128):
        assert scan(lib, states=states, b_stride=256, c_stride=256) == -2 and scan(lib, True, states=states, b_stride=256, c_stride=256) == -2
    assert scan(lib, ptrs=dict(cu=0)) == -1 and scan(lib, True, ptrs=dict(state_in=0)) == -1
    assert scan(lib, num_seqs=0) == 0 and scan(lib, True, num_seqs=0) == 0


def cache(bases=(P, P), page_bytes=64, **kw):
    d = L.CacheDesc()
    pools = (L.Pool * max(1, len(bases)))()
    for i, b in enumerate(bases):
        pools[i].base, pools[i].page_bytes = b, page_bytes
    d.pools, d.num_pools, d.num_pages, d.page_tokens, d.num_rows, d.row_pages = pools, len(bases), 8, 16, 4, 4
    d.workspace, d.workspace_bytes = P, 4096
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def refusals(lib, d, names, count=2, p=P):
    """What these calls answer, each of which has to be refused: with a GPU, one that is not would run on memory of the host's."""
    r = ctypes.byref(d)
    calls = {"copy": lambda: lib.gdn_cache_copy(r, p, p, count), "fork": lambda: lib.gdn_cache_fork(r, p, p, p, p, p, count),
             "free": lambda: lib.gdn_cache_free(r, p, p, p, count), "compact": lambda: lib.gdn_cache_compact(r, p, p, p, p, p, p)}
    return {calls[n]() for n in names}


@pytest.mark.parametrize("kw", [dict(num_pages=0), dict(bases=(P, 0)), dict(bases=(P + 8,)), dict(page_bytes=24), dict(page_bytes=0), dict(num_pools=-1)])
def test_cache_refuses_pools(lib, kw):
    d = cache(**kw)
    r = ctypes.byref(d)
    assert lib.gdn_cache_copy(r, P, P, 1) == -1
    assert lib.gdn_cache_fork(r, P, P, P, P, P, 1) == -1
    assert lib.gdn_cache_compact(r, P, P, P, P, P, P) == -1


def test_cache_refuses(lib):
    every, tables = ("copy", "fork", "free", "compact"), ("fork", "free", "compact")
    assert refusals(lib, cache(), every, p=P + 2) == {-1} and refusals(lib, cache(), every, p=0) == {-1}
    assert lib.gdn_cache_copy(None, P, P, 1) == -1 and lib.gdn_cache_free(None, P, P, P, 1) == -1
    for kw in (dict(num_rows=0), dict(row_pages=0)):
        assert refusals(lib, cache(**kw), tables) == {-1}
    assert refusals(lib, cache(status_word=P + 1), every) == {-1}
    assert refusals(lib, cache(num_rows=1 << 20, row_pages=1 << 20), tables) == {-2}
    assert refusals(lib, cache(num_rows=262145), ("fork",)) == {-2}
    assert refusals(lib, cache(), ("fork",), count=4097) == {-2}
    assert refusals(lib, cache(page_tokens=0), ("fork",)) == {-1}
    assert refusals(lib, cache(), ("copy", "fork", "free"), count=-1) == {-1}
    for kw in (dict(workspace=None), dict(workspace_bytes=8)):
        assert refusals(lib, cache(**kw), ("fork", "compact")) == {-3}
    assert refusals(lib, cache(workspace=P + 4), ("fork", "compact")) == {-1}
    d = cache()
    assert lib.gdn_cache_copy(ctypes.byref(d), 0, 0, 0) == 0 and lib.gdn_cache_fork(ctypes.byref(d), 0, 0, 0, 0, 0, 0) == 0
    assert lib.gdn_cache_free(ctypes.byref(d), 0, 0, 0, 0) == 0


def test_cache_workspace_size(lib):
    d = cache(num_pages=1000)
    assert lib.gdn_cache_workspace_size(ctypes.byref(d), 0) >= 12000 + 256
    assert lib.gdn_cache_workspace_size(ctypes.byref(d), 33) >= 33 * 20 and lib.gdn_cache_workspace_size(ctypes.byref(d), 33) % 256 == 0
    assert lib.gdn_cache_workspace_size(None, 0) == 0 and lib.gdn_cache_workspace_size(ctypes.byref(d), -1) == 0


def test_status_strings_of_device_errors(lib):
    assert "index" in gdn.status_string(-7) and "pages" in gdn.status_string(-8)


# The binding, with host memory: an error, never a launch and never a crash.
def test_host_tensors_raise(lib, monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, w, s, cu = torch.zeros(4, 8), torch.zeros(8, 4), torch.zeros(4, 3, 8), torch.tensor([0, 4], dtype=torch.int32)
    bc, a, h = torch.zeros(4, 1, 16), torch.zeros(8, 16), torch.zeros(4, 8, 16)
    i, t = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 4, dtype=torch.int32)
    for call in (lambda: gdn.gdn_short_conv(x, w, None, cu, torch.zeros(4, 8)), lambda: gdn.gdn_short_conv_step(x, w, None, s, x, s),
                 lambda: gdn.gdn_selective_scan(x, x, a, bc, bc, cu, x), lambda: gdn.gdn_selective_scan_step(x, x, a, bc, bc, h, x, h),
                 lambda: gdn.gdn_cache_copy([t], i, i), lambda: gdn.gdn_cache_fork([t], 16, i, t, i, i, i),
                 lambda: gdn.gdn_cache_free(i, t, i), lambda: gdn.gdn_cache_compact([t], i, t, i, t, i, i[:1])):
        with pytest.raises(ValueError, match="current device"):
            call()
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        gdn.gdn_short_conv(x.half(), w, None, cu, x)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        gdn.gdn_selective_scan_step(x.double(), x, a, bc, bc, h, x, h)
    with pytest.raises(ValueError, match="at least one pool"):
        gdn.gdn_cache_copy([], i, i)


# A tensor without sizes or storage ends in an error of torch's, in a process of its own: no C++ exception passes a C entry.
ODD = """
import torch, paper_2608_30310_b200 as gdn
gdn.load_library()
n = torch.nested.nested_tensor([torch.zeros(3, 8), torch.zeros(5, 8)])
i, t = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 4, dtype=torch.int32)
for call in (lambda: gdn.gdn_short_conv(n, n, n, n, n), lambda: gdn.gdn_short_conv_step(n, n, n, n, n, n),
             lambda: gdn.gdn_selective_scan(n, n, n, n, n, n, n), lambda: gdn.gdn_selective_scan_step(n, n, n, n, n, n, n, n),
             lambda: gdn.gdn_cache_copy([n], n, n), lambda: gdn.gdn_cache_copy([t.to_sparse()], i, i), lambda: gdn.gdn_cache_free(n, n, n),
             lambda: gdn.gdn_cache_fork([n], 16, n, n, n, n, n), lambda: gdn.gdn_cache_compact([n], n, n, n, n, n, n),
             lambda: gdn.gdn_cache_copy(3, i, i), lambda: gdn.gdn_short_conv(None, n, n, n, n)):
    try:
        call()
        print("no error")
    except (RuntimeError, ValueError, TypeError, AttributeError):
        pass
print("raised")
"""


def test_odd_tensors_raise():
    r = subprocess.run([sys.executable, "-c", ODD], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.strip() == "raised", r.stdout + r.stderr[-2000:]
