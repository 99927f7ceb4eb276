"""Binding of the recurrent layers' operators (short convolution, selective scan) and of the cache's pages.

As in ``_binding``: a call whose arguments are in order is marshalled in ``csrc/native.cpp``; what that does not take comes here, where
the checks raise the errors and the workspace grows.  Device tensors on the current device; asynchronous on the current (or given) stream."""
from __future__ import annotations

import ctypes

from . import _binding as B


class ConvDesc(ctypes.Structure):
    """Mirror of ``struct gdn_conv_desc`` in include/gdn_tail_replay.h."""
    _fields_ = [
        ("channels", ctypes.c_int32), ("width", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
        ("total_tokens", ctypes.c_int64), ("x_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
        ("silu", ctypes.c_int32), ("num_init_states", ctypes.c_int32), ("num_out_states", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("init_slots", ctypes.c_void_p), ("out_slots", ctypes.c_void_p), ("status_word", ctypes.c_void_p), ("stream", ctypes.c_void_p),
    ]


class ScanDesc(ctypes.Structure):
    """Mirror of ``struct gdn_scan_desc``."""
    _fields_ = [
        ("channels", ctypes.c_int32), ("states", ctypes.c_int32), ("groups", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
        ("num_seqs", ctypes.c_int32), ("softplus", ctypes.c_int32), ("total_tokens", ctypes.c_int64),
        ("x_stride", ctypes.c_int64), ("dt_stride", ctypes.c_int64), ("b_stride", ctypes.c_int64), ("c_stride", ctypes.c_int64),
        ("z_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
        ("num_init_states", ctypes.c_int32), ("num_out_states", ctypes.c_int32),
        ("init_slots", ctypes.c_void_p), ("out_slots", ctypes.c_void_p), ("status_word", ctypes.c_void_p), ("stream", ctypes.c_void_p),
    ]


class Pool(ctypes.Structure):
    """Mirror of ``struct gdn_pool``."""
    _fields_ = [("base", ctypes.c_void_p), ("page_bytes", ctypes.c_int64)]


class CacheDesc(ctypes.Structure):
    """Mirror of ``struct gdn_cache_desc``."""
    _fields_ = [
        ("pools", ctypes.POINTER(Pool)), ("num_pools", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
        ("num_rows", ctypes.c_int32), ("row_pages", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("status_word", ctypes.c_void_p), ("stream", ctypes.c_void_p),
    ]


# in the order that the native argument path takes their addresses
ENTRIES = ("gdn_short_conv", "gdn_short_conv_step", "gdn_selective_scan", "gdn_selective_scan_step",
           "gdn_cache_copy", "gdn_cache_fork", "gdn_cache_free", "gdn_cache_compact", "gdn_cache_workspace_size")


def declare(lib):
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    for name, desc, pointers in (("gdn_short_conv", ConvDesc, 7), ("gdn_short_conv_step", ConvDesc, 6),
                                 ("gdn_selective_scan", ScanDesc, 12), ("gdn_selective_scan_step", ScanDesc, 11),
                                 ("gdn_cache_compact", CacheDesc, 6)):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = i32, [ctypes.POINTER(desc)] + [vp] * pointers
    for name, pointers in (("gdn_cache_copy", 2), ("gdn_cache_fork", 5), ("gdn_cache_free", 3)):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = i32, [ctypes.POINTER(CacheDesc)] + [vp] * pointers + [i32]
    lib.gdn_cache_workspace_size.restype = ctypes.c_size_t
    lib.gdn_cache_workspace_size.argtypes = [ctypes.POINTER(CacheDesc), i32]


def _native(entry, *args):
    """The status of a call marshalled natively, or None."""
    if B._native is None:
        B.load_library()
    return getattr(B._native, entry)(*args) if B._native else None


def _finish(rc, name, check):
    if rc != B.GDN_OK and check:
        raise B.GdnError(rc, name)
    return rc


def _io(x):
    import torch
    if x.dtype == torch.bfloat16:
        return B.GDN_BF16
    if x.dtype == torch.float32:
        return B.GDN_F32
    raise TypeError("x must be bfloat16 or float32")


def _check(name, t, shape, dtype, rows=False):
    """Raises unless ``t`` is a device tensor of this shape (None: any size) and dtype, packed, or with ``rows`` in packed rows; its row stride."""
    import torch
    if t.dtype != dtype:
        raise TypeError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
    if t.dim() != len(shape) or any(s is not None and s != g for s, g in zip(shape, t.shape)):
        raise ValueError("%s must have the shape [%s], not %s" % (name, ", ".join("any" if s is None else str(s) for s in shape), list(t.shape)))
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError("%s must be on the current device" % name)
    values = 1
    for size, stride in zip(t.shape[:0:-1], t.stride()[:0:-1]):
        if rows and size != 1 and stride != values:
            raise ValueError("%s must be packed within a row" % name)
        values *= size
    if not rows and not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    stride = t.stride(0) if t.shape[0] > 1 else values
    if rows and stride < values:
        raise ValueError("the rows of %s overlap" % name)
    return stride


def _status(status_word):
    import torch
    if status_word is not None and (not status_word.is_cuda or status_word.device.index != torch.cuda.current_device() or
                                    status_word.numel() * status_word.element_size() < 4):
        raise ValueError("status_word must be an int32 on the current device")
    return B._ptr(status_word)


def _handle(stream):
    import torch
    return int((torch.cuda.current_stream() if stream is None else stream).cuda_stream)


def _optional(name, t, *args, **kw):
    return None if t is None else _check(name, t, *args, **kw)


def _slots(desc, num, init_slots, out_slots):
    import torch
    _optional("init_slots", init_slots, (num,), torch.int32)
    _optional("out_slots", out_slots, (num,), torch.int32)
    desc.init_slots, desc.out_slots = B._ptr(init_slots), B._ptr(out_slots)


def _conv(step, x, weight, bias, cu, init_state, out, out_state, silu, init_slots, out_slots, status_word, stream, check):
    rc = _native("conv", step, x, weight, bias, cu, init_state, out, out_state, silu, init_slots, out_slots, status_word, stream)
    name = "gdn_short_conv_step" if step else "gdn_short_conv"
    if rc is not None:
        return _finish(rc, name, check)
    import torch
    lib, d = B.load_library(), ConvDesc()
    d.io_dtype = _io(x)
    d.x_stride = _check("x", x, (None, None), x.dtype, rows=True)
    T, C = x.shape
    _check("weight", weight, (C, None), x.dtype)
    K = weight.shape[1]
    _optional("bias", bias, (C,), x.dtype)
    d.out_stride = _check("out", out, (T, C), x.dtype, rows=True)
    if step and (init_state is None or out_state is None):
        raise ValueError("a step needs state_in and state_out")
    _optional("state_in" if step else "init_state", init_state, (None, K - 1, C), x.dtype)
    _optional("state_out" if step else "out_state", out_state, (None, K - 1, C), x.dtype)
    if not step:
        _check("cu_tail_lens", cu, (None,), torch.int32)
    d.num_seqs = T if step else cu.numel() - 1
    d.channels, d.width, d.total_tokens, d.silu = C, K, T, int(bool(silu))
    d.num_init_states = 0 if init_state is None else init_state.shape[0]
    d.num_out_states = 0 if out_state is None else out_state.shape[0]
    _slots(d, d.num_seqs, init_slots, out_slots)
    d.status_word, d.stream = _status(status_word), _handle(stream)
    p = B._ptr
    if step:
        rc = lib.gdn_short_conv_step(ctypes.byref(d), p(x), p(weight), p(bias), p(init_state), p(out), p(out_state))
    else:
        rc = lib.gdn_short_conv(ctypes.byref(d), p(x), p(weight), p(bias), p(cu), p(init_state), p(out), p(out_state))
    return _finish(int(rc), name, check)


def gdn_short_conv(x, weight, bias, cu_tail_lens, out, *, silu=True, init_state=None, out_state=None, init_slots=None, out_slots=None,
                   status_word=None, stream=None, check=True) -> int:
    """Depthwise causal convolution over packed prompts: out[t] = silu(bias + sum_j weight[:, j] x[t - width + 1 + j]); see the header.

    x, out [T, C] (rows may be strided), weight [C, width], bias [C] or None, all bf16 or all fp32; cu_tail_lens [N + 1] int32, whose last
    entry may be below T.  init_state, out_state [slots, width - 1, C]: pools of the width - 1 rows before a request and of its last
    ones; init_slots, out_slots [N] int32 name the requests' slots in them (None: slot n; negative: a zero start, no state kept).
    A slot past a pool's end counts as negative and sets GDN_ERR_BAD_INDEX in status_word.  out may not overlap x."""
    return _conv(False, x, weight, bias, cu_tail_lens, init_state, out, out_state, silu, init_slots, out_slots, status_word, stream, check)


def gdn_short_conv_step(x, weight, bias, state_in, out, state_out, *, silu=True, slots=None, status_word=None, stream=None, check=True) -> int:
    """``gdn_short_conv`` for one token per request: x, out [N, C]; request n has slot slots[n] (None: n) of both pools, which may be the
    same tensor.  A request with a negative slot is padding: its row of out and the states are left as they were."""
    return _conv(True, x, weight, bias, None, state_in, out, state_out, silu, slots, None, status_word, stream, check)


def _scan(step, x, dt, a, b, c, cu, init_state, out, out_state, d_skip, z, dt_bias, softplus, init_slots, out_slots, status_word, stream, check):
    rc = _native("scan", step, x, dt, a, b, c, d_skip, z, dt_bias, cu, init_state, out, out_state, softplus, init_slots, out_slots,
                 status_word, stream)
    name = "gdn_selective_scan_step" if step else "gdn_selective_scan"
    if rc is not None:
        return _finish(rc, name, check)
    import torch
    lib, d, f32 = B.load_library(), ScanDesc(), torch.float32
    d.io_dtype = _io(x)
    d.x_stride = _check("x", x, (None, None), x.dtype, rows=True)
    T, C = x.shape
    d.dt_stride = _check("dt", dt, (T, C), x.dtype, rows=True)
    _check("a", a, (C, None), f32)
    S = a.shape[1]
    d.b_stride = _check("b", b, (T, None, S), x.dtype, rows=True)
    G = b.shape[1]
    d.c_stride = _check("c", c, (T, G, S), x.dtype, rows=True)
    _optional("d", d_skip, (C,), f32)
    _optional("dt_bias", dt_bias, (C,), f32)
    d.z_stride = _optional("z", z, (T, C), x.dtype, rows=True) or 0
    d.out_stride = _check("out", out, (T, C), x.dtype, rows=True)
    if step and (init_state is None or out_state is None):
        raise ValueError("a step needs state_in and state_out")
    _optional("state_in" if step else "init_state", init_state, (None, C, S), f32)
    _optional("state_out" if step else "out_state", out_state, (None, C, S), f32)
    if not step:
        _check("cu_tail_lens", cu, (None,), torch.int32)
    d.num_seqs = T if step else cu.numel() - 1
    d.channels, d.states, d.groups, d.total_tokens, d.softplus = C, S, G, T, int(bool(softplus))
    d.num_init_states = 0 if init_state is None else init_state.shape[0]
    d.num_out_states = 0 if out_state is None else out_state.shape[0]
    _slots(d, d.num_seqs, init_slots, out_slots)
    d.status_word, d.stream = _status(status_word), _handle(stream)
    p = B._ptr
    head = (ctypes.byref(d), p(x), p(dt), p(a), p(b), p(c), p(d_skip), p(z), p(dt_bias))
    if step:
        rc = lib.gdn_selective_scan_step(*head, p(init_state), p(out), p(out_state))
    else:
        rc = lib.gdn_selective_scan(*head, p(cu), p(init_state), p(out), p(out_state))
    return _finish(int(rc), name, check)


def gdn_selective_scan(x, dt, a, b, c, cu_tail_lens, out, *, d=None, z=None, dt_bias=None, softplus=True, init_state=None, out_state=None,
                       init_slots=None, out_slots=None, status_word=None, stream=None, check=True) -> int:
    """Selective state space scan over packed prompts: h = exp(dt a) h + dt x b, out = (c . h + d x) silu(z), dt = softplus(dt + dt_bias).

    x, dt, z, out [T, C], b, c [T, G, S] (rows may be strided) all bf16 or all fp32; a [C, S], d, dt_bias [C] fp32; S in {8, 16, 32, 64}; G
    divides C.  init_state, out_state [slots, C, S] fp32 pools, with slots as in ``gdn_short_conv``.  out may be x, dt or z."""
    return _scan(False, x, dt, a, b, c, cu_tail_lens, init_state, out, out_state, d, z, dt_bias, softplus, init_slots, out_slots,
                 status_word, stream, check)


def gdn_selective_scan_step(x, dt, a, b, c, state_in, out, state_out, *, d=None, z=None, dt_bias=None, softplus=True, slots=None,
                            status_word=None, stream=None, check=True) -> int:
    """``gdn_selective_scan`` for one token per request: x, dt, z, out [N, C], b, c [N, G, S]; slots as in ``gdn_short_conv_step``."""
    return _scan(True, x, dt, a, b, c, None, state_in, out, state_out, d, z, dt_bias, softplus, slots, None, status_word, stream, check)


def _pools(desc, pools):
    """Fills in the pools: [pages, ...] each, packed, of one number of pages.  Returns what has to outlive the call."""
    pools = list(pools)
    if not pools:
        raise ValueError("a cache has at least one pool")
    array = (Pool * len(pools))()
    for i, t in enumerate(pools):
        if t.dim() < 2 or t.shape[0] < 1:
            raise ValueError("a pool has the shape [pages, ...]")
        _check("pool %d" % i, t, (pools[0].shape[0],) + tuple(t.shape[1:]), t.dtype)
        array[i].base, array[i].page_bytes = t.data_ptr(), t.numel() * t.element_size() // t.shape[0]
    desc.pools, desc.num_pools, desc.num_pages = array, len(pools), pools[0].shape[0]
    return array


def _scratch(lib, desc, count, workspace, stream):
    """The workspace's buffer for the stream; returns what has to outlive the call."""
    import torch
    need = int(lib.gdn_cache_workspace_size(ctypes.byref(desc), count))
    if workspace is None:
        workspace = B.Workspace(device="cuda")
    if type(workspace) is not B.Workspace:                # (a caller's own, as the replay takes it)
        desc.workspace, desc.workspace_bytes = workspace.ensure(need)
        return workspace
    current = stream is None
    if current:
        stream = torch.cuda.current_stream()
    buf = workspace.reserve(need, stream, current, device_call=True)
    if not buf.is_cuda or buf.device.index != torch.cuda.current_device():
        raise ValueError("workspace must be on the current device")
    desc.workspace, desc.workspace_bytes = B._aligned(buf)
    return buf


def gdn_cache_copy(pools, src, dst, *, status_word=None, stream=None, check=True) -> int:
    """Page src[i] to page dst[i] in every pool; see the header.

    pools: a list of packed tensors [pages, ...], one per layer say, of the same number of pages, a page a multiple of 16 bytes; src, dst
    [n] int32.  The dst pages differ from each other and from all src pages."""
    rc = _native("cache_copy", pools, src, dst, status_word, stream)
    if rc is None:
        import torch
        lib, d = B.load_library(), CacheDesc()
        keep = _pools(d, pools)
        _check("src", src, (None,), torch.int32)
        _check("dst", dst, (src.shape[0],), torch.int32)
        d.status_word, d.stream = _status(status_word), _handle(stream)
        rc = int(lib.gdn_cache_copy(ctypes.byref(d), B._ptr(src), B._ptr(dst), src.numel()))
        del keep
    return _finish(rc, "gdn_cache_copy", check)


def gdn_cache_fork(pools, page_tokens, refcounts, tables, parents, children, tokens, *, workspace=None, status_word=None, stream=None,
                   check=True) -> int:
    """Row children[i] of the tables becomes a branch of row parents[i] after tokens[i] tokens; see the header.

    Whole pages are shared, a partial last one is copied to the lowest-numbered free page, what the children held before is given back.
    refcounts [pages], tables [rows, row_pages], parents, children, tokens [n], all int32.  A fork that names what is not there is left
    out (GDN_ERR_BAD_INDEX in status_word); without a free page for it a child's row ends empty (GDN_ERR_NO_PAGES)."""
    rc = _native("cache_fork", pools, page_tokens, refcounts, tables, parents, children, tokens, workspace, status_word, stream)
    if rc is None:
        import torch
        lib, d = B.load_library(), CacheDesc()
        keep = [_pools(d, pools)]
        _check("refcounts", refcounts, (d.num_pages,), torch.int32)
        _check("tables", tables, (None, None), torch.int32)
        _check("parents", parents, (None,), torch.int32)
        for name, t in (("children", children), ("tokens", tokens)):
            _check(name, t, (parents.shape[0],), torch.int32)
        d.page_tokens, (d.num_rows, d.row_pages) = int(page_tokens), tables.shape
        keep.append(_scratch(lib, d, parents.numel(), workspace, stream))
        d.status_word, d.stream = _status(status_word), _handle(stream)
        rc = int(lib.gdn_cache_fork(ctypes.byref(d), B._ptr(refcounts), B._ptr(tables), B._ptr(parents), B._ptr(children), B._ptr(tokens),
                                    parents.numel()))
        del keep
    return _finish(rc, "gdn_cache_fork", check)


def gdn_cache_free(refcounts, tables, rows, *, status_word=None, stream=None, check=True) -> int:
    """The rows rows[i] of the tables give their pages back: counts go down, the entries become -1; see the header."""
    rc = _native("cache_free", refcounts, tables, rows, status_word, stream)
    if rc is None:
        import torch
        lib, d = B.load_library(), CacheDesc()
        _check("refcounts", refcounts, (None,), torch.int32)
        _check("tables", tables, (None, None), torch.int32)
        _check("rows", rows, (None,), torch.int32)
        d.num_pages, (d.num_rows, d.row_pages) = refcounts.shape[0], tables.shape
        d.status_word, d.stream = _status(status_word), _handle(stream)
        rc = int(lib.gdn_cache_free(ctypes.byref(d), B._ptr(refcounts), B._ptr(tables), B._ptr(rows), rows.numel()))
    return _finish(rc, "gdn_cache_free", check)


def gdn_cache_compact(pools, refcounts, tables, out_refcounts, out_tables, page_map, live, *, workspace=None, status_word=None, stream=None,
                      check=True) -> int:
    """Brings the live pages to the front of the pools; see the header.

    out_refcounts and out_tables receive counts and tables afterwards (they may be the inputs), page_map [pages] each page's new number (-1:
    free), live [1] how many there are; all int32."""
    rc = _native("cache_compact", pools, refcounts, tables, out_refcounts, out_tables, page_map, live, workspace, status_word, stream)
    if rc is None:
        import torch
        lib, d = B.load_library(), CacheDesc()
        keep = [_pools(d, pools)]
        for name, t in (("refcounts", refcounts), ("out_refcounts", out_refcounts), ("page_map", page_map)):
            _check(name, t, (d.num_pages,), torch.int32)
        _check("tables", tables, (None, None), torch.int32)
        _check("out_tables", out_tables, tuple(tables.shape), torch.int32)
        _check("live", live, (1,), torch.int32)
        d.num_rows, d.row_pages = tables.shape
        keep.append(_scratch(lib, d, 0, workspace, stream))
        d.status_word, d.stream = _status(status_word), _handle(stream)
        rc = int(lib.gdn_cache_compact(ctypes.byref(d), B._ptr(refcounts), B._ptr(tables), B._ptr(out_refcounts), B._ptr(out_tables),
                                       B._ptr(page_map), B._ptr(live)))
        del keep
    return _finish(rc, "gdn_cache_compact", check)
