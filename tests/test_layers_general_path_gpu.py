"""The recurrent layers' operators and the cache's pages through the binding's general path, as with an extension built for another torch: the
same results as through the native one."""
import pytest
import torch

from layer_utils import cu_of, scan_inputs

pytestmark = pytest.mark.gpu


def results():
    import paper_2608_30310_b200 as gdn
    lens, out = [30, 0, 50], []
    m = {k: v.cuda() for k, v in scan_inputs(80, 48, 16, 2, torch.bfloat16, 5).items()}
    cu, w, b = cu_of(lens).cuda(), torch.randn(48, 4, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda(), None
    slots = torch.tensor([2, 0, 4], dtype=torch.int32, device="cuda")
    conv, scan = torch.ones(5, 3, 48, dtype=torch.bfloat16, device="cuda"), torch.ones(5, 48, 16, device="cuda")
    status, stream = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    x, y = torch.empty_like(m["x"]), torch.empty_like(m["x"])
    kw = dict(init_slots=slots, out_slots=slots, status_word=status, stream=stream)
    gdn.gdn_short_conv(m["x"], w, b, cu, x, init_state=conv, out_state=conv, **kw)
    gdn.gdn_selective_scan(x, m["dt"], m["a"], m["b"], m["c"], cu, y, d=m["d"], z=m["z"], dt_bias=m["dt_bias"], init_state=scan, out_state=scan, **kw)
    kw = dict(slots=slots, status_word=status, stream=stream)
    t = {k: v[:3] if k not in ("a", "d", "dt_bias") else v for k, v in m.items()}
    u = torch.empty_like(t["x"])
    gdn.gdn_short_conv_step(t["x"], w, b, conv, u, conv, silu=False, **kw)
    v = torch.empty_like(u)
    gdn.gdn_selective_scan_step(u, t["dt"], t["a"], t["b"], t["c"], scan, v, scan, d=t["d"], dt_bias=t["dt_bias"], softplus=True, **kw)
    pools = [torch.arange(40 * 32, device="cuda").view(40, 32) + i for i in range(3)]
    counts, tables = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.full((4, 6), -1, dtype=torch.int32, device="cuda")
    tables[0, :5] = torch.tensor([39, 7, 20, 3, 11])
    counts[[39, 7, 20, 3, 11]] = 1
    stream.wait_stream(torch.cuda.current_stream())

    def i32(*n):
        return torch.tensor(n, dtype=torch.int32, device="cuda")
    src, dst, parents, kids, tokens, rows = i32(7, 3), i32(30, 31), i32(0, 0), i32(1, 2), i32(37, 70), i32(2)
    stream.wait_stream(torch.cuda.current_stream())
    kw = dict(status_word=status, stream=stream)
    gdn.gdn_cache_copy(tuple(pools), src, dst, **kw)
    gdn.gdn_cache_fork(pools, 16, counts, tables, parents, kids, tokens, workspace=gdn.Workspace(), **kw)
    gdn.gdn_cache_free(counts, tables, rows, **kw)
    page_map, live = torch.empty_like(counts), torch.empty(1, dtype=torch.int32, device="cuda")
    gdn.gdn_cache_compact(pools, counts, tables, counts, tables, page_map, live, **kw)
    stream.synchronize()
    assert int(status) == 0
    return [x, y, u, v, conv, scan, counts, tables, page_map, live, *pools]


def test_the_general_path_gives_the_same(monkeypatch):
    from paper_2608_30310_b200 import _binding as B
    want = results()
    assert B._native
    monkeypatch.setattr(B, "_native", False)
    for got, ref in zip(results(), want):
        assert torch.equal(got, ref)
