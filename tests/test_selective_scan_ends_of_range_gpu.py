"""The selective scan with decays at the ends of the range: a of minus infinity (a state that holds one token), and of the type's lowest value."""
import pytest
import torch

from layer_utils import cu_of, scan_inputs, scan_ref, within

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# channels and requests' lengths: one request of few states, many of many; blocks of 32 rows that are full, and that are not
CALLS = [(64, [1]), (64, [5]), (64, [32, 64]), (64, [33, 0, 7]), (512, [70, 31, 2, 40]), (4096, [9, 33])]


def check(m, a, lens, softplus, init):
    """The call with ``a``; the reference with m's."""
    import paper_2608_30310_b200 as gdn
    d = {k: v.cuda() for k, v in m.items()}
    out, pool = torch.empty_like(d["x"]), init.cuda()
    bias = m["dt_bias"] if softplus else None
    gdn.gdn_selective_scan(d["x"], d["dt"], a.cuda(), d["b"], d["c"], cu_of(lens).cuda(), out, d=d["d"], z=d["z"], dt_bias=None if bias is None else bias.cuda(),
                           softplus=softplus, init_state=pool, out_state=pool)
    ref, bound, h, hb = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], lens, m["d"], m["z"], bias, softplus, init)
    within(out, ref, bound, "out")
    within(pool, h, hb, "state")
    # one token more
    n = len(lens)
    t = {k: (v[:n] if k in ("x", "dt", "z", "b", "c") else v) for k, v in m.items()}
    if t["x"].shape[0] < n:
        return
    before = pool.cpu()
    e = {k: v.cuda() for k, v in t.items()}
    step = torch.empty_like(e["x"])
    gdn.gdn_selective_scan_step(e["x"], e["dt"], a.cuda(), e["b"], e["c"], pool, step, pool, d=e["d"], z=e["z"], dt_bias=None if bias is None else bias.cuda(),
                                softplus=softplus)
    ref, bound, h, hb = scan_ref(t["x"], t["dt"], t["a"], t["b"], t["c"], [1] * n, t["d"], t["z"], bias, softplus, before)
    within(step, ref, bound, "token")
    within(pool, h, hb, "state after the token")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("C,lens", CALLS, ids=str)
def test_a_of_minus_infinity(dtype, S, C, lens):
    """Its decay is 0 for every time step above 0; at a = -1e30 the reference has the same decays, and bounds that are numbers."""
    m = scan_inputs(sum(lens), C, S, 1, dtype, S)
    init = torch.randn((len(lens), C, S), generator=torch.Generator().manual_seed(2))
    m["a"][:, S // 3] = -1e30
    m["a"][C // 2] = -1e30
    a = m["a"].clone()
    a[a == -1e30] = -float("inf")
    check(m, a, lens, True, init)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("C,lens", CALLS, ids=str)
def test_a_at_the_lowest_value(dtype, S, C, lens):
    """Time steps of 0 leave the state as it is whatever a is; others leave nothing of it."""
    m = scan_inputs(sum(lens), C, S, 1, dtype, S + 1)
    init = torch.randn((len(lens), C, S), generator=torch.Generator().manual_seed(3))
    low = torch.finfo(torch.float32).min
    m["a"][:, S // 3] = low
    m["a"][C // 2] = low
    m["dt"] = m["dt"].abs() + 0.01
    m["dt"][::2] = 0
    check(m, m["a"], lens, False, init)
