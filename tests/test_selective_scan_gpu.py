"""The selective scan against its definition in 64 bits, with a running bound of what fp32 arithmetic may lose: packed prompts in every
form of the kernel, single tokens, slots, strides, borders."""
import numpy as np
import pytest
import torch

from layer_utils import cu_of, scan_inputs, scan_ref, within

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def gdn():
    import paper_2608_30310_b200 as m
    return m


def run(m, lens, init=None, gate=True, skip=True, bias=True, softplus=True, pad=0):
    C, S, N, T = *m["a"].shape, len(lens), sum(lens)
    g = torch.Generator().manual_seed(1)
    slots = torch.randperm(N + 3, generator=g)[:N].to(torch.int32)
    dev = {k: v.cuda() for k, v in m.items()}
    if pad:
        for k in ("x", "dt", "z", "b", "c"):
            dev[k] = torch.cat([dev[k], torch.full((pad, *dev[k].shape[1:]), float("nan"), dtype=dev[k].dtype, device="cuda")])
    out = torch.full((T + pad, C), 7.0, dtype=m["x"].dtype, device="cuda")
    pool = torch.full((N + 3, C, S), 3.0, device="cuda")
    kw = dict(out_state=pool, out_slots=slots.cuda())
    if init is not None:
        src = torch.zeros_like(pool)
        src[slots.long().cuda()] = init.cuda()
        kw.update(init_state=src, init_slots=slots.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gdn().gdn_selective_scan(dev["x"], dev["dt"], dev["a"], dev["b"], dev["c"], cu_of(lens).cuda(), out, d=dev["d"] if skip else None,
                             z=dev["z"] if gate else None, dt_bias=dev["dt_bias"] if bias else None, softplus=softplus, status_word=status, **kw)
    torch.cuda.synchronize()
    assert gdn().last_launch_count() == 1 and int(status) == 0
    assert bool((out[T:] == 7).all())
    rest = [i for i in range(N + 3) if i not in slots.tolist()]
    assert bool((pool[rest] == 3).all())
    return out[:T], pool[slots.long().cuda()]


def check(m, lens, init=None, gate=True, skip=True, bias=True, softplus=True, pad=0):
    out, st = run(m, lens, init, gate, skip, bias, softplus, pad)
    ref, bound, h, hb = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], lens, m["d"] if skip else None, m["z"] if gate else None,
                                 m["dt_bias"] if bias else None, softplus, init)
    within(out, ref, bound, "out")
    within(st, h, hb, "state")


LENS = [[1], [0, 3, 0], [31, 32, 33, 0, 65, 1], [130, 7]]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("C,G", [(1, 1), (7, 1), (24, 2), (72, 3), (64, 1)])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_prompts(dtype, S, C, G, lens):
    m = scan_inputs(sum(lens), C, S, G, dtype, seed=S + C)
    init = torch.randn((len(lens), C, S), generator=torch.Generator().manual_seed(9)) if C != 24 else None
    check(m, lens, init, gate=C != 72, skip=C != 7, bias=C != 64, pad=4 if C in (1, 64) else 0)


# From few states in a call to many: every form of the kernel for each number of states, with channels that fill its tiles and that do not.
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("values", [5e3, 3e4, 1e5, 2.5e5, 5e5, 1.3e6])
@pytest.mark.parametrize("C,G", [(128, 2), (100, 1)])
def test_every_form(dtype, S, values, C, G):
    N = max(1, int(values / (C * S)))
    lens = [int(v) for v in np.random.default_rng(N).integers(0, 75, size=N)]
    lens[0] = 74
    m = scan_inputs(sum(lens), C, S, G, dtype, seed=S)
    check(m, lens, torch.randn((N, C, S), generator=torch.Generator().manual_seed(2)))


@pytest.mark.parametrize("N,most", [(63, 12), (64, 12), (65, 12), (300, 12), (2, 500), (33, 350), (64, 320)])
def test_many_requests(N, most):
    """Up to 64 requests of 128 tokens and more in the mean are taken longest first, others in the order given."""
    lens = [int(v) for v in np.random.default_rng(N).integers(0, most, size=N)]
    lens[-1] = most
    check(scan_inputs(sum(lens), 40, 16, 1, BF, N), lens, torch.randn((N, 40, 16), generator=torch.Generator().manual_seed(2)))


def test_without_softplus_and_with_extreme_time_steps():
    m = scan_inputs(90, 32, 16, 1, F32, 5)
    m["dt"] = torch.rand(m["dt"].shape, generator=torch.Generator().manual_seed(1)) * 0.2 + 1e-3
    check(m, [90], softplus=False, bias=False)
    m = scan_inputs(90, 32, 16, 1, F32, 6)
    m["dt"][:, ::2] = -30.0                                                # time steps of 1e-13: the state stays, to the last digit
    m["dt"][:, 1::4] = 25.0                                                # and of 25: nothing of it is left
    check(m, [50, 40], torch.randn((2, 32, 16), generator=torch.Generator().manual_seed(2)), bias=False)


def test_a_group_for_every_channel_and_rows_before_the_first_request():
    """As many groups as channels; and cu_tail_lens that begins above zero, as a slice of a longer batch's does: other rows stay."""
    lens = [20, 45]
    m = scan_inputs(65, 9, 8, 9, F32, 8)
    check(m, lens)
    ref, bound, _, _ = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], lens, m["d"], m["z"], m["dt_bias"])
    d = {k: v.cuda() for k, v in m.items()}
    out = torch.full_like(d["x"], 6.0)
    gdn().gdn_selective_scan(d["x"], d["dt"], d["a"], d["b"], d["c"], torch.tensor([20, 65], dtype=torch.int32, device="cuda"), out, d=d["d"], z=d["z"],
                             dt_bias=d["dt_bias"])
    assert bool((out[:20] == 6).all())
    within(out[20:], ref[20:], bound[20:])


def test_slow_decay_over_a_long_request():
    """Time steps of 0.001 over 6,000 tokens: the states hold sums over a thousand tokens."""
    m = scan_inputs(6000, 4, 16, 1, F32, 7)
    m["dt"].zero_()
    m["dt_bias"].fill_(float(np.log(np.expm1(1e-3))))
    check(m, [6000])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("off,extra", [(0, 0), (8, 16), (4, 4), (1, 3), (2, 2)])
def test_strided_rows(dtype, off, extra):
    """Slices of wider arrays, as a layer's projections are; the odd offsets leave no alignment."""
    lens, C, S = [9, 0, 40], 64, 16
    m = scan_inputs(sum(lens), C, S, 1, dtype, 11)
    T = sum(lens)

    def inside(t):
        flat = t.reshape(T, -1)
        wide = torch.full((T, flat.shape[1] + off + extra), float("nan"), dtype=dtype, device="cuda")
        wide[:, off:off + flat.shape[1]] = flat.cuda()
        return wide[:, off:off + flat.shape[1]].unflatten(1, t.shape[1:])
    x, dt, z, b, c = (inside(m[k]) for k in ("x", "dt", "z", "b", "c"))
    res = torch.full((T, C + off + extra), 5.0, dtype=dtype, device="cuda")
    gdn().gdn_selective_scan(x, dt, m["a"].cuda(), b, c, cu_of(lens).cuda(), res[:, off:off + C], d=m["d"].cuda(), z=z, dt_bias=m["dt_bias"].cuda())
    ref, bound, _, _ = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], lens, m["d"], m["z"], m["dt_bias"])
    within(res[:, off:off + C], ref, bound)
    assert bool((res[:, :off] == 5).all()) and bool((res[:, off + C:] == 5).all())


@pytest.mark.parametrize("name", ["x", "dt", "z"])
def test_in_place(name):
    lens = [70, 3, 40]
    m = scan_inputs(sum(lens), 96, 16, 1, BF, 12)
    ref, _ = run(m, lens)
    dev = {k: v.cuda() for k, v in m.items()}
    gdn().gdn_selective_scan(dev["x"], dev["dt"], dev["a"], dev["b"], dev["c"], cu_of(lens).cuda(), dev[name], d=dev["d"], z=dev["z"], dt_bias=dev["dt_bias"])
    assert torch.equal(dev[name], ref)


@pytest.mark.parametrize("N", [5, 400])
def test_other_requests_values_do_not_matter(N):
    lens = ([40, 3, 70, 0, 11] * N)[:N]
    m = scan_inputs(sum(lens), 64, 16, 1, BF, 13)
    cu = cu_of(lens).tolist()
    clean, s0 = run(m, lens)
    for n, v in ((0, float("inf")), (2, float("nan")), (4, -3e38)):
        y = {k: t.clone() for k, t in m.items()}
        for k in ("x", "dt", "z", "b", "c"):
            y[k][cu[n]:cu[n + 1]] = v
        out, s1 = run(y, lens)
        for r in range(N):
            if r != n:
                assert torch.equal(out[cu[r]:cu[r + 1]], clean[cu[r]:cu[r + 1]]) and torch.equal(s1[r], s0[r]), (n, r)


def test_a_channels_nan_stays_in_it():
    m = scan_inputs(50, 64, 16, 1, F32, 14)
    clean, s0 = run(m, [50])
    m["x"][20, 5] = float("nan")
    out, s1 = run(m, [50])
    rest = [c for c in range(64) if c != 5]
    assert torch.equal(out[:, rest], clean[:, rest]) and torch.equal(out[:20], clean[:20]) and bool(torch.isnan(out[20:, 5]).all())
    assert torch.equal(s1[:, rest], s0[:, rest]) and bool(torch.isnan(s1[:, 5]).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("N,C,G", [(1, 5, 1), (1, 512, 1), (37, 24, 2), (150, 1024, 1), (151, 1000, 4)])
def test_single_tokens(dtype, S, N, C, G):
    m = scan_inputs(N, C, S, G, dtype, 20)
    g = torch.Generator().manual_seed(4)
    pool = torch.randn((N + 2, C, S), generator=g)
    slots = torch.randperm(N + 2, generator=g)[:N].to(torch.int32)
    if N > 1:
        slots[3] = -1
    use = [n for n in range(N) if slots[n] >= 0]
    full = C != 512
    ref, bound, h, hb = scan_ref(*(m[k][use] if k != "a" else m[k] for k in ("x", "dt", "a", "b", "c")), [1] * len(use), m["d"] if full else None,
                                 m["z"][use] if full else None, m["dt_bias"] if full else None, True, pool[slots[use].long()])
    for in_place in (False, True):
        dev = {k: v.cuda() for k, v in m.items()}
        src = pool.cuda()
        dst = src if in_place else pool.cuda()
        out = dev["x"] if in_place else torch.full_like(dev["x"], 9)
        gdn().gdn_selective_scan_step(dev["x"], dev["dt"], dev["a"], dev["b"], dev["c"], src, out, dst, d=dev["d"] if full else None,
                                      z=dev["z"] if full else None, dt_bias=dev["dt_bias"] if full else None, slots=slots.cuda())
        within(out[use], ref, bound, "out")
        within(dst[slots[use].long().cuda()], h, hb, "state")
        rest = [i for i in range(N + 2) if i not in slots[use].tolist()]
        assert torch.equal(dst[rest].cpu(), pool[rest])
        if N > 1:
            assert torch.equal(out[3].cpu(), m["x"][3] if in_place else torch.full_like(m["x"][3], 9))


def test_prompt_then_tokens_is_one_pass():
    lens, more = [50, 3, 0, 130], 5
    full = [l + more for l in lens]
    m = scan_inputs(sum(full), 72, 16, 1, F32, 30)
    cu = cu_of(full).tolist()
    ref, bound, h, hb = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], full, m["d"], m["z"], m["dt_bias"])
    rows = torch.cat([torch.arange(cu[n], cu[n] + lens[n]) for n in range(4)])
    head = {k: v[rows] if k in ("x", "dt", "z", "b", "c") else v for k, v in m.items()}
    _, st = run(head, lens)
    st = st.contiguous()
    for t in range(more):
        r = torch.tensor([cu[n] + lens[n] + t for n in range(4)])
        tok = {k: (v[r] if k in ("x", "dt", "z", "b", "c") else v).cuda() for k, v in m.items()}
        out = torch.empty_like(tok["x"])
        gdn().gdn_selective_scan_step(tok["x"], tok["dt"], tok["a"], tok["b"], tok["c"], st, out, st, d=tok["d"], z=tok["z"], dt_bias=tok["dt_bias"])
        within(out, ref[r], bound[r], "token %d" % t)
    within(st, h, hb, "state")


def test_slots():
    lens, C = [4, 2, 1, 0, 6], 16
    m = scan_inputs(sum(lens), C, 16, 1, F32, 40)
    pool = torch.randn(6, C, 16, generator=torch.Generator().manual_seed(3))
    init, keep = torch.tensor([2, -1, 4, 0, 99], dtype=torch.int32), torch.tensor([2, 5, -1, 0, 77], dtype=torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev, out, d = pool.cuda(), torch.empty(sum(lens), C, device="cuda"), {k: v.cuda() for k, v in m.items()}
    gdn().gdn_selective_scan(d["x"], d["dt"], d["a"], d["b"], d["c"], cu_of(lens).cuda(), out, init_state=dev, out_state=dev, init_slots=init.cuda(),
                             out_slots=keep.cuda(), status_word=status)
    zero = torch.zeros(C, 16)
    ref, bound, h, hb = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], lens, init=torch.stack([pool[2], zero, pool[4], pool[0], zero]))
    within(out, ref, bound)
    got = dev.cpu()
    within(got[[2, 5, 0]], h[[0, 1, 3]], hb[[0, 1, 3]])
    assert torch.equal(got[[1, 3, 4]], pool[[1, 3, 4]]) and int(status) == -7
    status.zero_()
    gdn().gdn_selective_scan_step(d["x"][:2], d["dt"][:2], d["a"], d["b"][:2], d["c"][:2], dev, out[:2], dev,
                                  slots=torch.tensor([1, 6], dtype=torch.int32, device="cuda"), status_word=status)
    assert int(status) == -7


def test_two_streams_and_a_thread_each():
    """Calls at once, from two threads on two streams, share nothing."""
    import threading
    jobs = []
    for i in range(2):
        lens = [300 + 100 * i, 50, 7]
        m = scan_inputs(sum(lens), 256, 16, 1, BF, 80 + i)
        ref, st = run(m, lens)
        jobs.append((lens, {k: v.cuda() for k, v in m.items()}, ref, st, torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]

    def work(i):
        lens, d, _, _, stream = jobs[i]
        cu = cu_of(lens).cuda()
        torch.cuda.synchronize()
        for _ in range(40):
            o, p = torch.empty_like(d["x"]), torch.empty(3, 256, 16, device="cuda")
            torch.cuda.current_stream().synchronize()
            gdn().gdn_selective_scan(d["x"], d["dt"], d["a"], d["b"], d["c"], cu, o, d=d["d"], z=d["z"], dt_bias=d["dt_bias"], out_state=p, stream=stream)
            outs[i].append((o, p))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    for i in range(2):
        assert len(outs[i]) == 40
        for o, p in outs[i]:
            assert torch.equal(o, jobs[i][2]) and torch.equal(p, jobs[i][3])


def test_no_rows():
    m = {k: v.cuda() for k, v in scan_inputs(12, 8, 8, 1, F32, 1).items()}
    for T in (0, 12):
        out, old, pool = torch.full((T, 8), 2.0, device="cuda"), torch.randn(3, 8, 8, device="cuda"), torch.zeros(3, 8, 8, device="cuda")
        args = (m["x"][:T], m["dt"][:T], m["a"], m["b"][:T], m["c"][:T])
        gdn().gdn_selective_scan(*args, torch.zeros(4, dtype=torch.int32, device="cuda"), out, init_state=old, out_state=pool)
        assert torch.equal(pool, old) and bool((out == 2).all())
        gdn().gdn_selective_scan(*args, torch.zeros(1, dtype=torch.int32, device="cuda"), out)
        assert bool((out == 2).all())


def test_offsets_past_32_bits():
    T, C, S, stride = 2200, 8, 8, 1 << 20
    m = scan_inputs(T, C, S, 1, BF, 50)
    wide = torch.empty(T * stride, dtype=BF, device="cuda").view(T, stride)
    views = {}
    for i, k in enumerate(("x", "dt", "z", "b", "c")):
        views[k] = wide[:, 64 * i:64 * i + 8]
        views[k].copy_(m[k].reshape(T, 8))
    pool = torch.empty((34000000, C, S), device="cuda")                      # 2.18 G values
    last = pool.shape[0] - 1
    pool[last] = 1.5
    slot = torch.tensor([last], dtype=torch.int32, device="cuda")
    out = wide[:, 1024:1024 + C]
    gdn().gdn_selective_scan(views["x"], views["dt"], m["a"].cuda(), views["b"][:, None], views["c"][:, None], cu_of([T]).cuda(), out, z=views["z"],
                             dt_bias=m["dt_bias"].cuda(), init_state=pool, init_slots=slot, out_state=pool, out_slots=slot)
    ref, bound, h, hb = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], [T], z=m["z"], dt_bias=m["dt_bias"], init=torch.full((1, C, S), 1.5))
    within(out, ref, bound)
    within(pool[last:], h, hb)
    before = pool[last].cpu()
    gdn().gdn_selective_scan_step(views["x"][:1], views["dt"][:1], m["a"].cuda(), views["b"][:1, None], views["c"][:1, None], pool, out[:1], pool, slots=slot)
    _, _, h, hb = scan_ref(m["x"][:1], m["dt"][:1], m["a"], m["b"][:1], m["c"][:1], [1], init=before[None])
    within(pool[last:], h, hb)


def test_captured_and_on_another_stream():
    lens = [33, 0, 90]
    m = scan_inputs(sum(lens), 64, 16, 1, BF, 60)
    d = {k: v.cuda() for k, v in m.items()}
    cu, out, pool, side = cu_of(lens).cuda(), torch.zeros_like(d["x"]), torch.zeros(3, 64, 16, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()

    def call():
        gdn().gdn_selective_scan(d["x"], d["dt"], d["a"], d["b"], d["c"], cu, out, d=d["d"], z=d["z"], dt_bias=d["dt_bias"], out_state=pool, stream=side)
    call()
    side.synchronize()
    ref, bound, h, hb = scan_ref(m["x"], m["dt"], m["a"], m["b"], m["c"], lens, m["d"], m["z"], m["dt_bias"])
    within(out, ref, bound)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
        call()
    m2 = scan_inputs(sum(lens), 64, 16, 1, BF, 61)
    for k in d:
        d[k].copy_(m2[k])
    graph.replay()
    torch.cuda.synchronize()
    ref, bound, h, hb = scan_ref(m2["x"], m2["dt"], m2["a"], m2["b"], m2["c"], lens, m2["d"], m2["z"], m2["dt_bias"])
    within(out, ref, bound)
    within(pool, h, hb)


def test_refused_tensors():
    m = {k: v.cuda() for k, v in scan_inputs(8, 16, 16, 2, F32, 1).items()}
    cu, ok = cu_of([8]).cuda(), torch.empty(8, 16, device="cuda")

    def call(out=ok, **kw):
        a = dict(m, **kw)
        gdn().gdn_selective_scan(a["x"], a["dt"], a["a"], a["b"], a["c"], cu, out, d=a["d"], z=a["z"], dt_bias=a["dt_bias"], **a.get("more", {}))
    call()
    for kw, name in ((dict(dt=m["dt"][:7]), "dt"), (dict(a=m["a"].t().contiguous().t()), "a "), (dict(b=m["b"].transpose(1, 2).contiguous().transpose(1, 2)), "b "),
                     (dict(c=m["c"][:, :1]), "c "), (dict(d=m["d"][:3]), "d "), (dict(z=m["z"][:, ::2]), "z "), (dict(out=torch.empty(1, 16, device="cuda").expand(8, 16)), "out"),
                     (dict(more=dict(out_state=torch.zeros(1, 16, 8, device="cuda"))), "out_state"),
                     (dict(more=dict(out_state=torch.zeros(1, 16, 16, device="cuda"), out_slots=torch.zeros(3, dtype=torch.int32, device="cuda"))), "out_slots")):
        with pytest.raises(ValueError, match=name):
            call(**kw)
    for kw, name in ((dict(b=m["b"].to(BF)), "b "), (dict(a=m["a"].double()), "a "), (dict(x=m["x"].half()), "x must be")):
        with pytest.raises(TypeError, match=name):
            call(**kw)
    with pytest.raises(gdn().GdnError, match="invalid argument"):                # three groups of sixteen channels
        call(b=torch.zeros(8, 3, 16, device="cuda"), c=torch.zeros(8, 3, 16, device="cuda"))
    with pytest.raises(gdn().GdnError, match="unsupported"):
        call(a=torch.zeros(16, 12, device="cuda"), b=torch.zeros(8, 2, 12, device="cuda"), c=torch.zeros(8, 2, 12, device="cuda"))
