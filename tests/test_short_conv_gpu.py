"""The short causal convolution against its definition in 64 bits: packed prompts and single tokens, slots, strides, borders."""
import numpy as np
import pytest
import torch

from layer_utils import conv_ref, cu_of, within

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def gdn():
    import paper_2608_30310_b200 as m
    return m


def inputs(T, C, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)

    def n(*shape):
        return torch.randn(shape, generator=g)
    return n(T, C).to(dtype), (n(C, K) / K ** 0.5).to(dtype), n(C).to(dtype)


def run(x, w, b, lens, init=None, act=True, pad=0):
    """States go to shuffled slots of a larger pool; what is not named keeps its pattern."""
    C, K, N = x.shape[1], w.shape[1], len(lens)
    g = torch.Generator().manual_seed(1)
    slots = torch.randperm(N + 3, generator=g)[:N].to(torch.int32)
    T = sum(lens)
    xd = torch.cat([x, torch.full((pad, C), float("nan"), dtype=x.dtype)]).cuda()
    out = torch.full((T + pad, C), 7.0, dtype=x.dtype, device="cuda")
    pool = torch.full((N + 3, K - 1, C), 3.0, dtype=x.dtype, device="cuda")
    kw = dict(out_state=pool, out_slots=slots.cuda())
    if init is not None:
        from_pool = torch.zeros_like(pool)
        from_pool[slots.long().cuda()] = init.cuda()
        kw.update(init_state=from_pool, init_slots=slots.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gdn().gdn_short_conv(xd, w.cuda(), None if b is None else b.cuda(), cu_of(lens).cuda(), out, silu=act, status_word=status, **kw)
    torch.cuda.synchronize()
    assert gdn().last_launch_count() == 1 and int(status) == 0
    assert bool((out[T:] == 7).all())
    rest = [i for i in range(N + 3) if i not in slots.tolist()]
    assert bool((pool[rest] == 3).all())
    return out[:T], pool[slots.long().cuda()].cpu()


LENS = [[1], [2, 1, 3], [0, 5, 0, 0, 64, 1, 0], [7, 8, 9, 63, 130, 0], [300]]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("C", [1, 8, 36, 136])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_prompts(dtype, K, C, lens):
    x, w, b = inputs(sum(lens), C, K, dtype, seed=C + K)
    init = torch.randn((len(lens), K - 1, C), generator=torch.Generator().manual_seed(9)).to(dtype) if C != 8 else None
    out, states = run(x, w, b if C != 36 else None, lens, init, act=C != 136, pad=5 if C in (1, 136) else 0)
    ref, bound, rs = conv_ref(x, w, b if C != 36 else None, lens, init, act=C != 136)
    within(out, ref, bound, "out")
    assert torch.equal(states, rs)


@pytest.mark.parametrize("rows", [60000, 9000])
def test_long_walks(rows):
    """Enough rows that a thread walks as many as it ever does, over borders of requests anywhere inside."""
    lens = [int(v) for v in np.random.default_rng(3).integers(0, 900, size=400)]
    while sum(lens) > rows:
        lens.pop()
    x, w, b = inputs(sum(lens), 1024 if rows < 10000 else 2048, 4, BF, 5)
    out, states = run(x, w, b, lens)
    cols = torch.randperm(x.shape[1], generator=torch.Generator().manual_seed(2))[:9]
    ref, bound, rs = conv_ref(x[:, cols], w[cols], b[cols], lens)
    within(out.cpu()[:, cols], ref, bound, "out")
    assert torch.equal(states[:, :, cols], rs)


@pytest.mark.parametrize("dtype,C,off", [(BF, 64, 0), (BF, 64, 8), (BF, 64, 3), (F32, 20, 4), (F32, 20, 1)])
def test_strided_rows(dtype, C, off):
    """x and out are slices of wider arrays; the offsets of 3 and 1 values leave no alignment."""
    lens = [9, 0, 40]
    x, w, b = inputs(sum(lens), C, 4, dtype, 11)
    wide = torch.full((sum(lens), C + 24), float("nan"), dtype=dtype, device="cuda")
    res = torch.full((sum(lens), C + 16), 5.0, dtype=dtype, device="cuda")
    wide[:, off:off + C] = x.cuda()
    gdn().gdn_short_conv(wide[:, off:off + C], w.cuda(), b.cuda(), cu_of(lens).cuda(), res[:, off:off + C])
    ref, bound, _ = conv_ref(x, w, b, lens)
    within(res[:, off:off + C], ref, bound)
    assert bool((res[:, :off] == 5).all()) and bool((res[:, off + C:] == 5).all())


def test_other_requests_values_do_not_matter():
    lens, bad = [40, 3, 70, 0, 11], [float("inf"), float("nan")]
    x, w, b = inputs(sum(lens), 64, 4, BF, 12)
    cu = cu_of(lens).tolist()
    clean, s0 = run(x, w, b, lens)
    for n in (0, 2, 4):
        y = x.clone()
        y[cu[n]:cu[n + 1]] = bad[n % 2]
        out, s1 = run(y, w, b, lens)
        for m in range(len(lens)):
            if m != n:
                assert torch.equal(out[cu[m]:cu[m + 1]].view(torch.int16), clean[cu[m]:cu[m + 1]].view(torch.int16)) and torch.equal(s1[m], s0[m])


def test_rows_before_the_first_request():
    """cu_tail_lens that begins above zero, as a slice of a longer batch's does: other rows are neither read nor written."""
    x, w, b = inputs(200, 16, 4, F32, 13)
    y = x.clone()
    y[:77] = float("nan")
    out = torch.full((200, 16), 6.0, device="cuda")
    gdn().gdn_short_conv(y.cuda(), w.cuda(), b.cuda(), torch.tensor([77, 90, 190], dtype=torch.int32, device="cuda"), out)
    ref, bound, _ = conv_ref(x[77:190], w, b, [13, 100])
    assert bool((out[:77] == 6).all()) and bool((out[190:] == 6).all())
    within(out[77:190], ref, bound)


def test_values_at_the_ends_of_the_range():
    """Large negative results vanish, infinities and NaN stay where the formula has them."""
    x = torch.tensor([[1e4], [-1e4], [float("inf")], [0.0], [0.0], [0.0], [-200.0], [float("nan")], [1.0]])
    w, out = torch.tensor([[0.0, 1.0]]), torch.empty(9, 1, device="cuda")
    gdn().gdn_short_conv(x.cuda(), w.cuda(), None, cu_of([9]).cuda(), out)
    got = out.cpu()[:, 0]
    assert got[0] == 1e4 and got[1].abs() < 1e-30 and got[2] == float("inf")
    assert torch.isnan(got[3]) and got[4] == 0 and got[6].abs() < 1e-30 and torch.isnan(got[7]) and torch.isnan(got[8])    # (0 inf, 0 nan)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("N,C", [(1, 5), (1, 2048), (37, 24), (200, 512)])
def test_single_tokens(dtype, K, N, C):
    x, w, b = inputs(N, C, K, dtype, 20)
    g = torch.Generator().manual_seed(4)
    pool = torch.randn((N + 2, K - 1, C), generator=g).to(dtype)
    slots = torch.randperm(N + 2, generator=g)[:N].to(torch.int32)
    if N > 1:
        slots[3] = -1
    use = [n for n in range(N) if slots[n] >= 0]
    ref, bound, rs = conv_ref(x[use], w, b, [1] * len(use), pool[slots[use].long()])
    want = pool.clone()
    want[slots[use].long()] = rs
    for in_place in (False, True):
        src = pool.cuda()
        dst = src if in_place else pool.cuda()
        xd = x.cuda()
        out = xd if in_place else torch.full_like(xd, 9)
        gdn().gdn_short_conv_step(xd, w.cuda(), b.cuda(), src, out, dst, slots=slots.cuda())
        within(out[use], ref, bound)
        assert torch.equal(dst.cpu(), want)
        if N > 1:
            assert torch.equal(out[3].cpu(), x[3] if in_place else torch.full_like(x[3], 9))


def test_prompt_then_tokens_is_one_pass_bit_for_bit():
    lens, more = [50, 3, 0, 130], 5
    x, w, b = inputs(sum(lens) + more * len(lens), 72, 4, BF, 30)
    full = [l + more for l in lens]
    whole, states = run(x, w, b, full)
    cu = cu_of(full).tolist()
    head = torch.cat([x[cu[n]:cu[n] + lens[n]] for n in range(4)])
    _, s = run(head, w, b, lens)
    pool = s.cuda()
    for t in range(more):
        xt = torch.stack([x[cu[n] + lens[n] + t] for n in range(4)]).cuda()
        out = torch.empty_like(xt)
        gdn().gdn_short_conv_step(xt, w.cuda(), b.cuda(), pool, out, pool)
        assert torch.equal(out, torch.stack([whole[cu[n] + lens[n] + t] for n in range(4)]))
    assert torch.equal(pool.cpu(), states)


def test_slots():
    """In place, a zero start by a negative slot, states not kept, slots past the pool's end."""
    lens, C = [4, 2, 1, 0, 6], 16
    x, w, b = inputs(sum(lens), C, 4, F32, 40)
    pool = torch.randn(6, 3, C, generator=torch.Generator().manual_seed(3))
    init, keep = torch.tensor([2, -1, 4, 0, 99], dtype=torch.int32), torch.tensor([2, 5, -1, 0, 77], dtype=torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev, out = pool.cuda(), torch.empty(sum(lens), C, device="cuda")
    gdn().gdn_short_conv(x.cuda(), w.cuda(), b.cuda(), cu_of(lens).cuda(), out, init_state=dev, out_state=dev, init_slots=init.cuda(),
                         out_slots=keep.cuda(), status_word=status)
    start = torch.stack([pool[2], torch.zeros(3, C), pool[4], pool[0], torch.zeros(3, C)])
    ref, bound, rs = conv_ref(x, w, b, lens, start)
    within(out, ref, bound)
    want = pool.clone()
    want[2], want[5], want[0] = rs[0], rs[1], rs[3]
    assert torch.equal(dev.cpu(), want) and int(status) == -7
    status.zero_()
    gdn().gdn_short_conv_step(x[:2].cuda(), w.cuda(), b.cuda(), dev, out[:2], dev, slots=torch.tensor([1, 6], dtype=torch.int32, device="cuda"), status_word=status)
    assert int(status) == -7


@pytest.mark.parametrize("dtype,C", [(BF, 8), (F32, 3), (BF, 512)])
@pytest.mark.parametrize("K", [2, 3, 4])
def test_states_in_place_wherever_requests_begin(dtype, C, K):
    """Requests of all short lengths, one behind the other, so that they begin at every place of a thread's share of rows: the thread that
    replaces a start state is the only one that reads it."""
    rng = np.random.default_rng(K)
    lens = [int(v) for v in rng.permutation(np.repeat(np.arange(0, 21), 30))] + [40]
    x, w, b = inputs(sum(lens), C, K, dtype, 70)
    N = len(lens)
    init = torch.randn((N, K - 1, C), generator=torch.Generator().manual_seed(6)).to(dtype)
    cols = list(range(C))[:5]
    ref, bound, rs = conv_ref(x[:, cols], w[cols], b[cols], lens, init[:, :, cols])
    xd, wd, bd, cu = x.cuda(), w.cuda(), b.cuda(), cu_of(lens).cuda()
    first = None
    for _ in range(5):
        pool, out = init.cuda(), torch.empty_like(xd)
        gdn().gdn_short_conv(xd, wd, bd, cu, out, init_state=pool, out_state=pool)
        within(out.cpu()[:, cols], ref, bound)
        assert torch.equal(pool[:, :, cols].cpu(), rs)
        assert first is None or torch.equal(out, first)
        first = out


def test_a_request_alone_in_a_longer_batch_array():
    """No rows at all, no requests, only empty requests."""
    w, b = (t.cuda() for t in inputs(0, 8, 4, F32, 1)[1:])
    for T in (0, 12):
        x, out, pool = torch.ones(T, 8, device="cuda"), torch.full((T, 8), 2.0, device="cuda"), torch.zeros(3, 3, 8, device="cuda")
        old = torch.randn(3, 3, 8, device="cuda")
        gdn().gdn_short_conv(x, w, b, torch.zeros(4, dtype=torch.int32, device="cuda"), out, init_state=old, out_state=pool)
        assert torch.equal(pool, old) and bool((out == 2).all())
        gdn().gdn_short_conv(x, w, b, torch.zeros(1, dtype=torch.int32, device="cuda"), out)
        assert bool((out == 2).all())


def test_offsets_past_32_bits():
    T, C, stride = 2200, 8, 1 << 20
    x, w, b = inputs(T, C, 4, BF, 50)
    wide = torch.empty(T * stride, dtype=BF, device="cuda").view(T, stride)
    wide[:, 64:64 + C] = x.cuda()
    pool = torch.empty((90000000, 3, C), dtype=BF, device="cuda")            # 2.16 G values
    last = pool.shape[0] - 1
    pool[last] = 1.5
    slot = torch.tensor([last], dtype=torch.int32, device="cuda")
    out = wide[:, 1024:1024 + C]
    gdn().gdn_short_conv(wide[:, 64:64 + C], w.cuda(), b.cuda(), cu_of([T]).cuda(), out, init_state=pool, init_slots=slot, out_state=pool, out_slots=slot)
    ref, bound, rs = conv_ref(x, w, b, [T], torch.full((1, 3, C), 1.5, dtype=BF))
    within(out, ref, bound)
    assert torch.equal(pool[last].cpu(), rs[0])


def test_captured_and_on_another_stream():
    lens = [33, 0, 90]
    x, w, b = inputs(sum(lens), 64, 4, BF, 60)
    ref, bound, rs = conv_ref(x, w, b, lens)
    xd, wd, bd, cu = x.cuda(), w.cuda(), b.cuda(), cu_of(lens).cuda()
    out, pool = torch.zeros_like(xd), torch.zeros(3, 3, 64, dtype=BF, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    gdn().gdn_short_conv(xd, wd, bd, cu, out, out_state=pool, stream=side)
    side.synchronize()
    within(out, ref, bound)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        gdn().gdn_short_conv(xd, wd, bd, cu, out, out_state=pool, stream=side)
        gdn().gdn_short_conv_step(out[:3], wd, bd, pool, out[:3], pool, stream=side)
    y = torch.randn(x.shape, generator=torch.Generator().manual_seed(8)).to(BF)
    xd.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    ref, bound, rs = conv_ref(y, w, b, lens)
    within(out[3:], ref[3:], bound[3:])
    assert torch.equal(pool[:, :2].cpu(), rs[:, 1:])


def test_refused_tensors():
    x, w, cu = torch.zeros(8, 16, device="cuda"), torch.zeros(16, 4, device="cuda"), cu_of([8]).cuda()
    ok = torch.empty_like(x)
    with pytest.raises(ValueError, match="overlap"):
        gdn().gdn_short_conv(x, w, None, cu, torch.empty(1, 16, device="cuda").expand(8, 16))
    with pytest.raises(ValueError, match="packed within a row"):
        gdn().gdn_short_conv(torch.zeros(8, 32, device="cuda")[:, ::2], w, None, cu, ok)
    with pytest.raises(ValueError, match="weight"):
        gdn().gdn_short_conv(x, w[:8], None, cu, ok)
    with pytest.raises(TypeError, match="weight"):
        gdn().gdn_short_conv(x, w.to(BF), None, cu, ok)
    with pytest.raises(ValueError, match="out_state"):
        gdn().gdn_short_conv(x, w, None, cu, ok, out_state=torch.zeros(1, 4, 16, device="cuda"))
    with pytest.raises(ValueError, match="init_slots"):
        gdn().gdn_short_conv(x, w, None, cu, ok, init_state=torch.zeros(1, 3, 16, device="cuda"), init_slots=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(gdn().GdnError, match="invalid argument"):
        gdn().gdn_short_conv(x, w, None, cu, x)
    with pytest.raises(gdn().GdnError, match="unsupported"):
        gdn().gdn_short_conv(x, torch.zeros(16, 5, device="cuda"), None, cu, ok)
    with pytest.raises(ValueError, match="status_word"):
        gdn().gdn_short_conv(x, w, None, cu, ok, status_word=torch.zeros(1, dtype=torch.int32))
    assert gdn().gdn_short_conv(x, w, None, cu, x, check=False) == -1
