"""Weights and biases of the short convolution at every place that their values may begin: views into a larger buffer, as a model's parameters are."""
import pytest
import torch

from layer_utils import conv_ref, cu_of, within

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def at(t, off):
    """The values of ``t``, packed, ``off`` values into a buffer that begins on 256 bytes."""
    flat = torch.full((t.numel() + off,), float("nan"), dtype=t.dtype, device="cuda")
    assert flat.data_ptr() % 256 == 0
    flat[off:] = t.reshape(-1).cuda()
    return flat[off:].view(t.shape)


def inputs(T, C, K, dtype):
    g = torch.Generator().manual_seed(C + K)
    return (torch.randn(T, C, generator=g).to(dtype), (torch.randn(C, K, generator=g) / 2).to(dtype), torch.randn(C, generator=g).to(dtype),
            torch.randn((3, K - 1, C), generator=g).to(dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("C", [4, 64, 516, 21])
@pytest.mark.parametrize("w_off,b_off", [(1, 0), (2, 0), (4, 0), (12, 0), (0, 1), (0, 2), (0, 4), (4, 4), (8, 12)])
def test_offsets(dtype, K, C, w_off, b_off):
    import paper_2608_30310_b200 as gdn
    lens = [19, 0, 33]
    x, w, b, init = inputs(sum(lens), C, K, dtype)
    wd, bd, pool, xd = at(w, w_off), at(b, b_off), init.cuda(), x.cuda()
    out = torch.empty_like(xd)
    gdn.gdn_short_conv(xd, wd, bd, cu_of(lens).cuda(), out, init_state=pool, out_state=pool)
    ref, bound, states = conv_ref(x, w, b, lens, init)
    within(out, ref, bound, "prompt")
    assert torch.equal(pool.cpu(), states)
    step = torch.empty_like(xd[:3])
    gdn.gdn_short_conv_step(xd[:3], wd, bd, pool, step, pool)
    ref, bound, after = conv_ref(x[:3], w, b, [1, 1, 1], states)
    within(step, ref, bound, "step")
    assert torch.equal(pool.cpu(), after)


@pytest.mark.parametrize("K", [2, 4])
@pytest.mark.parametrize("first", [1, 2, 4])
def test_a_part_of_a_layers_channels(K, first):
    """w[first:]: an odd number of rows of weights cut off."""
    import paper_2608_30310_b200 as gdn
    C = 64
    x, w, b, _ = inputs(40, C + first, K, BF)
    xd, wd, bd = x[:, first:].contiguous().cuda(), w.cuda()[first:], b.cuda()[first:]
    out = torch.empty_like(xd)
    gdn.gdn_short_conv(xd, wd, bd, cu_of([40]).cuda(), out)
    ref, bound, _ = conv_ref(x[:, first:], w[first:], b[first:], [40])
    within(out, ref, bound)
