"""The operators as a server uses them: a request hits another one's prefix, takes over pages and states, replays its own tail through a
layer of each kind, and goes on token by token."""
import numpy as np
import pytest
import torch

import oracle
from gpu_utils import TOL, state_rel_fro
from layer_utils import conv_ref, cu_of, f64, scan_inputs, scan_ref, within

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


def test_a_hit_continues_as_if_it_had_been_one_request():
    """Request 0 leaves its states in slot 0 of the pools.  Requests 1 and 2 branch off: key/value pages forked, state pages copied; each runs
    its own tail and three tokens, while the first goes on as well.  All equal the whole sequences in one pass, in 64 bits."""
    import paper_2608_30310_b200 as gdn
    C, S, K, prefix, tails, more = 48, 16, 4, 90, [0, 25, 40], 3
    T = prefix + sum(tails) + 3 * more
    m = scan_inputs(T, C, S, 1, F32, 3)
    g = torch.Generator().manual_seed(5)
    u, w, bias = torch.randn(T, C, generator=g), torch.randn(C, K, generator=g) / 2, torch.randn(C, generator=g)
    begin = np.concatenate([[prefix], prefix + np.cumsum([t + more for t in tails])])
    own = [list(range(begin[n], begin[n + 1])) for n in range(3)]            # each request's rows after the shared prefix
    # one pass over each whole sequence: the convolution's output is the scan's input
    whole = [list(range(prefix)) + own[n] for n in range(3)]
    lens = [len(r) for r in whole]
    rows = torch.tensor(sum(whole, []))
    xc, xb, _ = conv_ref(u[rows], w, bias, lens)
    pick = {k: v[rows] if k in ("dt", "z", "b", "c") else v for k, v in m.items()}
    # (the scan is linear in x: its own bound, and the convolution's errors carried through the magnitudes)
    ref, bound, h, hb = scan_ref(xc, pick["dt"], m["a"], pick["b"], pick["c"], lens, m["d"], pick["z"], m["dt_bias"])
    wide, _, hw, _ = scan_ref(xb + xc.abs() * 2.0 ** -24, pick["dt"], m["a"], pick["b"].abs(), pick["c"].abs(), lens, m["d"].abs(), None, m["dt_bias"])
    zabs = f64(pick["z"])
    bound = scan_bound_in_fp32(bound, ref) + wide.abs() * (zabs / (1 + torch.exp(-zabs))).abs() * 1.01
    hb = hb + hw.abs() * 1.01 + h.abs() * 2.0 ** -22
    at = np.concatenate([[0], np.cumsum(lens)])

    dev = {k: v.cuda() for k, v in m.items()}
    ud, wd, bd = u.cuda(), w.cuda(), bias.cuda()
    slots = 6
    conv_pool, scan_pool = torch.zeros(slots, K - 1, C, device="cuda"), torch.zeros(slots, C, S, device="cuda")
    kv = torch.arange(64 * 16, device="cuda", dtype=F32).view(64, 16)
    counts, tables = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.full((4, 12), -1, dtype=torch.int32, device="cuda")
    tables[0, :6] = torch.arange(20, 26, device="cuda")                       # 90 tokens in pages of 16: five and a part
    counts[20:26] = 1

    def i32(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def layer(rows, cu, init, keep):
        r = torch.tensor(rows, device="cuda")
        x = torch.empty(len(rows), C, device="cuda")
        gdn.gdn_short_conv(ud[r], wd, bd, cu.cuda(), x, init_state=conv_pool, out_state=conv_pool, init_slots=init, out_slots=keep)
        gdn.gdn_selective_scan(x, dev["dt"][r], dev["a"], dev["b"][r], dev["c"][r], cu.cuda(), x, d=dev["d"], z=dev["z"][r], dt_bias=dev["dt_bias"],
                               init_state=scan_pool, out_state=scan_pool, init_slots=init, out_slots=keep)
        return x
    first = layer(range(prefix), cu_of([prefix]), i32(-1), i32(0))
    within(first, ref[:prefix], bound[:prefix], "prefix")
    # the hit: pages shared, the part of a page and the states copied
    gdn.gdn_cache_fork([kv], 16, counts, tables, i32(0, 0), i32(1, 2), i32(prefix, prefix))
    gdn.gdn_cache_copy([conv_pool, scan_pool], i32(0, 0), i32(3, 5))
    assert tables[1, :6].tolist() == [20, 21, 22, 23, 24, 0] and tables[2, :6].tolist() == [20, 21, 22, 23, 24, 1]
    assert counts[[20, 24, 25, 0, 1]].tolist() == [3, 3, 1, 1, 1] and torch.equal(kv[0], kv[25]) and torch.equal(kv[1], kv[25])
    tail = layer(own[1][:tails[1]] + own[2][:tails[2]], cu_of(tails), i32(0, 3, 5), i32(0, 3, 5))
    for n, lo in ((1, 0), (2, tails[1])):
        within(tail[lo:lo + tails[n]], ref[at[n] + prefix:at[n] + prefix + tails[n]], bound[at[n] + prefix:at[n] + prefix + tails[n]], "tail %d" % n)
    # the states' pages are brought together before the requests go on: slots 0, 3, 5 become 0, 1, 2
    held, slot_rows = i32(1, 0, 0, 1, 0, 1), i32(0, 3, 5).view(3, 1)
    page_map, live = torch.zeros_like(held), i32(0)
    gdn.gdn_cache_compact([conv_pool, scan_pool], held, slot_rows, held, slot_rows, page_map, live)
    assert slot_rows[:, 0].tolist() == [0, 1, 2] and int(live) == 3
    slot = slot_rows[:, 0].contiguous()
    for t in range(more):
        r = torch.tensor([own[n][tails[n] + t] for n in range(3)], device="cuda")
        x = ud[r]
        gdn.gdn_short_conv_step(x, wd, bd, conv_pool, x, conv_pool, slots=slot)
        gdn.gdn_selective_scan_step(x, dev["dt"][r], dev["a"], dev["b"][r], dev["c"][r], scan_pool, x, scan_pool, d=dev["d"], z=dev["z"][r],
                                    dt_bias=dev["dt_bias"], slots=slot)
        e = torch.tensor([at[n] + prefix + tails[n] + t for n in range(3)])
        within(x, ref[e], bound[e], "token %d" % t)
    within(scan_pool[slot.long()], h, hb, "states")
    gdn.gdn_cache_free(counts, tables, i32(1, 2))
    assert counts[20:26].tolist() == [1] * 6 and int(counts.sum()) == 6


def scan_bound_in_fp32(bound, ref):
    """scan_ref saw its x in 64 bits and bounded the last rounding by that type's step: fp32's on top."""
    return bound + ref.abs() * 2.0 ** -23


def test_convolution_before_the_gated_delta_net():
    """q, k and v of a layer through one strided convolution each, then the replay with its input stage: tail and two tokens."""
    import paper_2608_30310_b200 as gdn
    Hq, Hv, D, K, lens = 2, 4, 64, 4, [70, 0, 33]
    N, T, widths = len(lens), 103, (2 * 64, 2 * 64, 4 * 64)
    g = torch.Generator().manual_seed(8)
    proj, w = torch.randn(T, sum(widths), generator=g), torch.randn(sum(widths), K, generator=g) / 2
    gate, beta = torch.rand(T, Hv, generator=g) * 4 + 2.5, torch.randn(T, Hv, generator=g)
    pd, wd, cu = proj.cuda(), w.cuda(), cu_of(lens).cuda()
    parts, off = [], 0
    for n in widths:
        out = torch.empty(T, n, device="cuda")
        gdn.gdn_short_conv(pd[:, off:off + n], wd[off:off + n], None, cu, out)
        ref, bound, _ = conv_ref(proj[:, off:off + n], w[off:off + n], None, lens)
        within(out, ref, bound)
        parts.append(out.view(T, n // D, D))
        off += n
    o, st = torch.empty(T, Hv, D, device="cuda"), torch.empty(N, Hv, D, D, device="cuda")
    gdn.gdn_tail_replay(*parts, gate.cuda(), beta.cuda(), cu, 64, o, st, raw_inputs=True)
    q, k, v = (p.cpu().numpy().astype(np.float64) for p in parts)
    qn, kn, gl, bt = oracle.prologue(q, k, gate.numpy().astype(np.float64), beta.numpy().astype(np.float64))
    ro, rst = oracle.gdn_forward_f64(qn, kn, v, gl, bt, np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
    assert np.abs(o.cpu().numpy() - ro).max() <= TOL["f32"]["o_max_abs"]
    assert state_rel_fro(st.cpu().numpy().astype(np.float64), rst)[0] <= TOL["f32"]["state_rel_fro"]
