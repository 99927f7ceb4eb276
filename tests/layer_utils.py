"""64-bit definitions of the recurrent layers' operators, with the error that fp32 arithmetic may make beside each value, and of the
bookkeeping of the cache's pages in plain Python.

The bounds count roundings.  u = 2^-24 is half a step of fp32.  CUDA's documented errors: exp(x) by __expf (2 + 1.173 |x|) steps of 2^-23,
__fdividef 2 steps, ex2.approx 2^-22.  What is rounded to the io dtype is off by half a step more, eps / 2 of its value."""
import numpy as np
import torch

U = 2.0 ** -24


def silu(y):
    return y / (1 + torch.exp(-y))


def silu_rel(y):
    """exp weighs in with at most its own error; the sum 1, the quotient 2 steps, and a step of slack."""
    return (6 + 1.2 * y.abs()) * 2 * U


def rounding(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return None if t is None else t.detach().cpu().double()


def conv_ref(x, weight, bias, lens, init=None, act=True):
    """x [T, C], lens the requests' lengths, init [N, K - 1, C] or None.  (out, bound, states), states in x's dtype."""
    K, dtype = weight.shape[1], x.dtype
    xs, w = f64(x), f64(weight)
    b = torch.zeros(w.shape[0], dtype=torch.float64) if bias is None else f64(bias)
    out, bound = torch.zeros_like(xs), torch.zeros_like(xs)
    states, at = [], 0
    for n, length in enumerate(lens):
        old = torch.zeros((K - 1, w.shape[0]), dtype=torch.float64) if init is None else f64(init[n])
        rows = torch.cat([old, xs[at:at + length]])
        for t in range(length):
            win = rows[t:t + K].T
            y, size = b + (win * w).sum(1), b.abs() + (win * w).abs().sum(1)
            err = (K + 1) * U * size
            if act:
                out[at + t] = silu(y)
                err = 1.1 * err + out[at + t].abs() * silu_rel(y)          # |silu'| < 1.1
            else:
                out[at + t] = y
            bound[at + t] = 1.01 * (err + rounding(dtype) * (out[at + t].abs() + err)) + 1e-30
        states.append(rows[length:].to(dtype))
        at += length
    return out, bound, torch.stack(states)


def scan_ref(x, dt, a, b, c, lens, d=None, z=None, dt_bias=None, softplus=True, init=None):
    """(out, bound, states, bound of the states): all requests side by side, token by token."""
    dtype, N, (C, S), G = x.dtype, len(lens), a.shape, b.shape[1]
    xs, ds, bs, cs, av = f64(x), f64(dt), f64(b), f64(c), f64(a)
    begin = np.concatenate([[0], np.cumsum(lens)])[:-1]
    h = torch.zeros((N, C, S), dtype=torch.float64) if init is None else f64(init).clone()
    err = torch.zeros_like(h)
    out, bound = torch.zeros_like(xs), torch.zeros_like(xs)
    for t in range(max(lens, default=0)):
        who = [n for n in range(N) if lens[n] > t]
        r = torch.tensor([begin[n] + t for n in who])
        v = ds[r] + (0 if dt_bias is None else f64(dt_bias))
        step, rel = v, 2 * U * torch.ones_like(v)
        if softplus:
            # log1p's part: exp, quotient, series (4 steps), sums; v's own rounding moves the result by at most |v| u of its value
            step = torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))
            rel = (10 + 2 * v.abs()) * 2 * U
        else:
            rel = rel + U * (ds[r].abs() + (0 if dt_bias is None else f64(dt_bias).abs())) / v.abs().clamp(min=1e-300)
        B, Cc = (m[r].repeat_interleave(C // G, 1) for m in (bs, cs))
        arg = step[:, :, None] * av
        decay = torch.exp(arg)
        add = (step * xs[r])[:, :, None] * B
        old, olde = h[who], err[who]
        new = decay * old + add
        # the exponent's roundings (dt, a log2(e), their product) and ex2's own; dt x and its product with b; the fma
        drel = 4 * U + arg.abs() * (rel[:, :, None] + 4 * U)
        newe = decay * (1 + drel) * olde + decay * drel * old.abs() + add.abs() * (rel[:, :, None] + 4 * U)
        newe = newe + U * (new.abs() + newe)
        h[who], err[who] = new, newe
        y = (new * Cc).sum(-1)
        size = (new * Cc).abs().sum(-1)
        e = (newe * Cc.abs()).sum(-1) + (S + 2) * U * (size + (newe * Cc.abs()).sum(-1))
        if d is not None:
            y = y + f64(d) * xs[r]
            e = e + 2 * U * (f64(d) * xs[r]).abs()
        if z is not None:
            g = silu(f64(z)[r])
            e = e * g.abs() * 1.001 + (y * g).abs() * (silu_rel(f64(z)[r]) + 2 * U)
            y = y * g
        out[r] = y
        bound[r] = 1.01 * (e + rounding(dtype) * (y.abs() + e)) + 1e-30
    return out, bound, h, 1.01 * err + 1e-30


def within(got, ref, bound, what=""):
    got = f64(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), what + ": not finite"
    over = ((got - ref).abs() / bound)
    assert not over.numel() or over.max().item() <= 1, "%s: %.3g times the bound at %s" % (what, over.max().item(), np.unravel_index(int(over.argmax()), over.shape))


def cu_of(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))


def scan_inputs(T, C, S, G, dtype, seed, device="cpu"):
    g = torch.Generator().manual_seed(seed)

    def n(*shape):
        return torch.randn(shape, generator=g)
    m = {"x": n(T, C).to(dtype), "dt": (0.5 * n(T, C)).to(dtype), "z": n(T, C).to(dtype), "b": n(T, G, S).to(dtype), "c": n(T, G, S).to(dtype),
         "a": -torch.arange(1, S + 1, dtype=torch.float32) * torch.exp(0.1 * n(C, S)), "d": 1 + 0.1 * n(C),
         "dt_bias": torch.log(torch.expm1(torch.exp(torch.rand(C, generator=g) * 4.6 - 6.9)))}
    return {k: v.to(device) for k, v in m.items()}


# ---- pages, in plain Python on lists

def release(count, table, row):
    for j, p in enumerate(table[row]):
        if p >= 0:
            count[p] -= 1
        table[row][j] = -1


def fork_ref(count, table, parents, children, tokens, page_tokens):
    """The page moves [(src, dst)] of a call; count and table change.  Whether a fork was left out, or found no page."""
    pages, rows, W = len(count), len(table), len(table[0])
    named = [c for c in children if 0 <= c < rows]
    forks, bad = [], False
    for p, c, n in zip(parents, children, tokens):
        need = -(-n // page_tokens) if n >= 0 else -1
        ok = 0 <= p < rows and 0 <= c < rows and 0 <= need <= W and named.count(c) == 1 and p not in named and \
            all(0 <= e < pages for e in table[p][:need])
        bad |= not ok
        if ok:
            forks.append((p, c, n))
    for _, c, _ in forks:
        release(count, table, c)
    free = [p for p in range(pages) if count[p] <= 0]
    moves, short = [], False
    for p, c, n in forks:
        whole, part = n // page_tokens, n % page_tokens > 0
        if part:
            if not free:
                short = True
                continue
            new = free.pop(0)
            moves.append((table[p][whole], new))
            table[c][whole] = new
            count[new] = 1
        for j in range(whole):
            table[c][j] = table[p][j]
            count[table[p][j]] += 1
    return moves, bad, short


def compact_ref(count, table):
    pages = len(count)
    M = sum(c > 0 for c in count)
    moves = list(zip([p for p in range(M, pages) if count[p] > 0], [p for p in range(M) if count[p] <= 0]))
    to = {p: p for p in range(M) if count[p] > 0}
    to.update(dict(moves))
    out = [0] * pages
    for p, q in to.items():
        out[q] = count[p]
    table = [[to.get(e, -1) if e >= 0 else -1 for e in row] for row in table]
    return moves, out, table, [to.get(p, -1) for p in range(pages)], M
