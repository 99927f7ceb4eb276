"""Operators beside the tail replay: the short causal convolution and the selective state space scan of recurrent layers, for packed
prompts and for single tokens, and the pages of the cache that their states and the attention layers' keys and values live in.

A case is a dict of plain values; ``op`` says which call it is:

    conv, conv_step    depthwise causal convolution over the last ``width`` rows, with SiLU
    scan, scan_step    h = exp(dt a) h + dt x b,  y = c . h + d x,  y silu(z), with dt = softplus(dt + dt_bias)
    copy               pages of every layer's pool from one place to another
    fork               requests that begin as branches of others: whole pages shared, the last, partial one copied
    branch             the same, and the branches given up again
    compact            live pages moved to the front of the pools

Prompts are packed (``lo`` to ``hi`` tokens a request); states live in pools and requests name their slots.  x and z are halves of one
projection, b and c slices of another, as a layer has them.
"""
import math
import random

import torch

own = False


def _case(op, name=None, **kw):
    c = {"op": op}
    if op in ("conv", "conv_step", "scan", "scan_step"):
        c.update(requests=1, lo=1, hi=1, channels=4096, io="bf16", resume=False)
        c.update({"width": 4} if op.startswith("conv") else {"states": 16, "groups": 1, "gated": True})
    else:
        c.update(pools=12, pages=1024, page=8192)                          # page: bf16 values of one pool's page
        c.update({"copy": {"moved": 1}, "compact": {"live": 512, "moved": 128, "rows": 64}}.get(
            op, {"parents": 1, "children": 1, "row": 64, "page_tokens": 16}))
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # q, k and v of a linear-attention layer (2 x 16 + 32 heads of 128), the tails of four hits
        _case("conv", "conv_4_hits", requests=4, lo=1569, hi=3185, channels=8192, resume=True),
        # the same layer, one user, one token: a call's latency
        _case("conv_step", "conv_step_1", channels=8192),
        # one layer of one hit: 5 % of a 32K prefix, from a zero state
        _case("scan", "scan_tail_1638", lo=1638, hi=1638),
        # eight concurrent hits with ragged tails, continued from states of the cache
        _case("scan", "scan_8_hits", requests=8, lo=410, hi=3277, resume=True),
        # a small fp32 layer (4 heads of 64), 512 tokens
        _case("scan", "scan_tiny_fp32", lo=512, hi=512, channels=256, io="f32"),
        # a full serving batch, one token each
        _case("scan_step", "scan_step_256", requests=256),
        # one request's recurrent states (36 layers of 4,096 x 16 fp32) kept at a page boundary
        _case("copy", "copy_1_state", pools=36, pages=16, page=131072, moved=1),
        # pages brought together for a batch of hits: 12 attention layers
        _case("copy", "copy_400_pages", pages=1024, page=32768, moved=400),
        # one request continues from another one's prefix of a thousand tokens
        _case("fork", "fork_1"),
        # 64 branches of 8 long prefixes (32K tokens), two key/value heads per layer
        _case("fork", "fork_64", pages=20480, page=8192, parents=8, children=64, row=2048),
        # 32 branches for one step of sampling, given up again
        _case("branch", "branch_32", pages=4096, page=16384, parents=4, children=32, row=256),
        # a half-empty cache brought to the front
        _case("compact", "compact_2048", pages=2048, page=32768, live=1024, moved=512, rows=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["conv", "conv_step", "scan", "scan", "scan", "scan_step", "copy", "fork", "branch", "compact"])
    io = rng.choice(["bf16", "bf16", "f32"])
    if op in ("conv", "conv_step"):
        c = _case(op, requests=_log_int(rng, 1, 64 if op == "conv" else 256), channels=_log_int(rng, 60, 8192), io=io, width=rng.randint(2, 4),
                  resume=rng.random() < 0.5)
        if rng.random() < 0.6:
            c["channels"] = (c["channels"] + 7) // 8 * 8
        if op == "conv":
            c["hi"] = max(1, min(_log_int(rng, 1, 3300), 9000 // c["requests"]))
            c["lo"] = max(0, c["hi"] // rng.randint(1, 8))
        return c
    if op in ("scan", "scan_step"):
        c = _case(op, requests=_log_int(rng, 1, 32 if op == "scan" else 256), channels=_log_int(rng, 60, 4096), io=io,
                  states=rng.choice([8, 16, 16, 16, 32, 64]), gated=rng.random() < 0.7, resume=rng.random() < 0.5)
        if rng.random() < 0.6:
            c["channels"] = (c["channels"] + 63) // 64 * 64
            c["groups"] = rng.choice([1, 1, 2, 4])
        most = 7 * 10 ** 8 // (c["channels"] * c["states"])                # no more than the listed batch of eight hits
        if op == "scan":
            c["requests"] = max(1, min(c["requests"], most // 8))
            c["hi"] = max(1, min(_log_int(rng, 1, 3300), most // c["requests"]))
            c["lo"] = max(0, c["hi"] // rng.randint(1, 8))
        else:
            c["requests"] = max(1, min(c["requests"], 2 ** 24 // (c["channels"] * c["states"])))
        return c
    c = _case(op, pools=rng.choice([1, 4, 12, 24, 36]), pages=_log_int(rng, 64, 16384), page=8 * _log_int(rng, 16, 4096))
    c["pages"] = max(64, min(c["pages"], 4 * 10 ** 8 // (c["pools"] * c["page"])))
    if op == "copy":
        c["moved"] = _log_int(rng, 1, c["pages"] // 2)
    elif op == "compact":
        c["live"] = rng.randint(1, c["pages"])
        c["moved"] = rng.randint(0, min(c["live"], c["pages"] - c["live"]))
        c["rows"] = _log_int(rng, 1, 200)
    else:
        c["page_tokens"] = rng.choice([1, 16, 16, 32, 64])
        c["children"] = _log_int(rng, 1, min(64, c["pages"] // 4))
        c["parents"] = max(1, c["children"] // rng.randint(1, 8))
        c["row"] = max(1, min(_log_int(rng, 1, 1024), (c["pages"] - c["children"]) // c["parents"]))
    return c


def _tails(case):
    """Lengths of the requests: fixed by the sizes of the case, so that work() and prepare() agree."""
    r = random.Random("%d/%d/%d" % (case["requests"], case["lo"], case["hi"]))
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["requests"] - 1)] + [case["hi"]]


def _tokens(case):
    """Tokens that each child takes over from its parent: up to the parent's whole row, most of them ending inside a page."""
    r = random.Random("%d/%d/%d" % (case["children"], case["row"], case["page_tokens"]))
    return [r.randint(max(1, case["row"] * case["page_tokens"] // 2), case["row"] * case["page_tokens"]) for _ in range(case["children"])]


# ---- inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    s = {"op": case["op"]}
    if case["op"] in ("copy", "compact", "fork", "branch"):
        return _prepare_pages(case, seed, s, gen, dev)
    dt = torch.bfloat16 if case["io"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=gen, device=dev, dtype=torch.float32) * (hi - lo) + lo

    step = case["op"].endswith("_step")
    lens = [1] * case["requests"] if step else _tails(case)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    N, T, C = len(lens), cu[-1], case["channels"]
    if not step:
        s["cu"], s["longest"] = torch.tensor(cu, dtype=torch.int32, device=dev), max(lens)
    slots = torch.randperm(N + 4, generator=gen, device=dev)[:N].to(torch.int32)   # the pool has room for others
    s["slots"] = slots
    s["resume"] = case["resume"] or step
    if case["op"].startswith("conv"):
        K = case["width"]
        s["x"] = normal(T, C).to(dt)
        s["weight"], s["bias"] = uniform(-K ** -0.5, K ** -0.5, C, K).to(dt), uniform(-K ** -0.5, K ** -0.5, C).to(dt)
        s["out"] = torch.zeros((T, C), dtype=dt, device=dev)
        s["state"] = normal(N + 4, K - 1, C).to(dt)
        s["out_state"] = s["state"] if step else torch.zeros_like(s["state"])
        return s
    S, G = case["states"], case["groups"]
    R = (C + 15) // 16                                                     # rank of the projection that dt comes from
    both = normal(T, 2 * C).to(dt)
    s["x"], s["z"] = both[:, :C], both[:, C:] if case["gated"] else None
    s["dt"] = (0.5 * normal(T, C)).to(dt)
    proj = normal(T, R + 2 * G * S).to(dt)
    s["b"], s["c"] = proj[:, R:R + G * S].unflatten(1, (G, S)), proj[:, R + G * S:].unflatten(1, (G, S))
    # time steps of 0.001 to 0.1 at dt = 0; decays 1 to S, spread as training leaves them
    s["dt_bias"] = torch.log(torch.expm1(torch.exp(uniform(math.log(1e-3), math.log(1e-1), C))))
    s["a"] = -torch.arange(1, S + 1, device=dev, dtype=torch.float32) * torch.exp(0.1 * normal(C, S))
    s["d"] = 1 + 0.1 * normal(C)
    s["out"] = torch.zeros((T, C), dtype=dt, device=dev)
    s["state"] = normal(N + 4, C, S)
    s["out_state"] = s["state"] if step else torch.zeros_like(s["state"])
    return s


def _prepare_pages(case, seed, s, gen, dev):
    L, P, E = case["pools"], case["pages"], case["page"]
    r = random.Random(seed)
    s["store"] = torch.randn((L, P, E), generator=gen, device=dev, dtype=torch.float32 if L * P * E < 10 ** 8 else torch.bfloat16).to(torch.bfloat16)
    s["pools"] = [s["store"][i] for i in range(L)]

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    if case["op"] == "copy":
        ids = r.sample(range(P), 2 * case["moved"])
        s["src"], s["dst"] = ints(ids[:case["moved"]]), ints(ids[case["moved"]:])
        return s
    if case["op"] == "compact":
        M, k, R = case["live"], case["moved"], case["rows"]
        live = r.sample(range(M), M - k) + r.sample(range(M, P), k)
        r.shuffle(live)
        width = -(-M // R)
        table, count = [[-1] * (width + 2) for _ in range(R)], [0] * P
        for i, p in enumerate(live):
            table[i % R][i // R] = p
            count[p] += 1
        for i in range(R):                                                 # a page that two rows share
            table[i][width] = live[i % M]
            count[live[i % M]] += 1
        s["refcounts"], s["tables"] = ints(count), ints(table)
        s["out_refcounts"], s["out_tables"] = torch.zeros_like(s["refcounts"]), torch.zeros_like(s["tables"])
        s["moved"] = k
        s["page_map"], s["live"] = torch.zeros_like(s["refcounts"]), torch.zeros(1, dtype=torch.int32, device=dev)
        return s
    A, B, W = case["parents"], case["children"], case["row"]
    used = r.sample(range(P), A * W)
    rows = list(range(A + B + 2))
    r.shuffle(rows)
    table, count = [[-1] * (W + 1) for _ in rows], [0] * P
    for i, p in enumerate(used):
        table[rows[i // W]][i % W] = p
        count[p] = 1
    s["refcounts"], s["tables"] = ints(count), ints(table)
    s["page_tokens"] = case["page_tokens"]
    s["parents"], s["children"] = ints([rows[i % A] for i in range(B)]), ints(rows[A:A + B])
    s["tokens"] = ints(_tokens(case))
    return s


# ---- one pass

def run(s):
    if own:
        return _run_own(s)
    return {"conv": _conv, "conv_step": _conv, "scan": _scan, "scan_step": _scan, "copy": _copy, "fork": _fork, "branch": _branch,
            "compact": _compact}[s["op"]](s)


def _run_own(s):
    import paper_2608_30310_b200 as gdn
    op = s["op"]
    if op == "conv":
        gdn.gdn_short_conv(s["x"], s["weight"], s["bias"], s["cu"], s["out"], init_state=s["state"] if s["resume"] else None,
                           init_slots=s["slots"] if s["resume"] else None, out_state=s["out_state"], out_slots=s["slots"])
        return s["out"], s["out_state"]
    if op == "conv_step":
        gdn.gdn_short_conv_step(s["x"], s["weight"], s["bias"], s["state"], s["out"], s["out_state"], slots=s["slots"])
        return s["out"], s["out_state"]
    if op == "scan":
        gdn.gdn_selective_scan(s["x"], s["dt"], s["a"], s["b"], s["c"], s["cu"], s["out"], d=s["d"], z=s["z"], dt_bias=s["dt_bias"],
                               init_state=s["state"] if s["resume"] else None, init_slots=s["slots"] if s["resume"] else None,
                               out_state=s["out_state"], out_slots=s["slots"])
        return s["out"], s["out_state"]
    if op == "scan_step":
        gdn.gdn_selective_scan_step(s["x"], s["dt"], s["a"], s["b"], s["c"], s["state"], s["out"], s["out_state"], d=s["d"], z=s["z"],
                                    dt_bias=s["dt_bias"], slots=s["slots"])
        return s["out"], s["out_state"]
    if op == "copy":
        gdn.gdn_cache_copy(s["pools"], s["src"], s["dst"])
        return s["store"]
    if "workspace" not in s:
        s["workspace"] = gdn.Workspace()
    if op == "compact":
        gdn.gdn_cache_compact(s["pools"], s["refcounts"], s["tables"], s["out_refcounts"], s["out_tables"], s["page_map"], s["live"],
                              workspace=s["workspace"])
        return s["store"], s["out_refcounts"], s["out_tables"], s["page_map"], s["live"]
    gdn.gdn_cache_fork(s["pools"], s["page_tokens"], s["refcounts"], s["tables"], s["parents"], s["children"], s["tokens"],
                       workspace=s["workspace"])
    if op == "branch":
        gdn.gdn_cache_free(s["refcounts"], s["tables"], s["children"])
    return s["store"], s["refcounts"], s["tables"]


def _silu(x):
    return x / (1 + torch.exp(-x))


def _requests_of(s):
    """Request of each row, and its first row."""
    if "cu" not in s:
        t = torch.arange(s["x"].shape[0], device=s["x"].device)
        return t, t, t, t + 1
    cu = s["cu"].long()
    t = torch.arange(s["x"].shape[0], device=cu.device)
    req = torch.searchsorted(cu, t, right=True) - 1
    return req, cu[req], cu[:-1], cu[1:]


def _conv(s):
    x, w, K = s["x"].float(), s["weight"].float(), s["weight"].shape[1]
    T = x.shape[0]
    slots = s["slots"].long()
    hist = s["state"][slots].float() if s["resume"] else torch.zeros((len(slots), K - 1, x.shape[1]), device=x.device)
    req, first, begin, end = _requests_of(s)
    row = torch.arange(T, device=x.device)
    y = s["bias"].float() + w[:, K - 1] * x
    for j in range(K - 1):
        at = row - (K - 1) + j                                             # before the request's first row: its history
        before = hist[req, (at - first + K - 1).clamp(0, K - 2)]
        y = y + w[:, j] * torch.where((at >= first)[:, None], x[at.clamp(min=0)], before)
    i = torch.arange(K - 1, device=x.device)
    at = end[:, None] - (K - 1) + i
    old = torch.gather(hist, 1, ((end - begin)[:, None] + i).clamp(max=K - 2)[:, :, None].expand(-1, -1, x.shape[1]))
    new = torch.where((at >= begin[:, None])[:, :, None], x[at.clamp(min=0)] if T else old, old)
    s["out_state"][slots] = new.to(s["out_state"].dtype)
    s["out"].copy_(_silu(y))
    return s["out"], s["out_state"]


def _scan(s):
    x, a = s["x"].float(), s["a"]
    T, C = x.shape
    dt = s["dt"].float() + s["dt_bias"]
    dt = dt.clamp(min=0) + torch.log1p(torch.exp(-dt.abs()))               # softplus
    each = C // s["b"].shape[1]
    decay = torch.exp(dt[:, :, None] * a)
    h = (dt * x)[:, :, None] * s["b"].float().repeat_interleave(each, 1)
    slots = s["slots"].long()
    start = s["state"][slots] if s["resume"] else torch.zeros((len(slots), C, a.shape[1]), device=x.device)
    req, first, begin, end = _requests_of(s)
    # h_t = decay_t h_{t-1} + h_t by doubling: after a pass of step k every row has taken in the 2 k rows up to it; a request's first
    # row takes in the start state, and nothing before it
    there = (end > begin)
    at = begin.clamp(max=max(T - 1, 0))
    if T:
        h = h.index_add(0, at, torch.where(there[:, None, None], decay[at] * start, torch.zeros_like(start)))
    if "cu" in s:
        decay = torch.where((torch.arange(T, device=x.device) == first)[:, None, None], torch.zeros_like(decay[:1]), decay)
        k = 1
        while k < s["longest"]:
            h = torch.cat([h[:k], torch.addcmul(h[k:], decay[k:], h[:-k])])
            decay = torch.cat([decay[:k], decay[k:] * decay[:-k]])
            k *= 2
    y = (h * s["c"].float().repeat_interleave(each, 1)).sum(-1) + s["d"] * x
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    last = torch.where(there[:, None, None], h[(end - 1).clamp(min=0)], start) if T else start
    s["out_state"][slots] = last
    s["out"].copy_(y)
    return s["out"], s["out_state"]


def _copy(s):
    s["store"][:, s["dst"].long()] = s["store"][:, s["src"].long()]
    return s["store"]


def _release(s, rows):
    """Entries of these rows given back: their counts go down, the rows are empty."""
    e = s["tables"][rows].reshape(-1).long()
    s["refcounts"].index_add_(0, e.clamp(min=0), -(e >= 0).to(torch.int32))
    s["tables"][rows] = -1


def _fork(s):
    parents, children, tokens = s["parents"].long(), s["children"].long(), s["tokens"].long()
    _release(s, children)
    whole, part = tokens // s["page_tokens"], tokens % s["page_tokens"] > 0
    row = s["tables"][parents]
    W = row.shape[1]
    kept = torch.where(torch.arange(W, device=row.device) < whole[:, None], row, torch.full_like(row, -1))
    # partial last pages: the lowest-numbered free pages, in the order of the forks
    order = torch.cumsum(part.long(), 0) - 1
    free = torch.argsort((s["refcounts"] > 0).to(torch.int32), stable=True)
    new = free[order.clamp(min=0)]
    at = whole.clamp(max=W - 1)
    src = torch.gather(row, 1, at[:, None])[:, 0].long()
    kept.scatter_(1, at[:, None], torch.where(part, new, torch.gather(kept, 1, at[:, None])[:, 0].long()).to(torch.int32)[:, None])
    e = kept.reshape(-1).long()
    s["refcounts"].index_add_(0, e.clamp(min=0), (e >= 0).to(torch.int32))
    s["tables"][children] = kept
    src = torch.where(part, src, row[:, 0].long())                         # (a fork without one: a page in use onto itself)
    s["store"][:, torch.where(part, new, src)] = s["store"][:, src]
    return s["store"], s["refcounts"], s["tables"]


def _branch(s):
    _fork(s)
    _release(s, s["children"].long())
    return s["store"], s["refcounts"], s["tables"]


def _compact(s):
    count = s["refcounts"]
    P = count.shape[0]
    page = torch.arange(P, device=count.device)
    alive = count > 0
    M = alive.sum()
    dst, src = (torch.argsort((~m).to(torch.int32), stable=True)[:s["moved"]] for m in (~alive & (page < M), alive & (page >= M)))
    to = torch.where(alive, page, torch.full_like(page, -1))
    to[src] = dst
    s["store"][:, dst] = s["store"][:, src]
    out = torch.where(alive & (page < M), count, torch.zeros_like(count))
    out[dst] = count[src]
    s["out_refcounts"].copy_(out)
    t = s["tables"].long()
    s["out_tables"].copy_(torch.where(t >= 0, to[t.clamp(min=0)], t))
    s["page_map"].copy_(to)
    s["live"].copy_(M[None])
    return s["store"], s["out_refcounts"], s["out_tables"], s["page_map"], s["live"]


# ---- what a pass cannot do without

def work(case):
    if case["op"] in ("conv", "conv_step", "scan", "scan_step"):
        step = case["op"].endswith("_step")
        N, C, e = case["requests"], case["channels"], 2 if case["io"] == "bf16" else 4
        T = N if step else sum(_tails(case))
        ways = 2 if step or case["resume"] else 1                          # states written, and read where there are any
        if case["op"].startswith("conv"):
            K = case["width"]
            return {"bytes": e * (2 * T * C + (K + 1) * C + ways * N * (K - 1) * C), "flops": (2.0 * K + 4) * T * C}
        S = case["states"]
        arrays = 4 if case["gated"] else 3
        # an exponential, three products and two sums a state; the time step and the gate
        return {"bytes": e * (arrays * T * C + 2 * T * case["groups"] * S) + 4 * (C * S + 2 * C) + 4 * ways * N * C * S,
                "flops": 6.0 * T * C * S + 12.0 * T * C}
    page = 2 * case["pools"] * case["page"]
    if case["op"] == "copy":
        return {"bytes": 2 * case["moved"] * page + 8 * case["moved"], "flops": 0.0}
    if case["op"] == "compact":
        entries = case["rows"] * (-(-case["live"] // case["rows"]) + 2)
        return {"bytes": 2 * case["moved"] * page + 12 * case["pages"] + 8 * entries, "flops": 0.0}
    copied = sum(n % case["page_tokens"] > 0 for n in _tokens(case))
    shared = sum(n // case["page_tokens"] for n in _tokens(case))
    # rows of the parents read, of the children written, counts up (and down again)
    return {"bytes": 2 * copied * page + (16 + (12 if case["op"] == "branch" else 0)) * shared + 12 * case["children"], "flops": 0.0}


# ---- the definitions in 64 bits, request by request or token by token

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("conv"):
        return _exact_conv(s)
    if case["op"].startswith("scan"):
        return _exact_scan(s)
    return _exact_pages(s)


def _bounds(s):
    return s["cu"].tolist() if "cu" in s else list(range(s["x"].shape[0] + 1))


def _exact_conv(s):
    cu, K = _bounds(s), s["weight"].shape[1]
    w = s["weight"].double()
    y, out = torch.zeros(s["x"].shape, dtype=torch.float64, device=w.device), s["out_state"].double().clone()
    for n, slot in enumerate(s["slots"].tolist()):
        old = s["state"][slot].double() if s["resume"] else torch.zeros((K - 1, w.shape[0]), dtype=torch.float64, device=w.device)
        rows = torch.cat([old, s["x"][cu[n]:cu[n + 1]].double()])
        if cu[n + 1] > cu[n]:
            acc = s["bias"].double() + (rows.unfold(0, K, 1) * w).sum(-1)
            y[cu[n]:cu[n + 1]] = acc * torch.sigmoid(acc)
        out[slot] = rows[rows.shape[0] - (K - 1):]
    return y, out


def _exact_scan(s):
    cu = _bounds(s)
    dev = s["a"].device
    dt = torch.nn.functional.softplus(s["dt"].double() + s["dt_bias"].double(), threshold=100)
    x, a, G = s["x"].double(), s["a"].double(), s["b"].shape[1]
    each = a.shape[0] // G
    lens = torch.tensor([v - u for u, v in zip(cu, cu[1:])], device=dev)
    begin = torch.tensor(cu[:-1], device=dev)
    h = s["state"][s["slots"].long()].double() if s["resume"] else torch.zeros((len(lens), *a.shape), dtype=torch.float64, device=dev)
    y = torch.zeros(x.shape, dtype=torch.float64, device=dev)
    most = max([v - u for u, v in zip(cu, cu[1:])])
    by_length = sorted(range(len(lens)), key=lambda n: cu[n] - cu[n + 1])     # longest first: those still running come first
    order = torch.tensor(by_length, device=dev)
    h, begin, length = h[order], begin[order], [cu[n + 1] - cu[n] for n in by_length]
    running = len(length)
    for t in range(most):
        while running and length[running - 1] <= t:
            running -= 1
        r = begin[:running] + t
        b, c = (s[k][r].double().repeat_interleave(each, 1) for k in ("b", "c"))
        h[:running] = torch.exp(dt[r][:, :, None] * a) * h[:running] + (dt[r] * x[r])[:, :, None] * b
        y[r] = (h[:running] * c).sum(-1)
    y += s["d"].double() * x
    if s["z"] is not None:
        y *= s["z"].double() * torch.sigmoid(s["z"].double())
    out = s["out_state"].double().clone()
    out[s["slots"].long()[order]] = h
    return y, out


def _exact_pages(s):
    """The pages' values; counts and tables are whole numbers and have no other value than the one computed."""
    moves = []
    if s["op"] == "copy":
        moves = list(zip(s["src"].tolist(), s["dst"].tolist()))
        return _moved(s, moves)
    count = s["refcounts"].tolist()
    if s["op"] == "compact":
        M = sum(c > 0 for c in count)
        holes = [p for p in range(M) if count[p] == 0]
        moves = list(zip([p for p in range(M, len(count)) if count[p] > 0], holes))
        return _moved(s, moves), None, None, None, None
    table, free = s["tables"].tolist(), (p for p in range(len(count)) if count[p] == 0)
    for p, n in zip(s["parents"].tolist(), s["tokens"].tolist()):
        if n % s["page_tokens"]:
            moves.append((table[p][n // s["page_tokens"]], next(free)))
    return _moved(s, moves), None, None


def _moved(s, moves):
    out = s["store"].double()
    for src, dst in moves:
        out[:, dst] = s["store"][:, src].double()
    return out
