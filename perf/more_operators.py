"""Cases of the operators that answer from a cache: rotated queries and keys, attention over a paged cache, the
weights that its rows have gathered, and eviction by them.

`listed()` names the cases, `draw(rng)` gives more of the same ranges, `prepare(case, seed)` makes what a program
has in hand before the call, `run(state)` is one pass.  With `own` false a pass is written in elementary torch
operations in 32 bits (angles in 64), rounded once at the end; with `own` true it makes the calls a user makes of
this package.  `exact(case, seed)` states the same results in 64 bits.

Operators
  rotary      per head x * rsqrt(mean x^2 + eps) * gamma (or x as it is), then the rotation of every pair of columns
              by position * frequency, each pair with one of up to three position axes; "fwd" returns (q', k'),
              "bwd" (dq, dk, dgamma_q, dgamma_k), "append" q' and the cache with the rows of k' and v written
  attention   the new tokens of every sequence over its rows of a paged cache, each query up to its own row;
              returns (out, lse)
  weights     prior + the softmax weight that every cache row gets from the new tokens, per key / value head
  evict       rows kept by weight, first and last rows protected, moved in their order to other pages; returns
              (kept, lens, weights, key pages, value pages)
"""
import math

import torch

own = False

EPS = 1e-6
SCORES = 1 << 28        # scores of one step of the plain form


# ------------------------------------------------------------------ cases
def _rotary(name, direction, tokens, heads, head_dim, axes=1, norm=True, interleaved=False, dtype="bf16", fused=False, page=16):
    c = {"op": "rotary", "direction": direction, "tokens": tokens, "heads_q": heads[0], "heads_kv": heads[1],
         "head_dim": head_dim, "axes": axes, "norm": norm, "interleaved": interleaved, "dtype": dtype, "fused": fused, "page": page}
    return dict(c, name=name) if name else c


def _text(v):
    return " ".join(str(n) for n in v)


def _cached(op, name, new, lens, heads, head_dim, page, dtype="bf16"):
    c = {"op": op, "new": _text(new), "lens": _text(lens), "heads_q": heads[0], "heads_kv": heads[1], "head_dim": head_dim,
         "page": page, "dtype": dtype}
    return dict(c, name=name) if name else c


def _evict(name, lens, heads_kv, head_dim, page, budget, sinks, recent, dtype="bf16"):
    c = {"op": "evict", "lens": _text(lens), "heads_q": heads_kv, "heads_kv": heads_kv, "head_dim": head_dim, "page": page,
         "budget": budget, "sinks": sinks, "recent": recent, "dtype": dtype}
    return dict(c, name=name) if name else c


# cache lengths of 48 conversations that are being answered together, from a short question to many images
BATCH = (37, 2184, 616, 1501, 8877, 640, 4390, 1847, 93, 5702, 883, 1366, 2986, 2518, 601, 1660,
         3208, 953, 719, 6501, 1117, 7640, 390, 2847, 4093, 702, 1883, 366, 986, 518, 2601, 160,
         1208, 4953, 2719, 501, 3117, 1640, 1390, 847, 2093, 3702, 483, 5366, 1986, 1518, 4601, 1160)


def listed():
    return [
        # the tokens that 16 conversations have just sampled, far into their contexts: a call's latency
        _rotary("rotary-append-decode", "append", 16, (32, 8), 128),
        # the fine-tuning batch, 8 x 616 tokens with (time, height, width) positions, q / k / v views of one projection
        _rotary("rotary-fwd-tuning-batch", "fwd", 4928, (32, 8), 128, axes=3, fused=True),
        # four high-resolution samples at the 13B shape in training
        _rotary("rotary-bwd-documents", "bwd", 4 * 2344, (40, 40), 128),
        # vision tower in 32 bits: 8 images with (height, width) positions, no norm
        _rotary("rotary-fwd-tower-fp32", "fwd", 4616, (16, 16), 64, axes=2, norm=False, dtype="fp32"),
        # one conversation, one token: latency
        _cached("attention", "attention-one-token", (1,), (657,), (32, 8), 128, 16),
        # the next token of 48 conversations
        _cached("attention", "attention-decode-batch", (1,) * 48, BATCH, (32, 8), 128, 16),
        # the next token of one very long context
        _cached("attention", "attention-decode-long", (1,), (130001,), (32, 8), 128, 64),
        # prompt chunks that share the pass with conversations being answered
        _cached("attention", "attention-mixed-chunks", (2000, 500) + (1,) * 30, (14345, 500) + BATCH[:30], (32, 8), 128, 32),
        # weights that one token of each conversation gives to the rows of its cache
        _cached("weights", "weights-decode-batch", (1,) * 48, BATCH, (32, 8), 128, 16),
        # the last tokens of a prompt as observers of all of it, every head with its own keys
        _cached("weights", "weights-observers", (64, 64, 33), (6100, 2984, 16381), (40, 40), 128, 64),
        # one prompt cut down to 2048 rows per head before it is answered
        _evict("evict-one-prompt", (16381,), 8, 128, 64, 2048, 4, 256),
        # a batch cut down together; some are short enough to keep all
        _evict("evict-batch", BATCH, 8, 128, 16, 1024, 4, 128),
    ]


def _log(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: single tokens to long chunks, one conversation to dozens, caches from one row (now and then
    none) to a hundred thousand, shared heads of many group sizes, both types, pages of many sizes."""
    dtype = rng.choice(("bf16",) * 4 + ("fp32",))
    heads = rng.choice(((32, 8), (40, 40), (16, 16), (8, 1), (28, 4), (12, 4), (64, 8), (10, 2), (1, 1)))
    head_dim = rng.choice((128, 128, 64, 64, 96, 80, 40))
    page = rng.choice((16, 16, 32, 64, 128, 24, 256))
    op = rng.choice(("rotary", "rotary", "attention", "attention", "attention", "weights", "evict"))
    if op == "rotary":
        tokens, axes = _log(rng, 1, 20000), rng.choice((1, 1, 2, 3))
        direction, norm, interleaved, fused = rng.choice(("fwd", "bwd", "append")), rng.random() < 0.7, rng.random() < 0.25, rng.random() < 0.4
        case = _rotary(None, direction, tokens, heads, head_dim, axes, norm, interleaved, dtype, fused, page)
        while work(case)["bytes"] > 400e6:
            case["tokens"] //= 2
        return case
    count = _log(rng, 1, 64)
    lens = [_log(rng, 1, 100000 if count < 3 else 9000) for _ in range(count)]
    if op == "evict":
        budget = _log(rng, 16, 4096)
        sinks, recent = rng.choice((0, 4, budget // 16)), rng.choice((0, 1, budget // 8, budget // 4))
        make = lambda: _evict(None, lens, heads[1], head_dim, page, budget, sinks, recent, dtype)
        new = [0] * count
    else:
        kind = rng.choice(("decode", "decode", "few", "chunks")) if op == "attention" else rng.choice(("decode", "few"))
        most = {"decode": 1, "few": 8 if op == "attention" else 48, "chunks": 2000}[kind]
        new = [min(n, _log(rng, 1, most)) for n in lens]
        if count > 1 and rng.random() < 0.2:            # nothing new in one conversation, nothing at all in another
            new[0] = new[1] = lens[1] = 0
        if not sum(new):
            new[-1] = lens[-1] = 1
        make = lambda: _cached(op, None, new, lens, heads, head_dim, page, dtype)
    row = heads[1] * head_dim * (4 if dtype == "bf16" else 8)     # bytes of a row of k and v
    flops = 2e11 if dtype == "bf16" else 1e10
    while sum(lens) * row > 500e6 or work(make())["bytes"] > 400e6 or work(make())["flops"] > flops:
        if len(lens) > 1 and (op == "evict" or sum(new[:-1])):
            lens.pop()
            new.pop()
        else:                                           # the one that is left, or the only one with new tokens
            lens[-1] = max(1, lens[-1] // 2)
            new[-1] = min(new[-1], lens[-1])
            lens[:-1] = [n // 2 for n in lens[:-1]]
    return make()


# ------------------------------------------------------------------ inputs
def _ints(text):
    return [int(n) for n in text.split()]


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _sections(case):
    """Frequency pairs of each axis: contiguous sections, the first one the smaller."""
    pairs, axes = case["head_dim"] // 2, case["axes"]
    if axes == 1:
        return [pairs]
    if axes == 2:
        return [pairs // 2, pairs - pairs // 2]
    return [pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8]


def _frequencies(case):
    """Frequency of each pair (64 bits) and its axis: one ladder over all sections, with two axes one ladder each."""
    pairs = case["head_dim"] // 2
    axis = [a for a, n in enumerate(_sections(case)) for _ in range(n)]
    if case["axes"] == 2:
        freq = [100.0 ** (-j / n) for n in _sections(case) for j in range(n)]
    else:
        freq = [10000.0 ** (-j / pairs) for j in range(pairs)]
    return freq, axis


def _pages(lens, page, g):
    """(table [sequences, width], pages): pages handed out in random order, some of them never used."""
    need = [max(1, -(-n // page)) for n in lens]
    total = sum(need) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(lens), max(need), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, total


def _normal(g, dt, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dt)


def _inputs(case, seed):
    """The case's tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _dtype(case)
    hq, hk, d, page = case["heads_q"], case["heads_kv"], case["head_dim"], case["page"]
    if case["op"] == "rotary":
        n = case["tokens"]
        # projections have a few strong columns
        q, k, v = (_normal(g, torch.float32, n, h, d) * (1.0 + 4.0 * (torch.rand(d, generator=g, device="cuda") > 0.97)) for h in (hq, hk, hk))
        q, k, v = q.to(dt), k.to(dt), v.to(dt)
        if case["fused"]:                               # one projection's output: [n, (hq + 2 hk) d]
            q, k, v = torch.cat((q, k, v), dim=1).split((hq, hk, hk), dim=1)
        far = 24 if case["axes"] == 2 else (120000 if case["direction"] == "append" else 32000)
        pos = torch.randint(0, far, (case["axes"], n), generator=g, device="cuda", dtype=torch.int32)
        s = {"q": q, "k": k, "v": v, "positions": pos, "gamma_q": None, "gamma_k": None}
        if case["norm"]:
            s["gamma_q"], s["gamma_k"] = ((1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2))
        if case["direction"] == "bwd":
            s["dq"], s["dk"] = _normal(g, dt, n, hq, d, std=0.1), _normal(g, dt, n, hk, d, std=0.1)
        if case["direction"] == "append":               # one new row for each of n conversations
            s["lens_list"] = [1 + 89 * i % 400 for i in range(n)]
            s["new_list"] = [1] * n
            s["table"], pages = _pages(s["lens_list"], page, g)
            s["k_pages"], s["v_pages"] = (_normal(g, dt, pages, page, hk, d) for _ in range(2))
        return s
    lens = _ints(case["lens"])
    table, pages = _pages(lens, page, g)
    s = {"lens_list": lens, "table": table, "k_pages": _normal(g, dt, pages, page, hk, d), "v_pages": _normal(g, dt, pages, page, hk, d)}
    if case["op"] == "evict":
        width = max(lens)
        # softmax weights summed over many queries: a few rows gather most, many hardly any, some none
        w = torch.exp(2.0 * torch.randn(len(lens), hk, width, generator=g, device="cuda"))
        s["weights"] = torch.where(torch.rand(len(lens), hk, width, generator=g, device="cuda") < 0.05, torch.zeros_like(w), w)
        budget = case["budget"]
        s["dst_table"], pages = _pages([min(n, budget) for n in lens], page, g)
        s["k_dst"], s["v_dst"] = (torch.zeros(pages, page, hk, d, dtype=dt, device="cuda") for _ in range(2))
        s["new_list"] = [0] * len(lens)
        return s
    s["new_list"] = _ints(case["new"])
    n = sum(s["new_list"])
    s["q"] = _normal(g, dt, n, hq, d, std=1.5)
    if case["op"] == "weights":
        s["prior"] = torch.rand(len(lens), hk, max(lens), generator=g, device="cuda")
        s["lse"] = torch.empty(n, hq, device="cuda")    # an input of this operator: the attention's own result
        at = 0
        for i, (m, length) in enumerate(zip(s["new_list"], lens)):
            for a in range(0, m, 16):
                b = min(m, a + 16)
                z = _scores(s["q"][at + a:at + b], _gather(s["k_pages"], table[i], length).float(), length - m + a)
                s["lse"][at + a:at + b] = torch.logsumexp(z, -1).permute(2, 0, 1).reshape(b - a, hq)
            at += m
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["op"] == "rotary":
        freq, axis = _frequencies(case)
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        s["axis"] = torch.tensor(axis, device="cuda")
    if "table" in s:
        new, lens = s["new_list"], s["lens_list"]
        s["cu"] = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if own:
        import paper_2503_21817_b200 as sk
        if case["op"] == "rotary":
            s["rotary"] = sk.RotaryQK(case["heads_q"], case["heads_kv"], case["head_dim"], sections=_sections(case),
                                      inv_freq=freq, interleaved=case["interleaved"], eps=EPS)
        if "table" in s:
            s["cache"] = sk.PagedCache(s["k_pages"], s["v_pages"], s["table"], s["cu"], s["lens"], max(s["new_list"]))
        if case["op"] == "evict":
            s["into"] = sk.PagedCache(s["k_dst"], s["v_dst"], s["dst_table"], s["cu"], s["lens"], 0)
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if case["op"] == "rotary":
        norms = (state["gamma_q"], state["gamma_k"])
        if own:
            rotary = state["rotary"]
            if case["direction"] == "fwd":
                return rotary.forward(state["q"], state["k"], state["positions"], *norms)
            if case["direction"] == "bwd":
                return rotary.backward(state["dq"], state["dk"], state["q"], state["k"], state["positions"], *norms)
            q = rotary.append(state["cache"], state["q"], state["k"], state["v"], state["positions"], *norms)
            return q, state["k_pages"], state["v_pages"]
        return _plain_rotary(state, case, *norms)
    if case["op"] == "attention":
        if own:
            return state["cache"].attention(state["q"])
        return _plain_attention(state)
    if case["op"] == "weights":
        if own:
            return state["cache"].weights(state["q"], state["lse"], prior=state["prior"])
        return _plain_weights(state)
    if own:
        kept, lens, weights = state["cache"].evict(state["weights"], case["budget"], sinks=case["sinks"], recent=case["recent"],
                                                   into=state["into"])
        return kept, lens, weights, state["k_dst"], state["v_dst"]
    return _plain_evict(state, case)


def _halves(x, interleaved):
    if interleaved:
        return x[..., 0::2], x[..., 1::2]
    return x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:]


def _joined(a, b, interleaved):
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def _plain_rotary(state, case, gamma_q, gamma_k):
    inter, dt, d = case["interleaved"], state["q"].dtype, case["head_dim"]
    angle = state["positions"][state["axis"]].t().double() * state["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def forward(x, gamma):
        x = x.float()
        if gamma is not None:
            x = x * (1.0 / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)) * gamma.float()
        a, b = _halves(x, inter)
        return _joined(a * cos - b * sin, b * cos + a * sin, inter).to(dt)

    def backward(dy, x, gamma):
        a, b = _halves(dy.float(), inter)
        dn = _joined(a * cos + b * sin, b * cos - a * sin, inter)
        if gamma is None:
            return dn.to(dt), None
        x = x.float()
        r = 1.0 / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
        dgamma = (dn * (x * r)).sum((0, 1)).to(dt)
        u = dn * gamma.float()
        return (r * (u - x * (r * r * ((u * x).sum(-1, keepdim=True) / d)))).to(dt), dgamma

    if case["direction"] == "fwd":
        return forward(state["q"], gamma_q), forward(state["k"], gamma_k)
    if case["direction"] == "bwd":
        dq, dgq = backward(state["dq"], state["q"], gamma_q)
        dk, dgk = backward(state["dk"], state["k"], gamma_k)
        return dq, dk, dgq, dgk
    q, k = forward(state["q"], gamma_q), forward(state["k"], gamma_k)
    last = state["lens"].long() - 1                     # one new row per sequence: its last
    page = state["table"].gather(1, (last // case["page"])[:, None])[:, 0].long()
    state["k_pages"][page, last % case["page"]] = k
    state["v_pages"][page, last % case["page"]] = state["v"]
    return q, state["k_pages"], state["v_pages"]


def _gather(pages, row, length):
    """Rows 0 .. length - 1 of one sequence: [length, heads, d]."""
    page = pages.shape[1]
    return pages[row[:-(-length // page)].long()].flatten(0, 1)[:length]


def _scores(q, k, first):
    """Scaled scores [heads_kv, group, rows, length] in 32 bits; query i sees keys up to first + i."""
    n, hq, d = q.shape
    hk = k.shape[1]
    qf = q.float().reshape(n, hk, hq // hk, d).permute(1, 2, 0, 3).reshape(hk, -1, d)
    s = ((qf @ k.permute(1, 2, 0)) * (1.0 / math.sqrt(d))).view(hk, hq // hk, n, k.shape[0])
    if first < k.shape[0] - 1:
        late = torch.arange(k.shape[0], device=q.device)[None, :] > torch.arange(first, first + n, device=q.device)[:, None]
        s.masked_fill_(late, -math.inf)
    return s


def _steps(state):
    """(sequence, its new tokens, its length, first row of q, first token, end token) of steps whose scores fit in memory."""
    at, hq = 0, state["q"].shape[1]
    for i, (m, length) in enumerate(zip(state["new_list"], state["lens_list"])):
        rows = max(1, SCORES // max(1, hq * length))
        for a in range(0, m, rows):
            yield i, m, length, at, a, min(m, a + rows)
        at += m


def _plain_attention(state):
    q = state["q"]
    n, hq, d = q.shape
    hk = state["k_pages"].shape[2]
    out, lse = torch.empty_like(q), torch.empty(n, hq, device=q.device)
    for i, m, length, at, a, b in _steps(state):
        k, v = (_gather(state[p], state["table"][i], length).float() for p in ("k_pages", "v_pages"))
        s = _scores(q[at + a:at + b], k, length - m + a)
        top = s.amax(-1, keepdim=True)
        p = s.sub_(top).exp_()
        den = p.sum(-1, keepdim=True)
        o = (p.view(hk, -1, length) @ v.transpose(0, 1)).view(hk, hq // hk, b - a, d) / den
        out[at + a:at + b] = o.permute(2, 0, 1, 3).reshape(b - a, hq, d).to(q.dtype)
        lse[at + a:at + b] = (top + den.log()).squeeze(-1).permute(2, 0, 1).reshape(b - a, hq)
    return out, lse


def _plain_weights(state):
    q, prior = state["q"], state["prior"]
    hk = prior.shape[1]
    w = torch.zeros_like(prior)
    for i, length in enumerate(state["lens_list"]):
        w[i, :, :length] = prior[i, :, :length]
    for i, m, length, at, a, b in _steps(state):
        s = _scores(q[at + a:at + b], _gather(state["k_pages"], state["table"][i], length).float(), length - m + a)
        l = state["lse"][at + a:at + b].view(b - a, hk, -1).permute(1, 2, 0).unsqueeze(-1)
        w[i, :, :length] += s.sub_(l).exp_().sum((1, 2))
    return w


def _plain_evict(state, case):
    w, budget, sinks, recent = state["weights"], case["budget"], case["sinks"], case["recent"]
    n, hk, _ = w.shape
    page = state["k_dst"].shape[1]
    kept = torch.full((n, hk, budget), -1, dtype=torch.int32, device=w.device)
    new_w = torch.zeros(n, hk, budget, device=w.device)
    for i, length in enumerate(state["lens_list"]):
        m = min(length, budget)
        if length > budget:
            key = w[i, :, :length].clone()
            key[:, :sinks] = math.inf
            key[:, length - recent:] = math.inf
            rows = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :budget].sort(dim=1).values
        else:
            rows = torch.arange(length, device=w.device).expand(hk, length)
        kept[i, :, :m] = rows
        new_w[i, :, :m] = w[i].gather(1, rows)
        to = torch.arange(m, device=w.device)
        to_page, to_row = state["dst_table"][i, to // page].long()[None], (to % page)[None]
        head = torch.arange(hk, device=w.device)[:, None]
        src_page, src_row = state["table"][i][rows // page].long(), rows % page
        for src, dst in (("k_pages", "k_dst"), ("v_pages", "v_dst")):
            state[dst][to_page, to_row, head] = state[src][src_page, src_row, head]
    return kept, state["lens"].clamp(max=budget), new_w, state["k_dst"], state["v_dst"]


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(case, s)
    if case["op"] == "evict":
        return _exact_evict(case, s)
    hq, hk, d, page = case["heads_q"], case["heads_kv"], case["head_dim"], case["page"]
    group, n = hq // hk, s["q"].shape[0]
    out = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(n, hq, dtype=torch.float64, device="cuda")
    gathered = torch.zeros(len(s["lens_list"]), hk, max(s["lens_list"]), dtype=torch.float64, device="cuda")
    at = 0
    for i, (m, length) in enumerate(zip(s["new_list"], s["lens_list"])):
        row = torch.arange(length, device="cuda")
        where, inside = s["table"][i].long()[row // page], row % page
        if case["op"] == "weights":
            gathered[i, :, :length] = s["prior"][i, :, :length].double()
        for h in range(hk if m else 0):
            k = s["k_pages"][where, inside, h].double()
            v = s["v_pages"][where, inside, h].double() if case["op"] == "attention" else None
            for a in range(0, m, 1024):
                b = min(m, a + 1024)
                q = s["q"][at + a:at + b, h * group:(h + 1) * group].double()
                z = torch.einsum("igd,jd->igj", q, k) / d ** 0.5
                sees = row[None, :] <= torch.arange(length - m + a, length - m + b, device="cuda")[:, None]
                z = torch.where(sees[:, None, :], z, torch.full_like(z, -math.inf))
                if case["op"] == "weights":
                    given = s["lse"][at + a:at + b, h * group:(h + 1) * group].double()
                    gathered[i, h, :length] += torch.exp(z - given.unsqueeze(-1)).sum((0, 1))
                else:
                    out[at + a:at + b, h * group:(h + 1) * group] = torch.softmax(z, -1) @ v
                    lse[at + a:at + b, h * group:(h + 1) * group] = torch.logsumexp(z, -1)
        at += m
    return gathered if case["op"] == "weights" else (out, lse)


def _exact_rotary(case, s):
    """The rotation as multiplication by a complex number of modulus one; gradients by differentiation."""
    freq, axis = _frequencies(case)
    angle = torch.stack([s["positions"][a].double() * f for f, a in zip(freq, axis)], dim=1)
    turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
    pairs = case["head_dim"] // 2

    def rotated(x, gamma):
        if gamma is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gamma
        if case["interleaved"]:
            z = torch.view_as_complex(x.unflatten(-1, (pairs, 2)).contiguous()) * turn
            return torch.view_as_real(z).flatten(-2)
        z = torch.complex(x[..., :pairs].contiguous(), x[..., pairs:].contiguous()) * turn
        return torch.cat((z.real, z.imag), dim=-1)

    bwd = case["direction"] == "bwd"
    q, k, gq, gk = (None if s[i] is None else s[i].double().requires_grad_(bwd) for i in ("q", "k", "gamma_q", "gamma_k"))
    if bwd:
        if gq is None:
            dq, = torch.autograd.grad(rotated(q, gq), (q,), s["dq"].double())
            dk, = torch.autograd.grad(rotated(k, gk), (k,), s["dk"].double())
            return dq, dk, None, None
        dq, dgq = torch.autograd.grad(rotated(q, gq), (q, gq), s["dq"].double())
        dk, dgk = torch.autograd.grad(rotated(k, gk), (k, gk), s["dk"].double())
        return dq, dk, dgq, dgk
    q, k = rotated(q, gq), rotated(k, gk)
    if case["direction"] == "fwd":
        return q, k
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    for i, length in enumerate(s["lens_list"]):
        page = int(s["table"][i, (length - 1) // case["page"]])
        kp[page, (length - 1) % case["page"]] = k[i]
        vp[page, (length - 1) % case["page"]] = s["v"][i].double()
    return q, kp, vp


def _exact_evict(case, s):
    """Row by row on the host: sorted by (protected, weight, lower row)."""
    import numpy as np
    budget, sinks, recent, page = case["budget"], case["sinks"], case["recent"], case["page"]
    w = s["weights"].cpu().numpy()
    n, hk, _ = w.shape
    kept = np.full((n, hk, budget), -1, dtype=np.int32)
    new_w = np.zeros((n, hk, budget))
    table, dst = s["table"].cpu().numpy(), s["dst_table"].cpu().numpy()
    pools = [(s["k_pages"], s["k_dst"]), (s["v_pages"], s["v_dst"])]
    moved = [b.double() for _, b in pools]
    for i, length in enumerate(s["lens_list"]):
        row = np.arange(length)
        safe = (row < sinks) | (row >= length - recent)
        for h in range(hk):
            rows = np.sort(np.lexsort((row, -w[i, h, :length].astype(np.float64), ~safe))[:budget])
            kept[i, h, :rows.size] = rows
            new_w[i, h, :rows.size] = w[i, h, rows]
            to = np.arange(rows.size)
            a, b = (torch.from_numpy(t[i][r // page].astype(np.int64)).cuda() for t, r in ((table, rows), (dst, to)))
            ra, rb = (torch.from_numpy(r % page).cuda() for r in (rows, to))
            for (src, _), res in zip(pools, moved):
                res[b, rb, h] = src[a, ra, h].double()
    lens = torch.tensor([min(m, budget) for m in s["lens_list"]], dtype=torch.int32, device="cuda")
    return torch.from_numpy(kept).cuda(), lens, torch.from_numpy(new_w).cuda(), *moved


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    hq, hk, d = case["heads_q"], case["heads_kv"], case["head_dim"]
    if case["op"] == "rotary":
        n = case["tokens"]
        x = n * (hq + hk) * d
        small = 4 * case["axes"] * n + 2 * d * b * case["norm"]
        if case["direction"] == "fwd":                  # q, k -> q', k'
            return {"bytes": 2 * x * b + small, "flops": 9 * x}
        if case["direction"] == "bwd":                  # dq', dk', q, k -> dq, dk, dgamma (without a norm q, k are not needed)
            return {"bytes": (3 if case["norm"] else 2) * x * b + 2 * small, "flops": 16 * x}
        return {"bytes": 2 * (x + n * hk * d) * b + small + 12 * n, "flops": 9 * x}
    lens = _ints(case["lens"])
    rows = sum(lens) * hk
    if case["op"] == "evict":                           # weights; the kept rows of k and v read and written; kept, weights
        m = sum(min(n, case["budget"]) for n in lens) * hk
        cut = sum(n for n in lens if n > case["budget"]) * hk
        return {"bytes": 4 * (cut + m) + 4 * m * d * b + 8 * len(lens) * hk * case["budget"], "flops": 4 * cut}
    new = _ints(case["new"])
    live = sum(n for m, n in zip(new, lens) if m) * hk
    pairs = sum(m * n - m * (m - 1) // 2 for m, n in zip(new, lens))
    if case["op"] == "weights":                         # q, lse, k, prior -> weights
        return {"bytes": sum(new) * hq * (d * b + 4) + live * d * b + 4 * rows + 4 * len(lens) * hk * max(lens), "flops": (2 * d + 2) * hq * pairs}
    return {"bytes": sum(new) * hq * (2 * d * b + 4) + 2 * live * d * b, "flops": 4 * hq * d * pairs}
