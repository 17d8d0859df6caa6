"""Cases of the operators around the Skip-FFN sublayer: packed attention and layer normalisation.

`listed()` names the cases, `draw(rng)` gives more of the same ranges, `prepare(case, seed)` makes
what a program has in hand before the call, `run(state)` is one pass.  With `own` false a pass is
written in elementary torch operations in 32 bits, rounded once at the end; with `own` true it makes
the calls a user makes of this package.  `exact(case, seed)` states the same results in 64 bits.

Operators
  attention   softmax(scale * Q K^T) V inside each sequence of a packed batch, causal (decoder) or
              bidirectional (vision tower), `heads_q` query heads sharing `heads_kv` key / value
              heads; forward returns (out, lse), backward (dq, dk, dv)
  layernorm   (x - mean) / sqrt(var + eps) * gamma + beta per row; forward returns (y, mean, rstd),
              backward (dx, dgamma, dbeta)
"""
import math

import torch

own = False

EPS = 1e-5
SCORES = 1 << 28        # scores of one step of the plain form


# ------------------------------------------------------------------ cases
def _attention(name, direction, lens, heads, head_dim, causal=True, dtype="bf16", fused=False):
    c = {"op": "attention", "direction": direction, "lens": " ".join(str(n) for n in lens), "heads_q": heads[0],
         "heads_kv": heads[1], "head_dim": head_dim, "causal": causal, "dtype": dtype, "fused": fused}
    return dict(c, name=name) if name else c


def _layernorm(name, direction, rows, cols, dtype="bf16"):
    c = {"op": "layernorm", "direction": direction, "rows": rows, "cols": cols, "dtype": dtype}
    return dict(c, name=name) if name else c


# text + visual tokens of a packed batch of documents with 4 to 20 tiles of 144 visual tokens each
RAGGED = (1208, 2953, 719, 1501, 2117, 640, 2390, 1847, 1093, 2702, 883, 1366, 1986, 2518, 601, 1660)


def listed():
    return [
        # one question of 40 text tokens through the decoder: a call's latency
        _attention("fwd-one-question", "fwd", (40,), (32, 8), 128),
        # the fine-tuning batch: 8 x (576 visual + 40 text) tokens, 8B-shaped decoder
        _attention("fwd-tuning-batch", "fwd", (616,) * 8, (32, 8), 128),
        # packed documents of different lengths, 13B-shaped decoder (every head its own keys), q / k / v as
        # views of one fused projection
        _attention("fwd-packed-documents", "fwd", RAGGED, (40, 40), 128, fused=True),
        # one long interleaved prompt
        _attention("fwd-long-prompt", "fwd", (16381,), (32, 8), 128),
        # vision tower: 8 images of 24 x 24 patches and a class token, bidirectional
        _attention("fwd-vision-tower", "fwd", (577,) * 8, (16, 16), 64, causal=False),
        # the training step of the same layers
        _attention("bwd-tuning-batch", "bwd", (616,) * 8, (32, 8), 128),
        _attention("bwd-packed-documents", "bwd", RAGGED, (32, 8), 128, fused=True),
        _attention("bwd-vision-tower", "bwd", (577,) * 8, (16, 16), 64, causal=False),
        # a check run in 32 bits: three short sequences, one of them a single token
        _attention("bwd-fp32-check", "bwd", (33, 1, 200), (8, 2), 64, dtype="fp32"),
        # normalisation of one image's patches in the tower
        _layernorm("norm-fwd-one-image", "fwd", 577, 1024),
        # four high-resolution samples at the decoder's width
        _layernorm("norm-fwd-batch", "fwd", 4 * 2344, 4096),
        # its training step at the 13B width, an odd number of rows
        _layernorm("norm-bwd-batch", "bwd", 4927, 5120),
    ]


def _log(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: lengths from one token (now and then none) to thousands, packed batches, shared
    heads of many group sizes, head sizes up to 128, both directions and types."""
    if rng.random() < 0.35:
        rows = _log(rng, 1, 20000)
        cols = 8 * _log(rng, 4, 1024)
        while rows * cols > 48 << 20:
            rows = max(1, rows // 2)
        return _layernorm(None, rng.choice(("fwd", "bwd")), rows, cols, rng.choice(("bf16", "bf16", "fp32")))
    direction = rng.choice(("fwd", "bwd"))
    dtype = rng.choice(("bf16",) * 4 + ("fp32",))
    heads = rng.choice(((32, 8), (40, 40), (16, 16), (8, 1), (28, 4), (12, 4), (64, 8), (10, 2), (1, 1)))
    head_dim = rng.choice((128, 128, 64, 64, 96, 80, 40, 32))
    most = 600 if dtype == "fp32" else (6000 if direction == "fwd" else 4000)
    lens = [_log(rng, 1, most) for _ in range(_log(rng, 1, 16))]
    if rng.random() < 0.2:
        lens[rng.randrange(len(lens))] = 0
    if not sum(lens):
        lens[0] = 1
    while sum(lens) > 24000:
        lens.pop()
    return _attention(None, direction, lens, heads, head_dim, causal=rng.random() < 0.7, dtype=dtype, fused=rng.random() < 0.4)


# ------------------------------------------------------------------ inputs
def _lens(case):
    return [int(n) for n in case["lens"].split()]


def _offsets(case):
    cu = [0]
    for n in _lens(case):
        cu.append(cu[-1] + n)
    return cu


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    """The case's tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _dtype(case)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    if case["op"] == "layernorm":
        n, c = case["rows"], case["cols"]
        # activations of a residual stream: a few strong channels, rows of different size and offset
        x = normal(n, c) * (1.0 + 8.0 * (torch.rand(c, generator=g, device="cuda") > 0.98)) * (0.3 + normal(n, 1).abs())
        x = x + normal(c, std=0.5) + normal(n, 1, std=2.0)
        return {"x": x.to(dt), "gamma": (1.0 + normal(c, std=0.2)).to(dt), "beta": normal(c, std=0.2).to(dt),
                "dy": normal(n, c, std=0.1).to(dt) if case["direction"] == "bwd" else None}
    n, hq, hk, d = sum(_lens(case)), case["heads_q"], case["heads_kv"], case["head_dim"]
    q, k, v = normal(n, hq, d, std=1.5).to(dt), normal(n, hk, d).to(dt), normal(n, hk, d).to(dt)
    if case["fused"]:                                   # one projection's output: [n, (hq + 2 hk) d]
        q, k, v = torch.cat((q, k, v), dim=1).split((hq, hk, hk), dim=1)
    return {"q": q, "k": k, "v": v, "dout": normal(n, hq, d, std=0.1).to(dt) if case["direction"] == "bwd" else None}


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["op"] == "layernorm":
        if case["direction"] == "bwd":
            _, s["mean"], s["rstd"] = _plain_layernorm(s["x"], s["gamma"], s["beta"])
        return s
    s["cu"] = _offsets(case)
    if case["direction"] == "bwd":
        s["out"], s["lse"] = _plain_attention(s["q"], s["k"], s["v"], s["cu"], case["causal"])
    if own:
        import paper_2503_21817_b200 as sk
        s["attention"] = sk.PackedAttention(s["cu"], case["heads_q"], case["heads_kv"], case["head_dim"],
                                            dtype=sk.BF16 if case["dtype"] == "bf16" else sk.FP32, causal=case["causal"])
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if case["op"] == "layernorm":
        if case["direction"] == "fwd":
            a = (state["x"], state["gamma"], state["beta"])
            if own:
                import paper_2503_21817_b200 as sk
                return sk.layernorm_forward(*a, eps=EPS)
            return _plain_layernorm(*a)
        a = (state["dy"], state["x"], state["gamma"], state["mean"], state["rstd"])
        if own:
            import paper_2503_21817_b200 as sk
            return sk.layernorm_backward(*a)
        return _plain_layernorm_backward(*a)
    a = (state["q"], state["k"], state["v"])
    if case["direction"] == "fwd":
        if own:
            return state["attention"].forward(*a)
        return _plain_attention(*a, state["cu"], case["causal"])
    if own:
        return state["attention"].backward(state["dout"], *a, state["out"], state["lse"])
    return _plain_attention_backward(state["dout"], *a, state["lse"], state["cu"], case["causal"])


def _plain_layernorm(x, gamma, beta):
    xf = x.float()
    mean = xf.sum(1) / x.shape[1]
    z = xf - mean[:, None]
    rstd = 1.0 / torch.sqrt((z * z).sum(1) / x.shape[1] + EPS)
    return (z * rstd[:, None] * gamma.float() + beta.float()).to(x.dtype), mean, rstd


def _plain_layernorm_backward(dy, x, gamma, mean, rstd):
    dyf, n = dy.float(), x.shape[1]
    xh = (x.float() - mean[:, None]) * rstd[:, None]
    t = dyf * gamma.float()
    dx = rstd[:, None] * (t - t.sum(1, keepdim=True) / n - xh * ((t * xh).sum(1, keepdim=True) / n))
    return dx.to(x.dtype), (dyf * xh).sum(0).to(x.dtype), dyf.sum(0).to(x.dtype)


def _steps(cu, heads_q):
    """(first token, end, first query, end query) of steps whose scores fit in memory."""
    for lo, hi in zip(cu, cu[1:]):
        rows = max(1, SCORES // max(1, heads_q * (hi - lo)))
        for a in range(lo, hi, rows):
            yield lo, hi, a, min(hi, a + rows)


def _rows(t, heads_kv):
    """[rows, heads, d] -> [heads_kv, group * rows, d] in 32 bits, the heads of a group one after the other."""
    n, h, d = t.shape
    return t.float().reshape(n, heads_kv, h // heads_kv, d).permute(1, 2, 0, 3).reshape(heads_kv, -1, d)


def _back(t, n):
    """The inverse of _rows: [heads_kv, group * n, d] -> [n, heads, d]."""
    h, d = t.shape[0], t.shape[2]
    return t.reshape(h, -1, n, d).permute(2, 0, 1, 3).reshape(n, -1, d)


def _plain_scores(q, k, lo, hi, a, b, causal):
    """Scaled scores [heads_kv, group, b - a, hi - lo], minus infinity where a key comes after its query."""
    hk = k.shape[1]
    s = (_rows(q[a:b], hk) @ k[lo:hi].float().permute(1, 2, 0)) * (1.0 / math.sqrt(q.shape[2]))
    s = s.view(hk, -1, b - a, hi - lo)
    if causal:
        late = torch.arange(lo, hi, device=q.device)[None, :] > torch.arange(a, b, device=q.device)[:, None]
        s.masked_fill_(late, -math.inf)
    return s


def _plain_attention(q, k, v, cu, causal):
    n, hq, d = q.shape
    out = torch.empty(n, hq, d, dtype=q.dtype, device=q.device)
    lse = torch.empty(n, hq, dtype=torch.float32, device=q.device)
    for lo, hi, a, b in _steps(cu, hq):
        s = _plain_scores(q, k, lo, hi, a, b, causal)
        top = s.amax(-1, keepdim=True)
        p = s.sub_(top).exp_()
        den = p.sum(-1, keepdim=True)
        o = (p.view(p.shape[0], -1, hi - lo) @ v[lo:hi].float().transpose(0, 1)) / den.reshape(p.shape[0], -1, 1)
        out[a:b] = _back(o, b - a).to(q.dtype)
        lse[a:b] = (top + den.log()).squeeze(-1).permute(2, 0, 1).reshape(b - a, hq)
    return out, lse


def _plain_attention_backward(dout, q, k, v, lse, cu, causal):
    n, hq, d = q.shape
    hk, scale = k.shape[1], 1.0 / math.sqrt(d)
    dq = torch.empty(n, hq, d, dtype=q.dtype, device=q.device)
    dk = torch.zeros(hk, n, d, device=q.device)
    dv = torch.zeros(hk, n, d, device=q.device)
    for lo, hi, a, b in _steps(cu, hq):
        p = _plain_scores(q, k, lo, hi, a, b, causal)
        p = p.sub_(lse[a:b].view(b - a, hk, -1).permute(1, 2, 0).unsqueeze(-1)).exp_().view(hk, -1, hi - lo)
        do, kf = _rows(dout[a:b], hk), k[lo:hi].float().transpose(0, 1)
        dv[:, lo:hi] += p.transpose(1, 2) @ do
        ds = do @ v[lo:hi].float().permute(1, 2, 0)
        ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * scale
        dq[a:b] = _back(ds @ kf, b - a).to(q.dtype)
        dk[:, lo:hi] += ds.transpose(1, 2) @ _rows(q[a:b], hk)
    return dq, dk.transpose(0, 1).to(q.dtype), dv.transpose(0, 1).to(q.dtype)


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    grad = case["direction"] == "bwd"
    if case["op"] == "layernorm":
        x, gamma, beta = (s[i].double().requires_grad_(grad) for i in ("x", "gamma", "beta"))
        var, mean = torch.var_mean(x, dim=1, unbiased=False)
        rstd = (var + EPS).rsqrt()
        y = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1) * gamma + beta
        return torch.autograd.grad(y, (x, gamma, beta), s["dy"].double()) if grad else (y, mean, rstd)
    n, hq, hk, d = sum(_lens(case)), case["heads_q"], case["heads_kv"], case["head_dim"]
    group = hq // hk
    res = {i: torch.empty_like(s[j], dtype=torch.float64, memory_format=torch.contiguous_format)
           for i, j in (("dq", "q"), ("dk", "k"), ("dv", "v"), ("out", "q"))}
    lse = torch.empty(n, hq, dtype=torch.float64, device="cuda")
    cu = _offsets(case)
    for lo, hi in zip(cu, cu[1:]):
        length = hi - lo
        for h in range(hk if length else 0):
            k, v = (s[i][lo:hi, h].double().requires_grad_(grad) for i in ("k", "v"))
            for j in range(h * group, (h + 1) * group):
                for a in range(0, length, 4096):
                    b = min(length, a + 4096)
                    q = s["q"][lo + a:lo + b, j].double().requires_grad_(grad)
                    z = torch.einsum("id,jd->ij", q, k) / d ** 0.5
                    if case["causal"]:
                        z = z + torch.full((b - a, length), -math.inf, dtype=z.dtype, device="cuda").triu(a + 1)
                    o = torch.softmax(z, dim=1) @ v
                    if not grad:
                        res["out"][lo + a:lo + b, j] = o
                        lse[lo + a:lo + b, j] = torch.logsumexp(z, dim=1)
                        continue
                    gq, gk, gv = torch.autograd.grad(o, (q, k, v), s["dout"][lo + a:lo + b, j].double())
                    res["dq"][lo + a:lo + b, j] = gq
                    first = j == h * group and a == 0
                    for i, t in (("dk", gk), ("dv", gv)):
                        res[i][lo:hi, h] = t if first else res[i][lo:hi, h] + t
    return (res["dq"], res["dk"], res["dv"]) if grad else (res["out"], lse)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "layernorm":
        n, c = case["rows"], case["cols"]
        if case["direction"] == "fwd":                  # x, gamma, beta -> y, mean, rstd
            return {"bytes": 2 * n * c * b + 2 * c * b + 8 * n, "flops": 7 * n * c}
        return {"bytes": 3 * n * c * b + 3 * c * b + 8 * n, "flops": 14 * n * c}
    n, hq, hk, d = sum(_lens(case)), case["heads_q"], case["heads_kv"], case["head_dim"]
    pairs = sum(m * (m + 1) // 2 if case["causal"] else m * m for m in _lens(case))
    if case["direction"] == "fwd":                      # q, k, v -> out, lse; two products
        return {"bytes": (2 * hq + 2 * hk) * n * d * b + 4 * n * hq, "flops": 4 * hq * d * pairs}
    # dout, q, k, v, out, lse -> dq, dk, dv; five products
    return {"bytes": (4 * hq + 4 * hk) * n * d * b + 4 * n * hq, "flops": 10 * hq * d * pairs}
