"""Performance cases of the operators that train and score a readout.

A readout (a square matrix and an offset in front of the model's own final norm and unembedding) is
fitted by distilling the full model's answers into it, and judged by the log probabilities it gives.
A program that does that calls, per batch of rows:

  kind      what a user does
  linear    `linear` (bias, activation and residual in the product's epilogue), and for training
            `linear_backward`
  norm      `rms_norm` and `rms_norm_backward`, the gain's gradient included
  logprobs  `token_logprobs`: log probabilities of given tokens, entropy, the k best alternatives
  distill   `distill_topk` and `distill_topk_backward`, or both in one call, `distill_topk_step`

`run` computes them in plain 32-bit torch operations, or with the package's operators where `own` is
true.  Shapes are the repository's workloads (0.5b, 1.5b, 3b, their vocabulary), and odd sizes.
"""
from __future__ import annotations

import math

import torch

own = False

VOCAB = 151936
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6


def listed():
    return [
        # one token through a wide projection of the 0.5B shape: the serving form, latency counts
        {"name": "linear_token", "kind": "linear", "rows": 1, "n_in": 896, "n_out": 4864, "type": "bf16", "out": "bf16",
         "act": "silu", "bias": True, "residual": False, "backward": "none", "pad": 0},
        # a ragged batch, odd widths, half precision, everything in the epilogue
        {"name": "linear_ragged", "kind": "linear", "rows": 37, "n_in": 1001, "n_out": 2051, "type": "fp16",
         "out": "fp16", "act": "gelu", "bias": True, "residual": True, "backward": "none", "pad": 3},
        # a readout's map and its gradients at the 1.5B width, the weight's in 32 bits for the optimiser
        {"name": "linear_train", "kind": "linear", "rows": 2048, "n_in": 1536, "n_out": 1536, "type": "bf16",
         "out": "bf16", "act": "none", "bias": True, "residual": True, "backward": "all", "pad": 0},
        # the frozen unembedding in training: logits, and the gradient to its input alone
        {"name": "linear_vocab", "kind": "linear", "rows": 1024, "n_in": 1536, "n_out": VOCAB, "type": "bf16",
         "out": "bf16", "act": "none", "bias": False, "residual": False, "backward": "dx", "pad": 0},
        # a handful of rows, 32-bit residuals normalised to bf16
        {"name": "norm_few", "kind": "norm", "rows": 5, "d": 896, "type": "fp32", "out": "bf16", "backward": True,
         "pad": 0},
        # a training batch at the 3B width
        {"name": "norm_train", "kind": "norm", "rows": 8192, "d": 2048, "type": "bf16", "out": "bf16", "backward": True,
         "pad": 0},
        # one decoded token's log probability and alternatives, as a server returns them
        {"name": "logprobs_token", "kind": "logprobs", "rows": 1, "vocab": VOCAB, "type": "fp32", "k": 20,
         "temperature": 1.0, "masked": 0, "pad": 0},
        # odd vocabulary with a padded row, banned tokens, a temperature
        {"name": "logprobs_odd", "kind": "logprobs", "rows": 333, "vocab": 50257, "type": "fp16", "k": 5,
         "temperature": 0.7, "masked": 300, "pad": 47},
        # scoring a stretch of text and keeping the teacher's alternatives for distillation
        {"name": "logprobs_corpus", "kind": "logprobs", "rows": 2048, "vocab": VOCAB, "type": "bf16", "k": 64,
         "temperature": 1.0, "masked": 271, "pad": 0},
        # a small model's few rows, the loss and then, apart, its gradient
        {"name": "distill_few", "kind": "distill", "rows": 7, "vocab": 4096, "type": "fp32", "k": 8, "temperature": 1.0,
         "tail": False, "mode": "split", "pad": 0},
        # odd vocabulary in half precision, the rest of the vocabulary as a bucket of its own
        {"name": "distill_odd", "kind": "distill", "rows": 515, "vocab": 50257, "type": "fp16", "k": 17,
         "temperature": 1.0, "tail": True, "mode": "split", "pad": 0},
        # a training batch over the whole vocabulary: loss and gradient in one call
        {"name": "distill_train", "kind": "distill", "rows": 4096, "vocab": VOCAB, "type": "bf16", "k": 64,
         "temperature": 2.0, "tail": True, "mode": "step", "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "norm", "logprobs", "logprobs", "distill", "distill"])
    if kind == "linear":
        rows = _log_int(rng, 1, 4096)
        n_in = rng.choice([256, 896, 1536, 2048, _log_int(rng, 65, 2500)])
        n_out = rng.choice([688, 1536, 4864, 8960, _log_int(rng, 65, 40000), _log_int(rng, 65, 40000)])
        kind16 = rng.choice(["bf16", "bf16", "fp16"])
        back = rng.choice(["none", "none", "dx", "all"])
        act = rng.choice(["none", "none", "relu", "silu", "gelu"])
        most = 1024 * 1536 * VOCAB // 2
        while rows * n_in * n_out > most:
            rows = max(1, rows // 2)
        return {"kind": kind, "rows": rows, "n_in": n_in, "n_out": n_out, "type": kind16,
                "out": rng.choice([kind16, kind16, "fp32"]) if back == "none" else kind16, "act": act,
                "bias": rng.random() < 0.6, "residual": rng.random() < 0.4, "backward": back,
                "pad": rng.choice([0, 0, 8, 5])}
    if kind == "norm":
        d = rng.choice([256, 896, 1536, 2048, _log_int(rng, 33, 8192)])
        kx = rng.choice(["bf16", "fp16", "fp32"])
        return {"kind": kind, "rows": min(_log_int(rng, 1, 16384), 8192 * 2048 * 2 // (d * BYTES[kx])), "d": d, "type": kx,
                "out": rng.choice([kx, "bf16" if kx == "fp32" else kx]), "backward": rng.random() < 0.7,
                "pad": rng.choice([0, 0, 8, 3])}
    kx = rng.choice(["bf16", "fp16", "fp32"])
    vocab = rng.choice([4096, 32000, 50257, VOCAB, _log_int(rng, 300, VOCAB)])
    most = (2048 if kind == "logprobs" else 4096) * VOCAB * 2
    rows = max(1, min(_log_int(rng, 1, 4096), most // (vocab * BYTES[kx])))
    if kind == "logprobs":
        return {"kind": kind, "rows": rows, "vocab": vocab, "type": kx, "k": rng.choice([0, 1, 5, 20, rng.randint(2, 64)]),
                "temperature": rng.choice([1.0, 1.0, 0.7, 1.5]), "masked": rng.choice([0, 0, vocab // 50]),
                "pad": rng.choice([0, 0, 64, 7])}
    return {"kind": kind, "rows": rows, "vocab": vocab, "type": kx, "k": rng.choice([1, 8, 64, rng.randint(2, 64)]),
            "temperature": rng.choice([1.0, 1.0, 2.0]), "tail": rng.random() < 0.5,
            "mode": rng.choice(["forward", "split", "step", "step"]), "pad": rng.choice([0, 0, 64, 7])}


# ------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, rows, cols, kind, std=1.0, pad=0):
    """rows x cols N(0, std^2), its rows `pad` elements further apart than they are long."""
    t = torch.randn((rows, cols + pad), generator=g, device="cuda", dtype=torch.float32).mul_(std).to(TYPES[kind])
    return t[:, :cols]


def prepare(case, seed):
    """What the program holds before the call: activations, frozen or trained weights, the teacher's lists."""
    c, g = case, _gen(seed)
    s = {"case": c}
    if c["kind"] == "linear":
        s["x"] = _normal(g, c["rows"], c["n_in"], c["type"], 1.0, c["pad"])
        s["w"] = _normal(g, c["n_out"], c["n_in"], c["type"], c["n_in"] ** -0.5)
        s["b"] = _normal(g, 1, c["n_out"], c["type"], 0.5)[0] if c["bias"] else None
        s["r"] = _normal(g, c["rows"], c["n_out"], c["out"], 1.0, c["pad"]) if c["residual"] else None
        if c["backward"] != "none":
            s["dy"] = _normal(g, c["rows"], c["n_out"], c["type"], 1.0, c["pad"])
    elif c["kind"] == "norm":
        s["x"] = _normal(g, c["rows"], c["d"], c["type"], 2.0, c["pad"])
        s["gain"] = _normal(g, 1, c["d"], "bf16", 0.3)[0].add_(1.0)
        if c["backward"]:
            s["dy"] = _normal(g, c["rows"], c["d"], c["out"], 1.0)
    elif c["kind"] == "logprobs":
        z = _normal(g, c["rows"], c["vocab"], c["type"], 3.0, c["pad"])
        if c["masked"]:  # the columns that pad the vocabulary, or banned tokens
            z[:, c["vocab"] - c["masked"]:] = float("-inf")
        s["logits"] = z
        s["ids"] = torch.randint(0, c["vocab"] - c["masked"], (c["rows"],), generator=g, device="cuda", dtype=torch.int32)
        s["ids"][3::11] = -1  # prompt and padding positions have no token to score
    else:
        z = _normal(g, c["rows"], c["vocab"], c["type"], 3.0, c["pad"])
        s["logits"] = z
        k = min(c["k"], c["vocab"])
        ids = torch.empty((c["rows"], k), dtype=torch.int32, device="cuda")
        lps = torch.empty((c["rows"], k), dtype=torch.float32, device="cuda")
        for r0 in range(0, c["rows"], 256):  # the teacher: related to the student, its best tokens kept
            zt = z[r0:r0 + 256].float()
            zt = (zt * 0.8 + torch.randn(zt.shape, generator=g, device="cuda") * 2.0) / c["temperature"]
            top, idx = zt.topk(k, dim=-1)
            lps[r0:r0 + 256] = top - torch.logsumexp(zt, -1, keepdim=True)
            ids[r0:r0 + 256] = idx.to(torch.int32)
        if k > 4:
            ids[1::5, k - 3:] = -1  # lists that were cut shorter
        s["ids"], s["teacher"] = ids, lps
        w = torch.ones(c["rows"], device="cuda")
        w[5::9] = 0.0  # rows outside the batch's text
        # a mean over the batch; half precision trains with a scaled loss
        s["weight"] = w * ((1024.0 if c["type"] == "fp16" else 1.0) / c["rows"])
    return s


# ------------------------------------------------------------------ one pass


def _act(u, kind):
    if kind == "relu":
        return u * (u > 0)
    if kind == "silu":
        return u / (1 + torch.exp(-u))
    if kind == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    return u


def _act_slope(u, kind):
    if kind == "relu":
        return (u > 0).to(u.dtype)
    if kind == "silu":
        g = 1 / (1 + torch.exp(-u))
        return g * (1 + u * (1 - g))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) * (2 * math.pi) ** -0.5
    return torch.ones_like(u)


def _plain_linear(s, c):
    x, w = s["x"].float(), s["w"].float()
    u = x @ w.t()
    if s["b"] is not None:
        u = u + s["b"].float()
    y = _act(u, c["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    out = [y.to(TYPES[c["out"]])]
    if c["backward"] != "none":
        du = s["dy"].float()
        if c["act"] != "none":
            du = du * _act_slope(u, c["act"])
        out.append((du @ w).to(s["x"].dtype))
        if c["backward"] == "all":
            out.append((du.t() @ x).to(_dw_type(c)))
            out.append(du.sum(0))
    return out


def _dw_type(c):
    """The weight's gradient comes in 32 bits, behind an activation in the operands' type."""
    return torch.float32 if c["act"] == "none" else TYPES[c["type"]]


def _plain_norm(s, c):
    x, g = s["x"].float(), s["gain"].float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    out = [(x * r * g).to(TYPES[c["out"]])]
    if c["backward"]:
        dy = s["dy"].float()
        gdy = dy * g
        out.append((r * (gdy - x * (r * r * (gdy * x).mean(-1, keepdim=True)))).to(s["x"].dtype))
        out.append((dy * x * r).sum(0))
    return out


def _order_keys(z):
    """One 64-bit key per logit: larger values first, equal ones by the lower index."""
    bits = (z.float() + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return (bits << 24) - torch.arange(z.shape[-1], device=z.device)


def _plain_logprobs(s, c):
    z = s["logits"]
    x = z.float() / c["temperature"]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    p = e / total
    ent = -torch.where(p > 0, p * (x - lse), 0.0).sum(-1)
    ids = s["ids"].long()
    lp = x.gather(1, ids.clamp(min=0)[:, None]) - lse
    lp = torch.where(ids >= 0, lp[:, 0], 0.0)
    out = [lp, ent, lse[:, 0]]
    if c["k"]:
        top = _order_keys(z).topk(c["k"], dim=-1).indices
        out += [x.gather(1, top) - lse, top.to(torch.int32)]
    return out


def _plain_distill(s, c):
    x, T = s["logits"].float() / c["temperature"], c["temperature"]
    ids = s["ids"].long()
    here = ids >= 0
    at = ids.clamp(min=0)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    lse = m + torch.log(e.sum(-1, keepdim=True))
    lp = x.gather(1, at) - lse
    t = torch.where(here, s["teacher"], float("-inf"))
    if not c["tail"]:
        tm = t.amax(-1, keepdim=True)
        t = t - tm - torch.log(torch.exp(t - tm).sum(-1, keepdim=True))
    q = torch.exp(t)
    loss = torch.where(q > 0, q * (t - lp), 0.0).sum(-1)
    if c["tail"]:
        # an entry that is not there marks the column past the vocabulary
        mark = torch.zeros((x.shape[0], x.shape[1] + 1), dtype=torch.bool, device=x.device)
        mark.scatter_(1, torch.where(here, ids, x.shape[1]), True)
        rest = torch.where(mark[:, :-1], 0.0, e)
        lse0 = m + torch.log(rest.sum(-1, keepdim=True))
        q0 = (1 - q.sum(-1)).clamp(min=0.0)
        loss = loss + torch.where(q0 > 0, q0 * (torch.log(q0) - (lse0 - lse)[:, 0]), 0.0)
    out = [loss * (T * T)]
    if c["mode"] != "forward":
        grad = torch.exp(x - lse)
        total = q.sum(-1, keepdim=True)
        if c["tail"]:
            total = total + q0[:, None]
        grad = grad * total
        if c["tail"]:
            grad = grad - q0[:, None] * torch.where(mark[:, :-1], 0.0, torch.exp(x - lse0))
        grad = grad.scatter_add(1, at, torch.where(here, -q, 0.0))
        out.append((grad * (s["weight"][:, None] * T)).to(s["logits"].dtype))
    return out


def _own_linear(ee, s, c):
    act = c["act"]
    back = c["backward"] != "none"
    if not back or act == "none":
        y = ee.linear(s["x"], s["w"], s["b"], s["r"], activation=act, out_dtype=TYPES[c["out"]])
        u = None
    else:
        y, u = ee.linear(s["x"], s["w"], s["b"], s["r"], activation=act, out_dtype=TYPES[c["out"]], keep_preact=True)
    if not back:
        return [y]
    if c["backward"] == "dx":
        dx, _, _ = ee.linear_backward(s["dy"], None, s["w"], activation=act, preact=u, dw=False, dbias=False)
        return [y, dx]
    return [y, *ee.linear_backward(s["dy"], s["x"], s["w"], activation=act, preact=u, dw_dtype=_dw_type(c))]


def _own_norm(ee, s, c):
    y, rstd = ee.rms_norm(s["x"], s["gain"], EPS, out_dtype=TYPES[c["out"]])
    if not c["backward"]:
        return [y]
    return [y, *ee.rms_norm_backward(s["dy"], s["x"], s["gain"], rstd)]


def _own_logprobs(ee, s, c):
    lp, ent, lse, top_lp, top_ids = ee.token_logprobs(s["logits"], s["ids"], k=c["k"], temperature=c["temperature"])
    return [lp, ent, lse, top_lp, top_ids] if c["k"] else [lp, ent, lse]


def _own_distill(ee, s, c):
    kw = {"temperature": c["temperature"], "tail": c["tail"]}
    if c["mode"] == "step":
        return list(ee.distill_topk_step(s["logits"], s["ids"], s["teacher"], s["weight"], **kw))
    loss, stats = ee.distill_topk(s["logits"], s["ids"], s["teacher"], **kw)
    if c["mode"] == "forward":
        return [loss]
    return [loss, ee.distill_topk_backward(s["weight"], s["logits"], s["ids"], s["teacher"], stats, **kw)]


def run(state):
    c = state["case"]
    if own:
        import paper_2609_14144_gb300 as ee

        return {"linear": _own_linear, "norm": _own_norm, "logprobs": _own_logprobs,
                "distill": _own_distill}[c["kind"]](ee, state, c)
    return {"linear": _plain_linear, "norm": _plain_norm, "logprobs": _plain_logprobs,
            "distill": _plain_distill}[c["kind"]](state, c)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    if c["kind"] == "linear":
        n, i, o, b = c["rows"], c["n_in"], c["n_out"], BYTES[c["type"]]
        nbytes = b * (n * i + i * o) + BYTES[c["out"]] * n * o * (2 if c["residual"] else 1) + (b * o if c["bias"] else 0)
        flops = 2.0 * n * i * o
        if c["backward"] != "none":
            nbytes += b * (n * o + n * i)
            flops += 2.0 * n * i * o
        if c["backward"] == "all":
            nbytes += (4 if c["act"] == "none" else b) * i * o + 4 * o
            flops += 2.0 * n * i * o
        return {"bytes": nbytes, "flops": flops}
    if c["kind"] == "norm":
        n, d, bx, by = c["rows"], c["d"], BYTES[c["type"]], BYTES[c["out"]]
        nbytes = n * d * (bx + by) + 2 * d
        flops = 4.0 * n * d
        if c["backward"]:
            nbytes += n * d * (bx + by) + 4 * d
            flops += 9.0 * n * d
        return {"bytes": nbytes, "flops": flops}
    n, v, b = c["rows"], c["vocab"], BYTES[c["type"]]
    if c["kind"] == "logprobs":
        return {"bytes": n * v * b + n * (4 + 12 + 8 * c["k"]), "flops": 5.0 * n * v}
    nbytes = n * v * b * (1 if c["mode"] == "forward" else 2) + n * (8 * c["k"] + 8)
    return {"bytes": nbytes, "flops": (3.0 if c["mode"] == "forward" else 7.0) * n * v}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    c, s = case, prepare(case, seed)
    return {"linear": _exact_linear, "norm": _exact_norm, "logprobs": _exact_logprobs,
            "distill": _exact_distill}[c["kind"]](c, s)


def _exact_linear(c, s):
    x, w = s["x"].double(), s["w"].double()
    u = torch.einsum("ni,oi->no", x, w)
    if c["bias"]:
        u += s["b"].double()
    erf = torch.erf(u / 2.0 ** 0.5) if c["act"] == "gelu" else None
    y = {"none": lambda: u, "relu": lambda: u.clamp(min=0), "silu": lambda: u * torch.sigmoid(u),
         "gelu": lambda: u * (1 + erf) / 2}[c["act"]]()
    out = [y + s["r"].double() if c["residual"] else y]
    if c["backward"] == "none":
        return out
    du = s["dy"].double()
    if c["act"] == "relu":
        du = torch.where(u > 0, du, 0.0)
    elif c["act"] == "silu":
        du = du * (torch.sigmoid(u) + u * torch.sigmoid(u) * torch.sigmoid(-u))
    elif c["act"] == "gelu":
        du = du * ((1 + erf) / 2 + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi))
    out.append(torch.einsum("no,oi->ni", du, w))
    if c["backward"] == "all":
        out += [torch.einsum("no,ni->oi", du, x), du.sum(0)]
    return out


def _exact_norm(c, s):
    x, g = s["x"].double(), s["gain"].double()
    rms = torch.sqrt(x.square().sum(-1, keepdim=True) / c["d"] + EPS)
    xh = x / rms
    out = [xh * g]
    if c["backward"]:
        dxh = s["dy"].double() * g
        out.append((dxh - xh * ((dxh * xh).sum(-1, keepdim=True) / c["d"])) / rms)
        out.append((s["dy"].double() * xh).sum(0))
    return out


def _exact_logprobs(c, s):
    parts = []
    for r0 in range(0, c["rows"], 512):
        z = s["logits"][r0:r0 + 512].double()
        ids = s["ids"][r0:r0 + 512].long()
        lse = torch.logsumexp(z / c["temperature"], -1)
        logp = z / c["temperature"] - lse[:, None]
        given = logp.gather(1, ids.clamp(min=0)[:, None])[:, 0]
        part = [torch.where(ids < 0, 0.0, given), torch.special.entr(torch.exp(logp)).sum(-1), lse]
        if c["k"]:
            order = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :c["k"]]
            part += [logp.gather(1, order), order.to(torch.int32)]
        parts.append(part)
    return [torch.cat(p) for p in zip(*parts)]


def _exact_distill(c, s):
    T, V = c["temperature"], c["vocab"]
    parts = []
    for r0 in range(0, c["rows"], 256):
        rows = slice(r0, r0 + 256)
        u = s["logits"][rows].double() / T
        ids, weight = s["ids"][rows].long(), s["weight"][rows].double()
        logp = torch.log_softmax(u, -1)
        t = s["teacher"][rows].double().masked_fill(ids < 0, float("-inf"))
        q = t.exp() if c["tail"] else torch.softmax(t, -1)
        # the teacher over the vocabulary, zero outside its list (a spare column takes absent entries)
        full = torch.zeros((u.shape[0], V + 1), dtype=torch.float64, device=u.device)
        full.scatter_(1, torch.where(ids < 0, V, ids), q)
        full = full[:, :V]
        loss = (torch.special.xlogy(full, full) - full * logp).sum(-1)
        p = logp.exp()
        grad = p * full.sum(-1, keepdim=True) - full
        if c["tail"]:
            free = torch.ones((u.shape[0], V + 1), dtype=torch.bool, device=u.device)
            free.scatter_(1, torch.where(ids < 0, V, ids), False)
            free = free[:, :V]
            q0 = (1 - q.sum(-1)).clamp(min=0.0)
            lse0 = torch.logsumexp(u.masked_fill(~free, float("-inf")), -1)
            logp0 = lse0 - torch.logsumexp(u, -1)
            loss = loss + torch.special.xlogy(q0, q0) - torch.where(q0 > 0, q0 * logp0, 0.0)
            inside = torch.where(free, torch.exp(u - lse0[:, None]), 0.0)
            grad = grad + q0[:, None] * (p - inside)
        part = [loss * T * T]
        if c["mode"] != "forward":
            part.append(grad * (T * weight[:, None]))
        parts.append(part)
    return [torch.cat(p) for p in zip(*parts)]
