"""Cases of the operators at the two ends of a network over tokens, and of its normalisations.

`listed()` gives the named cases, `draw(rng)` more of the same ranges.  A case is a dict; `op` says which operator:

  embed       y_i = scale table[id_i]; an id outside of the table gives a row of zeros
  embed_grad  G_v = scale (sum over i with id_i = v of dy_i), for every row of the table, or added to a gradient that is
              there already (`add`: a table that is also the last layer's matrix)
  norm        y = (x - mean) rstd w + b for each row, mean and rstd kept; rstd = 1 / sqrt(var + eps)
  norm_grad   its gradient: with h = (x - mean) rstd and u = dy w,  dx = rstd (u - avg(u) - h avg(u h)),
              dw = the column sums of dy h, db those of dy
  xent        loss_i = log(sum over j of exp(z_ij)) - z_i,t_i with z = x W^T + b; x: rows x k, W: vocab x k; a target outside of
              the vocabulary marks a row that does not count (loss 0)
  xent_grad   the same, and the gradient of sum over i of g_i loss_i: with e_ij = g_i (exp(z_ij - lse_i) - [j = t_i]),
              dx = e W, dW = e^T x, db = the column sums of e.  `keep`: the forward pass leaves what spares the backward
              pass the first product

`pad` is by how many elements the rows of a matrix stand further apart than they are long.
With `own` false `run` is written in elementary torch operations, in 32 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
IGNORED = -100
PADDING = 0.04          # part of the tokens that are padding
ROWS_AT_ONCE = 1024     # of the 64-bit logits


def _embed(name, op, dtype, rows, vocab, width, index="i64", out="", scale=1.0, add=False, pad=0):
    c = dict(op=op, dtype=dtype, rows=rows, vocab=vocab, width=width, index=index, out=out or dtype, scale=scale, add=add, pad=pad)
    return dict(c, name=name) if name else c


def _norm(name, op, dtype, rows, cols, out="", affine=True, pad=0):
    c = dict(op=op, dtype=dtype, rows=rows, cols=cols, out=out or dtype, affine=affine, pad=pad)
    return dict(c, name=name) if name else c


def _xent(name, op, dtype, rows, vocab, k, index="i64", out="", bias=False, keep=False, pad=0):
    c = dict(op=op, dtype=dtype, rows=rows, vocab=vocab, k=k, index=index, out=out or dtype, bias=bias, keep=keep, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: the next token of each of a handful of requests
        _embed("embed_f16_7_tokens", "embed", "f16", 7, 32000, 4096, scale=64.0),
        # a batch of texts, rows that fit nothing
        _embed("embed_bf16_16384_tokens", "embed", "bf16", 16384, 50003, 1500, index="i32"),
        # a training step's gradient of the whole table, tokens as frequent as in texts
        _embed("embed_grad_bf16_16384_tokens", "embed_grad", "bf16", 16384, 50003, 1024, out="f32", scale=32.0),
        # the same table as the last layer's: added to that gradient; odd sizes
        _embed("embed_grad_f32_add_odd", "embed_grad", "f32", 4099, 5003, 777, index="i32", add=True),
        # serving: one token
        _norm("norm_bf16_one_row", "norm", "bf16", 1, 4096),
        # a batch of texts
        _norm("norm_bf16_16384_rows", "norm", "bf16", 16384, 4096),
        # a small network in 32 bits, odd sizes
        _norm("norm_grad_f32_777_rows_odd", "norm_grad", "f32", 777, 1301),
        # a training step of a large one
        _norm("norm_grad_bf16_16384_rows", "norm_grad", "bf16", 16384, 4096, out="f32"),
        # what a few tokens cost a model: perplexity of a short text
        _xent("xent_bf16_5_rows", "xent", "bf16", 5, 50003, 1024, index="i32"),
        # evaluation, rows that fit nothing
        _xent("xent_f16_1000_rows_odd", "xent", "f16", 1000, 31999, 1501, bias=True),
        # a training step of a small network, nothing kept
        _xent("xent_grad_bf16_4096_rows", "xent_grad", "bf16", 4096, 50003, 1024),
        # a training step of a large one with memory to spare
        _xent("xent_grad_bf16_8192_rows_keep", "xent_grad", "bf16", 8192, 131072, 4096, keep=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "xent", "xent_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    out = rng.choice([dtype, "f32"])
    index, pad = rng.choice(["i64", "i32"]), rng.choice([0, 0, 0, 8, 3])
    whole = rng.random() < 0.5          # whole multiples are as common as odd sizes

    def size(lo, hi):
        n = _log(rng, lo, hi)
        return min(hi, -(-n // 64) * 64) if whole else n
    if op in ("embed", "embed_grad"):
        while True:
            rows, vocab, width = _log(rng, 1, 32768), size(100, 131072), size(16, 8192)
            if rows * width <= 1 << 25 and vocab * width <= 1 << 27:
                break
        return _embed(None, op, dtype, rows, vocab, width, index, out if op == "embed_grad" else "", rng.choice([1.0, 0.125, 45.25]),
                      op == "embed_grad" and rng.random() < 0.4, pad)
    if op in ("norm", "norm_grad"):
        while True:
            rows, cols = _log(rng, 1, 65536), size(16, 16384)
            if rows * cols <= 1 << 26:
                break
        return _norm(None, op, dtype, rows, cols, out if op == "norm_grad" else "", rng.random() < 0.8, pad)
    top = 2.7e11 if dtype == "f32" else 2.2e12
    while True:
        rows, vocab, k = _log(rng, 1, 8192), size(100, 131072), size(64, 4096)
        if rows * vocab * k <= top and vocab * k <= 1 << 28:
            break
    return _xent(None, op, dtype, rows, vocab, k, index, out if op == "xent_grad" else "", rng.random() < 0.4,
                 op == "xent_grad" and rng.random() < 0.5, pad)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _matrix(g, rows, cols, dtype, scale=1.0, pad=0):
    """Normal entries; its rows are cols + pad elements apart."""
    a = torch.empty(rows, cols + pad, dtype=TYPES[dtype], device="cuda")
    a.copy_(torch.randn(rows, cols + pad, generator=g, dtype=torch.float32, device="cuda").mul_(scale))
    return a[:, :cols]


def _tokens(g, rows, vocab, index, padding):
    """Tokens in the order of how frequent they are: number v with a probability of log((v + 2) / (v + 1)) / log(vocab + 1)."""
    u = torch.rand(rows, generator=g, dtype=torch.float64, device="cuda")
    ids = (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1)
    ids[torch.rand(rows, generator=g, device="cuda") < PADDING] = padding
    return ids.to(torch.int32 if index == "i32" else torch.int64)


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(seed)
    op, dtype, pad = c["op"], c["dtype"], c["pad"]
    if op in ("embed", "embed_grad"):
        s = {"ids": _tokens(g, c["rows"], c["vocab"], c["index"], -1)}
        if op == "embed":
            s["table"] = _matrix(g, c["vocab"], c["width"], dtype, 0.02, pad)
        else:
            s["dy"] = _matrix(g, c["rows"], c["width"], dtype, 1e-3, pad)
            s["dtable"] = _matrix(g, c["vocab"], c["width"], c["out"], 1e-3, pad) if c["add"] else None
    elif op in ("norm", "norm_grad"):
        rows, cols = c["rows"], c["cols"]
        x = torch.randn(rows, cols + pad, generator=g, device="cuda")
        # a residual stream: rows differ in size, a few columns stand out
        x *= torch.exp(torch.randn(rows, 1, generator=g, device="cuda") * 0.7)
        x += torch.randn(cols + pad, generator=g, device="cuda") * 0.3
        x[:, torch.randint(0, cols, (max(1, cols // 256),), generator=g, device="cuda")] *= 8
        s = {"x": x.to(TYPES[dtype])[:, :cols], "w": None, "b": None}
        if c["affine"]:
            s["w"] = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[dtype])
            s["b"] = (0.1 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[dtype])
        if op == "norm_grad":
            s["dy"] = _matrix(g, rows, cols, dtype, 1e-2, pad)
            s["mean"], s["rstd"] = _statistics(s["x"].float())
    else:
        rows, vocab, k = c["rows"], c["vocab"], c["k"]
        s = {"target": _tokens(g, rows, vocab, c["index"], IGNORED), "w": _matrix(g, vocab, k, dtype, 1 / math.sqrt(k), pad),
             "bias": _matrix(g, 1, vocab, dtype, 0.5)[0] if c["bias"] else None}
        # what a trained network has in front of its last layer: from no idea of the next token to being sure of it
        x = torch.randn(rows, k + pad, generator=g, device="cuda")
        sure = torch.rand(rows, 1, generator=g, device="cuda") * 14
        x[:, :k] += sure * s["w"][s["target"].long().clamp(min=0)].float()
        s["x"] = x.to(TYPES[dtype])[:, :k]
        # the mean over the rows that count, times what keeps gradients in 16-bit floats away from their least number
        count = (s["target"] >= 0).sum().clamp(min=1)
        s["g"] = ((s["target"] >= 0) / count * (4096.0 if dtype == "f16" else 1.0)).float()
    return dict(s, case=case)


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_embed(s, c):
    ids = s["ids"].long()
    inside = (ids >= 0) & (ids < c["vocab"])
    rows = s["table"][torch.where(inside, ids, 0)].float() * c["scale"]
    return torch.where(inside[:, None], rows, 0.0).to(TYPES[c["dtype"]])


def _plain_embed_grad(s, c):
    ids = s["ids"].long()
    inside = (ids >= 0) & (ids < c["vocab"])
    total = torch.zeros(c["vocab"] + 1, c["width"], device="cuda")          # the last row takes the padding
    total.index_add_(0, torch.where(inside, ids, c["vocab"]), s["dy"].float() * c["scale"])
    total = total[:-1]
    if not c["add"]:
        return total.to(TYPES[c["out"]])
    s["dtable"].copy_(s["dtable"].float() + total)
    return s["dtable"]


def _statistics(x):
    mean = x.mean(1)
    centred = x - mean[:, None]
    return mean, 1 / torch.sqrt((centred * centred).mean(1) + EPS)


def _plain_norm(s, c):
    x = s["x"].float()
    mean, rstd = _statistics(x)
    y = (x - mean[:, None]) * rstd[:, None]
    if c["affine"]:
        y = y * s["w"].float() + s["b"].float()
    return y.to(TYPES[c["dtype"]]), mean, rstd


def _plain_norm_grad(s, c):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    h = (x - s["mean"][:, None]) * rstd
    u = dy * s["w"].float() if c["affine"] else dy
    dx = rstd * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
    dw, db = ((dy * h).sum(0).to(TYPES[c["out"]]), dy.sum(0).to(TYPES[c["out"]])) if c["affine"] else (None, None)
    return dx.to(TYPES[c["dtype"]]), dw, db


def _plain_xent(s, c):
    w, x = s["w"].float(), s["x"].float()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    target = s["target"].long()
    counts = (target >= 0) & (target < c["vocab"])
    safe = torch.where(counts, target, 0)
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    loss = torch.where(counts, lse - z.gather(1, safe[:, None])[:, 0], 0.0)
    if c["op"] == "xent":
        return loss, lse
    e = z.sub_(lse[:, None]).exp_()
    e[torch.arange(c["rows"], device="cuda"), safe] -= 1
    e *= torch.where(counts, s["g"], 0.0)[:, None]
    t = TYPES[c["out"]]
    return loss, (e @ w).to(TYPES[c["dtype"]]), (e.t().contiguous() @ x).to(t), e.sum(0).to(t) if c["bias"] else None


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
         "xent": _plain_xent, "xent_grad": _plain_xent}


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return PLAIN[op](s, c)
    import paper_2503_04424_amd as M
    if op == "embed":
        return M.mdet_embedding_forward(s["ids"], s["table"], scale=c["scale"])
    if op == "embed_grad":
        return M.mdet_embedding_backward(s["dy"], s["ids"], c["vocab"], scale=c["scale"], dtable=s["dtable"], accumulate=c["add"],
                                         grad_dtype=TYPES[c["out"]])
    if op == "norm":
        return M.mdet_layernorm_forward(s["x"], s["w"], s["b"], eps=EPS)
    if op == "norm_grad":
        return M.mdet_layernorm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["w"], dw=c["affine"], db=c["affine"], grad_dtype=TYPES[c["out"]])
    if op == "xent":
        return M.mdet_xent_forward(s["x"], s["w"], s["target"], s["bias"])[:2]
    loss, lse, kept = M.mdet_xent_forward(s["x"], s["w"], s["target"], s["bias"], keep=c["keep"])
    return (loss, *M.mdet_xent_backward(s["g"], s["x"], s["w"], s["target"], lse, s["bias"], kept=kept, db=c["bias"], grad_dtype=TYPES[c["out"]]))


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it should return
# ---------------------------------------------------------------------------
def _distinct(rows, vocab):
    """How many different tokens are to be expected among `rows` of them."""
    v = torch.arange(vocab, dtype=torch.float64)
    p = torch.log1p(1 / (v + 1)) / math.log(vocab + 1) * (1 - PADDING)
    return float((1 - torch.exp(rows * torch.log1p(-p))).sum())


def work(case):
    c, t, o = case, BYTES[case["dtype"]], BYTES[case["out"]]
    op, rows = c["op"], c["rows"]
    if op in ("embed", "embed_grad"):
        size, used = rows * c["width"], _distinct(rows, c["vocab"]) * c["width"]
        ids = rows * (8 if c["index"] == "i64" else 4)
        if op == "embed":
            return {"bytes": int(ids + t * (used + size)), "flops": size}
        return {"bytes": int(ids + t * size + o * (2 * used if c["add"] else c["vocab"] * c["width"])), "flops": 2 * size}
    if op in ("norm", "norm_grad"):
        size, line = rows * c["cols"], c["cols"] if c["affine"] else 0
        if op == "norm":
            return {"bytes": 2 * t * size + 2 * t * line + 8 * rows, "flops": 8 * size}
        return {"bytes": 3 * t * size + (t + 2 * o) * line + 8 * rows, "flops": 16 * size}
    ids = rows * (8 if c["index"] == "i64" else 4)
    ends = rows * c["k"] + c["vocab"] * c["k"] + (c["vocab"] if c["bias"] else 0)
    product = 2 * rows * c["vocab"] * c["k"]
    if op == "xent":
        return {"bytes": t * ends + ids + 8 * rows, "flops": product}
    return {"bytes": t * ends + t * rows * c["k"] + o * (ends - rows * c["k"]) + ids + 8 * rows, "flops": 3 * product}


def _exact_embed(s, case):
    y = torch.zeros(case["rows"], case["width"], dtype=torch.float64, device="cuda")
    at = torch.nonzero((s["ids"] >= 0) & (s["ids"] < case["vocab"]))[:, 0]
    y[at] = torch.index_select(s["table"], 0, s["ids"][at].long()).double() * case["scale"]
    return y


def _exact_embed_grad(s, case):
    at = torch.nonzero((s["ids"] >= 0) & (s["ids"] < case["vocab"]))[:, 0]
    total = s["dtable"].double() if case["add"] else torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
    return total.index_add(0, s["ids"][at].long(), s["dy"].double()[at], alpha=case["scale"])


def _exact_norm(s, case):
    x = s["x"].double()
    var, mean = torch.var_mean(x, dim=1, unbiased=False)
    rstd = (var + EPS).rsqrt()
    y = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
    if case["affine"]:
        y = torch.addcmul(s["b"].double().expand_as(y), y, s["w"].double())
    return y, mean, rstd


def _exact_norm_grad(s, case):
    h = (s["x"].double() - s["mean"].double().unsqueeze(1)) * s["rstd"].double().unsqueeze(1)
    dy, cols = s["dy"].double(), case["cols"]
    u = dy.mul(s["w"].double()) if case["affine"] else dy
    # u without its parts along the row of ones and along h
    dx = u - (u.sum(1, keepdim=True) + h * (u * h).sum(1, keepdim=True)) / cols
    dx *= s["rstd"].double().unsqueeze(1)
    return (dx, (dy * h).sum(0), dy.sum(0)) if case["affine"] else (dx, None, None)


def _exact_xent(s, case):
    vocab, grad = case["vocab"], case["op"] == "xent_grad"
    w = s["w"].double()
    opt = dict(dtype=torch.float64, device="cuda")
    losses, lses, dxs = [], [], []
    dw, db = (torch.zeros(vocab, case["k"], **opt), torch.zeros(vocab, **opt)) if grad else (None, None)
    for first in range(0, case["rows"], ROWS_AT_ONCE):
        x, t, g = (s[name][first:first + ROWS_AT_ONCE] for name in ("x", "target", "g"))
        x, t = x.double(), t.long()
        logits = torch.matmul(x, w.mT)
        if case["bias"]:
            logits += s["bias"].double()
        lse = torch.logsumexp(logits, 1)
        hit = torch.nonzero((t >= 0) & (t < vocab))[:, 0]
        loss = torch.zeros_like(lse)
        loss[hit] = lse[hit] - logits[hit, t[hit]]
        losses.append(loss)
        lses.append(lse)
        if grad:
            weight = torch.zeros_like(lse)
            weight[hit] = g[hit].double()
            slope = torch.softmax(logits, 1).mul_(weight[:, None])
            slope[hit, t[hit]] -= weight[hit]
            dxs.append(torch.matmul(slope, w))
            dw.addmm_(slope.mT.contiguous(), x)
            db += slope.sum(0)
    loss = torch.cat(losses)
    return (loss, torch.cat(dxs), dw, db if case["bias"] else None) if grad else (loss, torch.cat(lses))


EXACT = {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "norm": _exact_norm, "norm_grad": _exact_norm_grad,
         "xent": _exact_xent, "xent_grad": _exact_xent}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed), case)
