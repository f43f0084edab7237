"""Cases of the operators that train a network and form the Gram matrix of its Jacobian.

`listed()` gives the named cases, `draw(rng)` more of the same ranges.  A case is a dict; `op` says which operator:

  linear   y = act(x W^T + b) + r; x: rows x k, W: cols x k
  grad     its gradient: dz = dy act'(z), dx = dz W, dW = dz^T x, db = the column sums of dz
  adamw    one step over `count` tensors, states in 32 or 8 bits, gradients in type `gtype`, optionally a copy of the
           parameters in 16 bits (`copy`)
  ntk      K = sum over layers (a a^T + 1) * (g g^T) (elementwise), lower triangle; a: n x (inputs of the layer),
           g: n d x (outputs of the layer), d network outputs

`pad` is by how many elements the rows of a matrix stand further apart than they are long.
With `own` false `run` is written in elementary torch operations, in 32 bits (64 where the operands have 64).
"""
import math

import torch

own = False

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f64": 8, "f32": 4, "f16": 2, "bf16": 2}
BLOCK = 256             # elements that share a scale in an 8-bit state
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=10)


def _linear(name, op, dtype, rows, cols, k, act, bias=True, residual=False, pad=0):
    c = dict(op=op, dtype=dtype, rows=rows, cols=cols, k=k, act=act, bias=bias, residual=residual, pad=pad)
    return dict(c, name=name) if name else c


def _adamw(name, state, ptype, gtype, copy, count, size, tight=False):
    c = dict(op="adamw", state=state, ptype=ptype, gtype=gtype, copy=copy, count=count, size=size, tight=tight)
    return dict(c, name=name) if name else c


def _ntk(name, dtype, out, n, d, layers, first, width):
    c = dict(op="ntk", dtype=dtype, out=out, n=n, d=d, layers=layers, first=first, width=width)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: one token through a projection back to the residual stream
        _linear("linear_bf16_one_row", "linear", "bf16", 1, 4096, 4096, "none", residual=True),
        # serving a handful of requests, sizes that fit nothing
        _linear("linear_f16_7_rows_odd", "linear", "f16", 7, 1999, 1001, "silu"),
        # an ordinary batch, ragged
        _linear("linear_bf16_333_rows", "linear", "bf16", 333, 1500, 1000, "gelu", residual=True),
        # a network trained in 32 bits
        _linear("linear_f32_2048", "linear", "f32", 2048, 2048, 2048, "gelu_tanh", residual=True),
        # the first half of a large block's two products, many tokens
        _linear("linear_bf16_8192_rows", "linear", "bf16", 8192, 16384, 4096, "gelu"),
        # the gradient of a small network's layer in 32 bits, odd sizes
        _linear("grad_f32_777_rows_odd", "grad", "f32", 777, 1301, 515, "silu"),
        # the gradient of a layer, many tokens
        _linear("grad_bf16_4096_rows", "grad", "bf16", 4096, 8192, 4096, "gelu"),
        # a small network, everything in 32 bits
        _adamw("adamw_f32_24_tensors", 32, "f32", "f32", "", 24, 100_000),
        # many parameters: states in 8 bits, gradients in 16, the forward pass's 16-bit copy written beside
        _adamw("adamw_8bit_32_tensors", 8, "f32", "bf16", "bf16", 32, 3_000_000),
        # the benchmark's smallest order in 32 bits, a network of three layers
        _ntk("ntk_f32_n512", "f32", "f32", 512, 1, 3, 100, 256),
        # the benchmark's n = 8192 order in 64 bits
        _ntk("ntk_f64_n8192", "f64", "f64", 8192, 1, 3, 784, 512),
        # a classifier with 10 outputs, activations in 16 bits
        _ntk("ntk_bf16_n1000_d10", "bf16", "f32", 1000, 10, 4, 777, 512),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "grad", "adamw", "ntk"])
    if op in ("linear", "grad"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        top = 1.37e11 if dtype == "f32" else 5.5e11
        while True:
            rows, cols, k = _log(rng, 1, 8192), _log(rng, 64, 16384), _log(rng, 64, 8192)
            if rng.random() < 0.5:      # whole multiples are as common as odd sizes
                cols, k = -(-cols // 64) * 64, -(-k // 64) * 64
            if rows * cols * k * 2 <= top:
                break
        return _linear(None, op, dtype, rows, cols, k, rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                       bias=rng.random() < 0.7, residual=op == "linear" and rng.random() < 0.5, pad=rng.choice([0, 0, 0, 8, 3]))
    if op == "adamw":
        count = _log(rng, 1, 60)
        most = 45_000_000 // ((count + 1) // 2)
        return _adamw(None, rng.choice([32, 8]), rng.choice(["f32", "f32", "bf16"]), rng.choice(["f32", "bf16", "f16"]),
                      rng.choice(["", "bf16", "f16"]), count, _log(rng, 1000, most), rng.random() < 0.3)
    dtype, out = rng.choice([("f64", "f64"), ("f32", "f32"), ("f32", "f64"), ("bf16", "f32"), ("f16", "f32")])
    d = rng.choice([1, 1, 1, 3, 10])
    return _ntk(None, dtype, out, _log(rng, 100, 5000 // d), d, rng.randint(2, 4), _log(rng, 10, 1000), _log(rng, 32, 700))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _matrix(g, rows, cols, dtype, scale=1.0, pad=0):
    """Normal entries; its rows are cols + pad elements apart."""
    a = torch.empty(rows, cols + pad, dtype=TYPES[dtype], device="cuda")
    a.copy_(torch.randn(rows, cols + pad, generator=g, dtype=torch.float32, device="cuda").mul_(scale))
    return a[:, :cols]


def _sizes(case):
    """Sizes of the tensors of an optimiser step: matrices of about `size` elements, biases between them, odd ones."""
    return [max(1, case["size"] + 37 * i) if i % 2 == 0 else max(1, int(math.sqrt(case["size"])) + i)
            for i in range(case["count"])]


def _layers(case):
    """(inputs, outputs) of each layer; the last one's gradients are those of the network's outputs."""
    widths = [case["first"]] + [case["width"]] * (case["layers"] - 1) + [case["d"]]
    return list(zip(widths[:-1], widths[1:]))


def _prepare_adamw(case, g):
    sizes = _sizes(case)
    blocks = [-(-n // BLOCK) for n in sizes]
    at = [BLOCK * sum(blocks[:i]) for i in range(len(sizes) + 1)]
    opt = dict(generator=g, device="cuda")
    where = [sum(sizes[:i]) for i in range(len(sizes))] if case["tight"] else at[:-1]
    total = sum(sizes) if case["tight"] else at[-1]
    flat = torch.zeros(total, dtype=TYPES[case["ptype"]], device="cuda")
    for w, n in zip(where, sizes):
        flat[w:w + n] = torch.randn(n, **opt).mul_(0.02)
    s = {"flat": flat, "params": [flat[w:w + n] for w, n in zip(where, sizes)], "sizes": sizes, "where": where, "at": at,
         # gradients of a loss: tensors differ in scale, and elements by orders of magnitude
         "grads": [(torch.randn(n, **opt) * torch.randn(n, **opt) * 10.0 ** (-2 - i % 3)).to(TYPES[case["gtype"]])
                   for i, n in enumerate(sizes)],
         "seed": int(torch.randint(0, 2 ** 31, (1,), generator=g, device="cuda")), "copies": None, "scales": None}
    m = torch.randn(at[-1], **opt).mul_(1e-3)
    u = torch.randn(at[-1], **opt).abs_().mul_(2e-3).add_(1e-5)
    inside = torch.zeros(at[-1], dtype=torch.bool, device="cuda")
    for a, n in zip(at, sizes):
        inside[a:a + n] = True
    m.mul_(inside)
    u.mul_(inside)
    if case["state"] == 8:
        mb, ub = m.view(-1, BLOCK), u.view(-1, BLOCK)
        flat_scales = torch.stack([mb.abs().amax(1) / 127, ub.amax(1) / 255], 1).contiguous()
        s["m"] = (mb / flat_scales[:, :1]).round().to(torch.int8).view(-1)
        s["v"] = (ub / flat_scales[:, 1:]).round().clamp(1, 255).mul(inside.view(-1, BLOCK)).to(torch.uint8).view(-1)
        s["flat_scales"] = flat_scales
        s["scales"] = [flat_scales[a // BLOCK:a // BLOCK + b] for a, b in zip(at, blocks)]
        # number of each block's first element in its tensor, and number of the tensor
        s["first"] = torch.cat([torch.arange(b, dtype=torch.int32) * BLOCK for b in blocks]).cuda()
        s["tensor"] = torch.repeat_interleave(torch.arange(len(sizes), dtype=torch.int32), torch.tensor(blocks)).cuda()
    else:
        s["m"], s["v"] = m, u * u
    s["ms"] = [s["m"][a:a + n] for a, n in zip(at, sizes)]
    s["vs"] = [s["v"][a:a + n] for a, n in zip(at, sizes)]
    if case["copy"]:
        s["flat_copy"] = torch.zeros(total, dtype=TYPES[case["copy"]], device="cuda")
        s["copies"] = [s["flat_copy"][w:w + n] for w, n in zip(where, sizes)]
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "adamw":
        s = _prepare_adamw(case, g)
    elif case["op"] == "ntk":
        n, d = case["n"], case["d"]
        s = {"inputs": [_matrix(g, n, p, case["dtype"]) for p, _ in _layers(case)],
             "signals": [_matrix(g, n * d, q, case["dtype"], 1.0 / math.sqrt(q)) for _, q in _layers(case)],
             "scale": 1.0 / sum(p for p, _ in _layers(case)),
             "k": torch.zeros(n * d, n * d, dtype=TYPES[case["out"]], device="cuda")}
    else:
        rows, cols, k, dtype, pad = (case[v] for v in ("rows", "cols", "k", "dtype", "pad"))
        s = {"x": _matrix(g, rows, k, dtype, pad=pad), "w": _matrix(g, cols, k, dtype, 1.0 / math.sqrt(k), pad),
             "bias": _matrix(g, 1, cols, dtype, 0.1)[0] if case["bias"] else None,
             "residual": _matrix(g, rows, cols, dtype, pad=pad) if case["residual"] else None}
        if case["op"] == "grad":
            s["dy"] = _matrix(g, rows, cols, dtype, pad=pad)
            s["z"] = _matrix(g, rows, cols, dtype) if case["act"] != "none" else None
    return dict(s, case=case)


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
R2, R2PI, TANH_A, TANH_B = math.sqrt(0.5), 1.0 / math.sqrt(2.0 * math.pi), math.sqrt(2.0 / math.pi), 0.044715


def _act(name, z):
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * R2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(TANH_A * (z + TANH_B * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * R2)) + z * torch.exp(-0.5 * z * z) * R2PI
    if name == "gelu_tanh":
        t = torch.tanh(TANH_A * (z + TANH_B * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * TANH_A * (1 + 3 * TANH_B * z * z)
    if name == "silu":
        e = 1 / (1 + torch.exp(-z))
        return e * (1 + z * (1 - e))
    return torch.ones_like(z)


def _plain_linear(s, c):
    z = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(c["act"], z)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(TYPES[c["dtype"]])


def _plain_grad(s, c):
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_slope(c["act"], s["z"].float())
    t = TYPES[c["dtype"]]
    return (dz @ s["w"].float()).to(t), (dz.t().contiguous() @ s["x"].float()).to(t), dz.sum(0).to(t) if c["bias"] else None


def _bits(s):
    """32 random bits for each element, as int32: multiplications and shifts mix the element's number, the
    tensor's number and the seed."""
    def word(v):
        return v - 2 ** 32 if v >= 2 ** 31 else v
    key = s["tensor"] * word(0xA54FF53B) + word(s["seed"])
    h = (s["first"][:, None] + torch.arange(BLOCK, dtype=torch.int32, device="cuda")) * word(0x6A09E667) + key[:, None]
    h = (h ^ ((h >> 16) & 0xFFFF)) * word(0xBB67AE85)
    h = (h ^ ((h >> 15) & 0x1FFFF)) * word(0x3C6EF373)
    return h ^ ((h >> 16) & 0xFFFF)


def _factors():
    h = HYPER
    return dict(b1=h["beta1"], a1=1 - h["beta1"], b2=h["beta2"], a2=1 - h["beta2"], keep=1 - h["lr"] * h["weight_decay"],
                rate=h["lr"] / (1 - h["beta1"] ** h["step"]), root=1 / math.sqrt(1 - h["beta2"] ** h["step"]), eps=h["eps"])


def _step(p, g, m, v):
    """New p, m, v of an AdamW step, in the operands' type."""
    f = _factors()
    m = m * f["b1"] + g * f["a1"]
    v = v * f["b2"] + (g * f["a2"]) * g
    return p * f["keep"] - f["rate"] * (m / (torch.sqrt(v) * f["root"] + f["eps"])), m, v


def _padded(s, tensors, dtype=torch.float32):
    """The tensors one after the other, each filled up to whole blocks with zeros."""
    return torch.cat([torch.nn.functional.pad(t.to(dtype), (0, b - a - n))
                      for t, n, a, b in zip(tensors, s["sizes"], s["at"][:-1], s["at"][1:])])


def _tensors(s, flat):
    """The tensors out of what _padded gave, as they stand in the flat parameters."""
    if s["where"] == s["at"][:-1]:
        return flat
    return torch.cat([flat[a:a + n] for a, n in zip(s["at"], s["sizes"])])


def _quantise(m, u, bits, dtype):
    """Codes and scales of the blocks of m and u = sqrt(v)."""
    r1, r2 = (bits & 0xFFFF).to(dtype) / 65536, ((bits >> 16) & 0xFFFF).to(dtype) / 65536
    s1, s2 = m.abs().amax(1, keepdim=True) / 127, u.amax(1, keepdim=True) / 255
    c1 = torch.where(s1 > 0, torch.clamp(torch.floor(m / s1 + r1), -127, 127), torch.zeros_like(m))
    c2 = torch.where(s2 > 0, torch.clamp(torch.floor(u / s2 + r2), 0, 255), torch.zeros_like(u))
    return c1, torch.where((u > 0) & (s2 > 0), torch.clamp(c2, min=1), c2), s1, s2


def _values(s):
    """What the 8-bit states stand for: m and sqrt(v)."""
    return s["m"].view(-1, BLOCK) * s["flat_scales"][:, :1], s["v"].view(-1, BLOCK) * s["flat_scales"][:, 1:]


def _out_adamw(s, c):
    out = {"params": s["flat"]}
    if c["copy"]:
        out["copy"] = s["flat_copy"]
    if c["state"] == 8:
        out["m"], out["root_v"] = _values(s)
    else:
        out["m"], out["v"] = s["m"], s["v"]
    return out


def _plain_adamw(s, c):
    p, g = _padded(s, s["params"]), _padded(s, s["grads"])
    if c["state"] == 8:
        m, u = (x.reshape(-1) for x in _values(s))
        p, m, v = _step(p, g, m, u * u)
        c1, c2, s1, s2 = _quantise(m.view(-1, BLOCK), torch.sqrt(v).view(-1, BLOCK), _bits(s), torch.float32)
        s["m"].copy_(c1.view(-1))
        s["v"].copy_(c2.view(-1))
        s["flat_scales"].copy_(torch.cat([s1, s2], 1))
    else:
        p, m, v = _step(p, g, s["m"], s["v"])
        s["m"].copy_(m)
        s["v"].copy_(v)
    p = _tensors(s, p)
    s["flat"].copy_(p)
    if c["copy"]:
        s["flat_copy"].copy_(p)
    return _out_adamw(s, c)


def _ntk_sum(s, c, t):
    d = c["d"]
    k = 0
    for a, g in zip(s["inputs"], s["signals"]):
        a, g = a.to(t), g.to(t)
        first = a @ a.t() + 1
        if d > 1:
            first = first.repeat_interleave(d, 0).repeat_interleave(d, 1)
        k = k + first * (g @ g.t())
    return torch.tril(k * s["scale"])


def _plain_ntk(s, c):
    s["k"].copy_(_ntk_sum(s, c, TYPES[c["out"]]))
    return s["k"]


def run(s):
    c = s["case"]
    if not own:
        return {"linear": _plain_linear, "grad": _plain_grad, "adamw": _plain_adamw, "ntk": _plain_ntk}[c["op"]](s, c)
    import paper_2503_04424_amd as M
    if c["op"] == "linear":
        return M.mdet_linear_forward(s["x"], s["w"], s["bias"], s["residual"], c["act"])
    if c["op"] == "grad":
        return M.mdet_linear_backward(s["dy"], s["x"], s["w"], s["z"], c["act"], db=c["bias"])
    if c["op"] == "ntk":
        return M.mdet_ntk_gram(s["inputs"], s["signals"], s["k"], outputs=c["d"], scale=s["scale"])
    M.mdet_adamw_step(s["params"], s["grads"], s["ms"], s["vs"], scales=s["scales"], copies=s["copies"], seed=s["seed"], **HYPER)
    return _out_adamw(s, c)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it should return
# ---------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "adamw":
        each = 2 * BYTES[c["ptype"]] + BYTES[c["gtype"]] + (BYTES[c["copy"]] if c["copy"] else 0)
        # a state in 8 bits is read and written, and the values that it stands for are returned: codes read once more, 32 bits written
        each += 16 if c["state"] == 32 else 4 + 4 * 8 / BLOCK + 2 + 8
        n = sum(_sizes(c))
        return {"bytes": each * n, "flops": 15 * n}
    if c["op"] == "ntk":
        n, d, t = c["n"], c["d"], BYTES[c["dtype"]]
        big = n * d
        return {"bytes": sum(n * p + big * q for p, q in _layers(c)) * t + big * (big + 1) // 2 * BYTES[c["out"]],
                "flops": sum(n * (n + 1) * p + big * (big + 1) * q for p, q in _layers(c))}
    m, n, k, t = c["rows"], c["cols"], c["k"], BYTES[c["dtype"]]
    if c["op"] == "linear":
        return {"bytes": t * (m * k + n * k + m * n * (2 if c["residual"] else 1) + (n if c["bias"] else 0)), "flops": 2 * m * n * k}
    return {"bytes": t * (m * n * (1 if c["act"] == "none" else 2) + 2 * m * k + 2 * n * k + (n if c["bias"] else 0)),
            "flops": 4 * m * n * k}


def _exact_act(name, z):
    """act(z) and act'(z)."""
    if name == "relu":
        return torch.relu(z), torch.heaviside(z, torch.zeros_like(z))
    if name == "gelu":
        c = torch.special.ndtr(z)
        return z * c, c + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if name in ("gelu_tanh", "silu"):           # (1 + tanh(t)) / 2 is the logistic function of 2 t
        t, dt = (z, torch.ones_like(z)) if name == "silu" else (
            2 * TANH_A * (z + TANH_B * z.pow(3)), 2 * TANH_A * (1 + 3 * TANH_B * z.square()))
        q = torch.sigmoid(t)
        return z * q, q + z * q * torch.sigmoid(-t) * dt
    return z, torch.ones_like(z)


def _exact_linear(s, case):
    z = torch.matmul(s["x"].double(), s["w"].double().mT)
    if case["bias"]:
        z += s["bias"].double()[None, :]
    y = _exact_act(case["act"], z)[0]
    return y + s["residual"].double() if case["residual"] else y


def _exact_grad(s, case):
    dz = s["dy"].double()
    if case["act"] != "none":
        dz = dz * _exact_act(case["act"], s["z"].double())[1]
    return (torch.matmul(dz, s["w"].double()), torch.matmul(dz.mT.contiguous(), s["x"].double()),
            dz.sum(0) if case["bias"] else None)


def _exact_ntk(s, case):
    d, n = case["d"], case["n"]
    total = torch.zeros(n, d, n, d, dtype=torch.float64, device="cuda")
    for a, g in zip(s["inputs"], s["signals"]):
        a, g = a.double(), g.double()
        total += (a @ a.mT + 1)[:, None, :, None] * (g @ g.mT).view(n, d, n, d)
    return torch.tril(total.view(n * d, n * d)) * s["scale"]


def _exact_adamw(s, case):
    h, new = HYPER, {"m": [], "v": [], "params": s["flat"].double()}
    correct1, correct2 = 1 - h["beta1"] ** h["step"], 1 - h["beta2"] ** h["step"]
    for i, (p, g, w, a, n) in enumerate(zip(s["params"], s["grads"], s["where"], s["at"], s["sizes"])):
        p, g, m, v = p.double(), g.double(), s["ms"][i].double(), s["vs"][i].double()
        if case["state"] == 8:
            m = m * s["scales"][i][:, 0].double().repeat_interleave(BLOCK)[:n]
            v = (v * s["scales"][i][:, 1].double().repeat_interleave(BLOCK)[:n]).square()
        m = m.lerp(g, 1 - h["beta1"])
        v = v.lerp(g.square(), 1 - h["beta2"])
        new["params"][w:w + n] = p - h["lr"] * (h["weight_decay"] * p + m / correct1 / ((v / correct2).sqrt() + h["eps"]))
        fill = s["at"][i + 1] - a - n
        new["m"].append(torch.nn.functional.pad(m, (0, fill)))
        new["v"].append(torch.nn.functional.pad(v, (0, fill)))
    out = {"params": new["params"], "m": torch.cat(new["m"]), "v": torch.cat(new["v"])}
    if case["copy"]:
        out["copy"] = out["params"]
    if case["state"] == 8:                      # rounded up with the probability of what is left over
        low, high = (_bits(s).long() & 0xFFFFFFFF).remainder(65536), (_bits(s).long() & 0xFFFFFFFF).div(65536, rounding_mode="floor")
        for name, x, most, r in (("m", out["m"], 127, low), ("root_v", out.pop("v").sqrt(), 255, high)):
            x = x.view(-1, BLOCK)
            step = x.abs().amax(1, keepdim=True) / most
            units = torch.nan_to_num(x / step, nan=0.0)
            code = (units + r.double() / 65536).floor().clamp(-most, most)
            code = torch.where((units > 0) & (code < 1) & (most == 255), torch.ones_like(code), code)
            out[name] = code * step
    return out


def exact(case, seed):
    return {"linear": _exact_linear, "grad": _exact_grad, "adamw": _exact_adamw, "ntk": _exact_ntk}[case["op"]](prepare(case, seed), case)
