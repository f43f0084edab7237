"""A front end with the call shape of the paper's software appendix (``memdet(M, max_mem,
assume, triangle, overwrite, mixed_precision, ...)`` returning ``ld, sign, diag, perm[, info]``)
on top of the C ABI.  Argument marshalling only: it chooses the entry point and the flags,
lays a host matrix out in block columns, and turns the result struct into the tuple; every
step of the computation runs in the library.

Where the paper's call and this one differ:
  * ``M`` is a square CUDA tensor (resident: ``mdet_logdet_device``), or a CPU tensor / numpy
    array (``mdet_logdet_host`` on its packed block-column layout, streamed if it does not
    fit ``max_mem``).  Stores on disk go through ``mdet_logdet_file`` directly.
  * pivoting is off unless asked for (``pivot='leaf'`` or ``'block'``): ``perm`` is then the
    identity, and ``diag`` the pivots of the unpivoted factorisation (Sec. 2.2 pivots inside a
    block only; the determinant does not depend on it).
  * ``scratch_dir`` and ``parallel_io`` belong to the file entry point and are not taken here.
"""
import math
import re

from . import binding as B

_UNITS = {"": 1, "B": 1, "KB": 10 ** 3, "MB": 10 ** 6, "GB": 10 ** 9, "TB": 10 ** 12,
          "KIB": 2 ** 10, "MIB": 2 ** 20, "GIB": 2 ** 30, "TIB": 2 ** 40}


def parse_bytes(max_mem) -> int:
    """``'32GB'``, ``'16GiB'``, a number of bytes, or None / inf for no limit (0)."""
    if max_mem is None:
        return 0
    if isinstance(max_mem, str):
        m = re.fullmatch(r"\s*([0-9]*\.?[0-9]+)\s*([A-Za-z]*)\s*", max_mem)
        if not m or m.group(2).upper() not in _UNITS:
            raise ValueError(f"cannot read a size from {max_mem!r}")
        return int(float(m.group(1)) * _UNITS[m.group(2).upper()])
    if max_mem == float("inf"):
        return 0
    return int(max_mem)


def memdet(M, max_mem=None, assume="gen", triangle=None, overwrite=False, mixed_precision=None,
           block_size=0, pivot=None, return_info=False, stream=None):
    """``ld, sign, diag, perm`` (and ``info`` with ``return_info``) of the square matrix ``M``.

    assume: 'gen' (P M = L D U), 'sym' (L D L^T) or 'spd' (Cholesky form).
    triangle: for 'sym' / 'spd', 'l' or None reads the lower triangle, 'u' the upper one.
    mixed_precision: 'float64' runs fp64 arithmetic on a matrix stored in fp32 / fp16 / bf16
    (App. C); None or the matrix's own type computes in that type.
    """
    import numpy as np
    import torch
    if isinstance(M, np.ndarray):
        M = torch.from_numpy(M)
    if M.dim() != 2 or M.shape[0] != M.shape[1]:
        raise ValueError("a square matrix is expected")
    n = M.shape[0]
    if assume not in ("gen", "sym", "spd"):
        raise ValueError("assume must be 'gen', 'sym' or 'spd'")
    if triangle not in (None, "l", "u"):
        raise ValueError("triangle must be None, 'l' or 'u'")
    flags = {"gen": B.FLAG_GENERAL, "sym": 0, "spd": B.FLAG_ASSUME_SPD}[assume]
    if pivot is not None:
        if assume != "sym" or pivot not in ("leaf", "block"):
            raise ValueError("pivot='leaf' or 'block' goes with assume='sym'")
        flags |= B.FLAG_PIVOT if pivot == "leaf" else B.FLAG_PIVOT_BLOCK
    wide = mixed_precision in ("float64", "f64", torch.float64)
    if mixed_precision not in (None, "float64", "f64", torch.float64, "float32", "f32", torch.float32):
        raise ValueError("mixed_precision must be None, 'float32' or 'float64'")
    if wide and M.dtype != torch.float64:
        flags |= B.FLAG_COMPUTE_F64
    elif not wide and mixed_precision is not None and M.dtype != torch.float32:
        raise ValueError("arithmetic narrower than the storage is not offered")
    if triangle == "u" and assume != "gen":
        M = M.t()                       # the upper triangle of M is the lower triangle of its transpose
    budget = parse_bytes(max_mem)
    arith = torch.float64 if (flags & B.FLAG_COMPUTE_F64) else M.dtype
    want_perm = bool(flags & (B.FLAG_PIVOT | B.FLAG_PIVOT_BLOCK | B.FLAG_GENERAL))
    if M.is_cuda:
        a = M if (M.stride(1) == 1 or n <= 1) else M.contiguous()
        if a is not M:
            overwrite = True            # the library may work in the copy just made
        diag = torch.empty(n, dtype=arith, device="cuda")
        perm = torch.full((n,), -1, dtype=torch.int32, device="cuda") if want_perm else None
        r = B.mdet_logdet_device(a, block_size=block_size, mem_budget=budget, overwrite=overwrite, flags=flags,
                                 diag=diag, perm=perm, stream=stream, raise_on_error=False)
        diag = diag.cpu()
        perm = perm.cpu() if want_perm else None
    else:
        bs = B.mdet_plan(n, M.dtype, block_size, budget, flags=flags).block_size_used if n > 0 else 64
        pack = B.pack_general_block_columns if assume == "gen" else B.pack_lower_block_columns
        packed = pack(M, bs)
        diag = torch.empty(n, dtype=arith)
        perm = torch.full((n,), -1, dtype=torch.int32) if want_perm else None
        r = B.mdet_logdet_host(packed, n, bs, mem_budget=budget, overwrite=True, flags=flags, diag=diag,
                               perm=perm, stream=stream, raise_on_error=False)
    if r.status not in (B.Status.OK, B.Status.ESINGULAR):
        raise B.MemdetError(r.status, r)
    perm_out = perm.numpy().astype("int64") if want_perm else np.arange(n, dtype="int64")
    out = (r.logabsdet, r.sign, diag.numpy(), perm_out)
    if return_info:
        import dataclasses
        return out + (dataclasses.asdict(r),)
    return out


class FitLogdet:
    """The regression of Alg. 2 behind the ``fit`` / ``eval`` pair of the software appendix:
    ``fit(n, ell)`` takes consecutive integers ``n`` (the fit interval) and the log-determinants
    ``ell`` of the leading principal blocks of those orders (every d-th cumulative sum of
    ``log|diag|``, already sub-sampled by the caller as in the appendix); ``eval(n)`` returns the
    extrapolated log-determinants ``n * Lhat_n``.  Both run in the library (``mdet_flodance_fit``,
    ``mdet_flodance_eval``); this class only arranges the arrays."""

    def __init__(self, q: int = 0):
        self.q = int(q)
        self.coef = None

    def fit(self, n, ell):
        import numpy as np
        import torch
        n = np.asarray(n)
        ell = np.asarray(ell, dtype=np.float64)
        ni = np.rint(n).astype(np.int64)
        if n.ndim != 1 or n.shape != ell.shape or n.size < self.q + 3 or np.any(ni != n) or \
                np.any(np.diff(ni) != 1) or ni[0] < 1:
            raise ValueError("n must be consecutive integers >= 1, with one log-determinant each")
        # the library reads ell[j - 1] for j = n0 .. ns (one sample per order: d = 1)
        full = np.zeros(int(ni[-1]), dtype=np.float64)
        full[ni - 1] = ell
        self.coef = B.mdet_flodance_fit(torch.from_numpy(full).cuda(), 1, int(ni[0]), int(ni[-1]), self.q)
        return self

    def eval(self, n):
        import numpy as np
        import torch
        if self.coef is None:
            raise ValueError("fit first")
        nv = torch.from_numpy(np.asarray(n, dtype=np.float64).reshape(-1).copy()).cuda()
        lhat = B.mdet_flodance_eval(self.coef, self.q, nv)
        return (lhat * nv).cpu().numpy().reshape(np.shape(n))

    @property
    def parameters(self):
        """c_0, nu_0 .. nu_q, L_{n0}, residual norm, as the library returns them."""
        return None if self.coef is None else self.coef.cpu().numpy()


def _linear_function():
    """The autograd node of ``linear``, made at its first use (importing the package does not import torch)."""
    import torch

    class LinearFunction(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, bias, residual, activation):
            rows = _as_rows(x)
            keep = activation != "none" and any(ctx.needs_input_grad[:3])
            z = rows.new_empty((rows.shape[0], w.shape[0])) if keep else None
            y = _layer(rows, w, bias, residual, activation, z)
            ctx.save_for_backward(rows, w, z)
            ctx.activation, ctx.shape = activation, x.shape
            return y.view(*x.shape[:-1], w.shape[0])

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            x, w, z = ctx.saved_tensors
            need_x, need_w, need_b, need_r, _ = ctx.needs_input_grad
            dx = dw = db = None
            if need_x or need_w or need_b:
                dx, dw, db = B.mdet_linear_backward(_rows(_as_rows(dy)), _rows(x), _rows(w), z, ctx.activation,
                                                    dx=need_x, dw=need_w, db=need_b)
            return None if dx is None else dx.view(ctx.shape), dw, db, dy if need_r else None, None

    return LinearFunction


def _layer(rows, w, bias, residual, activation, z=None):
    """The layer on a matrix x; z: where what stands in front of the activation is kept."""
    return B.mdet_linear_forward(_rows(rows), _rows(w), None if bias is None else bias.contiguous(),
                                 None if residual is None else _rows(_as_rows(residual)), activation, preact=z)


def _as_rows(t):
    """The tensor as a matrix whose rows are its last axis (also where that or any other axis is empty)."""
    return t.reshape(math.prod(t.shape[:-1]), t.shape[-1])


def _rows(t):
    """Rows of consecutive elements that do not overlap: the matrix itself where it has them (views and slices do), or a
    copy.  Autograd hands over gradients that are one row, or one element, repeated (distances of zero)."""
    if (t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]):
        return t
    # an empty one as well, which contiguous() would leave as it is
    return t.new_empty(t.shape).copy_(t)


def _derivatives(*operands):
    """Whether a derivative can be asked for: gradients are on, or an operand carries a tangent of forward mode, which ``no_grad`` does not take
    away (the nodes have no forward mode: with them such a call raises)."""
    import torch
    if torch.is_grad_enabled():
        return True
    forward = torch.autograd.forward_ad
    if getattr(forward, "_current_level", 0) < 0:                # outside of forward mode there are none: a tenth of the time of asking each operand
        return False
    return any(t is not None and forward.unpack_dual(t).tangent is not None for t in operands)


_linear = None


def linear(x, w, bias=None, residual=None, activation="none"):
    """``act(x w^T + bias) + residual`` with its gradient (autograd): x (..., k), w (n, k), residual (..., n).
    activation: 'none', 'relu', 'gelu', 'gelu_tanh' or 'silu'.  One launch or two for the layer, up to six for its gradient;
    operands and gradients that are views of any kind, repeated rows among them, are laid out first where they have to be."""
    global _linear
    if x.dim() < 1 or w.dim() != 2:
        raise ValueError("x with rows of inputs as its last axis and a matrix w expected")
    if residual is not None and tuple(residual.shape) != (*x.shape[:-1], w.shape[0]):
        raise ValueError(f"residual: shape {(*x.shape[:-1], w.shape[0])} expected, not {tuple(residual.shape)}")
    if not _derivatives(x, w, bias, residual):
        # ctx.needs_input_grad is true for parameters here as well: nothing is kept for a gradient that cannot be asked for
        return _layer(_as_rows(x), w, bias, residual, activation).view(*x.shape[:-1], w.shape[0])
    if _linear is None:
        _linear = _linear_function()
    return _linear.apply(x, w, bias, residual, activation)


def _embedding_function():
    """The autograd node of ``embedding``."""
    import torch

    class EmbeddingFunction(torch.autograd.Function):
        @staticmethod
        def forward(ctx, table, ids, scale):
            flat = ids.reshape(-1).contiguous()
            ctx.save_for_backward(flat)
            ctx.vocab, ctx.scale = table.shape[0], scale
            return B.mdet_embedding_forward(flat, _rows(table), scale).view(*ids.shape, table.shape[1])

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            ids, = ctx.saved_tensors
            return B.mdet_embedding_backward(_rows(_as_rows(dy)), ids, ctx.vocab, ctx.scale), None, None

    return EmbeddingFunction


def _layer_norm_function():
    """The autograd node of ``layer_norm``."""
    import torch

    class LayerNormFunction(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, eps):
            rows = _rows(_as_rows(x))
            weight = None if weight is None else weight.contiguous()
            y, mean, rstd = B.mdet_layernorm_forward(rows, weight, None if bias is None else bias.contiguous(), eps)
            ctx.save_for_backward(rows, weight, mean, rstd)
            ctx.shape = x.shape
            return y.view(x.shape)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            x, weight, mean, rstd = ctx.saved_tensors
            need_x, need_w, need_b, _ = ctx.needs_input_grad
            dx, dw, db = B.mdet_layernorm_backward(_rows(_as_rows(dy)), x, mean, rstd, weight, dx=need_x, dw=need_w, db=need_b)
            return None if dx is None else dx.view(ctx.shape), dw, db, None

    return LayerNormFunction


def _cross_entropy_function():
    """The autograd node of ``linear_cross_entropy``."""
    import torch

    class CrossEntropyFunction(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, bias, target, ignore, reduction, keep):
            rows, mat = _rows(_as_rows(x)), _rows(w)
            bias = None if bias is None else bias.contiguous()
            loss, lse, kept = B.mdet_xent_forward(rows, mat, target, bias, ignore, keep=keep and any(ctx.needs_input_grad[:3]))
            rows_loss, weights = loss, None
            if reduction != "none":
                loss, weights = B.mdet_xent_reduce(loss, target, mat.shape[0], ignore, reduction == "mean")
            elif kept is None:
                loss = loss.clone()              # the caller's own, to be changed in place as any other result
            ctx.save_for_backward(rows, mat, bias, target, lse, rows_loss if kept is None else None, kept, weights)
            ctx.shape, ctx.ignore = x.shape, ignore
            return loss

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dloss):
            x, w, bias, target, lse, loss, kept, weights = ctx.saved_tensors
            dloss = dloss.contiguous() if weights is None else weights * dloss
            need_x, need_w, need_b = ctx.needs_input_grad[:3]
            dx, dw, db = B.mdet_xent_backward(dloss, x, w, target, lse, bias, ctx.ignore, kept, dx=need_x, dw=need_w, db=need_b,
                                              loss=loss)
            return None if dx is None else dx.view(ctx.shape), dw, db, None, None, None, None

    return CrossEntropyFunction


_functions = {}


def _function(make):
    """The node that make() makes, made once."""
    if make not in _functions:
        _functions[make] = make()
    return _functions[make]


def embedding(ids, table, scale=1.0):
    """``scale * table[ids]`` with its gradient by the table (autograd): ids (...) int32 or int64, table (vocab, width).  An id outside of the
    table gives a row of zeros, and has no part in the gradient."""
    if table.dim() != 2:
        raise ValueError("table: a matrix expected")
    if not _derivatives(table):
        return B.mdet_embedding_forward(ids.reshape(-1).contiguous(), _rows(table), scale).view(*ids.shape, table.shape[1])
    return _function(_embedding_function).apply(table, ids, scale)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last axis of x (..., n) with its gradient (autograd); weight and bias (n,)."""
    if x.dim() < 1:
        raise ValueError("x with rows as its last axis expected")
    if not _derivatives(x, weight, bias):
        return B.mdet_layernorm_forward(_rows(_as_rows(x)), None if weight is None else weight.contiguous(),
                                        None if bias is None else bias.contiguous(), eps, mean=False, rstd=False)[0].view(x.shape)
    return _function(_layer_norm_function).apply(x, weight, bias, eps)


def linear_cross_entropy(x, w, target, bias=None, ignore_index=-100, reduction="mean", keep=False):
    """Softmax cross entropy of ``x w^T + bias`` with its gradient (autograd), without that matrix in memory in the forward pass, and with one like it
    in the gradient, a piece of up to 2^29 elements (or 4096 of each row, if that is more) at a time: x (..., k), w (n, k), target (...) int32 or int64.  Targets that are ``ignore_index``, or outside of the vocabulary, do not count.  reduction: 'mean' over those that
    count (NaN if none does), 'sum', or 'none' (the losses, in float32, in target's shape).  ``keep`` spends x's rows times n elements between
    the two passes on sparing the gradient one of its three products."""
    if x.dim() < 1 or w.dim() != 2 or target.shape != x.shape[:-1]:
        raise ValueError(f"x with rows as its last axis, a matrix w and a target for each row expected, not {tuple(x.shape)}, {tuple(w.shape)} and "
                         f"{tuple(target.shape)}")
    if reduction not in ("mean", "sum", "none"):
        raise ValueError("reduction must be 'mean', 'sum' or 'none'")
    flat = target.reshape(-1).contiguous()
    if _derivatives(x, w, bias):
        loss = _function(_cross_entropy_function).apply(x, w, bias, flat, ignore_index, reduction, keep)
    else:
        loss = B.mdet_xent_forward(_rows(_as_rows(x)), _rows(w), flat, None if bias is None else bias.contiguous(), ignore_index, lse=False)[0]
        if reduction != "none":
            loss = B.mdet_xent_reduce(loss, flat, w.shape[0], ignore_index, reduction == "mean", weights=False)[0]
    return loss.view(target.shape) if reduction == "none" else loss


class AdamW:
    """AdamW over a list of CUDA tensors, updated in place by ``step()`` (``mdet_adamw_step``; asynchronous).

    state_bits: 32, or 8 for a mean and a root mean square in 8 bits each with two scales per 256 elements.
    copy_dtype: torch.bfloat16 or torch.float16 keeps a 16-bit copy of every tensor in ``copies``, written by the step and by ``load_state_dict``."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, copy_dtype=None, seed=0):
        import torch
        self.params = list(params)
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in self.params if p.numel())
        if any(b[0] < a[1] for a, b in zip(spans[:-1], spans[1:])):
            raise ValueError("a tensor twice, or tensors that overlap: a step would update the same memory from several places at once")
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self.state_bits, self.seed, self.steps = state_bits, int(seed), 0
        types = (torch.float32, torch.float32) if state_bits == 32 else (torch.int8, torch.uint8)
        self.exp_avg = [torch.zeros(p.shape, dtype=types[0], device=p.device) for p in self.params]
        self.exp_avg_sq = [torch.zeros(p.shape, dtype=types[1], device=p.device) for p in self.params]
        self.scales = None if state_bits == 32 else [torch.zeros((p.numel() + 255) // 256, 2, device=p.device) for p in self.params]
        self.copies = None if copy_dtype is None else [p.detach().to(copy_dtype) for p in self.params]

    def step(self, grads=None, grad_scale=None, stream=None):
        """One step with ``grads``, or with the tensors' own ``.grad``."""
        if grads is None:
            grads = [p.grad for p in self.params]
        if any(g is None for g in grads):
            raise ValueError("a gradient for every tensor expected")
        step = self.steps + 1
        B.mdet_adamw_step([p.detach() for p in self.params], grads, self.exp_avg, self.exp_avg_sq, lr=self.lr, step=step,
                          beta1=self.betas[0], beta2=self.betas[1], eps=self.eps, weight_decay=self.weight_decay,
                          scales=self.scales, copies=self.copies, grad_scale=grad_scale, seed=self.seed + step, stream=stream)
        self.steps = step                  # a step that was refused does not count

    def state_dict(self):
        return {"steps": self.steps, "seed": self.seed, "state_bits": self.state_bits, "exp_avg": list(self.exp_avg),
                "exp_avg_sq": list(self.exp_avg_sq), "scales": None if self.scales is None else list(self.scales)}

    def load_state_dict(self, state):
        """Takes over what ``state_dict`` gave, whole or not at all, and the parameters' present values into the copies."""
        names = ("exp_avg", "exp_avg_sq") + (("scales",) if self.state_bits == 8 else ())
        mine = [t for name in names for t in getattr(self, name)]
        other = [t for name in names for t in state[name] or ()]
        if state["state_bits"] != self.state_bits or [t.shape for t in mine] != [t.shape for t in other]:
            raise ValueError("a state of the same width for tensors of the same shapes expected")
        for a, b in zip(mine, other):
            a.copy_(b)
        for c, p in zip(self.copies or (), self.params):
            c.detach().copy_(p.detach())
        self.steps, self.seed = int(state["steps"]), int(state["seed"])
