"""Operators that train and serve the heads a cache certifies (argument
marshalling only; include/lipcache.h states the formulas).

* adapted_logits, adapted_logits_backward: logits of rows under a shared head
  and each row's own low-rank adapter, and their gradients;
* cross_entropy: per-row losses and the gradient of the logits in one call;
* orthogonalize, orthogonal_step: Newton-Schulz orthogonalisation of a
  matrix, and the optimiser step that uses it.

Tensors are float32 or bfloat16 on one GPU, up to 65,536 features and classes
(a cache takes float32 heads of up to 1,024); the work runs on the current
stream. Rows may be strided (a slice of a wider matrix); other layouts are
copied first. Scratch comes from PyTorch's allocator, so calls can be captured
into a CUDA graph. Autograd does not see the operators: gradients are what
adapted_logits_backward and cross_entropy return, and a tensor that requires
gradients is refused while they are recorded (call under torch.no_grad()).
"""
from __future__ import annotations

import ctypes as C
import functools
import struct

import torch

from . import _lib
from ._lib import Adapted, LipCacheError, check

TYPES = {torch.float32: _lib.F32, torch.bfloat16: _lib.BF16}
#: a, b, c of X <- aX + (bS + cSS)X, S = XX^T: singular values move fast to
#: about 1 (0.7 to 1.2) within five steps.
QUINTIC = (3.4445, -4.7750, 2.0315)

I32, F32 = torch.int32, torch.float32
_grads = torch.is_grad_enabled
#: tells autograd that tensors were written to, so that a gradient that needs the old values raises
_written = torch.autograd.graph.increment_version
#: struct lipcache_adapted, packed: half the time of filling ctypes' Adapted
_ADAPTED = struct.Struct("@6i9q")
assert _ADAPTED.size == C.sizeof(Adapted)


def _call(at: int, fn, *args) -> None:
    """fn on the current stream of GPU `at`, made current only where another one is."""
    if torch._C._cuda_getDevice() == at:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(at))
    else:
        with torch.cuda.device(at):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(at))
    if status:
        check(status)


def _type(t: torch.Tensor, name: str) -> int:
    try:
        return TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}") from None


def _check(t: torch.Tensor, name: str, dims: int, at: int, dtype: torch.dtype) -> None:
    if t.dtype == dtype and t.get_device() == at and t.dim() == dims:
        return
    if t.get_device() != at:
        raise ValueError(f"{name} must be on one GPU with the other tensors, not on {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    raise ValueError(f"{name} must have {dims} dimensions, not {t.dim()}")


def _recorded(**named) -> None:
    """Refuses the tensor that asks for gradients which autograd would not find."""
    for name, t in named.items():
        if t is not None and t.requires_grad:
            raise ValueError(f"{name} requires gradients, which autograd does not record here: call under torch.no_grad()")


def _gpu(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU, not on {t.device}")
    return t.get_device()


def _int32(*sizes: int) -> None:
    """Sizes that the C ABI takes as int32 (ctypes would cut larger ones off)."""
    if max(sizes) > 0x7fffffff:
        raise ValueError(f"sizes must be at most {0x7fffffff}, not {max(sizes)}")


def _rows(t: torch.Tensor):
    """`t` (2-D) with neighbours in a row next to each other in memory and rows
    that do not overlap, and its row stride."""
    n, width = t.shape
    if t.is_contiguous():
        return t, width
    if n > 1 and width > 1 and t.stride(1) == 1 and t.stride(0) >= width:
        return t, t.stride(0)
    return t.contiguous(), width


def _workspace(nbytes: int, device: torch.device) -> torch.Tensor:
    return torch.empty(nbytes if nbytes > 256 else 256, dtype=torch.uint8, device=device)


def _taken(nbytes: int) -> int:
    if nbytes < 0:
        raise LipCacheError(_lib.E_INVALID, _lib.load().lipcache_last_error().decode())
    return nbytes


# (sizes that are refused are asked for anew each time, for the library's message)
@functools.lru_cache(maxsize=1024)
def _adapted_bytes(ty: int, d: int, classes: int, G: int, r: int, n: int, backward: int) -> int:
    p = Adapted(ty, d, classes, G, r, 0, n)
    return _taken(_lib.load().lipcache_adapted_workspace(C.byref(p), backward))


@functools.lru_cache(maxsize=1024)
def _ortho_bytes(ty: int, batch: int, m: int, n: int) -> int:
    return _taken(_lib.load().lipcache_orthogonalize_workspace(ty, batch, m, n))


def _describe(x, W, A, B, adapter, scales, backward):
    """The operator's description, its sizes, scratch and device, and the tensors it points into."""
    dt, at = x.dtype, x.get_device()
    if not (dt in TYPES and at >= 0 and x.dim() == 2 and W.dtype == dt and W.get_device() == at and W.dim() == 2
            and A.dtype == dt and A.get_device() == at and A.dim() == 3 and B.dtype == dt and B.get_device() == at
            and B.dim() == 3 and adapter.dtype == I32 and adapter.get_device() == at and adapter.dim() == 1):
        _type(x, "x")
        _gpu(x, "x")
        for t, name, dims, dtype in ((x, "x", 2, dt), (W, "W", 2, dt), (A, "A", 3, dt), (B, "B", 3, dt),
                                     (adapter, "adapter", 1, I32)):
            _check(t, name, dims, at, dtype)
    if _grads() and (x.requires_grad or W.requires_grad or A.requires_grad or B.requires_grad
                    or scales is not None and scales.requires_grad):
        _recorded(x=x, W=W, A=A, B=B, scales=scales)
    (n, d), (classes, wide), (G, r, da) = x.shape, W.shape, A.shape
    if wide != d or da != d or B.shape != (G, classes, r) or len(adapter) != n:
        raise ValueError("x must be n x d, W C x d, A G x r x d, B G x C x r and adapter must have n entries")
    if scales is not None:
        _check(scales, "scales", 1, at, F32)
        if len(scales) != G:
            raise ValueError("scales must have an entry per adapter")
        scales = scales.contiguous()
    x, ldx = _rows(x)
    W, ldw = _rows(W)
    A, B, adapter = A.contiguous(), B.contiguous(), adapter.contiguous()
    ty, device = TYPES[dt], x.device
    try:
        p = _ADAPTED.pack(ty, d, classes, G, r, 0, n, x.data_ptr(), ldx, W.data_ptr(), ldw, A.data_ptr(), B.data_ptr(),
                          adapter.data_ptr(), 0 if scales is None else scales.data_ptr())
    except struct.error:
        _int32(d, classes, G, r)
        raise
    ws = _workspace(_adapted_bytes(ty, d, classes, G, r, n, backward), device)
    return p, n, d, classes, ws, at, device, (x, W, A, B, adapter, scales)


def adapted_logits(x: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor, adapter: torch.Tensor,
                   bias: torch.Tensor | None = None, scales: torch.Tensor | None = None,
                   out: torch.Tensor | None = None) -> torch.Tensor:
    """y_t = W x_t + bias + scales[g] B_g (A_g x_t), g = adapter[t].

    x: n x d; W: C x d; A: G x r x d; B: G x C x r; adapter: n (int32; a value
    outside [0, G) means no adapter); bias: C (float32); scales: G (float32);
    out must not overlap the other tensors."""
    p, n, _, classes, ws, at, device, keep = _describe(x, W, A, B, adapter, scales, 0)
    if bias is not None:
        _check(bias, "bias", 1, at, F32)
        if bias.requires_grad and _grads():
            _recorded(bias=bias)
        if len(bias) != classes:
            raise ValueError("bias must have C entries")
        bias = bias.contiguous()
    own = out is None
    if own:
        out, ldy = torch.empty(n, classes, dtype=x.dtype, device=device), classes
    else:
        _check(out, "out", 2, at, x.dtype)
        if out.requires_grad and _grads():
            _recorded(out=out)
        rows, ldy = _rows(out)
        if out.shape != (n, classes) or rows is not out:
            raise ValueError("out must be n x C with dense rows")
    _call(at, _lib.load().lipcache_adapted_logits, p, None if bias is None else bias.data_ptr(), out.data_ptr(), ldy,
          ws.data_ptr(), ws.numel())
    if not own:
        _written(out)
    return out


def adapted_logits_backward(dy: torch.Tensor, x: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                            adapter: torch.Tensor, scales: torch.Tensor | None = None, need_dx: bool = True,
                            need_dA: bool = True, need_dB: bool = True):
    """(dx, dA, dB) of adapted_logits for the gradient dy (n x C) of its
    result; W and bias are held fixed. An output that is not needed is None."""
    p, n, d, classes, ws, at, device, keep = _describe(x, W, A, B, adapter, scales, 1)
    dt = x.dtype
    _check(dy, "dy", 2, at, dt)
    if dy.requires_grad and _grads():
        _recorded(dy=dy)
    if dy.shape != (n, classes):
        raise ValueError("dy must be n x C")
    dy, lddy = _rows(dy)
    dx = torch.empty(n, d, dtype=dt, device=device) if need_dx else None
    dA = torch.empty(A.shape, dtype=dt, device=device) if need_dA else None
    dB = torch.empty(B.shape, dtype=dt, device=device) if need_dB else None
    _call(at, _lib.load().lipcache_adapted_logits_backward, p, dy.data_ptr(), lddy, dx.data_ptr() if need_dx else None, d,
          dA.data_ptr() if need_dA else None, dB.data_ptr() if need_dB else None, ws.data_ptr(), ws.numel())
    return dx, dA, dB


def cross_entropy(logits: torch.Tensor, target: torch.Tensor, weight: torch.Tensor | None = None,
                  need_grad: bool = True, in_place: bool = False):
    """(loss, dlogits): loss_t = weight_t (logsumexp(z_t) - z_t[target_t]) and
    the gradient of the losses' sum; dlogits is None without need_grad, and
    overwrites logits with in_place.

    logits: n x C; target: n (int32; a value outside [0, C) ignores the row);
    weight: n (float32)."""
    ty, at, dt = _type(logits, "logits"), _gpu(logits, "logits"), logits.dtype
    _check(logits, "logits", 2, at, dt)
    _check(target, "target", 1, at, I32)
    if _grads() and (logits.requires_grad or weight is not None and weight.requires_grad):
        _recorded(logits=logits, weight=weight)
    n, c = logits.shape
    _int32(c)
    if len(target) != n:
        raise ValueError("target must have an entry per row of logits")
    if weight is not None:
        _check(weight, "weight", 1, at, F32)
        if len(weight) != n:
            raise ValueError("weight must have an entry per row of logits")
        weight = weight.contiguous()
    z, ldz = _rows(logits)
    if in_place and z is not logits:
        raise ValueError("in_place needs logits with dense rows")
    target = target.contiguous()
    device = z.device
    loss = torch.empty(n, dtype=F32, device=device)
    dz, ldd = None, c
    if need_grad:
        dz, ldd = (z, ldz) if in_place else (torch.empty(n, c, dtype=dt, device=device), c)
    _call(at, _lib.load().lipcache_cross_entropy, ty, z.data_ptr(), ldz, n, c, target.data_ptr(),
          None if weight is None else weight.data_ptr(), loss.data_ptr(), None if dz is None else dz.data_ptr(), ldd)
    if in_place and need_grad:
        _written(dz)
    return loss, dz


def _polynomials(coefficients, steps: int):
    """The 3 * steps coefficients: one triple for all steps, or one a step."""
    if type(coefficients) is tuple and all(type(c) is float or type(c) is int for c in coefficients):
        return _triples(coefficients, int(steps))  # (numbers alone: what is in a tensor or a list can change)
    return _flat(coefficients, steps)


@functools.lru_cache(maxsize=64)
def _triples(coefficients: tuple, steps: int):
    return _flat(coefficients, steps)


def _flat(coefficients, steps: int):
    flat = []
    for c in coefficients:
        if hasattr(c, "tolist"):
            c = c.tolist()
        flat += [float(v) for v in (c if hasattr(c, "__len__") else (c,))]
    if len(flat) == 3:
        flat *= max(int(steps), 0)
    if len(flat) != 3 * steps:
        raise ValueError("coefficients must be (a, b, c), or such a triple for each step")
    return (C.c_double * len(flat))(*flat)


def _matrices(t: torch.Tensor, name: str):
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be rows x cols or batch x rows x cols")
    _int32(*t.shape[-2:])
    return (1, *t.shape) if t.dim() == 2 else tuple(t.shape)


def orthogonalize(G: torch.Tensor, steps: int = 5, coefficients=QUINTIC, eps: float = 1e-7,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """Each matrix of G (rows x cols, or batch x rows x cols) with its singular
    values moved towards 1 by `steps` Newton-Schulz products: X = G / (|G| +
    eps), X <- aX + (bS + cSS)X with S = XX^T (on the smaller side).
    coefficients: (a, b, c), or a triple for each step."""
    ty = _type(G, "G")
    at, device = _gpu(G, "G"), G.device
    if _grads() and (G.requires_grad or out is not None and out.requires_grad):
        _recorded(G=G, out=out)
    batch, m, n = _matrices(G, "G")
    coef = _polynomials(coefficients, steps)
    # rows of any stride, as long as the matrices follow one another in it
    ld = n if m == 1 else G.stride(-2)
    if not (n == 1 or G.stride(-1) == 1) or ld < n or (batch > 1 and G.stride(0) != m * ld):
        G = G.contiguous()
        ld = n
    own = out is None
    if own:
        out = torch.empty(G.shape, dtype=G.dtype, device=device)
    else:
        _check(out, "out", G.dim(), at, G.dtype)
        if out.shape != G.shape or not out.is_contiguous():
            raise ValueError("out must have G's shape and be contiguous")
    ws = _workspace(_ortho_bytes(ty, batch, m, n), device)
    _call(at, _lib.load().lipcache_orthogonalize, ty, G.data_ptr(), ld, batch, m, n, int(steps), coef, float(eps),
          out.data_ptr(), ws.data_ptr(), ws.numel())
    if not own:
        _written(out)
    return out


def orthogonal_step(weight: torch.Tensor, grad: torch.Tensor, momentum: torch.Tensor, lr: float, beta: float = 0.95,
                    nesterov: bool = True, weight_decay: float = 0.0, steps: int = 5, coefficients=QUINTIC,
                    eps: float = 1e-7, out: tuple[torch.Tensor, torch.Tensor] | None = None):
    """One optimiser step with an orthogonalised direction; returns (weight,
    momentum), updated in place, or written to the two tensors of `out`.

    momentum <- beta momentum + (1 - beta) grad; direction O of the momentum
    (nesterov: of beta momentum + (1 - beta) grad); weight <- (1 - lr
    weight_decay) weight - lr sqrt(max(1, rows / cols)) O. weight and grad:
    float32 or bfloat16; momentum: float32; all rows x cols, or batch x rows x
    cols, contiguous."""
    wt, gt, at = _type(weight, "weight"), _type(grad, "grad"), _gpu(weight, "weight")
    batch, m, n = _matrices(weight, "weight")
    ow, om = (weight, momentum) if out is None else out
    if _grads() and (weight.requires_grad or grad.requires_grad or momentum.requires_grad or ow.requires_grad
                    or om.requires_grad):
        _recorded(**{"weight": weight, "grad": grad, "momentum": momentum, "out[0]": ow, "out[1]": om})
    shape, dims = weight.shape, weight.dim()
    for t, name, dtype in ((weight, "weight", weight.dtype), (grad, "grad", grad.dtype),
                           (momentum, "momentum", F32), (ow, "out[0]", weight.dtype),
                           (om, "out[1]", F32)):
        _check(t, name, dims, at, dtype)
        if t.shape != shape or not (t.is_contiguous() or t is grad):
            raise ValueError(f"{name} must have the weight's shape and be contiguous")
    grad = grad.contiguous()
    coef = _polynomials(coefficients, steps)
    ws = _workspace(_ortho_bytes(wt, batch, m, n), weight.device)
    _call(at, _lib.load().lipcache_orthogonal_step, wt, gt, weight.data_ptr(), grad.data_ptr(), momentum.data_ptr(),
          ow.data_ptr(), om.data_ptr(), batch, m, n, float(lr), float(beta), int(bool(nesterov)), float(weight_decay),
          int(steps), coef, float(eps), ws.data_ptr(), ws.numel())
    _written((ow, om))
    return ow, om


def operator_errors(device: torch.device | int | None = None) -> int:
    """Bounded device waits of these operators that expired since the library
    was loaded (synchronises the current stream)."""
    n = C.c_int64()
    with torch.cuda.device(device):
        check(_lib.load().lipcache_operator_errors(C.byref(n), torch.cuda.current_stream().cuda_stream))
    return n.value
