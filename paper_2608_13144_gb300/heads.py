"""Operators that train and serve the heads a cache certifies (argument
marshalling only; include/lipcache.h states the formulas).

* adapted_logits, adapted_logits_backward: logits of rows under a shared head
  and each row's own low-rank adapter, and their gradients;
* cross_entropy: per-row losses and the gradient of the logits in one call;
* orthogonalize, orthogonal_step: Newton-Schulz orthogonalisation of a
  matrix, and the optimiser step that uses it.

Tensors are float32 or bfloat16 on one GPU; the work runs on the current
stream. Rows may be strided (a slice of a wider matrix); other layouts are
copied first. Scratch comes from PyTorch's allocator, so calls can be captured
into a CUDA graph.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import _lib
from ._lib import Adapted, LipCacheError, check

TYPES = {torch.float32: _lib.F32, torch.bfloat16: _lib.BF16}
#: a, b, c of X <- aX + (bS + cSS)X, S = XX^T: singular values move fast to
#: about 1 (0.7 to 1.2) within five steps.
QUINTIC = (3.4445, -4.7750, 2.0315)


def _stream(device: torch.device):
    return torch.cuda.current_stream(device).cuda_stream


def _type(t: torch.Tensor, name: str) -> int:
    try:
        return TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}") from None


def _check(t: torch.Tensor, name: str, dims: int, device: torch.device, dtype: torch.dtype) -> None:
    if t.dtype == dtype and t.dim() == dims and t.device == device:
        return
    if t.device != device:
        raise ValueError(f"{name} must be on one GPU with the other tensors, not on {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    raise ValueError(f"{name} must have {dims} dimensions, not {t.dim()}")


def _gpu(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU, not on {t.device}")
    return t.device


class _On:
    """The device a call runs on, made current only where another one is."""

    __slots__ = ("other",)

    def __init__(self, device: torch.device):
        self.other = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self.other is not None:
            self.other.__enter__()

    def __exit__(self, *exc):
        if self.other is not None:
            self.other.__exit__(*exc)


def _rows(t: torch.Tensor) -> torch.Tensor:
    """`t` (2-D) with neighbours in a row next to each other in memory and rows that do not overlap."""
    if t.shape[1] <= 1 or t.shape[0] <= 1:
        return t if t.is_contiguous() else t.contiguous()
    return t if t.stride(1) == 1 and t.stride(0) >= t.shape[1] else t.contiguous()


def _ld(t: torch.Tensor) -> int:
    return max(t.stride(0), t.shape[1]) if t.shape[0] > 1 else t.shape[1]


def _workspace(nbytes: int, device: torch.device) -> torch.Tensor:
    if nbytes < 0:
        raise LipCacheError(_lib.E_INVALID, _lib.load().lipcache_last_error().decode())
    return torch.empty(nbytes if nbytes > 256 else 256, dtype=torch.uint8, device=device)


@functools.lru_cache(maxsize=1024)
def _adapted_bytes(ty: int, d: int, classes: int, G: int, r: int, n: int, backward: int) -> int:
    p = Adapted(ty, d, classes, G, r, 0, n)
    return _lib.load().lipcache_adapted_workspace(C.byref(p), backward)


@functools.lru_cache(maxsize=1024)
def _ortho_bytes(ty: int, batch: int, m: int, n: int) -> int:
    return _lib.load().lipcache_orthogonalize_workspace(ty, batch, m, n)


def _describe(x, W, A, B, adapter, scales):
    """The operator's description, and the tensors it points into."""
    ty, dev, dt = _type(x, "x"), _gpu(x, "x"), x.dtype
    _check(x, "x", 2, dev, dt)
    _check(W, "W", 2, dev, dt)
    _check(A, "A", 3, dev, dt)
    _check(B, "B", 3, dev, dt)
    _check(adapter, "adapter", 1, dev, torch.int32)
    (n, d), classes, (G, r, _) = x.shape, W.shape[0], A.shape
    if W.shape[1] != d or tuple(A.shape) != (G, r, d) or tuple(B.shape) != (G, classes, r) or adapter.shape[0] != n:
        raise ValueError("x must be n x d, W C x d, A G x r x d, B G x C x r and adapter must have n entries")
    if scales is not None:
        _check(scales, "scales", 1, dev, torch.float32)
        if scales.shape[0] != G:
            raise ValueError("scales must have an entry per adapter")
        scales = scales.contiguous()
    x, W, A, B, adapter = _rows(x), _rows(W), A.contiguous(), B.contiguous(), adapter.contiguous()
    p = Adapted(ty, d, classes, G, r, 0, n, x.data_ptr(), _ld(x), W.data_ptr(), _ld(W), A.data_ptr(), B.data_ptr(),
                adapter.data_ptr(), scales.data_ptr() if scales is not None else None)
    return p, (x, W, A, B, adapter, scales)


def adapted_logits(x: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor, adapter: torch.Tensor,
                   bias: torch.Tensor | None = None, scales: torch.Tensor | None = None,
                   out: torch.Tensor | None = None) -> torch.Tensor:
    """y_t = W x_t + bias + scales[g] B_g (A_g x_t), g = adapter[t].

    x: n x d; W: C x d; A: G x r x d; B: G x C x r; adapter: n (int32; a value
    outside [0, G) means no adapter); bias: C (float32); scales: G (float32)."""
    p, keep = _describe(x, W, A, B, adapter, scales)
    if bias is not None:
        _check(bias, "bias", 1, x.device, torch.float32)
        if bias.shape[0] != p.classes:
            raise ValueError("bias must have C entries")
        bias = bias.contiguous()
    if out is None:
        out = torch.empty(p.tokens, p.classes, dtype=x.dtype, device=x.device)
    else:
        _check(out, "out", 2, x.device, x.dtype)
        if tuple(out.shape) != (p.tokens, p.classes) or _rows(out) is not out:
            raise ValueError("out must be n x C with dense rows")
    L = _lib.load()
    ws = _workspace(_adapted_bytes(p.type, p.d, p.classes, p.adapters, p.rank, p.tokens, 0), x.device)
    with _On(x.device):
        check(L.lipcache_adapted_logits(C.byref(p), bias.data_ptr() if bias is not None else None, out.data_ptr(),
                                        _ld(out), ws.data_ptr(), ws.numel(), _stream(x.device)))
    return out


def adapted_logits_backward(dy: torch.Tensor, x: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                            adapter: torch.Tensor, scales: torch.Tensor | None = None, need_dx: bool = True,
                            need_dA: bool = True, need_dB: bool = True):
    """(dx, dA, dB) of adapted_logits for the gradient dy (n x C) of its
    result; W and bias are held fixed. An output that is not needed is None."""
    p, keep = _describe(x, W, A, B, adapter, scales)
    _check(dy, "dy", 2, x.device, x.dtype)
    if tuple(dy.shape) != (p.tokens, p.classes):
        raise ValueError("dy must be n x C")
    dy = _rows(dy)
    dx = torch.empty(p.tokens, p.d, dtype=x.dtype, device=x.device) if need_dx else None
    dA = torch.empty(A.shape, dtype=x.dtype, device=x.device) if need_dA else None
    dB = torch.empty(B.shape, dtype=x.dtype, device=x.device) if need_dB else None
    L = _lib.load()
    ws = _workspace(_adapted_bytes(p.type, p.d, p.classes, p.adapters, p.rank, p.tokens, 1), x.device)
    with _On(x.device):
        check(L.lipcache_adapted_logits_backward(C.byref(p), dy.data_ptr(), _ld(dy),
                                                 dx.data_ptr() if need_dx else None, p.d,
                                                 dA.data_ptr() if need_dA else None,
                                                 dB.data_ptr() if need_dB else None, ws.data_ptr(), ws.numel(),
                                                 _stream(x.device)))
    return dx, dA, dB


def cross_entropy(logits: torch.Tensor, target: torch.Tensor, weight: torch.Tensor | None = None,
                  need_grad: bool = True, in_place: bool = False):
    """(loss, dlogits): loss_t = weight_t (logsumexp(z_t) - z_t[target_t]) and
    the gradient of the losses' sum; dlogits is None without need_grad, and
    overwrites logits with in_place.

    logits: n x C; target: n (int32; a value outside [0, C) ignores the row);
    weight: n (float32)."""
    ty, dev = _type(logits, "logits"), _gpu(logits, "logits")
    _check(logits, "logits", 2, dev, logits.dtype)
    _check(target, "target", 1, dev, torch.int32)
    n, c = logits.shape
    if target.shape[0] != n:
        raise ValueError("target must have an entry per row of logits")
    if weight is not None:
        _check(weight, "weight", 1, dev, torch.float32)
        if weight.shape[0] != n:
            raise ValueError("weight must have an entry per row of logits")
        weight = weight.contiguous()
    z = _rows(logits)
    if in_place and z is not logits:
        raise ValueError("in_place needs logits with dense rows")
    target = target.contiguous()
    loss = torch.empty(n, dtype=torch.float32, device=z.device)
    dz = None
    if need_grad:
        dz = z if in_place else torch.empty(n, c, dtype=z.dtype, device=z.device)
    with _On(dev):
        check(_lib.load().lipcache_cross_entropy(ty, z.data_ptr(), _ld(z), n, c, target.data_ptr(),
                                                 weight.data_ptr() if weight is not None else None, loss.data_ptr(),
                                                 dz.data_ptr() if need_grad else None, _ld(dz) if need_grad else c,
                                                 _stream(z.device)))
    return loss, dz


def _polynomials(coefficients, steps: int):
    """The 3 * steps coefficients: one triple for all steps, or one a step."""
    if isinstance(coefficients, tuple):
        return _triples(coefficients, int(steps))
    return _flat(coefficients, steps)


@functools.lru_cache(maxsize=64)
def _triples(coefficients: tuple, steps: int):
    return _flat(coefficients, steps)


def _flat(coefficients, steps: int):
    flat = [float(v) for c in coefficients for v in (c if hasattr(c, "__len__") else (c,))]
    if len(flat) == 3:
        flat *= max(int(steps), 0)
    if len(flat) != 3 * steps:
        raise ValueError("coefficients must be (a, b, c), or such a triple for each step")
    return (C.c_double * len(flat))(*flat)


def _matrices(t: torch.Tensor, name: str):
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be rows x cols or batch x rows x cols")
    return (1, *t.shape) if t.dim() == 2 else tuple(t.shape)


def orthogonalize(G: torch.Tensor, steps: int = 5, coefficients=QUINTIC, eps: float = 1e-7,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """Each matrix of G (rows x cols, or batch x rows x cols) with its singular
    values moved towards 1 by `steps` Newton-Schulz products: X = G / (|G| +
    eps), X <- aX + (bS + cSS)X with S = XX^T (on the smaller side).
    coefficients: (a, b, c), or a triple for each step."""
    ty = _type(G, "G")
    dev = _gpu(G, "G")
    batch, m, n = _matrices(G, "G")
    coef = _polynomials(coefficients, steps)
    # rows of any stride, as long as the matrices follow one another in it
    ld = n if m == 1 else G.stride(-2)
    if not (n == 1 or G.stride(-1) == 1) or ld < n or (batch > 1 and G.stride(0) != m * ld):
        G = G.contiguous()
        ld = n
    if out is None:
        out = torch.empty(G.shape, dtype=G.dtype, device=G.device)
    else:
        _check(out, "out", G.dim(), dev, G.dtype)
        if out.shape != G.shape or not out.is_contiguous():
            raise ValueError("out must have G's shape and be contiguous")
    L = _lib.load()
    ws = _workspace(_ortho_bytes(ty, batch, m, n), dev)
    with _On(dev):
        check(L.lipcache_orthogonalize(ty, G.data_ptr(), ld, batch, m, n, int(steps), coef, float(eps),
                                       out.data_ptr(), ws.data_ptr(), ws.numel(), _stream(G.device)))
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
    wt, gt, dev = _type(weight, "weight"), _type(grad, "grad"), _gpu(weight, "weight")
    batch, m, n = _matrices(weight, "weight")
    ow, om = (weight, momentum) if out is None else out
    for t, name, dtype in ((weight, "weight", weight.dtype), (grad, "grad", grad.dtype),
                           (momentum, "momentum", torch.float32), (ow, "out[0]", weight.dtype),
                           (om, "out[1]", torch.float32)):
        _check(t, name, weight.dim(), dev, dtype)
        if t.shape != weight.shape or (name != "grad" and not t.is_contiguous()):
            raise ValueError(f"{name} must have the weight's shape and be contiguous")
    grad = grad.contiguous()
    coef = _polynomials(coefficients, steps)
    L = _lib.load()
    ws = _workspace(_ortho_bytes(wt, batch, m, n), dev)
    with _On(dev):
        check(L.lipcache_orthogonal_step(wt, gt, weight.data_ptr(), grad.data_ptr(), momentum.data_ptr(),
                                         ow.data_ptr(), om.data_ptr(), batch, m, n, float(lr), float(beta),
                                         int(bool(nesterov)), float(weight_decay), int(steps), coef, float(eps),
                                         ws.data_ptr(), ws.numel(), _stream(weight.device)))
    return ow, om


def operator_errors(device: torch.device | int | None = None) -> int:
    """Bounded device waits of these operators that expired since the library
    was loaded (synchronises the current stream)."""
    n = C.c_int64()
    with torch.cuda.device(device):
        check(_lib.load().lipcache_operator_errors(C.byref(n), _stream(torch.device("cuda", torch.cuda.current_device()))))
    return n.value
