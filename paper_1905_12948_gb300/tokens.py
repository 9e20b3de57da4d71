"""Operators of a language model's post-training step, on torch tensors.

They produce the K workers' gradients that ``GMC.step`` takes: log-probabilities
of given tokens, the clipped policy loss and the preference loss with the
gradient of the logits, and dropout whose masks follow from (seed, t, worker,
site). include/gmc.h states each operator; here arguments are checked and
marshalled, and outputs allocated where none are given.

Logits are (n, vocab) CUDA tensors of float32, bfloat16 or float16 whose rows are
contiguous; a row stride larger than vocab is fine. Targets are int64, negative
where a token is not scored. Outputs are allocated on the stream of the call.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from . import gmc as _gmc
from .gmc import _check, _import_torch, load

_torch = None    # set with the library, on the first call
_lib = None
_f32 = _i64 = None
_DTYPES = {}     # torch dtype -> GMC_F32 / GMC_BF16 / GMC_F16
_current = None  # () -> the current device's index


def _setup() -> None:
    global _torch, _lib, _f32, _i64, _current
    torch = _import_torch()
    _f32, _i64 = torch.float32, torch.int64
    _DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    _current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _lib = load()
    _torch = torch


def _device(t, name: str) -> int:
    """The index of a CUDA tensor's device."""
    if _torch is None:
        _setup()
    if not isinstance(t, _torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    return t.get_device()


def _elsewhere(dev: int, stream):
    """None where the call can be made at once: on the current device and stream. Else
    the context to make it under, so that its outputs are allocated there too."""
    if stream is not None:
        if stream.device_index != dev:
            raise TypeError(f"stream must be one of cuda:{dev}")
        return _torch.cuda.stream(stream)
    return None if _current() == dev else _torch.cuda.device(dev)


def _rows(t, name: str):
    """Row stride of a 2-D CUDA tensor with contiguous rows."""
    if t.dim() != 2:
        raise TypeError(f"{name} must be 2-D")
    n, v = t.shape
    if t.is_contiguous():
        return n, v, v
    ld, step = t.stride()
    if step != 1 and v > 1:
        raise TypeError(f"{name}'s rows must be contiguous")
    if n <= 1:
        return n, v, v
    if ld < v:
        raise TypeError(f"{name}'s rows must not overlap")
    return n, v, ld


def _kind(t, name: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16")
    return code


def _vector(t, n: int, dtype, dev: int, name: str):
    if t is None:
        return None
    if not isinstance(t, _torch.Tensor) or not t.is_cuda or t.get_device() != dev:
        raise TypeError(f"{name} must be a CUDA tensor on cuda:{dev}")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor")
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements")
    return t.data_ptr()


def _gradient(logits, out, grad: bool, vocab: int):
    """(tensor, pointer, row stride) of the gradient's destination."""
    if not grad:
        return None, None, vocab
    if out is None:
        out = _torch.empty_like(logits, memory_format=_torch.contiguous_format)
        return out, out.data_ptr(), vocab
    if out is not logits and (not isinstance(out, _torch.Tensor) or out.shape != logits.shape
                              or out.dtype != logits.dtype or out.device != logits.device):
        raise TypeError("out must have the logits' shape, dtype and device")
    return out, out.data_ptr(), _rows(out, "out")[2]


def token_logp(logits, targets, *, scale: float = 1.0, return_stats: bool = False, stream=None):
    """Log-probability of each row's target under softmax(scale * logits): n float32
    (gmc_token_logp). With ``return_stats`` also the (n, 2) float32 that
    ``token_logp_backward`` takes."""
    dev = _device(logits, "logits")
    under = _elsewhere(dev, stream)
    if under is not None:
        with under:
            return token_logp(logits, targets, scale=scale, return_stats=return_stats)
    n, vocab, ld = _rows(logits, "logits")
    code = _kind(logits, "logits")
    tgt = _vector(targets, n, _i64, dev, "targets")
    where = logits.device
    logp = _torch.empty(n, dtype=_f32, device=where)
    stats = _torch.empty((n, 2), dtype=_f32, device=where) if return_stats else None
    _check(_lib.gmc_token_logp(logits.data_ptr(), code, n, vocab, ld, scale, tgt, logp.data_ptr(),
                               stats.data_ptr() if return_stats else None, _gmc._raw_stream(dev)), "gmc_token_logp")
    return (logp, stats) if return_stats else logp


def token_logp_backward(logits, targets, stats, dlogp, *, scale: float = 1.0, out=None, stream=None):
    """Gradient of sum(dlogp * logp) in the logits (gmc_token_logp_backward), of the
    logits' dtype; ``out`` may be the logits themselves."""
    dev = _device(logits, "logits")
    under = _elsewhere(dev, stream)
    if under is not None:
        with under:
            return token_logp_backward(logits, targets, stats, dlogp, scale=scale, out=out)
    n, vocab, ld = _rows(logits, "logits")
    code = _kind(logits, "logits")
    tgt = _vector(targets, n, _i64, dev, "targets")
    st = _vector(stats, 2 * n, _f32, dev, "stats")
    g = _vector(dlogp, n, _f32, dev, "dlogp")
    out, optr, old = _gradient(logits, out, True, vocab)
    _check(_lib.gmc_token_logp_backward(logits.data_ptr(), code, n, vocab, ld, scale, tgt, st, g, optr, old,
                                        _gmc._raw_stream(dev)), "gmc_token_logp_backward")
    return out


class PolicyLoss(NamedTuple):
    loss: object         # float32 scalar tensor: sum of weights * token_loss
    token_loss: object   # (n,) float32, 0 where a token is not scored
    logp: object         # (n,) float32, 0 where a token is not scored
    dlogits: object      # gradient of loss, or None


class PreferenceLoss(NamedTuple):
    loss: object         # float32 scalar tensor: sum of weights * pair_loss
    pair_loss: object    # (pairs,) float32
    seq_ratio: object    # (2 * pairs,) float32: summed log ratio of each sequence
    logp: object         # (n,) float32
    dlogits: object      # gradient of loss, or None


class TokenLoss:
    """Workspace of the two losses (gmc_loss_create), for up to ``max_rows`` rows and
    ``max_pairs`` pairs a call. Calls with one instance are ordered by the caller."""

    def __init__(self, max_rows: int, max_pairs: int = 0, device=None):
        if _torch is None:
            _setup()
        self.lib = _lib
        self.device = _torch.device(device if device is not None else "cuda")
        if self.device.index is None:
            self.device = _torch.device("cuda", _torch.cuda.current_device())
        self.index = self.device.index
        h = _gmc._c_p()
        with _torch.cuda.device(self.device):
            _check(_lib.gmc_loss_create(ctypes.byref(h), int(max_rows), int(max_pairs)), "gmc_loss_create")
        self.h = h

    def close(self) -> None:
        if getattr(self, "h", None):
            self.lib.gmc_loss_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _elsewhere(self, logits, stream):
        if _device(logits, "logits") != self.index:
            raise TypeError(f"logits must be on {self.device}")
        return _elsewhere(self.index, stream)

    def policy(self, logits, targets, old_logp, advantages, *, weights=None, ref_logp=None,
               clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0, scale: float = 1.0,
               grad: bool = True, out=None, stream=None) -> PolicyLoss:
        """Clipped policy loss with a KL term, and its gradient in the logits
        (gmc_policy_loss). ``out`` may be the logits themselves."""
        under = self._elsewhere(logits, stream)
        if under is not None:
            with under:
                return self.policy(logits, targets, old_logp, advantages, weights=weights, ref_logp=ref_logp,
                                   clip_low=clip_low, clip_high=clip_high, kl=kl, scale=scale, grad=grad, out=out)
        dev, where = self.index, self.device
        n, vocab, ld = _rows(logits, "logits")
        code = _kind(logits, "logits")
        tgt = _vector(targets, n, _i64, dev, "targets")
        old = _vector(old_logp, n, _f32, dev, "old_logp")
        adv = _vector(advantages, n, _f32, dev, "advantages")
        ref = _vector(ref_logp, n, _f32, dev, "ref_logp")
        w = _vector(weights, n, _f32, dev, "weights")
        out, optr, dld = _gradient(logits, out, grad, vocab)
        loss = _torch.empty((), dtype=_f32, device=where)
        token_loss = _torch.empty(n, dtype=_f32, device=where)
        logp = _torch.empty(n, dtype=_f32, device=where)
        _check(_lib.gmc_policy_loss(self.h, logits.data_ptr(), code, n, vocab, ld, scale, tgt, old, ref, adv, w,
                                    clip_low, clip_high, kl, loss.data_ptr(), token_loss.data_ptr(), logp.data_ptr(),
                                    optr, dld, _gmc._raw_stream(dev)), "gmc_policy_loss")
        return PolicyLoss(loss, token_loss, logp, out)

    def preference(self, logits, targets, offsets, *, beta: float, smoothing: float = 0.0, ref_logp=None,
                   weights=None, scale: float = 1.0, grad: bool = True, out=None, stream=None) -> PreferenceLoss:
        """Preference loss on paired log ratios, and its gradient in the logits
        (gmc_preference_loss). ``offsets``: int64, 2 * pairs + 1 row numbers on the
        device, the preferred sequence of a pair first. ``out`` may be the logits
        themselves."""
        under = self._elsewhere(logits, stream)
        if under is not None:
            with under:
                return self.preference(logits, targets, offsets, beta=beta, smoothing=smoothing, ref_logp=ref_logp,
                                       weights=weights, scale=scale, grad=grad, out=out)
        dev, where = self.index, self.device
        n, vocab, ld = _rows(logits, "logits")
        code = _kind(logits, "logits")
        tgt = _vector(targets, n, _i64, dev, "targets")
        if not isinstance(offsets, _torch.Tensor) or offsets.numel() % 2 != 1:
            raise ValueError("offsets must have 2 * pairs + 1 elements")
        pairs = offsets.numel() // 2
        off = _vector(offsets, 2 * pairs + 1, _i64, dev, "offsets")
        ref = _vector(ref_logp, n, _f32, dev, "ref_logp")
        w = _vector(weights, pairs, _f32, dev, "weights")
        out, optr, dld = _gradient(logits, out, grad, vocab)
        loss = _torch.empty((), dtype=_f32, device=where)
        each = _torch.empty(pairs, dtype=_f32, device=where)
        ratio = _torch.empty(2 * pairs, dtype=_f32, device=where)
        logp = _torch.empty(n, dtype=_f32, device=where)
        _check(_lib.gmc_preference_loss(self.h, logits.data_ptr(), code, n, vocab, ld, scale, tgt, off, pairs, ref, w,
                                        beta, smoothing, loss.data_ptr(), each.data_ptr(), ratio.data_ptr(),
                                        logp.data_ptr(), optr, dld, _gmc._raw_stream(dev)), "gmc_preference_loss")
        return PreferenceLoss(loss, each, ratio, logp, out)


def _workers(u, x, K: int, n: int, name: str):
    """(pointer, worker stride) of one of dropout's tensors."""
    if u is not x and (not isinstance(u, _torch.Tensor) or u.shape != x.shape or u.dtype != x.dtype
                       or u.device != x.device):
        raise TypeError(f"{name} must be a tensor of x's shape, dtype and device")
    if u.is_contiguous():
        return u.data_ptr(), n
    if K == 0 or not u[0].is_contiguous() or (K > 1 and u.stride(0) < n):
        raise TypeError(f"each worker's part of {name} must be contiguous, and none overlap")
    return u.data_ptr(), u.stride(0)


def dropout(x, p: float, *, seed: int, t: int = 0, worker: int = 0, site: int = 0, residual=None, out=None,
            stream=None):
    """``residual`` + dropout of x, the mask that of (seed, t, worker, site)
    (gmc_dropout). x's first dimension is the workers' (one worker: ``x[None]``): x[k],
    whose elements are contiguous, is drawn as worker ``worker`` + k. p is rounded to a
    multiple of 2**-16 and the kept elements are divided by the share kept. ``out`` may
    be x or the residual."""
    dev = _device(x, "x")
    under = _elsewhere(dev, stream)
    if under is not None:
        with under:
            return dropout(x, p, seed=seed, t=t, worker=worker, site=site, residual=residual, out=out)
    if x.dim() < 2:
        raise TypeError("x must have the workers as its first dimension")
    code = _kind(x, "x")
    K = x.shape[0]
    n = x.numel() // K if K else 0
    px, ldx = _workers(x, x, K, n, "x")
    pr, ldr = _workers(residual, x, K, n, "residual") if residual is not None else (None, 0)
    if out is None:
        out = _torch.empty_like(x, memory_format=_torch.contiguous_format)
        po, ldo = out.data_ptr(), n
    else:
        po, ldo = _workers(out, x, K, n, "out")
    _check(_lib.gmc_dropout(px, ldx, pr, ldr, po, ldo, code, worker, K, n, p, seed & ((1 << 64) - 1), t, site,
                            _gmc._raw_stream(dev)), "gmc_dropout")
    return out


def dropout_backward(dout, p: float, *, seed: int, t: int = 0, worker: int = 0, site: int = 0, out=None, stream=None):
    """Gradient of ``dropout`` in x, from that of its output: the same mask on ``dout``."""
    return dropout(dout, p, seed=seed, t=t, worker=worker, site=site, out=out, stream=stream)
