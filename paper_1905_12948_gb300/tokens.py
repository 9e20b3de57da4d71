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
from typing import NamedTuple, Optional

from .gmc import _check, _i64, _import_torch, _stream_ptr, load
from . import gmc as _gmc

_DTYPES = None   # torch dtype -> GMC_F32 / GMC_BF16 / GMC_F16


def _dtype(t, name: str) -> int:
    global _DTYPES
    if _DTYPES is None:
        torch = _import_torch()
        _DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16")
    return code


class _On:
    """The device and the stream of a call: outputs are allocated and the library is
    called under them."""

    def __init__(self, device, stream):
        torch = _import_torch()
        self.stream = stream
        self.swap = None
        if stream is not None:
            self.swap = torch.cuda.stream(stream)
        elif torch.cuda.current_device() != device.index:
            self.swap = torch.cuda.device(device)

    def __enter__(self):
        if self.swap is not None:
            self.swap.__enter__()
        return _stream_ptr(self.stream)

    def __exit__(self, *exc):
        if self.swap is not None:
            self.swap.__exit__(*exc)


def _rows(t, name: str, like=None):
    """(pointer, row stride) of a 2-D CUDA tensor with contiguous rows."""
    torch = _import_torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise TypeError(f"{name} must be 2-D with contiguous rows")
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise TypeError(f"{name} must have the shape, dtype and device of {like.shape}, {like.dtype}, {like.device}")
    n, v = t.shape
    ld = t.stride(0) if n > 1 else v
    if ld < v:
        raise TypeError(f"{name}'s rows must not overlap")
    return t.data_ptr(), ld


def _vector(t, n: int, dtype, device, name: str) -> Optional[int]:
    if t is None:
        return None
    torch = _import_torch()
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise TypeError(f"{name} must be a CUDA tensor on {device}")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor")
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements")
    return t.data_ptr()


def token_logp(logits, targets, *, scale: float = 1.0, return_stats: bool = False, stream=None):
    """Log-probability of each row's target under softmax(scale * logits): n float32
    (gmc_token_logp). With ``return_stats`` also the (n, 2) float32 that
    ``token_logp_backward`` takes."""
    torch = _import_torch()
    ptr, ld = _rows(logits, "logits")
    n, vocab = logits.shape
    dev = logits.device
    tgt = _vector(targets, n, torch.int64, dev, "targets")
    with _On(dev, stream) as s:
        logp = torch.empty(n, dtype=torch.float32, device=dev)
        stats = torch.empty((n, 2), dtype=torch.float32, device=dev) if return_stats else None
        _check(load().gmc_token_logp(ptr, _dtype(logits, "logits"), n, vocab, ld, scale, tgt, logp.data_ptr(),
                                     stats.data_ptr() if return_stats else None, s), "gmc_token_logp")
    return (logp, stats) if return_stats else logp


def token_logp_backward(logits, targets, stats, dlogp, *, scale: float = 1.0, out=None, stream=None):
    """Gradient of sum(dlogp * logp) in the logits (gmc_token_logp_backward), of the
    logits' dtype; ``out`` may be the logits themselves."""
    torch = _import_torch()
    ptr, ld = _rows(logits, "logits")
    n, vocab = logits.shape
    dev = logits.device
    tgt = _vector(targets, n, torch.int64, dev, "targets")
    st = _vector(stats, 2 * n, torch.float32, dev, "stats")
    g = _vector(dlogp, n, torch.float32, dev, "dlogp")
    with _On(dev, stream) as s:
        if out is None:
            out = torch.empty((n, vocab), dtype=logits.dtype, device=dev)
        optr, old = _rows(out, "out", logits)
        _check(load().gmc_token_logp_backward(ptr, _dtype(logits, "logits"), n, vocab, ld, scale, tgt, st, g, optr,
                                              old, s), "gmc_token_logp_backward")
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
        torch = _import_torch()
        self.lib = load()
        self.device = torch.device(device if device is not None else "cuda")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        h = _gmc._c_p()
        with torch.cuda.device(self.device):
            _check(self.lib.gmc_loss_create(ctypes.byref(h), int(max_rows), int(max_pairs)), "gmc_loss_create")
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

    def _logits(self, logits, targets):
        torch = _import_torch()
        ptr, ld = _rows(logits, "logits")
        if logits.device != self.device:
            raise TypeError(f"logits must be on {self.device}")
        return ptr, ld, _vector(targets, logits.shape[0], torch.int64, self.device, "targets")

    def _gradient(self, logits, out, grad: bool):
        torch = _import_torch()
        if not grad:
            return None, None, logits.shape[1]
        if out is None:
            out = torch.empty(logits.shape, dtype=logits.dtype, device=self.device)
        return (out, *_rows(out, "out", logits))

    def policy(self, logits, targets, old_logp, advantages, *, weights=None, ref_logp=None,
               clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0, scale: float = 1.0,
               grad: bool = True, out=None, stream=None) -> PolicyLoss:
        """Clipped policy loss with a KL term, and its gradient in the logits
        (gmc_policy_loss). ``out`` may be the logits themselves."""
        torch = _import_torch()
        ptr, ld, tgt = self._logits(logits, targets)
        n, vocab = logits.shape
        f32, dev = torch.float32, self.device
        old = _vector(old_logp, n, f32, dev, "old_logp")
        adv = _vector(advantages, n, f32, dev, "advantages")
        ref = _vector(ref_logp, n, f32, dev, "ref_logp")
        w = _vector(weights, n, f32, dev, "weights")
        with _On(dev, stream) as s:
            # one allocation for the loss and the rows' outputs
            buf = torch.empty(2 * n + 1, dtype=f32, device=dev)
            base = buf.data_ptr()
            out, optr, old_ = self._gradient(logits, out, grad)
            _check(self.lib.gmc_policy_loss(self.h, ptr, _dtype(logits, "logits"), n, vocab, ld, scale, tgt, old,
                                            ref, adv, w, clip_low, clip_high, kl, base + 8 * n, base, base + 4 * n,
                                            optr, old_, s), "gmc_policy_loss")
        return PolicyLoss(buf[2 * n], buf[:n], buf[n: 2 * n], out)

    def preference(self, logits, targets, offsets, *, beta: float, smoothing: float = 0.0, ref_logp=None,
                   weights=None, scale: float = 1.0, grad: bool = True, out=None, stream=None) -> PreferenceLoss:
        """Preference loss on paired log ratios, and its gradient in the logits
        (gmc_preference_loss). ``offsets``: int64, 2 * pairs + 1 row numbers on the
        device, the preferred sequence of a pair first. ``out`` may be the logits
        themselves."""
        torch = _import_torch()
        ptr, ld, tgt = self._logits(logits, targets)
        n, vocab = logits.shape
        f32, dev = torch.float32, self.device
        if not isinstance(offsets, torch.Tensor) or offsets.numel() % 2 != 1:
            raise ValueError("offsets must have 2 * pairs + 1 elements")
        pairs = offsets.numel() // 2
        off = _vector(offsets, 2 * pairs + 1, torch.int64, dev, "offsets")
        ref = _vector(ref_logp, n, f32, dev, "ref_logp")
        w = _vector(weights, pairs, f32, dev, "weights")
        with _On(dev, stream) as s:
            buf = torch.empty(n + 3 * pairs + 1, dtype=f32, device=dev)
            logp, seq, each, loss = buf.split([n, 2 * pairs, pairs, 1])
            out, optr, old_ = self._gradient(logits, out, grad)
            _check(self.lib.gmc_preference_loss(self.h, ptr, _dtype(logits, "logits"), n, vocab, ld, scale, tgt, off,
                                                pairs, ref, w, beta, smoothing, loss.data_ptr(), each.data_ptr(),
                                                seq.data_ptr(), logp.data_ptr(), optr, old_, s),
                   "gmc_preference_loss")
        return PreferenceLoss(loss[0], each, seq, logp, out)


def dropout(x, p: float, *, seed: int, t: int = 0, worker: int = 0, site: int = 0, residual=None, out=None,
            stream=None):
    """``residual`` + dropout of x, the mask that of (seed, t, worker, site)
    (gmc_dropout). x's first dimension is the workers' (one worker: ``x[None]``): x[k],
    whose elements are contiguous, is drawn as worker ``worker`` + k. p is rounded to a
    multiple of 2**-16 and the kept elements are divided by the share kept. ``out`` may
    be x or the residual."""
    torch = _import_torch()
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a CUDA tensor")
    if x.dim() < 2:
        raise TypeError("x must have the workers as its first dimension")
    dev, K = x.device, x.shape[0]
    n = x.numel() // K if K else 0
    code = _dtype(x, "x")
    with _On(dev, stream) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=dev)
        ptrs = []
        for u, name in ((x, "x"), (residual, "residual"), (out, "out")):
            if u is None:
                ptrs += [None, 0]
                continue
            if u is not x and (not isinstance(u, torch.Tensor) or u.shape != x.shape or u.dtype != x.dtype
                               or u.device != dev):
                raise TypeError(f"{name} must be a tensor of x's shape, dtype and device")
            if not u.is_contiguous() and (K == 0 or not u[0].is_contiguous() or (K > 1 and u.stride(0) < n)):
                raise TypeError(f"each worker's part of {name} must be contiguous, and none overlap")
            ptrs += [u.data_ptr(), n if u.is_contiguous() else u.stride(0)]
        _check(load().gmc_dropout(*ptrs, code, int(worker), K, n, float(p), int(seed) & ((1 << 64) - 1),
                                  int(t), int(site), s), "gmc_dropout")
    return out


def dropout_backward(dout, p: float, *, seed: int, t: int = 0, worker: int = 0, site: int = 0, out=None, stream=None):
    """Gradient of ``dropout`` in x, from that of its output: the same mask on ``dout``."""
    return dropout(dout, p, seed=seed, t=t, worker=worker, site=site, out=out, stream=stream)
