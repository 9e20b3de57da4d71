"""Operators of a language model's post-training step, on torch tensors.

They produce the K workers' gradients that ``GMC.step`` takes: log-probabilities
of given tokens, the clipped policy loss and the preference loss with the
gradient of the logits, and dropout whose masks follow from (seed, t, worker,
site). include/gmc.h states each operator; the compiled module behind this one checks
and marshals arguments and allocates outputs where none are given.

Logits are (n, vocab) CUDA tensors of float32, bfloat16 or float16 whose rows are
contiguous; a row stride larger than vocab is fine. Targets are int64, negative
where a token is not scored. Outputs are allocated on the stream of the call. A
gradient is contiguous where the logits are; beside a view with padded rows its rows
lie as the view's do, a few elements apart.

Nothing here is recorded by autograd: outputs have no grad_fn, also for logits that
require a gradient. It is had by ``logits.backward(result.dlogits)``, or from
``token_logp_backward``; a loss that is added to another one adds no gradient. Writing
into ``out`` raises that tensor's version, as torch's own writes in place do. With
``stream=`` the inputs are recorded on that stream (their memory is kept until the call
has run); what follows on another stream waits for it by the caller's own events.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import NamedTuple

from . import gmc as _gmc
from .gmc import GMCError, _check, _import_torch, load

MODULE_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_tokens.so")

_ops = None   # the compiled module, from the first call on


def _load():
    """Load _tokens.so (built in-tree) and hand it the library's entry points; raise
    ImportError if it is missing."""
    global _ops
    _import_torch()
    lib = load()
    if not os.path.exists(MODULE_PATH):
        raise ImportError(f"{MODULE_PATH} is not built; run `python -m paper_1905_12948_gb300.build`")
    spec = importlib.util.spec_from_file_location("_tokens", MODULE_PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.init(GMCError, *(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.gmc_token_logp, lib.gmc_token_logp_backward, lib.gmc_policy_loss, lib.gmc_preference_loss,
        lib.gmc_dropout)))
    module.init_more(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.gmc_token_scores, lib.gmc_token_scores_backward, lib.gmc_orthogonalize_workspace, lib.gmc_orthogonalize)))
    _ops = module
    return module


def _on(stream, t, name: str, *others):
    """The context of a call on another stream than the current one: the outputs belong to it, and the
    memory of t and the others is not handed out again before the call is done."""
    torch = _import_torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if stream.device_index != t.device.index:
        raise TypeError(f"stream must be one of {t.device}")
    for tensor in (t, *others):
        if isinstance(tensor, torch.Tensor) and tensor.is_cuda:
            tensor.record_stream(stream)
    return torch.cuda.stream(stream)


def token_logp(logits, targets, *, scale: float = 1.0, return_stats: bool = False, stream=None):
    """Log-probability of each row's target under softmax(scale * logits): n float32
    (gmc_token_logp). With ``return_stats`` also the (n, 2) float32 that
    ``token_logp_backward`` takes."""
    if stream is not None:
        with _on(stream, logits, "logits", targets):
            return token_logp(logits, targets, scale=scale, return_stats=return_stats)
    return (_ops or _load()).token_logp(logits, targets, scale, return_stats)


def token_logp_backward(logits, targets, stats, dlogp, *, scale: float = 1.0, out=None, stream=None):
    """Gradient of sum(dlogp * logp) in the logits (gmc_token_logp_backward), of the
    logits' dtype; ``out`` may be the logits themselves."""
    if stream is not None:
        with _on(stream, logits, "logits", targets, stats, dlogp, out):
            return token_logp_backward(logits, targets, stats, dlogp, scale=scale, out=out)
    return (_ops or _load()).token_logp_backward(logits, targets, stats, dlogp, scale, out)


class TokenScores(NamedTuple):
    """None in the place of what was not asked for. The float32 ones share one allocation: clone
    what is kept beyond the others, or saved without them (torch.save writes all of an allocation)."""
    logp: object         # float32 of the targets' shape, 0 where a token is not scored
    entropy: object      # (n,) float32
    top_logp: object     # (n, top) float32, larger ones first
    top_index: object    # (n, top) int64, the lower one first among equal logits
    stats: object        # (n, 4) float32, for token_scores_backward


def token_scores(logits, targets=None, *, top: int = 0, scale: float = 1.0, return_stats: bool = False,
                 stream=None) -> TokenScores:
    """Log-probabilities of given tokens, the entropy and the ``top`` most probable tokens of
    each row under softmax(scale * logits), in one pass (gmc_token_scores). ``targets``: (n,) or
    (n, given) int64, up to 64 a row; a row whose targets are all negative is not scored.
    Without targets every row is."""
    if stream is not None:
        with _on(stream, logits, "logits", targets):
            return token_scores(logits, targets, top=top, scale=scale, return_stats=return_stats)
    return TokenScores(*(_ops or _load()).token_scores(logits, targets, top, scale, return_stats))


def token_scores_backward(logits, targets, stats, dlogp=None, dentropy=None, *, scale: float = 1.0, out=None,
                          stream=None):
    """Gradient of sum(dlogp * logp) + sum(dentropy * entropy) in the logits
    (gmc_token_scores_backward), of the logits' dtype; ``out`` may be the logits themselves. The
    slopes of top alternatives are given as those of tokens: ``targets=scores.top_index`` (a row that is
    not finite, whose alternatives are -1, stays NaN)."""
    if stream is not None:
        with _on(stream, logits, "logits", targets, stats, dlogp, dentropy, out):
            return token_scores_backward(logits, targets, stats, dlogp, dentropy, scale=scale, out=out)
    return (_ops or _load()).token_scores_backward(logits, targets, stats, dlogp, dentropy, scale, out)


class PolicyLoss(NamedTuple):
    """loss, token_loss and logp share one allocation: clone what is kept beyond the others."""
    loss: object         # float32 scalar tensor: sum of weights * token_loss
    token_loss: object   # (n,) float32, 0 where a token is not scored
    logp: object         # (n,) float32, 0 where a token is not scored
    dlogits: object      # gradient of loss, or None


class PreferenceLoss(NamedTuple):
    """All but dlogits share one allocation: clone what is kept beyond the others."""
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
        if _ops is None:
            _load()
        self.lib = load()
        self.device = torch.device(device if device is not None else "cuda")
        if self.device.type != "cuda":
            raise ValueError("device must be a CUDA device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        h = _gmc._c_p()
        with torch.cuda.device(self.device):
            _check(self.lib.gmc_loss_create(ctypes.byref(h), int(max_rows), int(max_pairs)), "gmc_loss_create")
        self.h = h
        self._h = h.value

    def close(self) -> None:
        if getattr(self, "h", None):
            self.lib.gmc_loss_destroy(self.h)
            self.h = self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def policy(self, logits, targets, old_logp, advantages, *, weights=None, ref_logp=None,
               clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0, scale: float = 1.0,
               grad: bool = True, out=None, stream=None) -> PolicyLoss:
        """Clipped policy loss with a KL term, and its gradient in the logits
        (gmc_policy_loss). ``out`` may be the logits themselves."""
        if stream is not None:
            with _on(stream, logits, "logits", targets, old_logp, advantages, weights, ref_logp, out):
                return self.policy(logits, targets, old_logp, advantages, weights=weights, ref_logp=ref_logp,
                                   clip_low=clip_low, clip_high=clip_high, kl=kl, scale=scale, grad=grad, out=out)
        return PolicyLoss(*_ops.policy(self._h, self._index, logits, targets, old_logp, advantages, weights, ref_logp,
                                       clip_low, clip_high, kl, scale, grad, out))

    def preference(self, logits, targets, offsets, *, beta: float, smoothing: float = 0.0, ref_logp=None,
                   weights=None, scale: float = 1.0, grad: bool = True, out=None, stream=None) -> PreferenceLoss:
        """Preference loss on paired log ratios, and its gradient in the logits
        (gmc_preference_loss). ``offsets``: int64, 2 * pairs + 1 row numbers on the
        device, the preferred sequence of a pair first. ``out`` may be the logits
        themselves."""
        if stream is not None:
            with _on(stream, logits, "logits", targets, offsets, ref_logp, weights, out):
                return self.preference(logits, targets, offsets, beta=beta, smoothing=smoothing, ref_logp=ref_logp,
                                       weights=weights, scale=scale, grad=grad, out=out)
        return PreferenceLoss(*_ops.preference(self._h, self._index, logits, targets, offsets, beta, smoothing,
                                               ref_logp, weights, scale, grad, out))


def dropout(x, p: float, *, seed: int, t: int = 0, worker: int = 0, site: int = 0, residual=None, out=None,
            stream=None):
    """``residual`` + dropout of x, the mask that of (seed, t, worker, site)
    (gmc_dropout). x's first dimension is the workers' (one worker: ``x[None]``): x[k],
    whose elements are contiguous, is drawn as worker ``worker`` + k. p is rounded to a
    multiple of 2**-16 and the kept elements are divided by the share kept. ``out`` may
    be x or the residual."""
    if stream is not None:
        with _on(stream, x, "x", residual, out):
            return dropout(x, p, seed=seed, t=t, worker=worker, site=site, residual=residual, out=out)
    return (_ops or _load()).dropout(x, p, seed, t, worker, site, residual, out)


def dropout_backward(dout, p: float, *, seed: int, t: int = 0, worker: int = 0, site: int = 0, out=None, stream=None):
    """Gradient of ``dropout`` in x, from that of its output: the same mask on ``dout``."""
    return dropout(dout, p, seed=seed, t=t, worker=worker, site=site, out=out, stream=stream)
