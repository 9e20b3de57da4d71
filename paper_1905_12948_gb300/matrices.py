"""Operators on the gradients of weight matrices, on torch tensors.

``orthogonalize`` makes of the K workers' gradients of a matrix what ``GMC.step`` is to
compress: include/gmc.h states it; the compiled module behind this one checks and marshals
arguments, and allocates the output and the workspace on the stream of the call.

Nothing here is recorded by autograd. Writing into ``out`` raises that tensor's version,
as torch's own writes in place do. With ``stream=`` the inputs are recorded on that stream.
"""
from __future__ import annotations

from . import tokens as _tokens

# a, b, c of one step: those of the Muon optimiser
QUINTIC = (3.4445, -4.7750, 2.0315)


def orthogonalize(x, *, steps: int = 5, coefficients=QUINTIC, scale: float = 1.0, out=None, stream=None):
    """``scale`` * the orthogonalised matrices of x, by ``steps`` Newton-Schulz products
    X <- a X + (b A + c A^2) X, A = X X', from X = x / |x| (gmc_orthogonalize). x: (K, m, n), a
    matrix of each worker, or (m, n), of float32, bfloat16 or float16; a matrix's rows are
    contiguous, the workers' and the rows' strides are free, one matrix after the other or a row of each in
    turn: the part of a K x d gradient that is a
    matrix, ``grads[:, at: at + m * n].view(K, m, n)``, is taken as it lies.
    ``coefficients``: (a, b, c), or one such triple for each step. ``out`` may be x."""
    if stream is not None:
        with _tokens._on(stream, x, "x", out):
            return orthogonalize(x, steps=steps, coefficients=coefficients, scale=scale, out=out)
    return (_tokens._ops or _tokens._load()).orthogonalize(x, steps, coefficients, scale, out)
