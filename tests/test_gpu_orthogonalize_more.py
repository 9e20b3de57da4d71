"""Orthogonalised matrices: what waits order, time-outs, workspaces and strides. Bounds: scores_ref."""
import pytest

from test_gpu_orthogonalize import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,K,m,n", [("f32", 2, 200, 1000), ("f32", 1, 16, 5000), ("bf16", 2, 1000, 2050), ("f32", 3, 700, 2000)])
def test_other_matrices_in_turn(kind, K, m, n):
    """Diagonals and shares of sums come from other blocks, at the same places in each step and call: what an earlier
    step or matrix left there would show."""
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    some = [make(K, m, n, kind, seed=i, form=form) for i, form in enumerate(("noise", "layer", "noise"))]
    want = [orthogonalize(g) for g in some]
    for g, out in zip(some, want):
        check(g, out, kind)
    for _ in range(5):
        got = [orthogonalize(g) for g in some]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
