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


def errors_of_all(g, out, kind):
    """As test_gpu_orthogonalize_limits: errors of single small matrices are small by chance as well, so those of all are compared,
    and each with the largest."""
    import torch

    import scores_ref as ref
    want = ref.products(g)
    off, size = (out.double() - want).flatten(1).norm(dim=1), want.flatten(1).norm(dim=1)
    plain = (ref.in_float32(g) - want).flatten(1).norm(dim=1) + (ref.rounded(g, fine=kind != "bf16") - want).flatten(1).norm(dim=1)
    last = torch.finfo(out.dtype).eps / 2 * size
    assert off.norm() <= 2 * plain.norm() + last.norm()
    assert (off <= 2 * (plain / size).max() * size + last).all()


@pytest.mark.parametrize("kind,K,m,n", [("bf16", 9_001, 129, 131), ("f32", 5_003, 131, 129)])
def test_matrices_in_slices(kind, K, m, n):
    """More than one workspace holds: slices, the last of them smaller; in place."""
    import torch
    from paper_1905_12948_gb300 import load, orthogonalize
    code = {"f32": 0, "bf16": 1}[kind]
    need = load().gmc_orthogonalize_workspace
    assert need(code, K, m, n) < 0.75 * K / 1000 * need(code, 1000, m, n)
    g = make(K, m, n, kind)
    out = orthogonalize(g.clone())
    same = g.clone()
    assert torch.equal(orthogonalize(same, out=same), out)
    for at in range(0, K, 1_000):
        errors_of_all(g[at: at + 1_000], out[at: at + 1_000], kind)


@pytest.mark.parametrize("refused", [1, 2, 7])
@pytest.mark.parametrize("kind,K,m,n", [("f32", 300, 100, 700), ("bf16", 1_001, 130, 40)])
def test_small_matrices_in_a_context_without_room_for_clusters(kind, K, m, n, refused):
    """Slices of some tens, by way of the workspace."""
    from paper_1905_12948_gb300 import load, orthogonalize
    g = make(K, m, n, kind)
    load().gmc_test_refuse_cooperative(refused)
    try:
        out = orthogonalize(g)
    finally:
        load().gmc_test_refuse_cooperative(0)
    errors_of_all(g, out, kind)


@pytest.mark.parametrize("product", [0, 1, 2, 3, 7, 12, 13, 14])
@pytest.mark.parametrize("block,matrix", [(0, 0), (3, 0), (6, 1), (7, 1)])
@pytest.mark.parametrize("kind,m,n", [("bf16", 100, 500), ("bf16", 500, 100), ("f32", 30, 400)])
def test_a_wait_that_runs_out_in_a_cluster(kind, m, n, block, matrix, product):
    """Four blocks a matrix: one of them gives up, and all of the matrix is NaN, whichever product of whichever step it
    was; the other matrices are what they are."""
    import torch
    from paper_1905_12948_gb300 import load, orthogonalize
    lib = load()
    g = make(3, m, n, kind)
    want = orthogonalize(g)
    assert lib.gmc_test_withhold_product(5_000_000, block, product) == 0
    out = orthogonalize(g)
    torch.cuda.synchronize()
    assert out[matrix].isnan().all()
    others = [k for k in range(3) if k != matrix]
    assert torch.equal(out[others], want[others])
    assert torch.equal(orthogonalize(g), want)      # the next call is not affected


def test_one_block_whose_last_product_is_withheld():
    import torch
    from paper_1905_12948_gb300 import load, orthogonalize
    lib = load()
    for m, n in ((100, 90), (90, 100)):
        g = make(2, m, n, "f32")
        want = orthogonalize(g)
        assert lib.gmc_test_withhold_product(5_000_000, 1, 14) == 0
        out = orthogonalize(g)
        assert out[1].isnan().all() and torch.equal(out[0], want[0]) and torch.equal(orthogonalize(g), want)
    for bad in ((2_000_000_001, 0, 0), (1, -1, 0), (1, 0, -1)):
        assert lib.gmc_test_withhold_product(*bad) == 1
