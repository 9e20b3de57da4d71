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


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("K,m,n", [(3, 40, 50), (2, 500, 100), (3, 300, 260), (4, 1, 77), (2, 130, 1_100)])
def test_workers_rows_in_turn(kind, K, m, n):
    """The workers' rows lie between one another's (m, K, n), apart or not; into such a tensor, and in place. (Where a row begins
    at another offset from a 16-byte boundary, other 16 or 32 squares are added up in 32 bits before the 64 of the norm: a sum
    may be rounded otherwise, the results are held to the formula's bound.)"""
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    g = make(K, m, n, kind)
    want = orthogonalize(g)
    for pad in (0, 3, 8):
        buf = torch.full((m, K, n + pad), 7.0, dtype=g.dtype, device="cuda")
        x = buf[:, :, :n].transpose(0, 1)
        x.copy_(g)
        assert x.stride(0) == n + pad
        got = orthogonalize(x)
        check(g, got, kind)
        out = torch.full((m, K, n + pad), 7.0, dtype=g.dtype, device="cuda")
        view = out[:, :, :n].transpose(0, 1)
        assert orthogonalize(g, out=view).data_ptr() == view.data_ptr() and torch.equal(view, want)
        assert torch.equal(orthogonalize(x, out=x), got) and (buf[:, :, n:] == 7).all() and (out[:, :, n:] == 7).all()
    check(g, want, kind)


def test_rows_that_overlap_are_refused():
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    buf = torch.randn(10_000, device="cuda")
    before = buf.clone()
    for shape, strides in (((3, 4, 10), (9, 30, 1)), ((3, 4, 10), (10, 29, 1)), ((3, 4, 10), (39, 10, 1)), ((3, 4, 10), (40, 9, 1)),
                           ((3, 4, 10), (0, 10, 1)), ((3, 4, 10), (20, 20, 1)), ((3, 1, 10), (9, 10, 1)), ((3, 4, 10), (10, 0, 1))):
        x = buf.as_strided(shape, strides)
        with pytest.raises(TypeError, match="rows that do not overlap"):
            orthogonalize(x)
        with pytest.raises(TypeError, match="rows that do not overlap"):
            orthogonalize(torch.randn(shape, device="cuda"), out=x)
    torch.cuda.synchronize()
    assert torch.equal(buf, before)
