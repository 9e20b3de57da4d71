"""Workspaces of gmc_orthogonalize by their sizes (no GPU)."""
import pytest

from paper_1905_12948_gb300 import load

F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def need():
    return load().gmc_orthogonalize_workspace


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_many_small_matrices_want_little(need, dtype):
    """Small matrices do not go through the workspace, but for clusters that find no room; thin ones go in slices."""
    for m, n in ((16, 16), (3, 5), (128, 128), (1, 128), (128, 7)):
        assert 0 < need(dtype, 65535, m, n) <= 4096
    for m, n in ((5, 130), (128, 1024), (1000, 64), (1, 129)):
        assert 0 < need(dtype, 65535, m, n) <= 64 << 20
    for m, n in ((129, 131), (1, 10_000), (700, 1_000)):
        assert 0 < need(dtype, 65535, m, n) <= 4 << 30


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_workspaces_grow_with_their_matrices_alone(need, dtype):
    """Up to a slice: 8 bytes an element of X and 8 of A and B, sides padded to 256, sums of squares and diagonals, and the shares
    of the last round's tiles: at most 75 of 256 x 256 (of 76 pairs) in 16 shares."""
    for m, n in ((129, 1025), (500, 600), (1000, 4096), (4096, 4096), (16, 5000)):
        lo, hi = -(-min(m, n) // 256) * 256, -(-max(m, n) // 256) * 256
        for K in (1, 2, 8):
            assert 8 * K * m * n <= need(dtype, K, m, n) <= K * (8 * lo * hi + 8 * lo * lo + 4096 + 8 * lo) + 75 * 16 * 256 * 256 * 4 + 65536


@pytest.mark.parametrize("dtype,K,m,n,taken", [
    # 8 m n bytes of X, its successor beside it, 4 (bfloat16) or 8 of the shorter side's square: below 2^38 or not
    (BF16, 1, 1 << 14, 1 << 20, True), (BF16, 1, 1 << 15, 1 << 20, False), (F32, 1, 1 << 20, 1 << 15, False),
    (BF16, 1, 1 << 16, 1 << 18, True), (F16, 1, 1 << 18, 1 << 16, True), (BF16, 1, 1 << 17, 1 << 18, False), (F32, 1, 1 << 18, 1 << 18, False),
    (BF16, 1, 149_760, 149_760, True), (F32, 1, 149_760, 149_760, False),
    # matrices by their number: as many as 2^36 elements
    (BF16, 16, 1 << 16, 1 << 16, True), (BF16, 17, 1 << 16, 1 << 16, False),
    (BF16, 65535, 1, 10_000, True), (F32, 65535, 1, 1 << 20, True), (F32, 65535, 2, 1 << 20, False),
    (BF16, 65535, 1_020, 1_020, True), (BF16, 65535, 1_030, 1_020, False),
])
def test_the_largest_sizes(need, dtype, K, m, n, taken):
    bytes_ = need(dtype, K, m, n)
    assert (0 < bytes_ <= 1 << 38) if taken else bytes_ == -1
