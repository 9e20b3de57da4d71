"""Orthogonalised matrices, each way that their sizes may take, and waits that run out. Bounds: scores_ref."""
import pytest

import scores_ref as ref
from test_gpu_orthogonalize import check, make

pytestmark = pytest.mark.gpu
CODE = {"f32": 0, "bf16": 1, "f16": 2}


def way(kind, K, m, n):
    from paper_1905_12948_gb300 import load
    v = load().gmc_test_orthogonalize_course(CODE[kind], K, m, n)
    return "shared memory" if v == 0 else (("pairs" if v & 2 else "blocks"), bool(v & 4), bool(v & 8), v >> 4 & 255, bool(v >> 12))


WAYS = [   # (triangle of A, of B, shares, whole tiles beside them)
    ("f32", 1, 129, 127, "shared memory"), ("bf16", 5, 128, 1024, "shared memory"), ("f16", 2, 1024, 100, "shared memory"),
    ("f32", 1, 33, 513, "shared memory"), ("bf16", 300, 17, 250, "shared memory"),
    ("bf16", 1, 129, 1025, ("blocks", False, False, 4, False)),
    ("f32", 3, 300, 300, ("blocks", False, False, 1, False)), ("bf16", 30, 260, 300, ("blocks", False, False, 1, True)),
    ("f32", 2, 200, 1000, ("blocks", False, False, 4, False)), ("f32", 1, 16, 5000, ("blocks", False, False, 12, False)),
    ("f32", 2, 512, 4608, ("blocks", True, False, 7, False)), ("f32", 20, 500, 600, ("blocks", True, True, 3, True)),
    ("bf16", 12, 512, 900, ("blocks", True, True, 1, False)),
    ("bf16", 4, 1300, 1500, ("pairs", False, False, 1, True)), ("bf16", 2, 1000, 2050, ("pairs", False, False, 2, False)),
    ("f32", 3, 700, 9000, ("pairs", True, False, 4, False)), ("bf16", 8, 1000, 4096, ("pairs", True, False, 8, True)),
    ("f32", 8, 1000, 4096, ("pairs", True, False, 16, True)), ("f16", 5, 1100, 1200, ("pairs", True, True, 1, False)),
    ("bf16", 2, 1900, 1800, ("pairs", True, True, 1, False)), ("bf16", 1, 4096, 4096, ("pairs", True, True, 1, True)),
]


@pytest.mark.parametrize("kind,K,m,n,expected", WAYS)
def test_ways(kind, K, m, n, expected):
    from paper_1905_12948_gb300 import orthogonalize
    assert way(kind, K, m, n) == expected
    g = make(K, m, n, kind, form="layer")
    out = orthogonalize(g)
    check(g, out, kind)
    import torch
    assert torch.equal(orthogonalize(g), out)


@pytest.mark.parametrize("refused", [1, 2, 3])
@pytest.mark.parametrize("kind,K,m,n", [("bf16", 2, 100, 700), ("f32", 2, 512, 1100), ("bf16", 4, 1300, 1500), ("f32", 5, 1100, 1200)])
def test_a_context_without_room_for_all_blocks(kind, K, m, n, refused):
    """Launches whose blocks wait for one another are refused: products one by one, without clusters."""
    from paper_1905_12948_gb300 import load, orthogonalize
    g = make(K, m, n, kind, form="layer")
    load().gmc_test_refuse_cooperative(refused)
    try:
        out = orthogonalize(g)
    finally:
        load().gmc_test_refuse_cooperative(0)
    check(g, out, kind)


@pytest.mark.parametrize("kind,K,m,n", [("f32", 1, 100, 100), ("bf16", 1, 100, 700), ("f32", 2, 300, 300), ("bf16", 1, 600, 20_000),
                                        ("bf16", 4, 1300, 1500), ("f32", 3, 700, 9000)])
def test_waits_that_run_out(kind, K, m, n):
    import torch
    from paper_1905_12948_gb300 import load, orthogonalize
    g = make(K, m, n, kind)
    want = orthogonalize(g)
    assert load().gmc_test_withhold_phase(20_000_000) == 0
    out = orthogonalize(g)
    torch.cuda.synchronize()
    assert out.isnan().all()
    assert torch.equal(orthogonalize(g), want)      # the next call is not affected


def test_hook_refuses_and_disarms():
    import torch
    from paper_1905_12948_gb300 import load, orthogonalize
    lib = load()
    assert lib.gmc_test_withhold_phase(2_000_000_001) == 1
    assert lib.gmc_test_withhold_phase(1_000_000) == 0 and lib.gmc_test_withhold_phase(0) == 0
    assert orthogonalize(torch.randn(40, 50, device="cuda")).isfinite().all()
    assert lib.gmc_test_orthogonalize_course(3, 1, 10, 10) == -1
