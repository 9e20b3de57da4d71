"""Arguments that the post-training operators refuse before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_1905_12948_gb300 import load


@pytest.fixture(scope="module")
def lib():
    return load()


def test_dropout_in_place_with_another_stride(lib):
    """Workers' rows that are written where other rows are still to be read."""
    buf = ctypes.create_string_buffer(4096)
    p = ctypes.addressof(buf) + 16 - ctypes.addressof(buf) % 16

    def call(x, ldx, res, ldr, out, ldo, K):
        return lib.gmc_dropout(x, ldx, res, ldr, out, ldo, 0, 0, K, 8, 0.5, 0, 0, 0, None)

    assert call(p, 8, None, 0, p, 12, 2) == 1
    assert call(p, 12, None, 0, p, 8, 2) == 1
    assert call(p, 8, p + 1024, 9, p + 1024, 8, 2) == 1
    # (K = 0: nothing to do)
    for right in ((p, 8, None, 0, p, 8, 0), (p, 8, p + 1024, 9, p + 1024, 8, 0)):
        assert call(*right) == 0


def test_token_loss_wants_a_cuda_device(lib):
    pytest.importorskip("torch")
    from paper_1905_12948_gb300 import TokenLoss
    with pytest.raises(ValueError, match="CUDA device"):
        TokenLoss(4, device="cpu")
