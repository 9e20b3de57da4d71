"""Arguments that token scores and orthogonalize refuse before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_1905_12948_gb300 import load


@pytest.fixture(scope="module")
def lib():
    return load()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(1 << 16)
    test_keep.append(buf)
    return ctypes.addressof(buf) + 256 - ctypes.addressof(buf) % 256


test_keep = []


def test_scores(lib, p):
    def call(x=p, dtype=0, n=4, vocab=10, ld=10, scale=1.0, y=p, given=2, top=3, logp=p, h=p, best=p, index=p, stats=p):
        return lib.gmc_token_scores(x, dtype, n, vocab, ld, scale, y, given, top, logp, h, best, index, stats, None)

    for bad in (dict(dtype=3), dict(ld=9), dict(x=p + 2), dict(vocab=0), dict(scale=0.0), dict(scale=float("nan")), dict(x=None),
                dict(n=-1), dict(vocab=1 << 31, ld=1 << 31), dict(y=None), dict(y=p + 4), dict(given=-1), dict(given=65),
                dict(top=-1), dict(top=65, vocab=100, ld=100), dict(top=11), dict(best=None), dict(index=None), dict(index=p + 4),
                dict(best=p + 2), dict(stats=p + 8), dict(logp=p + 1), dict(h=p + 1), dict(n=(1 << 27) + 1)):
        assert call(**bad) == 1, bad
    assert call(x=None, y=None, n=0) == 0


def test_scores_backward(lib, p):
    def call(x=p, dtype=0, n=4, vocab=10, ld=10, scale=1.0, y=p, given=2, stats=p, g=p, h=p, dx=p + 1024, dld=10):
        return lib.gmc_token_scores_backward(x, dtype, n, vocab, ld, scale, y, given, stats, g, h, dx, dld, None)

    for bad in (dict(dtype=-1), dict(ld=9), dict(dld=9), dict(dx=p + 2), dict(dx=None), dict(stats=None), dict(stats=p + 8),
                dict(g=p + 2), dict(h=p + 2), dict(dx=p, dld=11), dict(y=None), dict(given=65), dict(scale=-1.0)):
        assert call(**bad) == 1, bad
    assert call(x=None, y=None, dx=None, stats=None, n=0) == 0


def test_orthogonalize(lib, p):
    three = (ctypes.c_float * 48)(*([3.0, -4.0, 2.0] * 16))
    need = lib.gmc_orthogonalize_workspace(0, 2, 4, 5)
    assert need > 0
    for bad in ((3, 2, 4, 5), (0, -1, 4, 5), (0, 65536, 4, 5), (0, 1, (1 << 20) + 1, 1), (0, 65535, 1 << 20, 1 << 20)):
        assert lib.gmc_orthogonalize_workspace(*bad) == -1, bad

    def call(x=p, ldk=20, ld=5, out=p + 4096, oldk=20, old=5, dtype=0, K=2, m=4, n=5, steps=5, c=three, scale=1.0, w=p,
             bytes=need):
        return lib.gmc_orthogonalize(x, ldk, ld, out, oldk, old, dtype, K, m, n, steps, c, scale, w, bytes, None)

    inf = (ctypes.c_float * 15)(*([float("inf")] * 15))
    for bad in (dict(x=None), dict(out=None), dict(x=p + 2), dict(out=p + 1), dict(ldk=19), dict(ld=4), dict(oldk=19), dict(old=4),
                dict(dtype=5), dict(K=-1), dict(steps=0), dict(steps=17), dict(c=None), dict(c=inf), dict(scale=float("nan")),
                dict(w=None), dict(w=p + 128), dict(bytes=need - 1), dict(out=p, oldk=24), dict(out=p, oldk=24, old=6)):
        assert call(**bad) == 1, bad
    for nothing in (dict(K=0), dict(m=0), dict(n=0)):
        assert call(x=None, out=None, w=None, bytes=0, **nothing) == 0


def test_python_refuses_what_is_not_on_a_gpu(lib):
    torch = pytest.importorskip("torch")
    from paper_1905_12948_gb300 import orthogonalize, token_scores, token_scores_backward
    with pytest.raises(TypeError, match="logits must be a CUDA tensor"):
        token_scores(torch.zeros(2, 3))
    with pytest.raises(TypeError, match="logits must be a CUDA tensor"):
        token_scores_backward(torch.zeros(2, 3), None, None)
    with pytest.raises(TypeError, match="x must be a CUDA tensor"):
        orthogonalize(torch.zeros(2, 3, 3))
    with pytest.raises(TypeError, match="x must be a CUDA tensor"):
        orthogonalize(3.0, stream=object())
