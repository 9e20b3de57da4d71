"""The ends of gmc_orthogonalize's ranges: many and thin matrices, far strides, in place, coefficients as arrays."""
import pytest

import scores_ref as ref
from test_gpu_orthogonalize import check

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def matrices(kind, *shape, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=gen).to(DTYPES[kind])


@pytest.mark.parametrize("kind, K, m, n", [
    ("bf16", 65535, 3, 5), ("f32", 65535, 2, 1), ("f32", 9000, 5, 130), ("bf16", 700, 130, 5), ("bf16", 1500, 129, 131)])
def test_many_matrices(kind, K, m, n):
    """Errors of single small matrices are small by chance as well: those of all are compared, and each with the
    largest."""
    from paper_1905_12948_gb300 import orthogonalize
    g = matrices(kind, K, m, n)
    out, want = orthogonalize(g), ref.products(g)

    def errors(x):
        return (x.double() - want).flatten(1).norm(dim=1)

    off, size = errors(out), want.flatten(1).norm(dim=1)
    plain = errors(ref.in_float32(g)) + errors(ref.rounded(g, fine=kind != "bf16"))
    last = torch.finfo(out.dtype).eps / 2 * size
    assert off.norm() <= 2 * plain.norm() + last.norm(), (off.norm(), plain.norm(), last.norm())
    assert (off <= 2 * (plain / size).max() * size + last).all(), ((off - last) / size).max()


@pytest.mark.parametrize("kind, m, n", [("f32", 1, 1 << 20), ("bf16", 1 << 20, 2), ("f16", 3, (1 << 20) - 1)])
def test_thin_matrices(kind, m, n):
    """A sum of one sign of 2^20 products, cut off after each 16 (bf16) or added up by parts of 128 in 32 bits. Cut off:
    2^16 times at most 2^-23 of a sum that is half as large on the mean, and half of that on the mean: 2^-9 of A. By parts: 2^13
    roundings of at most 2^-24 of a sum that is half as large, four times their root mean square 2^6.5 2^-25, and 24
    cuts in a part, 2^-19.6: 2^-16.3. The singular values of such matrices are 1 / sqrt(rows) at first, then
    between 0.6 and 1.25, where a step's relative change is at most that of A; steps together pass on 1.5
    times each at most (|s p'(s) / p(s)| along the five steps from 1: 1.03, 0.72, 2.0, 0.83, 1.2): 7.5 times in all."""
    from paper_1905_12948_gb300 import orthogonalize
    g = matrices(kind, m, n)
    out, want = orthogonalize(g).double(), ref.products(g[None])[0]
    off, last = (out - want).norm() / want.norm(), torch.finfo(g.dtype).eps / 2
    if kind == "f16":  # its smallest steps, 2^-24 apart
        last += 2.0 ** -25 * g.numel() ** 0.5 / want.norm().item()
    assert off <= last + 7.5 * 2.0 ** (-9 if kind == "bf16" else -16.3), off


@pytest.mark.parametrize("m, n", [(20, 30), (300, 200), (200, 1500)])
def test_offsets_past_32_bits(m, n):
    from paper_1905_12948_gb300 import orthogonalize
    far = (1 << 31) + 40
    whole = torch.empty(2 * far, dtype=torch.bfloat16, device="cuda")
    x = whole.as_strided((2, m, n), (far, n, 1))
    x.copy_(matrices("bf16", 2, m, n))
    g = x.contiguous()
    check(g, orthogonalize(x), "bf16")
    rows = (1 << 31) // m + 8  # a matrix's rows apart as well: the last one past 2^31 elements
    x = whole.as_strided((m, n), (rows + n, 1))
    x.copy_(g[0])
    assert orthogonalize(x, out=x) is not None
    check(g[:1], x.contiguous()[None], "bf16")


def test_in_place_with_other_strides_is_refused():
    from paper_1905_12948_gb300 import GMCError, orthogonalize
    whole = matrices("f32", 8 * 40 * 50)
    x, other = whole[:4 * 40 * 30].view(4, 40, 30), whole.as_strided((4, 40, 30), (1500, 31, 1))
    before = whole.clone()
    with pytest.raises(GMCError):
        orthogonalize(x, out=other)
    with pytest.raises(TypeError):
        orthogonalize(x, out=whole.as_strided((4, 40, 30), (0, 30, 1)))
    torch.cuda.synchronize()
    assert torch.equal(whole, before)


def test_coefficients_as_arrays():
    import numpy as np

    from paper_1905_12948_gb300 import orthogonalize
    g = matrices("f32", 2, 70, 90)
    three = [[3.4445, -4.775, 2.0315], [2.0, -1.5, 0.5], [1.5, -0.5, 0.0]]
    want = orthogonalize(g, steps=3, coefficients=three)
    for c in (np.array(three), torch.tensor(three, dtype=torch.float64), tuple(tuple(t) for t in three)):
        assert torch.equal(orthogonalize(g, steps=3, coefficients=c), want)
    want = orthogonalize(g, steps=3, coefficients=three[1])
    for c in (np.array(three[1]), torch.tensor(three[1], dtype=torch.float64), np.array([three[1]] * 3)):
        assert torch.equal(orthogonalize(g, steps=3, coefficients=c), want)
    for c in ((), (1.0, 2.0), [three[0], three[1]], [three[0], three[1], (1.0, 2.0)], ["a", "b", "c"], None):
        with pytest.raises((TypeError, ValueError)):
            orthogonalize(g, steps=3, coefficients=c)
