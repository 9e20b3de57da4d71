"""Orthogonalised matrices against the formula in 64 bits. Bounds: scores_ref."""
import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": "float32", "bf16": "bfloat16", "f16": "float16"}


def make(K, m, n, kind, seed=0, form="noise"):
    import torch
    gen = torch.Generator().manual_seed(seed)
    if form == "noise":
        g = torch.randn(K, m, n, generator=gen)
    else:      # a few directions and a little noise, as a layer's gradient
        r = max(1, min(m, n) // 8)
        g = (torch.randn(K, m, r, generator=gen) * torch.arange(1, r + 1) ** -0.5) @ torch.randn(K, r, n, generator=gen)
        g = (g + 0.3 * torch.randn(K, m, n, generator=gen)) * 1e-3
    return g.to(getattr(torch, DT[kind])).cuda()


def check(g, out, kind, **how):
    import torch
    scale = how.pop("scale", 1.0)
    assert out.shape == g.shape and out.dtype == g.dtype
    want = ref.products(g, **how)
    off32 = (ref.in_float32(g, **how) - want).flatten(1).norm(dim=1)
    own = (ref.rounded(g, fine=kind != "bf16", **how) - want).flatten(1).norm(dim=1)
    got = out.double() / scale
    off = (got - want).flatten(1).norm(dim=1)
    size = want.flatten(1).norm(dim=1)
    # the last rounding is off by half a step of each element at most; half's smallest steps are 2^-25 away
    last = torch.finfo(out.dtype).eps / 2 * size + (2.0 ** -25 / scale * g[0].numel() ** 0.5 if kind == "f16" else 0.0)
    assert (off <= 2 * (own + off32) + last).all(), ((off - last) / (own + off32), off / size)
    return want


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("K,m,n", [(1, 1, 1), (2, 1, 9), (2, 9, 1), (3, 2, 3), (2, 17, 33), (1, 64, 64), (4, 63, 65), (2, 128, 128),
                                   (1, 129, 127), (2, 200, 1000), (1, 1000, 64), (1, 256, 512), (1, 257, 511), (3, 300, 300),
                                   (1, 640, 520), (33, 40, 24), (1, 16, 5_000)])
def test_sizes(kind, K, m, n):
    from paper_1905_12948_gb300 import orthogonalize
    for form in ("noise", "layer"):
        g = make(K, m, n, kind, seed=m * n, form=form)
        check(g, orthogonalize(g), kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("K,m,n", [(1, 1024, 1024), (2, 1000, 2050), (1, 2100, 900), (2, 512, 4608), (9, 384, 700)])
def test_larger_sizes(kind, K, m, n):
    from paper_1905_12948_gb300 import orthogonalize
    g = make(K, m, n, kind, form="layer")
    check(g, orthogonalize(g), kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_steps_coefficients_and_scale(kind):
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    g = make(2, 70, 150, kind)
    for steps in (1, 2, 7):
        check(g, orthogonalize(g, steps=steps), kind, steps=steps)
    check(g, orthogonalize(g, scale=0.25), kind, scale=0.25)
    # the cubic iteration converges: rows become orthonormal
    cubic = (1.5, -0.5, 0.0)
    out = orthogonalize(g.float(), steps=16, coefficients=cubic)
    eye = out.double() @ out.double().transpose(1, 2)
    assert (eye - torch.eye(70, dtype=torch.double, device="cuda")).abs().max() < 1e-4
    each = [(3.0, -3.2, 1.2), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)]
    check(g, orthogonalize(g, steps=3, coefficients=each), kind, steps=3, coefficients=each)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n", [(48, 100), (100, 48), (300, 260), (7, 5)])
def test_the_part_of_a_flat_gradient_in_place(kind, m, n):
    """K x d gradients, the matrix somewhere in each row; what lies around it stays."""
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    K, at, d = 3, 37, 37 + m * n + 11
    grads = torch.randn(K, d, generator=torch.Generator().manual_seed(1)).to(getattr(torch, DT[kind])).cuda()
    before = grads.clone()
    part = grads[:, at: at + m * n].view(K, m, n)
    out = orthogonalize(part, out=part)
    assert out.data_ptr() == part.data_ptr()
    check(before[:, at: at + m * n].reshape(K, m, n), part, kind)
    assert torch.equal(grads[:, :at], before[:, :at]) and torch.equal(grads[:, at + m * n:], before[:, at + m * n:])


def test_rows_apart_and_one_matrix():
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    buf = torch.randn(2, 40, 101, generator=torch.Generator().manual_seed(1)).cuda()
    x = buf[:, 3:, 5:95]
    out = torch.full((2, 40, 120), 7.0, device="cuda")
    view = out[:, :37, 1:91]
    assert orthogonalize(x, out=view).data_ptr() == view.data_ptr()
    check(x, view, "f32")
    assert (out[:, 37:] == 7).all() and (out[:, :37, 0] == 7).all() and (out[:, :37, 91:] == 7).all()
    one = orthogonalize(x[1])
    assert one.shape == x[1].shape and torch.equal(one, view[1])


def test_zeros_and_numbers_that_are_not_finite():
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    for m, n in ((40, 50), (300, 400)):
        g = make(5, m, n, "f32")
        want = orthogonalize(g)
        g[1] = 0
        g[2, 3, 4] = torch.inf
        g[3, 5, 6] = torch.nan
        out = orthogonalize(g)
        assert (out[1] == 0).all() and out[2:4].isnan().all() and torch.equal(out[[0, 4]], want[[0, 4]])


def test_any_magnitude():
    """The norm's square may lie outside 32 bits."""
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    g = make(1, 60, 90, "f32")
    want = orthogonalize(g)
    for e in (100, -100):
        out = orthogonalize(g * 2.0 ** e)
        assert torch.equal(out, want)
    tiny = (g * 2.0 ** -140)                 # subnormal: with fewer bits, but no less a matrix
    check(tiny, orthogonalize(tiny), "f32")
    for kind in ("bf16", "f16"):
        x = make(1, 60, 90, kind)
        x = x / x.abs().max() * torch.finfo(x.dtype).max * 0.9
        check(x, orthogonalize(x), kind)


def test_rows_of_very_different_size():
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    for kind in ("f32", "bf16"):
        g = make(2, 130, 200, kind)
        g = g * (10.0 ** torch.linspace(-4, 0, 130, device="cuda"))[:, None].to(g.dtype)
        check(g, orthogonalize(g), kind)


def test_same_bits_twice_on_a_stream_and_in_a_graph():
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    inputs = [make(2, 100, 300, "bf16"), make(1, 700, 600, "f32"), make(3, 20, 30, "f16"), make(2, 600, 1100, "bf16")]
    want = [orthogonalize(g) for g in inputs]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [orthogonalize(g, stream=s) for g in inputs]
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):          # two graphs, replayed side by side
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = [orthogonalize(g) for g in inputs]
        graphs.append((graph, captured, torch.cuda.Stream()))
    for _, captured, _ in graphs:
        for t in captured:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, _, stream in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, captured, _ in graphs:
        assert all(torch.equal(a, b) for a, b in zip(captured, want))


def test_calls_side_by_side():
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    g = [make(2, 520, 700, "bf16", seed=i) for i in range(4)]
    want = [orthogonalize(x) for x in g]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in g]
    for _ in range(3):
        got = [orthogonalize(x, stream=s) for x, s in zip(g, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    import torch
    from paper_1905_12948_gb300 import orthogonalize
    g = make(2, 8, 9, "f32")
    for bad in (g.double(), g.cpu(), g[0, 0], g[None], g.transpose(1, 2), g[:, :, ::2], g.expand(2, 8, 9)[:1].expand(2, 8, 9)):
        with pytest.raises(TypeError):
            orthogonalize(bad)
    for how in (dict(steps=0), dict(steps=17), dict(coefficients=(1.0, 2.0)), dict(coefficients=[(1, 2, 3)] * 4),
                dict(coefficients=[(1, 2)] * 5)):
        with pytest.raises(ValueError):
            orthogonalize(g, **how)
    with pytest.raises(TypeError):
        orthogonalize(g, out=torch.empty(2, 9, 8, device="cuda"))
    from paper_1905_12948_gb300 import GMCError
    with pytest.raises(GMCError):
        orthogonalize(g, coefficients=(float("nan"), 1.0, 1.0))
    with pytest.raises(GMCError):
        orthogonalize(g, scale=float("inf"))
    assert orthogonalize(g[:0]).shape == (0, 8, 9) and orthogonalize(g[:, :0]).shape == (2, 0, 9)
