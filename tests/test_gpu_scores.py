"""Token scores (log-probabilities of given tokens, entropy, top alternatives) and their
gradient against plain statements in 64 bits, with the bounds of scores_ref."""
import numpy as np
import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": "float32", "bf16": "bfloat16", "f16": "float16"}


def torch_():
    import torch
    return torch


def make(n, V, kind, *, seed=0, spread=2.5, offset=0, pad=0):
    """Logits in a buffer of their own, their rows pad elements apart, beginning offset elements in."""
    torch = torch_()
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, V, generator=gen) * spread).to(getattr(torch, DT[kind]))
    buf = torch.zeros(offset + n * (V + pad), dtype=x.dtype, device="cuda")
    view = buf[offset:].view(n, V + pad)[:, :V] if pad else buf[offset:].view(n, V)
    view.copy_(x)
    return view


def given(n, V, k, seed=1, masked=0.0):
    torch = torch_()
    gen = torch.Generator().manual_seed(seed)
    y = torch.randint(0, V, (n, k), generator=gen)
    y[torch.rand(n, generator=gen) < masked] = -1
    return y.cuda()


def host(x):
    return x.double().cpu().numpy()


def check_forward(x, y, top, scale=1.0):
    from paper_1905_12948_gb300 import token_scores
    n = x.shape[0]
    r = token_scores(x, y, top=top, scale=scale, return_stats=True)
    ys = np.zeros((n, 0), np.int64) if y is None else y.cpu().numpy().reshape(n, -1)
    logp, h, best, index = ref.scores(host(x), ys, top, float(np.float32(scale)))
    if y is None:
        assert r.logp is None
    else:
        got = r.logp.double().cpu().numpy().reshape(n, -1)
        assert r.logp.shape == y.shape
        fin = np.isfinite(logp)
        assert np.array_equal(np.isneginf(logp), np.isneginf(got))
        assert (np.abs(got - logp)[fin] <= ref.LOGP + 2 * ref.U * np.abs(logp[fin])).all()
    got = host(r.entropy)
    assert (np.abs(got - h) <= ref.entropy_bound(h)).all(), np.abs(got - h).max()
    assert (got >= 0).all()
    if top:
        assert np.array_equal(r.top_index.cpu().numpy(), index)
        got = host(r.top_logp)
        fin = np.isfinite(best)
        assert np.array_equal(np.isneginf(best), np.isneginf(got))
        assert (np.abs(got - best)[fin] <= ref.LOGP + 2 * ref.U * np.abs(best[fin])).all()
    else:
        assert r.top_logp is None and r.top_index is None
    return r


def check_backward(x, y, kind, scale=1.0, seed=2, out=None, unit=1.0, entropy=True):
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    torch = torch_()
    n = x.shape[0]
    gen = torch.Generator().manual_seed(seed)
    g = None if y is None else (torch.randn(y.shape, generator=gen) * unit).cuda()
    h = (torch.randn(n, generator=gen) * unit).cuda() if entropy else None
    stats = token_scores(x, y, scale=scale, return_stats=True).stats
    before = host(x)
    d = token_scores_backward(x, y, stats, g, h, scale=scale, out=out)
    ys = np.zeros((n, 0), np.int64) if y is None else y.cpu().numpy().reshape(n, -1)
    gs = np.zeros((n, 0)) if y is None else host(g).reshape(n, -1)
    hs = host(h) if entropy else np.zeros(n)
    s = float(np.float32(scale))
    want = ref.gradient(before, ys, gs, hs, s)
    assert d.dtype == x.dtype and d.shape == x.shape
    off = np.abs(host(d) - want)
    bound = ref.gradient_bound(before, ys, gs, hs, s, kind)
    assert (off <= bound).all(), (off / bound).max()
    return d


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V", [(1, 1), (3, 2), (5, 7), (2, 33), (7, 64), (4, 1000), (3, 4096), (2, 8191), (3, 8200), (2, 16400),
                                 (1, 50257), (2, 131072)])
@pytest.mark.parametrize("top", [0, 1, 5, 64])
def test_forward_sizes(kind, n, V, top):
    check_forward(make(n, V, kind, seed=V), given(n, V, 1 + V % 3), min(top, V))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (5, 7, 3), (7, 64, 64), (4, 1000, 0), (3, 4099, 1), (2, 50257, 17), (2, 131072, 2)])
def test_backward_sizes(kind, n, V, k):
    check_backward(make(n, V, kind, seed=V), given(n, V, k) if k else None, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 5), (8, 24)])
@pytest.mark.parametrize("scale", [1.0, 1 / 0.7, 0.5])
def test_strides_and_scales(kind, offset, pad, scale):
    x = make(6, 2011, kind, offset=offset, pad=pad)
    y = given(6, 2011, 4)
    check_forward(x, y, 9, scale)
    check_backward(x, y, kind, scale)


@pytest.mark.parametrize("rows,V", [(20_000, 501), (9_000, 1_000), (700, 2_049), (700, 9_000), (1_200, 16_390), (300, 3_000)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_rows(rows, V, kind):
    """Numbers of rows and lengths that other groupings of threads take."""
    torch = torch_()
    x = make(rows, V, kind, seed=rows)
    y = given(rows, V, 2, masked=0.2)
    some = torch.linspace(0, rows - 1, 40).long().cuda()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    g, h = torch.randn(rows, 2, device="cuda"), torch.randn(rows, device="cuda")
    r = token_scores(x, y, top=6, return_stats=True)
    d = token_scores_backward(x, y, r.stats, g, h)
    part = check_forward(x[some], y[some], 6)
    for a, b in ((r.logp, part.logp), (r.entropy, part.entropy), (r.top_logp, part.top_logp)):
        want = host(b)
        # both within the bound of the exact value
        assert (np.abs(host(a[some]) - want) <= 2 * (ref.LOGP + 2 * ref.U * np.abs(want)) + 2 * ref.entropy_bound(want)).all()
    assert torch.equal(r.top_index[some], part.top_index)
    ys, gs, hs = y[some].cpu().numpy(), host(g[some]), host(h[some])
    want = ref.gradient(host(x[some]), ys, gs, hs, 1.0)
    assert (np.abs(host(d[some]) - want) <= ref.gradient_bound(host(x[some]), ys, gs, hs, 1.0, kind)).all()
    # what the sampled rows do not show: rows that do not count, and sums
    masked = (y < 0).all(1)
    assert (d[masked] == 0).all() and (r.entropy[masked] == 0).all() and (r.top_index[masked] == -1).all()
    assert (r.top_index[~masked] >= 0).all()
    assert torch.equal(x[torch.arange(rows, device="cuda")[:, None], r.top_index.clamp(min=0)][~masked],
                       torch.topk(x, 6, dim=1).values[~masked])


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "steps", "late"])
@pytest.mark.parametrize("V", [300, 5_000, 40_000])
@pytest.mark.parametrize("top", [1, 7, 64])
def test_orders_and_ties(kind, order, V, top):
    """Rows that put every element above all before it, and rows of few distinct values."""
    torch = torch_()
    i = torch.arange(V, dtype=torch.float32)
    rows = {"ascending": i / V * 8, "descending": -i / V * 8, "equal": torch.full((V,), 0.25), "steps": (i * 7919 % 13).floor(),
            "late": torch.where(i >= V - 70, i - V, torch.full_like(i, -200.0))}[order]
    x = torch.stack([rows, rows.flip(0)]).to(getattr(torch, DT[kind])).cuda()
    check_forward(x, None, top)


def test_zeros_of_either_sign_are_equal():
    torch = torch_()
    x = torch.full((1, 100), -1.0, device="cuda")
    x[0, [5, 70]] = -0.0
    x[0, [9, 60]] = 0.0
    r = check_forward(x, None, 4)
    assert r.top_index[0].tolist() == [5, 9, 60, 70]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [40, 9_000, 70_000])
def test_masked_logits(kind, V):
    """-inf and the type's lowest value in a row, all of it, all but one."""
    torch = torch_()
    x = make(8, V, kind, seed=5)
    y = given(8, V, 2)
    lowest = torch.finfo(x.dtype).min
    x[0, V // 3:] = -torch.inf
    x[1, : V // 2] = lowest
    x[2] = -torch.inf
    x[3] = lowest
    x[4] = -torch.inf
    x[4, V // 2] = 1.5
    x[5] = lowest
    x[5, 3] = 2.0
    y[0, 0], y[0, 1] = 1, V - 1          # the second one masked: -inf
    x[6, :] = -30.0
    x[6, V - 1] = 60.0                   # a one-hot row
    check_forward(x, y, min(20, V))
    check_forward(x, None, min(20, V))
    # the gradient of a masked token's -inf is taken through its softmax all the same
    check_backward(x, y, kind)


def test_large_logits_over_a_low_temperature():
    torch = torch_()
    x = torch.randn(4, 3000, generator=torch.Generator().manual_seed(3)).cuda() * 2e5
    x[1] += 3e6
    x[2, 5] = 4e6
    check = check_forward(x, None, 5, 8.0)
    assert (check.entropy[2] == 0).all()


def test_nan_and_inf_mark_their_row_alone():
    torch = torch_()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    for V in (50, 5_000, 40_000):
        x = make(6, V, "f32")
        y = given(6, V, 2)
        want = token_scores(x, y, top=3)
        x[1, V // 2] = torch.nan
        x[3, 7] = torch.inf
        x[4, 9] = -torch.nan
        r = token_scores(x, y, top=3, return_stats=True)
        bad, fine = [1, 3, 4], [0, 2, 5]
        for a, b in ((r.logp, want.logp), (r.entropy, want.entropy), (r.top_logp, want.top_logp)):
            assert a[bad].isnan().all() and torch.equal(a[fine], b[fine])
        assert (r.top_index[bad] == -1).all() and torch.equal(r.top_index[fine], want.top_index[fine])
        d = token_scores_backward(x, y, r.stats, torch.ones(6, 2, device="cuda"), torch.ones(6, device="cuda"))
        assert d[bad].isnan().all() and d[fine].isfinite().all()


def test_rows_that_do_not_count_are_not_read():
    torch = torch_()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    x = make(5, 3_001, "f32")
    y = given(5, 3_001, 3)
    y[1] = -1
    y[2, 1] = -5
    x[1] = torch.nan
    r = token_scores(x, y, top=2, return_stats=True)
    assert (r.logp[1] == 0).all() and r.entropy[1] == 0 and (r.top_index[1] == -1).all() and (r.top_logp[1] == 0).all()
    assert r.logp[2, 1] == 0 and r.logp[2, 0] != 0
    h = torch.full((5,), 0.3, device="cuda")
    g = torch.ones(5, 3, device="cuda")
    d = token_scores_backward(x, y, r.stats, g, h)
    assert (d[1] == 0).all() and d.isfinite().all()
    x[3] = torch.nan                       # no slope: not read
    g[3], h[3] = 0, 0
    d = token_scores_backward(x, y, r.stats, g, h)
    assert (d[3] == 0).all()


def test_target_outside_the_vocabulary_marks_its_gradient():
    torch = torch_()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    x = make(4, 2_000, "bf16")
    x[2] = -torch.inf
    y = given(4, 2_000, 2)
    y[1, 1] = 2_000
    y[2, 0] = 1 << 40
    r = token_scores(x, y, return_stats=True)
    assert r.logp[1, 1].isnan() and r.logp[1, 0].isfinite() and r.logp[2, 0].isnan() and r.entropy.isfinite().all()
    for g in (1.0, 0.0):
        d = token_scores_backward(x, y, r.stats, torch.full((4, 2), g, device="cuda"))
        assert d[1:3].isnan().all() and d[[0, 3]].isfinite().all()


def test_the_same_token_twice():
    torch = torch_()
    x = make(3, 700, "f32")
    y = given(3, 700, 5)
    y[0, 3] = y[0, 1]
    y[1, :] = y[1, 0]
    check_forward(x, y, 0)
    check_backward(x, y, "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 5_003, 60_000])
def test_in_place(kind, V):
    x = make(5, V, kind, offset=1, pad=3)
    y = given(5, V, 6)
    d = check_backward(x, y, kind, out=x)
    assert d.data_ptr() == x.data_ptr()


def test_gradient_against_differences():
    torch = torch_()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    x = make(4, 900, "f32")
    y = given(4, 900, 3)
    g, h = torch.randn(4, 3, device="cuda"), torch.randn(4, device="cuda")
    r = token_scores(x, y, scale=0.8, return_stats=True)
    d = host(token_scores_backward(x, y, r.stats, g, h, scale=0.8))
    way = np.random.default_rng(1).standard_normal(x.shape)
    x0, eps, s = host(x), 1e-4, float(np.float32(0.8))

    def value(z):
        logp, ent, _, _ = ref.scores(z, y.cpu().numpy(), 0, s)
        return (logp * host(g)).sum(1) + ent * host(h)

    # the difference's own error: eps^2 / 6 times a third derivative below 10 |way|^3, and 1e-16 / eps
    diff = (value(x0 + eps * way) - value(x0 - eps * way)) / (2 * eps)
    bound = (ref.gradient_bound(x0, y.cpu().numpy(), host(g), host(h), s, "f32") * np.abs(way)).sum(1) + 1e-5
    assert (np.abs((d * way).sum(1) - diff) <= bound).all()


def test_alternatives_slopes_through_given_tokens():
    """The slopes of top_logp are those of its tokens: against autograd in 64 bits."""
    torch = torch_()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    x = make(4, 2_000, "f32")
    r = token_scores(x, top=8, return_stats=True)
    g = torch.randn(4, 8, device="cuda")
    d = token_scores_backward(x, r.top_index, r.stats, g)
    z = x.double().requires_grad_()
    want, = torch.autograd.grad((torch.log_softmax(z, 1).gather(1, r.top_index) * g).sum(), z)
    bound = ref.gradient_bound(host(x), r.top_index.cpu().numpy(), host(g), np.zeros(4), 1.0, "f32")
    assert (np.abs(host(d) - host(want)) <= bound).all()


def test_agrees_with_token_logp():
    """One given token, without its entropy: the log-probability and the gradient of token_logp."""
    torch = torch_()
    from paper_1905_12948_gb300 import token_logp, token_logp_backward, token_scores, token_scores_backward
    x = make(64, 8_001, "bf16")
    y = given(64, 8_001, 1)[:, 0].contiguous()
    logp, stats = token_logp(x, y, return_stats=True)
    r = token_scores(x, y, return_stats=True)
    assert (logp - r.logp).abs().max() <= 2 * ref.LOGP + 4 * ref.U * logp.abs().max()
    g = torch.randn(64, device="cuda")
    a, b = token_logp_backward(x, y, stats, g).float(), token_scores_backward(x, y, r.stats, g).float()
    assert ((a - b).abs() <= 2 ** -7 * a.abs() + 1e-6).all()


def test_same_bits_twice_on_a_stream_and_in_a_graph():
    torch = torch_()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    cases = []
    for n, V in ((2, 60_000), (40, 20_000), (2_000, 900)):
        x = make(n, V, "bf16", seed=n)
        y = given(n, V, 2)
        g, h = torch.randn(n, 2, device="cuda"), torch.randn(n, device="cuda")
        cases.append((x, y, g, h))

    def calls(**stream):
        out = []
        for x, y, g, h in cases:
            r = token_scores(x, y, top=9, return_stats=True, **stream)
            out += [*r, token_scores_backward(x, y, r.stats, g, h, **stream)]
        return out

    want = [t.clone() for t in calls()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = calls(stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = calls()
    for t in captured:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, want))


def test_offsets_past_32_bits():
    torch = torch_()
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    far = (1 << 31) + 40
    buf = torch.zeros(far + 1_000, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, 1_000), (far, 1))
    x.copy_(make(2, 1_000, "bf16"))
    y = given(2, 1_000, 2)
    check_forward(x, y, 5)
    r = token_scores(x, y, return_stats=True)
    d = token_scores_backward(x, y, r.stats, torch.ones(2, 2, device="cuda"), out=x)
    assert d.data_ptr() == x.data_ptr()
    assert x[1].float().abs().sum() > 0.5 and not buf[1_000: far].any()


def test_refusals():
    torch = torch_()
    from paper_1905_12948_gb300 import GMCError, token_scores, token_scores_backward
    x, y = make(4, 100, "f32"), given(4, 100, 2)
    stats = token_scores(x, y, return_stats=True).stats
    g = torch.ones(4, 2, device="cuda")
    for bad in (dict(top=65), dict(top=-1), dict(targets=y[:3].contiguous()), dict(targets=given(4, 100, 65)),
                dict(targets=y[:, :0].contiguous())):
        with pytest.raises(ValueError):
            token_scores(x, **{"targets": y, **bad})
    with pytest.raises(ValueError):
        token_scores(x[:, :3], top=4)
    for bad in (y.int(), y.cpu(), y.t().contiguous().t()):
        with pytest.raises(TypeError):
            token_scores(x, bad)
    with pytest.raises(TypeError):
        token_scores(x.double(), y)
    with pytest.raises(GMCError):
        token_scores(x, y, scale=0.0)
    with pytest.raises(ValueError):
        token_scores_backward(x, y, stats)
    with pytest.raises(ValueError):
        token_scores_backward(x, None, stats, g)
    with pytest.raises(ValueError):
        token_scores_backward(x, y, stats[:3].contiguous(), g)
    with pytest.raises(TypeError):
        token_scores_backward(x, y, stats, g, out=torch.empty(4, 101, device="cuda"))
    r = token_scores(x[:0], top=2, return_stats=True)
    assert r.entropy.shape == (0,) and r.top_index.shape == (0, 2)
    assert token_scores_backward(x[:0], None, r.stats, None, r.entropy).shape == (0, 100)
