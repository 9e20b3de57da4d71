"""Token log-probabilities, policy loss and preference loss against their 64-bit
statements (token_ref), within the bounds derived there."""
import ctypes

import numpy as np
import pytest

import token_ref as ref

pytestmark = pytest.mark.gpu
KINDS = ["f32", "bf16", "f16"]
LO, HI = 0.2, 0.28
GMC_EINVAL = 1


def _torch_type(kind):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


def _place(x, kind, pad=0, shift=0):
    """x (n, V) on the device with row stride V + pad, its first element `shift`
    elements past an aligned address; and the values as they were rounded."""
    import torch
    n, V = x.shape
    buf = torch.full((max(n, 1) * (V + pad) + shift,), float("nan"), dtype=_torch_type(kind), device="cuda")
    t = buf[shift:].as_strided((n, V), (V + pad, 1))
    t.copy_(torch.from_numpy(np.ascontiguousarray(x)).cuda())
    return t, t.double().cpu().numpy()


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _f32(a):
    return np.asarray(a, np.float32).astype(np.float64)


def _logits(n, V, seed, kind, pad=0, shift=0):
    rng = np.random.default_rng([seed, n, V])
    x = rng.standard_normal((n, V)) * 2.5
    y = rng.integers(0, V, n)
    if n:
        x[np.arange(n), y] += rng.uniform(0, 9, n)
    t, x = _place(x, kind, pad, shift)
    return rng, t, x, y


def _check_logp(got, want):
    bound = ref.LOGP + 2 * ref.U * np.abs(want)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got))
    assert (np.abs(got[fine] - want[fine]) <= bound[fine]).all(), np.max(np.abs(got[fine] - want[fine]))


def _check_gradient(got, x, y, coef, dcoef, scale, kind):
    got = got.double().cpu().numpy()
    want = ref.gradient(x, y, coef, scale)
    bound = ref.gradient_bound(x, y, coef, dcoef, scale, kind)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], bound[bad][:5])


SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (3, 31), (1, 4096), (7, 1000), (33, 513), (2, 50_257),
         (1, 131_072), (3, 131_073), (1, 300_001), (400, 129), (700, 4_099)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,V", SIZES)
def test_token_logp_and_gradient(n, V, kind):
    from paper_1905_12948_gb300 import token_logp, token_logp_backward
    rng, t, x, y = _logits(n, V, 1, kind)
    scale = 1.0 if V % 2 else 0.75
    if n > 2:
        y[1] = -1
    g = _f32(rng.standard_normal(n))
    if n > 3:
        g[3] = 0.0
    tgt = _dev(y)
    logp, stats = token_logp(t, tgt, scale=scale, return_stats=True)
    _check_logp(logp.double().cpu().numpy(), ref.token_logp(x, y, scale))
    d = token_logp_backward(t, tgt, stats, _dev(g.astype(np.float32)), scale=scale)
    _check_gradient(d, x, y, g, np.zeros(n), scale, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pad,shift,opad,oshift", [(0, 1, 0, 1), (3, 0, 3, 0), (1, 5, 2, 3), (0, 0, 1, 0), (8, 3, 0, 0)])
@pytest.mark.parametrize("V", [5, 40, 1_021, 20_011])
def test_strides_and_alignments(V, pad, shift, opad, oshift, kind):
    """Rows that start at every offset from a 16-byte boundary, outputs at others;
    nothing is written beside the output's rows."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n = 6
    rng, t, x, y = _logits(n, V, 2, kind, pad, shift)
    lp = ref.token_logp(x, y, 1.0)
    old, rf = _f32(lp + 0.1), _f32(lp - 0.2)
    adv, w = _f32(rng.uniform(0.5, 1.5, n)), _f32(rng.uniform(0.1, 1.0, n))
    buf = torch.full((n * (V + opad) + oshift,), 7.0, dtype=_torch_type(kind), device="cuda")
    out = buf[oshift:].as_strided((n, V), (V + opad, 1))
    h = TokenLoss(n)
    r = h.policy(t, _dev(y), _dev(old, torch.float32), _dev(adv, torch.float32), weights=_dev(w, torch.float32),
                 ref_logp=_dev(rf, torch.float32), clip_low=LO, clip_high=HI, kl=0.1, out=out)
    assert r.dlogits is out
    _, _, coef = ref.policy(lp, y, old, adv, w, rf, LO, HI, 0.1)
    _check_gradient(out, x, y, coef, w * ref.policy_bound(lp, old, adv, rf, 0.1), 1.0, kind)
    flat = buf.float().cpu().numpy()
    beside = np.ones(flat.size, bool)
    for i in range(n):
        beside[oshift + i * (V + opad): oshift + i * (V + opad) + V] = False
    assert (flat[beside] == 7.0).all()
    h.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("kl", [0.0, 0.05])
@pytest.mark.parametrize("n,V", SIZES)
def test_policy(n, V, kl, kind):
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    rng, t, x, y = _logits(n, V, 3, kind)
    scale = 1 / 0.7 if V % 2 else 1.0
    lp = ref.token_logp(x, y, scale)
    # ratios away from the clip's ends and from 1, on both sides of each
    ratio = rng.choice([0.5, 0.75, 0.9, 1.1, 1.25, 1.4], n)
    old, rf = _f32(lp - np.log(ratio)), _f32(lp + rng.standard_normal(n) * 0.3)
    adv, w = _f32(rng.standard_normal(n)), _f32(rng.uniform(0.1, 1.0, n))
    if n > 2:
        y[0], w[2] = -1, 0.0
    f = torch.float32
    h = TokenLoss(max_rows=n + 5)
    r = h.policy(t, _dev(y), _dev(old, f), _dev(adv, f), weights=_dev(w, f), ref_logp=_dev(rf, f) if kl else None,
                 clip_low=LO, clip_high=HI, kl=kl, scale=scale)
    loss, each, coef = ref.policy(lp, y, old, adv, w, rf, LO, HI, kl)
    bound = ref.policy_bound(lp, old, adv, rf, kl)
    counts = (y >= 0) & (w != 0)
    _check_logp(r.logp.double().cpu().numpy(), np.where(counts, lp, 0.0))
    assert (np.abs(r.token_loss.double().cpu().numpy() - each) <= bound).all()
    assert abs(float(r.loss) - loss) <= (w * bound)[counts].sum() + 2 * ref.U * abs(loss)
    _check_gradient(r.dlogits, x, y, coef, w * bound, scale, kind)
    again = h.policy(t, _dev(y), _dev(old, f), _dev(adv, f), weights=_dev(w, f), ref_logp=_dev(rf, f) if kl else None,
                     clip_low=LO, clip_high=HI, kl=kl, scale=scale, out=t)       # in place, the same bits
    assert again.dlogits is t and torch.equal(t, r.dlogits)
    assert torch.equal(again.loss, r.loss) and torch.equal(again.token_loss, r.token_loss)
    h.close()


def test_policy_without_weights_and_without_gradient():
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n, V, f = 21, 333, torch.float32
    rng, t, x, y = _logits(n, V, 4, "f32")
    lp = ref.token_logp(x, y, 1.0)
    old, adv = _f32(lp), _f32(rng.standard_normal(n))
    h = TokenLoss(n)
    r = h.policy(t, _dev(y), _dev(old, f), _dev(adv, f), grad=False)
    assert r.dlogits is None
    loss, _, _ = ref.policy(lp, y, old, adv, np.full(n, 1 / n), lp, 0.2, 0.2, 0.0)
    assert abs(float(r.loss) - loss) <= ref.policy_bound(lp, old, adv, lp, 0.0).mean() + 4 * ref.U
    h.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths,V", [([1, 1], 9), ([0, 3], 50), ([4, 0, 0, 0], 130), ([2, 5, 1, 7, 3, 3], 50_257),
                                       ([17, 40, 33, 25], 4_099), ([300, 411], 517), ([3, 2] * 90, 40),
                                       ([1, 2], 131_073), ([9, 14, 11, 8], 32_000)])
def test_preference(lengths, V, kind):
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n, pairs, f = sum(lengths), len(lengths) // 2, torch.float32
    rng, t, x, y = _logits(n, V, 5, kind)
    scale, beta, eps = (0.8 if V % 2 else 1.0), 0.1, 0.05
    y[rng.random(n) < 0.2] = -1
    lp = ref.token_logp(x, y, scale)
    off = np.concatenate([[0], np.cumsum(lengths)])
    rf, w = _f32(lp + rng.standard_normal(n) * 0.4), _f32(rng.uniform(0.1, 1.0, pairs))
    if pairs > 2:
        w[1] = 0.0
    h = TokenLoss(n, pairs)
    args = dict(beta=beta, smoothing=eps, ref_logp=_dev(rf, f), weights=_dev(w, f), scale=scale)
    r = h.preference(t, _dev(y), _dev(off), **args)
    loss, each, ratio, coef = ref.preference(lp, y, off, rf, w, beta, eps, np.zeros(n, bool))
    row = np.where(y >= 0, ref.LOGP + 2 * ref.U * np.abs(lp), 0.0)
    off_ratio = np.array([row[off[s]: off[s + 1]].sum() for s in range(2 * pairs)])
    dm = beta * (off_ratio[0::2] + off_ratio[1::2]) + 2 * ref.U * beta * np.abs(ratio).max()
    _check_logp(r.logp.double().cpu().numpy(), lp)
    assert (np.abs(r.seq_ratio.double().cpu().numpy() - ratio) <= off_ratio + ref.U * np.abs(ratio)).all()
    assert (np.abs(r.pair_loss.double().cpu().numpy() - each) <= dm + 8 * ref.U * (1 + each)).all()
    assert abs(float(r.loss) - loss) <= (w * (dm + 8 * ref.U * (1 + each))).sum() + ref.U * loss
    # the slope's own slope is at most w beta / 4
    dc = np.zeros(n)
    for s in range(2 * pairs):
        dc[off[s]: off[s + 1]] = w[s // 2] * beta * (dm[s // 2] / 4 + 8 * ref.U)
    _check_gradient(r.dlogits, x, y, coef, dc, scale, kind)
    again = h.preference(t, _dev(y), _dev(off), out=t, **args)
    assert torch.equal(t, r.dlogits) and torch.equal(again.loss, r.loss) and torch.equal(again.seq_ratio, r.seq_ratio)
    h.close()


def test_preference_without_reference_weights_or_gradient_and_with_extreme_margins():
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    x = np.zeros((4, 3))
    x[0, 0], x[3, 0] = 3_000.0, 3_000.0    # the first pair's margin is far above 0, the second's far below
    y = np.array([0, 1, 1, 1])
    x[1, 2] = 2_000.0
    t, x = _place(x, "f32")
    h = TokenLoss(4, 2)
    off = np.arange(5)
    r = h.preference(t, _dev(y), _dev(off), beta=1.0)
    lp = ref.token_logp(x, y, 1.0)
    loss, each, _, coef = ref.preference(lp, y, off, np.zeros(4), np.full(2, 0.5), 1.0, 0.0, np.zeros(4, bool))
    np.testing.assert_allclose(r.pair_loss.cpu().numpy(), each, rtol=1e-5, atol=1e-7)
    np.testing.assert_allclose(float(r.loss), loss, rtol=1e-5)
    np.testing.assert_allclose(r.dlogits.cpu().numpy(), ref.gradient(x, y, coef, 1.0), rtol=1e-4, atol=1e-6)
    assert h.preference(t, _dev(y), _dev(off), beta=1.0, grad=False).dlogits is None
    h.close()


@pytest.mark.parametrize("V", [40, 2_999, 131_072])
@pytest.mark.parametrize("kind", KINDS)
def test_masked_rows_and_logits(kind, V):
    """-inf and the type's lowest value among the logits, rows of them alone, and rows
    that do not count holding NaN and infinities."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss, token_logp
    low = float(torch.finfo(_torch_type(kind)).min)
    rng = np.random.default_rng(6)
    n = 9
    x = rng.standard_normal((n, V)) * 2
    y = rng.integers(0, V // 2, n)
    x[0, V // 2:] = -np.inf          # a padded vocabulary
    x[1, V // 3:] = low
    y[1] = 0
    x[2] = low                       # all alike: uniform
    x[3] = -np.inf                   # no distribution
    x[4] = np.nan                    # not scored
    x[5] = np.inf                    # not scored
    x[6, :V - 1] = -np.inf           # one logit left, the target
    y[6] = V - 1
    x[7, y[7]] = -np.inf             # the target masked
    t, x = _place(x, kind)
    y[4] = -1
    w = np.ones(n)
    w[5] = 0.0
    f = torch.float32
    scale = 1.5
    with np.errstate(invalid="ignore", over="ignore"):
        lp = ref.log_softmax(x, scale)[np.arange(n), np.maximum(y, 0)]
    lp[4] = lp[5] = 0.0
    got = token_logp(t, _dev(y), scale=scale).double().cpu().numpy()
    _check_logp(np.where(np.arange(n) == 5, 0.0, got), lp)   # row 5 has a target: NaN there
    assert np.isnan(got[5])
    old = _f32(np.where(np.isfinite(lp), lp, -3.0) - 0.1)
    h = TokenLoss(n, 1)
    adv = np.ones(n)
    r = h.policy(t, _dev(y), _dev(old, f), _dev(adv, f), weights=_dev(w, f), clip_low=LO, clip_high=HI, scale=scale)
    xs = np.where(np.isnan(x) | np.isposinf(x), 0.0, x)
    loss, each, coef = ref.policy(lp, y, old, adv, w, lp, LO, HI, 0.0)
    fine = np.isfinite(lp)
    bound = np.where(fine, ref.policy_bound(np.where(fine, lp, 0), old, adv, lp, 0.0), 1e-6)
    np.testing.assert_array_less(np.abs(r.token_loss.double().cpu().numpy() - each), bound + 1e-30)
    assert abs(float(r.loss) - loss) <= bound.sum()
    _check_gradient(r.dlogits, xs, y, coef, bound, scale, kind)
    # a preference pair over rows 0..4 and 6: the empty row and the unscored one add nothing
    rows = [0, 1, 2, 3, 4, 6]
    tt = t[rows].contiguous()
    off = np.array([0, 3, 6])
    rl = _f32(np.where(np.isfinite(lp[rows]), lp[rows], 0.0) + 0.2)
    r = h.preference(tt, _dev(y[rows]), _dev(off), beta=0.5, ref_logp=_dev(rl, f), scale=scale)
    empty = np.isneginf(lp[rows])
    _, _, ratio, coef = ref.preference(np.where(empty, 0, lp[rows]), y[rows], off, rl, np.ones(1), 0.5, 0.0, empty)
    np.testing.assert_allclose(r.seq_ratio.cpu().numpy(), ratio, atol=1e-4)
    _check_gradient(r.dlogits, xs[rows], y[rows], coef, np.full(6, 1e-4), scale, kind)
    h.close()


def test_marked_targets_and_non_finite_rows():
    import torch
    from paper_1905_12948_gb300 import TokenLoss, token_logp, token_logp_backward
    x = np.random.default_rng(7).standard_normal((5, 100))
    x[3, 50] = np.nan
    x[4, 10] = np.inf
    t, x = _place(x, "f32")
    y = np.array([5, 100, 7, 3, 4])            # the second target is outside the vocabulary
    lp, st = token_logp(t, _dev(y), return_stats=True)
    bad = np.array([False, True, False, True, True])
    assert np.array_equal(np.isnan(lp.cpu().numpy()), bad)
    one = torch.ones(5, device="cuda")
    d = token_logp_backward(t, _dev(y), st, one).cpu().numpy()
    assert np.array_equal(np.isnan(d).all(1), bad) and np.isfinite(d[~bad]).all()
    h = TokenLoss(5, 1)
    r = h.policy(t, _dev(y), one, one)
    assert np.array_equal(np.isnan(r.token_loss.cpu().numpy()), bad) and np.isnan(float(r.loss))
    d = r.dlogits.cpu().numpy()
    assert np.array_equal(np.isnan(d).all(1), bad) and np.isfinite(d[~bad]).all()
    r = h.policy(t[:1], _dev(y[:1]), torch.full((1,), float("nan"), device="cuda"), one[:1])
    assert np.isnan(float(r.loss)) and torch.isnan(r.dlogits).all()      # a NaN input is not hidden by the clip
    h.close()


def test_differences_on_the_device():
    """The kernels' gradients against differences of the kernels' losses: d along a
    random direction, over 2^-6 (the third order: below 1e-3 of it here)."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    rng, t, x, y = _logits(12, 60, 8, "f32")
    f = torch.float32
    lp = ref.token_logp(x, y, 1.0)
    old = _dev(_f32(lp - np.log(rng.choice([0.5, 0.9, 1.1, 1.5], 12))), f)
    rf, adv = _dev(_f32(lp + 0.2), f), _dev(rng.standard_normal(12), f)
    u = _dev(rng.standard_normal(x.shape), f)
    off = _dev(np.array([0, 4, 7, 10, 12]))
    h = TokenLoss(12, 2)
    s = 2.0 ** -6

    def policy(v):
        return h.policy(v, _dev(y), old, adv, ref_logp=rf, kl=0.1)

    def preference(v):
        return h.preference(v, _dev(y), off, beta=0.5, ref_logp=rf, smoothing=0.1)

    for call in (policy, preference):
        want = float((call(t).dlogits.double() * u.double()).sum())
        got = (float(call(t + s * u).loss.double()) - float(call(t - s * u).loss.double())) / (2 * s)
        assert abs(got - want) <= 5e-3 * abs(want) + 1e-4, (got, want)
    h.close()


def test_empty_calls():
    import torch
    from paper_1905_12948_gb300 import TokenLoss, token_logp
    x = torch.empty((0, 17), device="cuda")
    y = torch.empty(0, dtype=torch.int64, device="cuda")
    e = torch.empty(0, device="cuda")
    assert token_logp(x, y).shape == (0,)
    h = TokenLoss(4, 4)
    assert float(h.policy(x, y, e, e).loss) == 0.0
    assert float(h.preference(x, y, torch.zeros(1, dtype=torch.int64, device="cuda"), beta=0.1).loss) == 0.0
    r = h.preference(x, y, torch.zeros(3, dtype=torch.int64, device="cuda"), beta=0.1)   # two empty sequences
    np.testing.assert_allclose(float(r.loss), np.log(2), rtol=1e-6)
    # rows outside every sequence: zero gradients
    r = h.preference(torch.randn((3, 17), device="cuda"), torch.ones(3, dtype=torch.int64, device="cuda"),
                     torch.tensor([1, 2, 2], device="cuda"), beta=0.1)
    assert (r.dlogits[0] == 0).all() and (r.dlogits[1] != 0).any() and (r.dlogits[2] == 0).all()
    h.close()


def test_offsets_beyond_32_bits():
    """Rows more than 2^31 elements apart."""
    import torch
    from paper_1905_12948_gb300 import token_logp, token_logp_backward
    n, V, ld = 3, 1_001, (1 << 30) + 3
    buf = torch.empty(2 * ld + V, dtype=torch.float16, device="cuda")
    t = buf.as_strided((n, V), (ld, 1))
    rng = np.random.default_rng(9)
    t.copy_(torch.from_numpy(rng.standard_normal((n, V))).cuda())
    x, y = t.double().cpu().numpy(), rng.integers(0, V, n)
    lp, st = token_logp(t, _dev(y), return_stats=True)
    _check_logp(lp.double().cpu().numpy(), ref.token_logp(x, y, 1.0))
    token_logp_backward(t, _dev(y), st, torch.ones(n, device="cuda"), out=t)
    _check_gradient(t, x, y, np.ones(n), np.zeros(n), 1.0, "f16")


def test_streams_and_graph():
    """On a side stream after work on the current one, and captured into a graph that
    is replayed on new logits."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n, V, f = 40, 5_003, torch.float32
    rng, t, x, y = _logits(n, V, 10, "bf16")
    lp = ref.token_logp(x, y, 1.0)
    old, adv = _dev(_f32(lp + 0.05), f), _dev(rng.standard_normal(n), f)
    tgt = _dev(y)
    h = TokenLoss(n, 1)
    want = h.policy(t, tgt, old, adv)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = h.policy(t, tgt, old, adv, stream=s)
    s.synchronize()
    assert torch.equal(got.dlogits, want.dlogits) and torch.equal(got.loss, want.loss)
    static, off = torch.zeros_like(t), _dev(np.array([0, 15, n]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a = h.policy(static, tgt, old, adv)
        b = h.preference(static, tgt, off, beta=0.2)
    for _ in range(2):
        static.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.dlogits, want.dlogits) and torch.equal(a.loss, want.loss)
        p = h.preference(t, tgt, off, beta=0.2)
        torch.cuda.synchronize()
        assert torch.equal(b.dlogits, p.dlogits) and torch.equal(b.loss, p.loss)
        static.zero_()
        g.replay()
    h.close()


def test_refusals():
    import torch
    from paper_1905_12948_gb300 import GMCError, TokenLoss, gmc, token_logp, token_logp_backward
    f = torch.float32
    x = torch.zeros((4, 10), device="cuda")
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    v = torch.zeros(4, device="cuda")
    off = torch.tensor([0, 2, 4], device="cuda")
    h = TokenLoss(4, 1)
    for bad in (x.double(), x.t(), x[0], x.cpu(), torch.zeros((1, 10), device="cuda").expand(4, 10)):
        with pytest.raises(TypeError):
            token_logp(bad, y)
    with pytest.raises(TypeError):
        token_logp(x, y.int())
    with pytest.raises(ValueError):
        token_logp(x, y[:3])
    with pytest.raises(TypeError):
        h.policy(x, y, v.double(), v)
    with pytest.raises(TypeError):
        h.policy(x, y, v, v, out=x.half())
    with pytest.raises(ValueError):
        h.preference(x, y, off[:2], beta=0.1)
    for bad in (dict(scale=0.0), dict(scale=float("nan")), dict(clip_low=-0.1), dict(clip_low=1.5),
                dict(clip_high=float("inf")), dict(kl=-1.0), dict(kl=0.1)):      # kl without a reference
        with pytest.raises(GMCError) as e:
            h.policy(x, y, v, v, **bad)
        assert e.value.status == GMC_EINVAL
    for bad in (dict(beta=0.0), dict(beta=float("inf")), dict(beta=0.1, smoothing=1.1), dict(beta=0.1, scale=-1.0)):
        with pytest.raises(GMCError):
            h.preference(x, y, off, **bad)
    big = torch.zeros((5, 10), device="cuda")
    with pytest.raises(GMCError):      # more rows, or pairs, than the handle was made for
        h.policy(big, torch.zeros(5, dtype=torch.int64, device="cuda"), big[:, 0].contiguous(), big[:, 0].contiguous())
    with pytest.raises(GMCError):
        h.preference(x, y, torch.tensor([0, 1, 2, 3, 4], device="cuda"), beta=0.1)
    st = torch.zeros((4, 2), device="cuda")
    with pytest.raises(TypeError):
        token_logp_backward(x, y, st, v, out=x[:2])
    lib = gmc.load()
    p, s = x.data_ptr(), 0
    assert lib.gmc_token_logp(p, 3, 4, 10, 10, 1.0, y.data_ptr(), v.data_ptr(), None, s) == GMC_EINVAL   # type
    assert lib.gmc_token_logp(p, 0, 4, 10, 9, 1.0, y.data_ptr(), v.data_ptr(), None, s) == GMC_EINVAL    # stride
    assert lib.gmc_token_logp(p + 2, 0, 4, 10, 10, 1.0, y.data_ptr(), v.data_ptr(), None, s) == GMC_EINVAL
    assert lib.gmc_token_logp(p, 0, 4, 10, 10, 1.0, y.data_ptr() + 4, v.data_ptr(), None, s) == GMC_EINVAL
    assert lib.gmc_token_logp(p, 0, -1, 10, 10, 1.0, y.data_ptr(), v.data_ptr(), None, s) == GMC_EINVAL
    assert lib.gmc_token_logp(p, 0, 4, 0, 10, 1.0, y.data_ptr(), v.data_ptr(), None, s) == GMC_EINVAL
    assert lib.gmc_token_logp(None, 0, 4, 10, 10, 1.0, y.data_ptr(), v.data_ptr(), None, s) == GMC_EINVAL
    # in place with another stride
    assert lib.gmc_token_logp_backward(p, 0, 4, 10, 10, 1.0, y.data_ptr(), st.data_ptr(), v.data_ptr(), p, 11,
                                       s) == GMC_EINVAL
    assert lib.gmc_policy_loss(None, p, 0, 4, 10, 10, 1.0, y.data_ptr(), v.data_ptr(), None, v.data_ptr(), None, 0.2,
                               0.2, 0.0, v.data_ptr(), None, None, None, 10, s) == GMC_EINVAL
    out = ctypes.c_void_p()
    for rows, pairs in ((0, 1), (-1, 0), (1, -1), ((1 << 27) + 1, 0)):
        assert lib.gmc_loss_create(ctypes.byref(out), rows, pairs) == GMC_EINVAL and out.value is None
    h.close()


def test_workspace_allocation_failure():
    import torch
    from paper_1905_12948_gb300 import GMCError, TokenLoss, gmc
    lib = gmc.load()
    torch.cuda.init()
    held = lib.gmc_test_fail_alloc(0)
    with pytest.raises(GMCError) as e:
        TokenLoss(100, 10)
    assert e.value.status == 2
    assert lib.gmc_test_fail_alloc(-1) == held
    h = TokenLoss(100, 10)
    assert lib.gmc_test_fail_alloc(-1) == held + 1
    h.close()
    assert lib.gmc_test_fail_alloc(-1) == held


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pad,shift", [(0, 3), (7, 0), (5, 2), (16, 8), (1, 0)])
def test_gradients_of_views(pad, shift, kind):
    """A gradient allocated for a view (padded rows, an odd start) has the view's shape,
    and its rows lie at the same offsets from a 16-byte boundary."""
    import torch
    from paper_1905_12948_gb300 import token_logp, token_logp_backward
    n, V = 5, 1_003
    rng, t, x, y = _logits(n, V, 11, kind, pad, shift)
    _, st = token_logp(t, _dev(y), return_stats=True)
    d = token_logp_backward(t, _dev(y), st, torch.ones(n, device="cuda"))
    assert d.shape == t.shape and d.dtype == t.dtype
    for i in range(n):
        assert (d[i].data_ptr() - t[i].data_ptr()) % 16 == 0
    _check_gradient(d, x, y, np.ones(n), np.zeros(n), 1.0, kind)


def test_one_row_views_and_requires_grad():
    """A row of a larger tensor, and logits that autograd follows: logits.backward takes
    the gradient."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n, V = 8, 77
    w = torch.randn((16, V), device="cuda", requires_grad=True)
    h = torch.randn((n, 16), device="cuda")
    logits = h @ w
    y = torch.arange(n, device="cuda")
    old, adv = torch.full((n,), -3.0, device="cuda"), torch.ones(n, device="cuda")
    loss = TokenLoss(n)
    r = loss.policy(logits, y, old, adv, clip_high=1e6)
    assert not r.loss.requires_grad
    logits.backward(r.dlogits)
    ratio = torch.exp(torch.log_softmax((h @ w.detach()).double(), -1)[y, y] - old.double())
    z = w.detach().double().requires_grad_()
    lp = torch.log_softmax(h.double() @ z, -1)[y, y]
    (-torch.exp(lp - old.double()).mean()).backward()
    # products of fp32 matrices: 16 terms of about 1, and a gradient good to P of itself
    np.testing.assert_allclose(w.grad.double().cpu().numpy(), z.grad.cpu().numpy(), rtol=1e-3, atol=1e-5 * float(ratio.max()))
    one = loss.policy(logits.detach()[3:4], y[3:4], old[3:4], adv[3:4], clip_high=1e6)
    assert torch.equal(one.logp, r.logp[3:4])
    loss.close()


@pytest.mark.parametrize("n,V", [(3, 50_257), (2, 300_001), (40, 8_192)])
def test_contexts_without_room_for_clusters(n, V):
    """Launches of clusters answered as in a context with too few SMs: the same results by
    one block a row."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss, gmc, token_logp
    rng, t, x, y = _logits(n, V, 12, "f32")
    lp = ref.token_logp(x, y, 1.0)
    old, adv = _f32(lp - 0.1), _f32(rng.uniform(0.5, 1.5, n))
    f, lib = torch.float32, gmc.load()
    h = TokenLoss(n, 1)
    want = np.full(n, 1 / n)
    loss, each, coef = ref.policy(lp, y, old, adv, want, lp, 0.2, 0.2, 0.0)
    off = np.array([0, n // 2, n])
    none = np.zeros(n, bool)
    _, _, ratio, pcoef = ref.preference(lp, y, off, np.zeros(n), np.ones(1), 0.1, 0.0, none)
    try:
        for refuse in (1, 2):      # the ring, and the clusters of the two-sweep kernel
            assert lib.gmc_test_refuse_cooperative(refuse) == 0
            r = h.policy(t, _dev(y), _dev(old, f), _dev(adv, f))
            _check_logp(r.logp.double().cpu().numpy(), lp)
            _check_gradient(r.dlogits, x, y, coef, want * ref.policy_bound(lp, old, adv, lp, 0.0), 1.0, "f32")
        assert lib.gmc_test_refuse_cooperative(1) == 0
        _check_logp(token_logp(t, _dev(y)).double().cpu().numpy(), lp)
        assert lib.gmc_test_refuse_cooperative(1) == 0
        r = h.preference(t, _dev(y), _dev(off), beta=0.1)
        _check_logp(r.logp.double().cpu().numpy(), lp)
        _check_gradient(r.dlogits, x, y, pcoef, np.full(n, 0.1 * 0.1 * (n * 2e-5) + 1e-7), 1.0, "f32")
    finally:
        lib.gmc_test_refuse_cooperative(0)
    h.close()


@pytest.mark.parametrize("n,V,kind", [(40, 50_257, "f32"), (200, 9_000, "bf16"), (3, 131_072, "bf16"), (700, 900, "f16"),
                                      (1, 40, "f32")])
def test_a_wait_that_runs_out(n, V, kind):
    """A row whose copy is withheld: every wait gives up, the loss is NaN, and the next call
    (and a new handle) is right again. By the ring with and without clusters, and a warp a row."""
    import time
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    rng, t, x, y = _logits(n, V, 13, kind)
    lp = ref.token_logp(x, y, 1.0)
    old, adv = _dev(_f32(lp - 0.1), torch.float32), _dev(_f32(rng.uniform(0.5, 1.5, n)), torch.float32)
    h = TokenLoss(n)
    want = h.policy(t, _dev(y), old, adv)
    assert h.lib.gmc_test_withhold_row(h.h, n // 2, 20_000_000) == 0
    t0 = time.time()
    assert np.isnan(float(h.policy(t, _dev(y), old, adv).loss))
    assert time.time() - t0 < 5
    for handle in (h, TokenLoss(n)):
        r = handle.policy(t, _dev(y), old, adv)
        assert torch.equal(r.loss, want.loss) and torch.equal(r.dlogits, want.dlogits)
        handle.close()


def test_withhold_refusals():
    from paper_1905_12948_gb300 import TokenLoss, gmc
    lib, h = gmc.load(), TokenLoss(10)
    assert lib.gmc_test_withhold_row(None, 0, 1000) == GMC_EINVAL
    for row, ns in ((-1, 1000), (10, 1000), (0, 0), (0, 2_000_000_001)):
        assert lib.gmc_test_withhold_row(h.h, row, ns) == GMC_EINVAL
    h.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,V,pad,shift", [(601, 1, 0, 0), (640, 2, 1, 0), (999, 15, 0, 1), (1_024, 61, 3, 5),
                                           (777, 1_021, 0, 0), (2_051, 5_003, 0, 0)])
def test_many_short_rows(n, V, pad, shift, kind):
    """Rows that a warp does: every offset from a 32-byte boundary, the last warps without
    a row, marked targets, masked logits, rows of nothing, nothing written beside the rows."""
    import torch
    from paper_1905_12948_gb300 import token_logp, token_logp_backward
    rng = np.random.default_rng([17, n, V])
    x, y = rng.standard_normal((n, V)) * 2.5, rng.integers(0, V, n)
    x[5, 1:] = -np.inf
    x[6] = -np.inf
    x[7] = np.nan
    y[5], y[7], y[n - 1] = 0, -1, -1
    t, x = _place(x, kind, pad, shift)
    logp, stats = token_logp(t, _dev(y), return_stats=True)
    with np.errstate(invalid="ignore"):
        want = ref.token_logp(x, y, 1.0)
    _check_logp(logp.double().cpu().numpy(), want)
    g = _f32(rng.standard_normal(n))
    g[[3, 6, 7]] = 0.0
    stride = V + pad + 1
    buf = torch.full((n * stride,), 7.0, dtype=_torch_type(kind), device="cuda")
    out = buf.as_strided((n, V), (stride, 1))
    token_logp_backward(t, _dev(y), stats, _dev(g, torch.float32), out=out)
    got = out.double().cpu().numpy()
    assert (got[[3, 6, 7, n - 1]] == 0).all()
    rows = np.setdiff1d(np.arange(n), [3, 6, 7, n - 1])
    _check_gradient(out[torch.from_numpy(rows).cuda()], x[rows], y[rows], g[rows], np.zeros(len(rows)), 1.0, kind)
    assert (buf.view(n, stride)[:, V:] == 7.0).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths,V", [([1] * 700, 33), ([0, 0] + [7, 3] * 65 + [0, 1, 0, 0], 257), ([900, 0], 1_021),
                                       ([0, 0] * 400 + [511, 513] + [0, 0] * 40, 5)])
def test_pairs_of_many_short_rows(lengths, V, kind):
    """A warp does a row, and the last one of a pair the pair: pairs with and without rows,
    with and without the gradient, the same bits each time."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n, pairs, f = sum(lengths), len(lengths) // 2, torch.float32
    rng, t, x, y = _logits(n, V, 18, kind)
    y[rng.random(n) < 0.2] = -1
    beta, eps = 0.1, 0.05
    lp = ref.token_logp(x, y, 1.0)
    off = np.concatenate([[0], np.cumsum(lengths)])
    rf, w = _f32(lp + rng.standard_normal(n) * 0.4), _f32(rng.uniform(0.1, 1.0, pairs))
    w[0] = 0.0 if pairs > 1 else w[0]
    h = TokenLoss(n, pairs)
    args = dict(beta=beta, smoothing=eps, ref_logp=_dev(rf, f), weights=_dev(w, f))
    r = h.preference(t, _dev(y), _dev(off), **args)
    loss, each, ratio, coef = ref.preference(lp, y, off, rf, w, beta, eps, np.zeros(n, bool))
    row = np.where(y >= 0, ref.LOGP + 2 * ref.U * np.abs(lp), 0.0)
    off_ratio = np.array([row[off[s]: off[s + 1]].sum() for s in range(2 * pairs)])
    dm = beta * (off_ratio[0::2] + off_ratio[1::2]) + 2 * ref.U * beta * np.abs(ratio).max()
    _check_logp(r.logp.double().cpu().numpy(), lp)
    assert (np.abs(r.seq_ratio.double().cpu().numpy() - ratio) <= off_ratio + ref.U * np.abs(ratio)).all()
    assert (np.abs(r.pair_loss.double().cpu().numpy() - each) <= dm + 8 * ref.U * (1 + each)).all()
    assert abs(float(r.loss) - loss) <= (w * (dm + 8 * ref.U * (1 + each))).sum() + ref.U * loss
    dc = np.zeros(n)
    for s in range(2 * pairs):
        dc[off[s]: off[s + 1]] = w[s // 2] * beta * (dm[s // 2] / 4 + 8 * ref.U)
    _check_gradient(r.dlogits, x, y, coef, dc, 1.0, kind)
    for _ in range(3):
        again = h.preference(t, _dev(y), _dev(off), grad=False, **args)
        assert torch.equal(again.loss, r.loss) and torch.equal(again.seq_ratio, r.seq_ratio)
        again = h.preference(t, _dev(y), _dev(off), **args)
        assert torch.equal(again.loss, r.loss) and torch.equal(again.dlogits, r.dlogits)
    h.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [60, 121, 200, 251, 256, 310, 500, 512, 700, 1_000, 1_024, 1_990, 2_048, 3_990])
def test_policy_of_many_short_rows(V, kind):
    """Rows that a warp does, over the sizes of its buffers: a block's shared memory goes from a
    few KB, over what a kernel has without asking, to all there is."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n, f = 700, torch.float32
    rng, t, x, y = _logits(n, V, 19, kind)
    y[rng.random(n) < 0.2] = -1
    lp = ref.token_logp(x, y, 1.0)
    old, rf = _f32(lp + 0.1 * rng.standard_normal(n)), _f32(lp - 0.2)
    adv, w = _f32(rng.uniform(-1.5, 1.5, n)), _f32(rng.uniform(0.1, 1.0, n))
    # no ratio within the rounding of its bounds
    close = np.abs(np.exp(lp - old)[:, None] - [1 - LO, 1 + HI]).min(1) < 1e-3
    old[close] = _f32(lp[close])
    h = TokenLoss(n)
    r = h.policy(t, _dev(y), _dev(old, f), _dev(adv, f), weights=_dev(w, f), ref_logp=_dev(rf, f), clip_low=LO,
                 clip_high=HI, kl=0.1)
    _check_logp(r.logp.double().cpu().numpy(), lp)
    _, _, coef = ref.policy(lp, y, old, adv, w, rf, LO, HI, 0.1)
    _check_gradient(r.dlogits, x, y, coef, w * ref.policy_bound(lp, old, adv, rf, 0.1), 1.0, kind)
    h.close()
