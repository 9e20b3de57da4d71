"""Values at the limits of what the post-training operators take."""
import numpy as np
import pytest

import token_ref as ref

pytestmark = pytest.mark.gpu
# Of a logp whose exponents are near 2^20, token_ref's bound with one term more: an exponent's rounding
# is that of its distance from the maximum (below 8 here) and of the last place of s log2 e in two
# words, 2^-46 of 2^20. logp itself is below 16 there.
LIMIT = ref.LOGP + 2.0 ** -24


def _type(kind):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _around(V, scale, sign, order, seed):
    """A row of float32 logits whose exponents scale * log2(e) * x lie on both sides of 2^20 (or
    -2^20), from which on the kernels take the difference to the maximum first: within 0.7 of it
    below, 0.05 to 1 of it above. order: where those above lie."""
    rng = np.random.default_rng(seed)
    limit = 2.0 ** 20 / (scale * np.log2(np.e))
    near, past = rng.uniform(0.05, 0.7, V) / scale, rng.uniform(0.05, 1.0, V) / scale
    above = {"first": np.arange(V) < V // 2, "last": np.arange(V) >= V // 2, "one": np.arange(V) == V // 3,
             "but one": np.arange(V) != V // 3, "mixed": rng.random(V) < 0.5}[order]
    return (sign * (limit + np.where(above, past, -near))).astype(np.float32)


@pytest.mark.parametrize("order", ["first", "last", "one", "but one", "mixed"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** 20, 2.0 ** -20, 1e5])
@pytest.mark.parametrize("n,V", [(5, 2), (5, 40), (3, 129), (2, 5_003), (1, 70_001), (700, 37), (700, 1_021)])
def test_rows_around_the_limit_of_the_exponents(n, V, scale, sign, order):
    """In a thread, across lanes, warps and blocks."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss, token_logp, token_logp_backward
    rng = np.random.default_rng([21, n, V])
    rows = min(n, 7)
    x = np.stack([_around(V, scale, sign, order, [i, V]) for i in range(rows)])[np.arange(n) % rows]
    y = rng.integers(0, V, n)
    t, tgt, f = _dev(x), _dev(y), torch.float32
    x = x.astype(np.float64)
    scale = float(np.float32(scale))
    lp = ref.token_logp(x, y, scale)
    logp, stats = token_logp(t, tgt, scale=scale, return_stats=True)
    off = abs(logp.double().cpu().numpy() - lp)
    assert (off <= LIMIT).all(), off.max()
    g = np.ones(n)
    d = token_logp_backward(t, tgt, stats, _dev(g, f), scale=scale).double().cpu().numpy()
    bound = ref.gradient_bound(x, y, g, np.zeros(n), scale, "f32")
    assert (abs(d - ref.gradient(x, y, g, scale)) <= bound).all()
    h = TokenLoss(n, 1)
    old = np.float32(lp + 0.05).astype(np.float64)
    r = h.policy(t, tgt, _dev(old, f), _dev(g, f), scale=scale, out=torch.empty_like(t))
    assert (abs(r.logp.double().cpu().numpy() - lp) <= LIMIT).all()
    _, _, coef = ref.policy(lp, y, old, g, g / n, lp, 0.2, 0.2, 0.0)
    bound = ref.gradient_bound(x, y, coef, ref.policy_bound(lp, old, g, lp, 0.0) / n, scale, "f32")
    assert (abs(r.dlogits.double().cpu().numpy() - ref.gradient(x, y, coef, scale)) <= bound).all()
    h.close()


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("scale", [100.0, 2.0 ** 9])
@pytest.mark.parametrize("n,V,kind", [(3, 130, "bf16"), (2, 5_003, "f16"), (1, 70_001, "bf16"), (700, 1_021, "f16")])
def test_rows_around_the_limit_in_16_bits(n, V, kind, scale, sign):
    """The type's values on either side of 2^20 exponents lie hundreds of exponents apart."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss, token_logp
    limit = 2.0 ** 20 / (scale * np.log2(np.e))
    ulp = 2.0 ** (np.floor(np.log2(limit)) - {"bf16": 7, "f16": 10}[kind])
    rng = np.random.default_rng([23, n, V])
    x = sign * ulp * (np.floor(limit / ulp) + rng.integers(-1, 3, (n, V)))
    y = rng.integers(0, V, n)
    t = _dev(x).to(_type(kind))
    assert np.array_equal(t.double().cpu().numpy(), x)
    lp = ref.token_logp(x, y, scale)
    one = torch.ones(n, device="cuda")
    for logp in (token_logp(t, _dev(y), scale=scale), TokenLoss(n).policy(t, _dev(y), -one, one, scale=scale).logp):
        assert (abs(logp.double().cpu().numpy() - lp) <= LIMIT + 2 * ref.U * abs(lp)).all()


@pytest.mark.parametrize("n,V,kind", [(400, 300, "bf16"), (9, 300, "f32"), (6, 50_257, "bf16"), (3, 300_001, "f32")])
def test_weights_that_are_not_finite_on_rows_that_add_nothing(n, V, kind):
    """A warp a row, the ring by one block and by several, and rows swept twice."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((n, V), generator=g, device="cuda").to(_type(kind))
    y = torch.randint(0, V, (n,), generator=g, device="cuda")
    old, adv, w = torch.full((n,), -8.0, device="cuda"), torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    y[1] = -1
    x[n - 1] = -float("inf")          # no distribution
    h = TokenLoss(n)
    want = h.policy(x, y, old, adv, weights=w)
    assert torch.isfinite(want.loss)
    for bad in (float("inf"), float("nan")):
        w[1] = w[n - 1] = bad
        r = h.policy(x, y, old, adv, weights=w)
        assert torch.equal(r.loss, want.loss) and torch.equal(r.dlogits, want.dlogits), bad
        assert torch.equal(r.token_loss, want.token_loss)
    h.close()


@pytest.mark.parametrize("n,V", [(400, 300), (4, 300), (4, 50_257), (3, 300_001)])
def test_target_outside_the_vocabulary_in_a_row_of_nothing(n, V):
    import torch
    from paper_1905_12948_gb300 import TokenLoss, token_logp, token_logp_backward
    x = torch.zeros((n, V), device="cuda")
    x[1] = -float("inf")
    y = torch.zeros(n, dtype=torch.int64, device="cuda")
    y[1] = V
    one = torch.ones(n, device="cuda")
    logp, stats = token_logp(x, y, return_stats=True)
    h = TokenLoss(n, 1)
    r = h.policy(x, y, logp.nan_to_num(), one)
    q = h.preference(x, y, torch.tensor([0, 2, 3], device="cuda"), beta=0.1)
    assert torch.isnan(logp[1]) and torch.isnan(token_logp_backward(x, y, stats, one)[1]).all()
    assert torch.isnan(r.token_loss[1]) and torch.isnan(r.loss) and torch.isnan(r.dlogits[1]).all()
    assert torch.isfinite(r.token_loss[[0, 2]]).all() and torch.isfinite(r.dlogits[[0, 2]]).all()
    assert torch.isnan(q.seq_ratio[0]) and torch.isfinite(q.seq_ratio[1]) and torch.isnan(q.loss)
    h.close()


@pytest.mark.parametrize("n", [60, 700])
def test_kl_term_near_the_reference(n):
    """Advantages of 0 leave the KL term alone: f(d) = exp(d) - d - 1 of d = ref - logp, and its
    slope, as good as 32 bits hold them at any distance. d is the kernel's own: the difference of two
    floats within a factor of two of each other (exact), or rounded once (u of d, which f'/f d, below
    2 + |d|, multiplies). f's series or difference takes some ten roundings, none larger than u of f
    (where it is a difference, from |d| = 1/2 on, of terms that are below 9 f): 40u of f cover them."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    rng = np.random.default_rng(22)
    V, kl, f = 50, 0.25, torch.float32
    x = rng.standard_normal((n, V)).astype(np.float32)
    y = rng.integers(0, V, n)
    x[np.arange(n), y] += np.where(np.arange(n) % 2, 12.0, 0.0).astype(np.float32)     # confident tokens too
    t, tgt, zero = _dev(x), _dev(y), torch.zeros(n, device="cuda")
    h = TokenLoss(n)
    logp = h.policy(t, tgt, zero, zero).logp.cpu().numpy()
    d = rng.choice([-1, 1], n) * 10.0 ** rng.uniform(-7.5, 1, n)
    d[:6] = 0.0, 0.5, -0.5, 0.4999, -0.4999, 1e-7
    rf = (logp.astype(np.float64) + d).astype(np.float32)
    r = h.policy(t, tgt, _dev(logp), zero, ref_logp=_dev(rf), kl=kl, weights=torch.ones(n, device="cuda"))
    assert np.array_equal(r.logp.cpu().numpy(), logp)
    d = rf.astype(np.float64) - logp.astype(np.float64)
    # to 64 bits: the series, or expm1 where its difference from d loses no more than 4 bits
    k = np.where(abs(d) < 0.5, d * d / 2 * sum(2.0 * d ** i / _factorial(i + 2) for i in range(20)), np.expm1(d) - d)
    got = r.token_loss.double().cpu().numpy()
    assert (got >= 0).all()
    assert (abs(got - kl * k) <= kl * k * (40 + abs(d)) * ref.U + 1e-44).all()
    coef = -kl * np.expm1(d)
    bound = ref.gradient_bound(x, y, coef, abs(kl * np.exp(d) * d) * 2 * ref.U + 8 * ref.U * abs(coef), 1.0, "f32")
    assert (abs(r.dlogits.double().cpu().numpy() - ref.gradient(x.astype(np.float64), y, coef, 1.0)) <= bound).all()
    h.close()


def _factorial(n):
    import math
    return math.factorial(n)


@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_pairs_whose_margin_is_infinite(smoothing):
    """A token masked by -inf in one of a pair's sequences: the margin is inf or -inf. What is not
    asked for (a weight of 0 on one of the two terms) does not make the loss NaN."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    x = torch.zeros((4, 8), device="cuda")
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    x[1, 0] = -float("inf")          # the first pair's other answer: margin inf
    x[2, 0] = -float("inf")          # the second pair's preferred one: margin -inf
    h = TokenLoss(4, 2)
    r = h.preference(x, y, torch.arange(5, device="cuda"), beta=0.5, smoothing=smoothing)
    up, down = (0.0 if smoothing == 0 else np.inf), (0.0 if smoothing == 1 else np.inf)
    assert np.array_equal(r.pair_loss.cpu().numpy(), np.array([up, down]))
    assert np.array_equal(r.seq_ratio.cpu().numpy()[[1, 2]], [-np.inf, -np.inf])
    assert float(r.loss) == np.inf
    assert torch.isfinite(r.dlogits).all()
    one = h.preference(x[:2], y[:2], torch.arange(3, device="cuda"), beta=0.5, smoothing=smoothing)
    assert float(one.loss) == up
    h.close()


@pytest.mark.parametrize("call", ["backward", "policy", "preference", "dropout"])
def test_autograd_is_told_of_writes_in_place(call):
    """Logits that a layer's backward pass has saved, and that an operator overwrote: backward refuses."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss, dropout, token_logp, token_logp_backward
    z = torch.randn((4, 32), device="cuda", requires_grad=True)
    logits = torch.tanh(z)            # its backward pass takes its output
    y = torch.arange(4, device="cuda")
    one, h = torch.ones(4, device="cuda"), TokenLoss(4, 1)
    before = logits._version
    if call == "backward":
        _, stats = token_logp(logits, y, return_stats=True)
        token_logp_backward(logits, y, stats, one, out=torch.empty_like(logits))
        assert logits._version == before
        d = token_logp_backward(logits, y, stats, one, out=logits)
    elif call == "policy":
        d = h.policy(logits, y, -one, one, out=logits).dlogits
    elif call == "preference":
        d = h.preference(logits, y, torch.tensor([0, 2, 4], device="cuda"), beta=0.1, out=logits).dlogits
    else:
        d = dropout(logits, 0.5, seed=1, out=logits)
    assert d is logits and logits._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        logits.backward(torch.ones_like(d))
    with torch.inference_mode():      # tensors without a version
        v = torch.randn((4, 32), device="cuda")
        h.policy(v, y, -one, one, out=v)
    h.policy(v, y, -one, one, out=v)
    h.close()
