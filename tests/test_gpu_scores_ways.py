"""Token scores and their gradient in each grouping of threads that numbers of rows and lengths may take, all
rows against plain statements in 64 bits.

The entropy's bound. Sums lie below a shift that may be up to 8 exponents below that of the row's largest logit, and
at most one above it: exponents e are at most 8, S >= 1/2. S is off by 8e-6 of itself (token_ref), and so is each term of
T = sum e 2^e; sum |e| 2^e <= |T| + 2 (8 S), the terms above 0 being at most 8 S. Hence H = log S - log 2 T / S is off by at most
8e-6 (1 + log 2 (|T / S| + 16) + log 2 |T / S|), where log 2 |T / S| = |log S - H| <= max(8 log 2, H + log 2): 8e-6 (12.1 + 2 (H + 5.6)).
"""
import numpy as np
import pytest

import scores_ref as ref
from test_gpu_scores import check_backward, check_forward, given, make

pytestmark = pytest.mark.gpu


def check_all_rows(x, y, top, scale=1.0):
    """As check_forward, the 64-bit side on the GPU."""
    import torch
    from paper_1905_12948_gb300 import token_scores
    r = token_scores(x, y, top=top, scale=scale)
    s = float(np.float32(scale))
    lp = torch.log_softmax(x.double() * s, 1)
    empty = (x == -torch.inf).all(1)
    lp[empty] = -torch.inf
    h = -torch.where(lp > -torch.inf, lp.exp() * lp, 0.0).sum(1)
    counts = (y >= 0).any(1)
    assert ((r.entropy - torch.where(counts, h, 0.0)).abs() <= 8e-6 * (12.1 + 2 * (h + 5.6))).all()
    pairs = [(r.logp, torch.where(y >= 0, lp.gather(1, y.clamp(min=0)), 0.0))]
    if top:
        order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(r.top_index, torch.where(counts[:, None], order, -1))
        pairs.append((r.top_logp, torch.where(counts[:, None], lp.gather(1, order), 0.0)))
    for got, want in pairs:
        fin = want.float() > -torch.inf      # (the lowest float, 1 / 0.7 times: no float is that low)
        assert torch.equal(got == -torch.inf, ~fin)
        assert ((got - want).abs()[fin] <= (ref.LOGP + 2 * ref.U * want.abs())[fin]).all()


def with_masks(x):
    """Rows of -inf and of the type's lowest value, whole and in part, and of one value."""
    import torch
    V, lowest = x.shape[1], torch.finfo(x.dtype).min
    x[0] = -torch.inf
    x[1] = lowest
    x[2, : V // 2] = -torch.inf
    x[3, V // 3:] = lowest
    x[4] = 0.25
    x[5] = -torch.inf
    x[5, V - 1] = 3
    return x


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V", [(2_000, 600), (1_500, 1_000), (1_600, 4_000), (1_500, 9_000), (1_403, 77)])
@pytest.mark.parametrize("top", [0, 1, 9, 20, 33, 64])
def test_short_rows_by_warps(kind, n, V, top):
    """Bounds from the lanes' largest logits (up to 8 best), from their batches' (9 to 64), and from all elements of a batch
    (33 to 64)."""
    check_all_rows(with_masks(make(n, V, kind, seed=V + top, spread=2.5 if top % 2 else 0.3)), given(n, V, 2, masked=0.1), top)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "steps"])
@pytest.mark.parametrize("V", [300, 2_100])
@pytest.mark.parametrize("top", [7, 40])
def test_orders_and_ties_by_warps(kind, order, V, top):
    """Rows that put every element above all before it, and rows of few distinct values: lists that are cut back many times."""
    import torch
    i = torch.arange(V, dtype=torch.float32)
    row = {"ascending": i / V * 8, "descending": -i / V * 8, "equal": torch.full((V,), 0.25), "steps": (i * 7919 % 13).floor()}[order]
    x = torch.stack([row, row.flip(0)]).repeat(750, 1).to(make(1, 1, kind).dtype).cuda()
    check_all_rows(x, given(1_500, V, 1), top)


@pytest.mark.parametrize("kind,n,V", [("bf16", 320, 70_000), ("f16", 310, 70_001), ("f32", 320, 40_000)])
@pytest.mark.parametrize("top", [0, 5, 64])
def test_long_rows_by_a_block_each(kind, n, V, top):
    check_all_rows(with_masks(make(n, V, kind, seed=V, spread=2.5)), given(n, V, 2, masked=0.1), top, 1 / 0.7)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V", [(8, 50_257), (7, 131_072), (100, 40_000)])
@pytest.mark.parametrize("top", [0, 3, 64])
def test_few_rows_with_and_without_room_for_clusters(kind, n, V, top):
    import torch
    from paper_1905_12948_gb300 import load
    x, y = with_masks(make(n, V, kind, seed=V)), given(n, V, 2)
    check_all_rows(x, y, top)
    load().gmc_test_refuse_cooperative(1)
    try:
        check_all_rows(x, y, top)
    finally:
        load().gmc_test_refuse_cooperative(0)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,k", [(700, 300, 2), (601, 333, 33), (1_300, 64, 64), (2_000, 1_001, 17)])
def test_gradient_by_warps_with_many_given_tokens(kind, n, V, k):
    """Every lane sums all of a row's slopes, and looks for its own token among all of them: what other lanes have put
    into shared memory. Tokens come twice in most of the rows, a fifth of which do not count."""
    check_backward(make(n, V, kind, seed=n), given(n, V, k, masked=0.2), kind)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V", [(6, 50), (6, 40_000), (700, 300)])
def test_alternatives_of_a_row_that_is_not_a_number(kind, n, V):
    """NaN and +inf make a row's alternatives -1: the gradient through them is NaN where the row has slopes, as with any
    other tokens, and not that of a row that does not count."""
    import torch
    from paper_1905_12948_gb300 import token_scores, token_scores_backward
    x = make(n, V, kind)
    x[1, V // 2] = torch.nan
    x[3, 7] = torch.inf
    bad = torch.tensor([1, 3], device="cuda")
    fine = torch.tensor([r for r in range(n) if r not in (1, 3)], device="cuda")
    r = token_scores(x, top=4, return_stats=True)
    assert (r.top_index[bad] == -1).all() and (r.top_index[fine] >= 0).all()
    ones = torch.ones(n, 4, device="cuda")
    h = torch.ones(n, device="cuda")
    for slopes in ((ones, None), (None, h), (ones, h)):
        d = token_scores_backward(x, r.top_index, r.stats, *slopes)
        assert d[bad].isnan().all() and d[fine].isfinite().all()
    ones[1], h[1] = 0, 0                         # without slopes it is not read
    d = token_scores_backward(x, r.top_index, r.stats, ones, h)
    assert (d[1] == 0).all() and d[3].isnan().all()
    # rows that did not count are told apart: zeros, whatever their logits and slopes
    y = given(n, V, 4)
    y[1] = -1
    r = token_scores(x, y, top=4, return_stats=True)
    slope = torch.full((n, 4), torch.nan, device="cuda")
    slope[2:] = 1
    d = token_scores_backward(x, r.top_index, r.stats, slope, h)
    assert (d[1] == 0).all() and d[3].isnan().all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("e", [-64, -40, 20, 30, 33, 34, 48, 64])
@pytest.mark.parametrize("n,V", [(3, 50), (3, 9_000), (1_500, 600)])
def test_any_scale(kind, e, n, V):
    """Scales up to the largest, of rows whose largest logit is 0 (that of a normalised row), or far from it: a logit that lies far
    below the largest adds nothing, however small a number of the type that is."""
    import torch
    x = make(n, V, kind, seed=V)
    x -= x.amax(1, keepdim=True)
    x[1] *= 2.0 ** -10          # (half: down to its subnormal numbers)
    x[2] += 5
    check_forward(x, None, 3, 2.0 ** e)
    check_forward(x, given(n, V, 2), 0, 2.0 ** e)


def test_results_are_saved_and_read():
    """A teacher's best tokens are kept in files: together, alone, and whole."""
    import io

    import torch
    from paper_1905_12948_gb300 import token_scores
    r = token_scores(make(5, 300, "bf16"), given(5, 300, 2), top=8, return_stats=True)
    for some in (tuple(r), (r.top_logp, r.top_index), r.top_index, r.logp):
        f = io.BytesIO()
        torch.save(some, f)
        f.seek(0)
        back = torch.load(f)
        pairs = [(some, back)] if torch.is_tensor(some) else zip(some, back)
        assert all(torch.equal(a, b) and a.dtype == b.dtype for a, b in pairs)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("e", [-64, -40, 20, 34, 64])
@pytest.mark.parametrize("n,V", [(4, 50), (4, 9_000), (700, 300)])
def test_gradient_at_any_scale(kind, e, n, V):
    """Slopes small enough for a large scale's gradient to fit the type."""
    x = make(n, V, kind, seed=V)
    x -= x.amax(1, keepdim=True)
    x[1] *= 2.0 ** -10
    x[2] += 5
    check_backward(x, given(n, V, 3), kind, 2.0 ** e, unit=2.0 ** -max(e, 0))
