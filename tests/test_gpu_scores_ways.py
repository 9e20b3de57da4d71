"""Token scores and their gradient in each grouping of threads that numbers of rows and lengths may take, all
rows against plain statements in 64 bits."""
import pytest

from test_gpu_scores import check_backward, check_forward, given, make

pytestmark = pytest.mark.gpu


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
