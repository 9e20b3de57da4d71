"""Token scores and their gradient in each grouping of threads that numbers of rows and lengths may take, all
rows against plain statements in 64 bits."""
import pytest

from test_gpu_scores import check_backward, given, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,k", [(700, 300, 2), (601, 333, 33), (1_300, 64, 64), (2_000, 1_001, 17)])
def test_gradient_by_warps_with_many_given_tokens(kind, n, V, k):
    """Every lane sums all of a row's slopes, and looks for its own token among all of them: what other lanes have put
    into shared memory. Tokens come twice in most of the rows, a fifth of which do not count."""
    check_backward(make(n, V, kind, seed=n), given(n, V, k, masked=0.2), kind)
