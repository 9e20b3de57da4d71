"""Waits of the policy loss that give up here and there: with a limit that ordinary waits reach."""
import pytest

pytestmark = pytest.mark.gpu

# the ring by one block and by 2, 4 and 8, and a warp a row
SHAPES = [(400, 15_001, "bf16"), (300, 50_257, "bf16"), (120, 70_003, "f16"), (60, 131_073, "f32"), (9_000, 2_001, "bf16")]


def _call(n, V, kind):
    """(a call, a row that does not count): the call's loss, token losses, logp and gradient."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    g = torch.Generator(device="cuda").manual_seed(31)
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]
    x = torch.randn((n, V), generator=g, device="cuda").to(dtype)
    y = torch.randint(0, V, (n,), generator=g, device="cuda")
    y[n // 3] = -1
    old, adv = -9 - torch.rand(n, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda") + 0.5
    h = TokenLoss(n)
    out = torch.empty_like(x)

    def call():
        out.fill_(7.0)      # what is not written stays
        return h.policy(x, y, old, adv, out=out)

    return h, call, n // 3


@pytest.mark.parametrize("n,V,kind", SHAPES)
def test_the_next_call_is_right(n, V, kind):
    import torch
    h, call, row = _call(n, V, kind)
    want = [t.clone() for t in call()]
    for limit in (1, 1, 500, 2_000, 10_000, 40_000, 150_000):
        assert h.lib.gmc_test_withhold_row(h.h, row, limit) == 0
        call()
        for got, right in zip(call(), want):
            assert torch.equal(got, right), limit
    h.close()


@pytest.mark.parametrize("n,V,kind", SHAPES)
def test_a_loss_that_is_a_number_has_its_gradient(n, V, kind):
    """Whichever waits give up (few: the hardware holds a wait for microseconds before it is asked again), in
    whichever block of a cluster: the loss is NaN, or every output is what it is without a limit."""
    import torch
    h, call, row = _call(n, V, kind)
    want = [t.clone() for t in call()]
    for limit in [int(10 * 1.3 ** i) for i in range(44)] * 3:      # 10 ns to 0.8 ms
        assert h.lib.gmc_test_withhold_row(h.h, row, limit) == 0
        got = call()
        if torch.isnan(got.loss):
            continue
        for a, b in zip(got, want):
            assert torch.equal(a, b), limit
    h.close()
