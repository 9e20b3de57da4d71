"""The policy loss where its kernels' loops turn: many rows a block, a cluster and a warp.
The 64-bit statement is formed on the device, in slices of rows, within token_ref's bounds."""
import pytest

import token_ref as ref

pytestmark = pytest.mark.gpu


def _type(kind):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


def _inputs(n, V, kind, seed, masked=0.0):
    """Logits with rows at V elements, targets, and the other arguments of a policy call. No ratio
    lies within 0.05 of a bound of the clip (0.8 and 1.28)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")
    x = (torch.randn((n, V), generator=g, device="cuda") * 2.5).to(_type(kind))
    y = torch.randint(0, V, (n,), generator=g, device="cuda")
    rows = torch.arange(n, device="cuda")
    x[rows, y] += 6 * rand(n).to(x.dtype)
    lp = torch.cat([torch.log_softmax(p.double(), 1).gather(1, q[:, None])[:, 0]
                    for p, q in zip(x.split(256), y.split(256))])
    old = (lp - torch.log(torch.tensor([0.5, 0.7, 0.9, 1.1, 1.4], device="cuda")[(5 * rand(n)).long()])).float()
    args = dict(weights=rand(n) + 0.1, ref_logp=(lp + 0.6 * rand(n) - 0.3).float(), clip_low=0.2, clip_high=0.28, kl=0.05)
    y = torch.where(rand(n) < masked, -1, y)
    return x, y, old, 2 * rand(n) - 1, args


@pytest.mark.parametrize("n,V", [(152, 16_384), (152, 65_536), (700, 1_024)])
def test_loss_of_alternating_calls(n, V):
    """Two inputs in turn with one handle: each call's loss is that of its own tokens, the same
    bits each time, whatever the call before left in the workspace."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    h = TokenLoss(n)
    calls = [_inputs(n, V, "bf16", seed) for seed in (1, 2)]
    first = []
    for x, y, old, adv, args in calls:
        r = h.policy(x, y, old, adv, **args)
        want = float((r.token_loss.double() * args["weights"].double()).sum())
        # the products and sums are formed in 64 bits and rounded once
        assert abs(float(r.loss) - want) <= 2 * ref.U * abs(want)
        first.append(r.loss)
    losses = [[h.policy(x, y, old, adv, **args).loss for x, y, old, adv, args in calls] for _ in range(100)]
    for pair in losses:
        assert torch.equal(pair[0], first[0]) and torch.equal(pair[1], first[1])
    h.close()
