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


def _check(r, x, y, old, adv, args, kind):
    """A call's outputs against the 64-bit statement."""
    import torch
    n = x.shape[0]
    weights, rf = args["weights"].double().cpu().numpy(), args["ref_logp"].double().cpu().numpy()
    lp = torch.cat([torch.log_softmax(p.double(), 1).gather(1, q.clamp(min=0)[:, None])[:, 0]
                    for p, q in zip(x.split(256), y.split(256))]).cpu().numpy()
    yn, o, a = y.cpu().numpy(), old.double().cpu().numpy(), adv.double().cpu().numpy()
    loss, each, coef = ref.policy(lp, yn, o, a, weights, rf, args["clip_low"], args["clip_high"], args["kl"])
    bound = ref.policy_bound(lp, o, a, rf, args["kl"])
    counts = yn >= 0
    got = r.logp.double().cpu().numpy()
    assert (abs(got - lp)[counts] <= (ref.LOGP + 2 * ref.U * abs(lp))[counts]).all() and (got[~counts] == 0).all()
    assert (abs(r.token_loss.double().cpu().numpy() - each) <= bound).all()
    assert abs(float(r.loss) - loss) <= (weights * bound)[counts].sum() + 2 * ref.U * abs(loss)
    rel, low = ref.ROUND[kind]
    k_all, dk_all = torch.from_numpy(coef).cuda(), torch.from_numpy(abs(weights * bound) * counts).cuda()
    for i in range(0, n, 256):      # ref.gradient and ref.gradient_bound, on the device
        p = torch.softmax(x[i: i + 256].double(), 1)
        k, dk, at = k_all[i: i + 256, None], dk_all[i: i + 256, None], y[i: i + 256].clamp(min=0)[:, None]
        want = -k * p
        want.scatter_add_(1, at, k)
        away = p.scatter(1, at, 1 - p.gather(1, at))
        off = dk * away + k.abs() * (ref.P * p + 2.0 ** -126)
        off.scatter_add_(1, at, k.abs() * (2 * ref.LOGP + 4 * ref.U))
        off = off + rel * (k.abs() * away + off) + low
        d = r.dlogits[i: i + 256].double()
        bad = ~((d - want).abs() <= off)
        assert not bad.any(), (i, bad.nonzero()[:5], d[bad][:5], want[bad][:5], off[bad][:5])
        assert (d[(y[i: i + 256] < 0)] == 0).all()


# parts: the blocks that share a row at these lengths; each takes more than 16 rows, so that its
# eight row slots, its ring and the two sets of messages are used again and again
RING = [(3_000, 15_001, "bf16", 1), (2_600, 15_000, "f16", 1), (2_600, 7_503, "f32", 1), (1_500, 50_257, "bf16", 2),
        (720, 70_003, "f16", 4), (360, 131_073, "f32", 8)]


@pytest.mark.parametrize("masked", [0.0, 0.2])
@pytest.mark.parametrize("n,V,kind,parts", RING)
def test_many_rows_a_cluster(n, V, kind, parts, masked):
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert n * parts > 16 * sms
    x, y, old, adv, args = _inputs(n, V, kind, 3, masked)
    h = TokenLoss(n)
    r = h.policy(x, y, old, adv, **args)
    _check(r, x, y, old, adv, args, kind)
    again = h.policy(x, y, old, adv, **args)
    assert torch.equal(again.loss, r.loss) and torch.equal(again.dlogits, r.dlogits)
    h.close()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,most", [(30_000, 301, 56), (20_000, 1_021, 56), (11_000, 4_999, 22)])
def test_many_rows_a_warp(n, V, most, kind):
    """most: warps of an SM at most, so that each takes rows in turn from one buffer."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert n > 2 * most * sms
    x, y, old, adv, args = _inputs(n, V, kind, 4, 0.2)
    h = TokenLoss(n)
    r = h.policy(x, y, old, adv, **args)
    _check(r, x, y, old, adv, args, kind)
    again = h.policy(x, y, old, adv, **args)
    assert torch.equal(again.loss, r.loss) and torch.equal(again.dlogits, r.dlogits)
    h.close()


@pytest.mark.parametrize("n,V,kind", [c[:3] for c in RING] + [(11_000, 4_999, "bf16"), (20_000, 301, "f16")])
def test_many_rows_in_place(n, V, kind):
    """The gradient in the logits' place: the same bits as beside them, call after call."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    x, y, old, adv, args = _inputs(n, V, kind, 5, 0.2)
    h = TokenLoss(n)
    want = h.policy(x, y, old, adv, **args)
    for _ in range(5):
        t = x.clone()
        r = h.policy(t, y, old, adv, out=t, **args)
        assert r.dlogits is t and torch.equal(t, want.dlogits)
        assert torch.equal(r.loss, want.loss) and torch.equal(r.logp, want.logp)
    h.close()


@pytest.mark.parametrize("y", [0, 69_000])
def test_marked_targets_and_nan_targets_of_a_cluster(y):
    """A target outside the vocabulary, and one whose logit is NaN, in a row that several blocks
    share: the row is NaN in all of its blocks' shares, the others are as they were."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss
    n, V = 4, 70_003
    x, tgt, old, adv, args = _inputs(n, V, "bf16", 6)
    h = TokenLoss(n)
    want = h.policy(x, tgt, old, adv, **args)
    bad = x.clone()
    bad[1, y] = float("nan")
    marked = tgt.clone()
    marked[1], marked[2] = y, V
    r = h.policy(bad, marked, old, adv, **args)
    assert torch.isnan(r.dlogits[1:3]).all() and torch.isnan(r.token_loss[1:3]).all() and torch.isnan(r.loss)
    for i in (0, 3):
        assert torch.equal(r.dlogits[i], want.dlogits[i]) and torch.equal(r.token_loss[i], want.token_loss[i])
    h.close()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,V,kind,refuse", [(400, 50_257, "bf16", True),
                                             (130, 300_001, "f32", False), (130, 540_003, "bf16", False)])
def test_many_rows_swept_twice(n, V, kind, refuse, in_place):
    """Rows over 1 MB by clusters of 8, and shorter ones where a launch of clusters is refused: more rows than
    two blocks an SM take at once."""
    import torch
    from paper_1905_12948_gb300 import TokenLoss, gmc
    x, y, old, adv, args = _inputs(n, V, kind, 8, 0.2)
    h = TokenLoss(n)
    t = x.clone()
    try:
        assert gmc.load().gmc_test_refuse_cooperative(int(refuse)) == 0
        r = h.policy(t, y, old, adv, out=t if in_place else None, **args)
    finally:
        gmc.load().gmc_test_refuse_cooperative(0)
    _check(r, x, y, old, adv, args, kind)
    h.close()
