"""Dropout from the counter stream: masks exactly, values within one rounding."""
import numpy as np
import pytest

import token_ref as ref

pytestmark = pytest.mark.gpu
KINDS = ["f32", "bf16", "f16"]
SEED, T, SITE = 0xFEDCBA9876543210, 12, 5


def _type(kind):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


def _want(x, res, p, worker=0, seed=SEED, t=T, site=SITE):
    q = round(p * 65536)
    out = np.zeros_like(x) if res is None else res.copy()
    for k in range(x.shape[0]):
        keep = ref.dropout_bits(seed, t, worker + k, site, x.shape[1]) >= q
        out[k] += np.where(keep, x[k] * (65536 / max(1, 65536 - q)), 0.0)
    return out


def _close(got, want, x, kind, p):
    """The product and the sum are rounded to 32 bits (gain and product: 2u of the
    product, u of the sum), then once to the type."""
    rel, low = ref.ROUND[kind]
    gain = 65536 / max(1, 65536 - round(p * 65536))
    bound = 2 * ref.U * np.abs(x) * gain + 2 * ref.U * np.abs(want)
    bound = bound + rel * (np.abs(want) + bound) + low
    assert (np.abs(got - want) <= bound).all()


def _make(K, n, kind, seed, pad=0, shift=0):
    import torch
    buf = torch.full((K * (n + pad) + shift,), float("nan"), dtype=_type(kind), device="cuda")
    t = buf[shift:].as_strided((K, n), (n + pad, 1))
    t.copy_(torch.from_numpy(np.random.default_rng([seed, K, n]).standard_normal((K, n))).cuda())
    return t


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("K,n", [(1, 1), (2, 3), (3, 4), (1, 5), (4, 8), (2, 1_023), (3, 2_049), (5, 4_097), (1, 70_001)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.9, 1.0])
def test_values(K, n, p, kind):
    from paper_1905_12948_gb300 import dropout, dropout_backward
    x, res = _make(K, n, kind, 1), _make(K, n, kind, 2)
    xd, rd = x.double().cpu().numpy(), res.double().cpu().numpy()
    args = dict(seed=SEED, t=T, site=SITE, worker=3)
    got = dropout(x, p, residual=res, **args).double().cpu().numpy()
    _close(got, _want(xd, rd, p, 3), xd, kind, p)
    got = dropout_backward(x, p, **args).double().cpu().numpy()
    want = _want(xd, None, p, 3)
    _close(got, want, xd, kind, p)
    assert np.array_equal(got == 0, want == 0)      # the mask itself


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pads", [(1, 1, 1), (0, 3, 0), (5, 0, 2), (8, 8, 8)])
@pytest.mark.parametrize("shifts", [(0, 0, 0), (1, 1, 1), (3, 2, 7), (0, 1, 0), (5, 5, 2)])
def test_strides_and_alignments(pads, shifts, kind):
    import torch
    from paper_1905_12948_gb300 import dropout
    K, n, p = 3, 1_501, 0.25
    x, res = _make(K, n, kind, 3, pads[0], shifts[0]), _make(K, n, kind, 4, pads[1], shifts[1])
    buf = torch.full((K * (n + pads[2]) + shifts[2],), 7.0, dtype=_type(kind), device="cuda")
    out = buf[shifts[2]:].as_strided((K, n), (n + pads[2], 1))
    xd, rd = x.double().cpu().numpy(), res.double().cpu().numpy()
    for r, rr in ((res, rd), (None, None)):
        assert dropout(x, p, seed=SEED, t=T, site=SITE, residual=r, out=out) is out
        _close(out.double().cpu().numpy(), _want(xd, rr, p), xd, kind, p)
        flat, beside = buf.float().cpu().numpy(), np.ones(buf.numel(), bool)
        for k in range(K):
            at = shifts[2] + k * (n + pads[2])
            beside[at: at + n] = False
        assert (flat[beside] == 7.0).all()


@pytest.mark.parametrize("kind", KINDS)
def test_in_place_and_rows_apart(kind):
    """The mask is worker's, wherever the row lies: stacked, alone, in place, in parts of
    another shape."""
    import torch
    from paper_1905_12948_gb300 import dropout
    x = _make(4, 3_002, kind, 5)
    res = _make(4, 3_002, kind, 6)
    args = dict(seed=1, t=0, site=0)
    want = dropout(x, 0.3, residual=res, worker=2, **args)
    for k in range(4):
        assert torch.equal(dropout(x[k: k + 1], 0.3, residual=res[k: k + 1], worker=2 + k, **args)[0], want[k])
    y = x.clone()
    assert dropout(y, 0.3, residual=res, worker=2, out=y, **args) is y and torch.equal(y, want)
    r = res.clone()
    assert torch.equal(dropout(x, 0.3, residual=r, worker=2, out=r, **args), want)
    shaped = dropout(x.view(4, 2, 19, 79), 0.3, residual=res.view(4, 2, 19, 79), worker=2, **args)
    assert torch.equal(shaped.view(4, -1), want)
    other = [dropout(x, 0.3, worker=2, **{**args, **c}) for c in ({}, {"seed": 2}, {"t": 1}, {"site": 1})]
    for i in range(4):
        for j in range(i):
            assert not torch.equal(other[i] == 0, other[j] == 0)


def test_dropped_values_are_not_computed_with():
    import torch
    from paper_1905_12948_gb300 import dropout
    n = 4_001
    keep = ref.dropout_bits(9, 0, 0, 0, n) >= round(0.5 * 65536)
    x = torch.from_numpy(np.where(keep, 1.0, np.nan)[None]).float().cuda()
    x[0, torch.from_numpy(~keep).cuda().nonzero()[::2, 0]] = float("inf")
    got = dropout(x, 0.5, seed=9, residual=torch.ones_like(x)).cpu().numpy()[0]
    assert np.array_equal(got, np.where(keep, 3.0, 1.0))
    assert (dropout(x, 1.0, seed=9) == 0).all()


def test_beyond_32_bits():
    """Elements past 2^31 of one row."""
    import torch
    from paper_1905_12948_gb300 import dropout
    n = (1 << 31) + 4_099
    x = torch.ones((1, n), dtype=torch.bfloat16, device="cuda")
    y = dropout(x, 0.5, seed=3, t=1, site=2)
    mask, gamma = (1 << 64) - 1, 0x9E3779B97F4A7C15

    def mix(z):
        z &= mask
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
        return z ^ (z >> 31)

    key = 3 ^ 0x44524F504F555421
    for number in (1, 1, 2):
        key = mix(key + gamma * (number + 1))
    tail = y[0, n - 4_099:].float().cpu().numpy()
    want = [2.0 if (mix(key + gamma * (i // 4 + 1)) >> (16 * (i % 4))) & 0xFFFF >= 32768 else 0.0
            for i in range(n - 4_099, n)]
    assert np.array_equal(tail, want)
    share = sum(int((part != 0).sum()) for part in y[0].split(1 << 28)) / n
    assert abs(share - 0.5) < 5 * 0.5 / n ** 0.5


def test_stream_and_empty():
    import torch
    from paper_1905_12948_gb300 import dropout
    x = _make(2, 5_000, "f32", 8)
    want = dropout(x, 0.2, seed=4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = dropout(x, 0.2, seed=4, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    assert dropout(x[:, :0], 0.2, seed=4).shape == (2, 0)
    assert dropout(x[:0], 0.2, seed=4).shape == (0, 5_000)


def test_refusals():
    import torch
    from paper_1905_12948_gb300 import GMCError, dropout, gmc
    x = torch.zeros((2, 8), device="cuda")
    for bad in (x.cpu(), x.double(), x[0], x.t(), x[:, ::2], x[:1].expand(2, 8)):
        with pytest.raises(TypeError):
            dropout(bad, 0.1, seed=0)
    with pytest.raises(TypeError):
        dropout(x, 0.1, seed=0, residual=x.half())
    with pytest.raises(TypeError):
        dropout(x, 0.1, seed=0, out=x[:1])
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(GMCError):
            dropout(x, p, seed=0)
    for bad in (dict(worker=-1), dict(t=-1), dict(site=-1)):
        with pytest.raises(GMCError):
            dropout(x, 0.1, seed=0, **bad)
    lib, p = gmc.load(), x.data_ptr()
    ok = dict(x=p, ldx=8, r=None, ldr=0, o=p, ldo=8, dtype=0, w=0, K=2, n=8, p=0.1, seed=0, t=0, site=0, s=0)
    assert lib.gmc_dropout(*ok.values()) == 0
    for bad in (dict(dtype=5), dict(ldx=7), dict(ldo=7), dict(r=p, ldr=4), dict(x=p + 1), dict(x=None), dict(K=-1),
                dict(n=-1), dict(n=1 << 41), dict(K=(1 << 20) + 1)):
        assert lib.gmc_dropout(*{**ok, **bad}.values()) == 1, bad
    torch.cuda.synchronize()
