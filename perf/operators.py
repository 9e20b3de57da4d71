"""The operators of a language model's post-training step, as cases that can be timed and compared.

A case is one call of an operator as a training program makes it, or the two
calls of its directions: the log-probabilities of given tokens from logits
(``token_logp``, and its backward pass), the clipped policy loss with a KL term
and the preference loss on paired log ratios (both with the gradient of the
logits), and dropout from the counter stream of (seed, t, worker, site), forward
with a residual and backward.

``run`` computes them in elementary torch operations in 32 bits, or, where
``own`` is true, through the library. ``exact`` does so in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
BETA, SMOOTH = 0.1, 0.05           # preference loss
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04
SEED, T, SITE = 0x5DEECE66D1234567, 41, 3   # of the dropout's stream


def _logp(name, n, V, dtype, grad, *, scale=1.0, padded=False):
    return {"name": name, "kind": "logp", "n": n, "V": V, "dtype": dtype, "grad": grad, "scale": scale,
            "padded": padded}


def _policy(name, n, V, dtype, *, scale=1.0, padded=False, masked=0.2):
    return {"name": name, "kind": "policy", "n": n, "V": V, "dtype": dtype, "scale": scale,
            "padded": padded, "masked": masked}


def _preference(name, pairs, lo, hi, V, dtype, *, scale=1.0, padded=False):
    return {"name": name, "kind": "preference", "pairs": pairs, "lo": lo, "hi": hi, "V": V,
            "dtype": dtype, "scale": scale, "padded": padded}


def _dropout(name, K, n, dtype, p):
    return {"name": name, "kind": "dropout", "K": K, "n": n, "dtype": dtype, "p": p}


def listed():
    return [
        # one token scored as it is sampled: the smallest call, a long row
        _logp("logp_token", 1, 131_072, "bf16", False),
        # rollouts scored under the old or the reference policy, no gradient
        _logp("logp_score", 8_192, 32_000, "bf16", False, scale=1 / 0.7),
        # the general building block of a loss, forward and backward, fp32 and an odd vocabulary
        _logp("logp_grad_f32", 4_096, 50_257, "f32", True),
        # a short batch: 64 tokens' policy step, where launches count
        _policy("policy_small", 64, 32_000, "bf16"),
        # an ordinary batch, every row at another alignment, a fifth of the tokens masked
        _policy("policy_odd", 3_001, 50_257, "bf16", scale=1 / 0.7),
        # fp32 logits with a vocabulary padded at its end (logits of -inf)
        _policy("policy_f32_padded", 1_024, 128_256, "f32", padded=True),
        # the largest: 8,192 tokens of a large vocabulary
        _policy("policy_large", 8_192, 131_072, "bf16", masked=0.1),
        # two short pairs
        _preference("pref_small", 2, 20, 40, 32_000, "bf16"),
        # an ordinary batch of ragged pairs, odd vocabulary
        _preference("pref_odd", 16, 40, 512, 50_257, "bf16"),
        # the largest: longer pairs of a large, padded vocabulary
        _preference("pref_large", 16, 100, 384, 128_256, "bf16", padded=True),
        # the activations of four workers' small model
        _dropout("dropout_small", 4, 65_536, "f32", 0.1),
        # eight workers' hidden states, 4,096 tokens of 4,096 channels each
        _dropout("dropout_large", 8, 4_096 * 4_096, "bf16", 0.1),
    ]


def _spread(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


def draw(rng):
    kind = rng.choice(["logp", "logp", "policy", "policy", "preference", "preference", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
    if kind == "dropout":
        K = _spread(rng, 1, 32)
        n = _spread(rng, 1_000, (1 << 27) * 2 // SIZES[dtype] // K)
        n -= n % 8 if rng.random() < 0.5 else 0
        c = _dropout("", K, n, dtype, rng.choice([0.0, 0.05, 0.1, 0.3]))
    else:
        V = _spread(rng, 2_000, 131_072)
        V -= V % 64 if rng.random() < 0.4 else 0
        scale, padded = rng.choice([1.0, 1.0, 1 / 0.7, 0.5]), rng.random() < 0.3
        most = (1 << 30) * 2 // SIZES[dtype] // V      # rows of the largest
        if kind == "preference":
            pairs = _spread(rng, 1, 32)
            hi = _spread(rng, 4, min(1_024, max(4, most // (2 * pairs))))
            c = _preference("", pairs, max(1, hi // 5), hi, V, dtype, scale=scale, padded=padded)
        elif kind == "policy":
            c = _policy("", _spread(rng, 1, min(most, 16_384)), V, dtype, scale=scale, padded=padded,
                        masked=rng.choice([0.0, 0.2, 0.5]))
        else:
            c = _logp("", _spread(rng, 1, min(most, 16_384)), V, dtype, rng.random() < 0.5, scale=scale,
                      padded=padded)
    del c["name"]
    return c


# -- inputs -------------------------------------------------------------------
def _lengths(case):
    """The lengths of the 2 * pairs sequences; part of the case, not of the seed."""
    rng = random.Random(case["pairs"] * 1_000_003 + case["lo"] * 1_009 + case["hi"])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(2 * case["pairs"])]


def _rows(case):
    return sum(_lengths(case)) if case["kind"] == "preference" else case["n"]


def _plain_logp(logits, targets, scale):
    """(log-probability, maximum, log of the sum) of each row, 32 bits."""
    x = logits.float()
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    z = (x - m).mul_(scale)
    t = z.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    s = z.exp_().sum(-1)
    ls = torch.where(s > 0, s.log(), 0.0)
    return torch.where(targets >= 0, t - ls, 0.0), m, ls


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    dtype = DTYPES[case["dtype"]]
    if case["kind"] == "dropout":
        shape = case["K"], case["n"]
        return {"x": normal(*shape).to(dtype), "residual": normal(*shape).to(dtype), "dy": normal(*shape).to(dtype)}
    n, V = _rows(case), case["V"]
    # logits of a model: a few units wide, the trained-on token usually among the larger ones
    targets = torch.randint(0, V - V // 200 if case["padded"] else V, (n,), generator=gen, device="cuda")
    x = normal(n, V).mul_(2.5)
    rows = torch.arange(n, device="cuda")
    x[rows, targets] += torch.rand(n, generator=gen, device="cuda") * 9
    if case["padded"]:
        x[:, V - V // 200:] = -math.inf
    s = {"logits": x.to(dtype), "targets": targets}
    if case["kind"] == "logp":
        s["dlogp"] = normal(n) * (1.0 if dtype == torch.float16 else 1 / n)
        return s
    logp = torch.cat([_plain_logp(s["logits"][i: i + 1_024], targets[i: i + 1_024], case["scale"])[0]
                      for i in range(0, n, 1_024)])
    if case["kind"] == "policy":
        # the rollout's policy a few updates old, the reference further off; rewards above a low baseline
        s["old_logp"] = logp + normal(n) * 0.15
        s["ref_logp"] = logp + normal(n) * 0.3
        s["advantages"] = normal(n) + 0.5
        keep = torch.rand(n, generator=gen, device="cuda") >= case["masked"]
        # 16-bit gradients of fp16 are kept in range by a loss scale
        s["weights"] = keep.float() * ((1024.0 if dtype == torch.float16 else 1.0) / n)
        return s
    lengths = _lengths(case)
    offsets = [0]
    for length in lengths:
        offsets.append(offsets[-1] + length)
    s["offsets"] = torch.tensor(offsets, dtype=torch.int64, device="cuda")
    s["longest"] = max(lengths)
    # the first quarter of a sequence is its prompt: no log-probability is taken there
    at = rows - torch.repeat_interleave(s["offsets"][:-1], s["offsets"].diff())
    long = torch.repeat_interleave(s["offsets"].diff(), s["offsets"].diff())
    s["targets"] = torch.where(at < long // 4, -1, targets)
    s["ref_logp"] = logp + normal(n) * 0.4
    s["weights"] = torch.full((case["pairs"],), (1024.0 if dtype == torch.float16 else 1.0) / case["pairs"],
                              device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own and case["kind"] in ("policy", "preference"):
        from paper_1905_12948_gb300 import TokenLoss
        s["loss"] = TokenLoss(max_rows=_rows(case), max_pairs=case.get("pairs", 0))
    return s


# -- the operators ------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_1905_12948_gb300 import dropout, dropout_backward, token_logp, token_logp_backward
    case = s["case"]
    if case["kind"] == "dropout":
        return {"out": dropout(s["x"], case["p"], seed=SEED, t=T, site=SITE, residual=s["residual"]),
                "dx": dropout_backward(s["dy"], case["p"], seed=SEED, t=T, site=SITE)}
    if case["kind"] == "logp":
        if not case["grad"]:
            return {"logp": token_logp(s["logits"], s["targets"], scale=case["scale"])}
        logp, stats = token_logp(s["logits"], s["targets"], scale=case["scale"], return_stats=True)
        return {"logp": logp, "dlogits": token_logp_backward(s["logits"], s["targets"], stats, s["dlogp"],
                                                             scale=case["scale"])}
    if case["kind"] == "policy":
        r = s["loss"].policy(s["logits"], s["targets"], s["old_logp"], s["advantages"], weights=s["weights"],
                             ref_logp=s["ref_logp"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl=KL,
                             scale=case["scale"])
        return {"loss": r.loss, "token_loss": r.token_loss, "logp": r.logp, "dlogits": r.dlogits}
    r = s["loss"].preference(s["logits"], s["targets"], s["offsets"], beta=BETA, smoothing=SMOOTH,
                             ref_logp=s["ref_logp"], weights=s["weights"], scale=case["scale"])
    return {"loss": r.loss, "pair_loss": r.pair_loss, "seq_ratio": r.seq_ratio, "dlogits": r.dlogits}


def _plain_gradient(logits, targets, m, ls, coef, scale):
    """d/dlogits of sum_n coef_n logp_n; zero where coef_n is."""
    p = (logits.float() - m).mul_(scale).sub_(ls[:, None]).exp_()
    p.mul_((-scale * coef)[:, None])
    p.scatter_add_(1, targets.clamp(min=0)[:, None], (scale * coef)[:, None])
    return torch.where((coef != 0)[:, None], p, 0.0).to(logits.dtype)


def _plain_mix(z):
    """SplitMix64's output function on int64, whose shifts to the right keep the sign."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * (0x94D049BB133111EB - (1 << 64))
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _plain_dropout(x, p, residual):
    K, n = x.shape
    gamma = 0x9E3779B97F4A7C15 - (1 << 64)
    worker = torch.arange(K, dtype=torch.int64, device=x.device)
    step = torch.full_like(worker, T)
    tag = 0x44524F504F555421                        # the key of a dropout site's stream
    key = _plain_mix(gamma * (step + 1) + (SEED ^ tag))
    key = _plain_mix(key + gamma * (worker + 2))
    key = _plain_mix(key + gamma * torch.full_like(worker, SITE + 1))
    i = torch.arange((n + 3) // 4, dtype=torch.int64, device=x.device)
    z = _plain_mix(key[:, None] + gamma * (i + 1))
    bits = (z[:, :, None] >> torch.arange(0, 64, 16, device=x.device)) & 0xFFFF
    q = round(p * 65536)
    keep = bits.reshape(K, -1)[:, :n] >= q
    y = torch.where(keep, x.float() * (65536 / (65536 - q)), 0.0)
    return (y if residual is None else residual.float() + y).to(x.dtype)


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "dropout":
        return {"out": _plain_dropout(s["x"], case["p"], s["residual"]),
                "dx": _plain_dropout(s["dy"], case["p"], None)}
    scale, targets = case["scale"], s["targets"]
    logp, m, ls = _plain_logp(s["logits"], targets, scale)
    if case["kind"] == "logp":
        if not case["grad"]:
            return {"logp": logp}
        return {"logp": logp, "dlogits": _plain_gradient(s["logits"], targets, m, ls, s["dlogp"], scale)}
    if case["kind"] == "policy":
        adv, w = s["advantages"], s["weights"]
        ratio = torch.exp(logp - s["old_logp"])
        plain, clipped = ratio * adv, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
        far = s["ref_logp"] - logp
        token_loss = torch.where(w != 0, KL * (far.exp() - far - 1) - torch.minimum(plain, clipped), 0.0)
        slope = KL * (1 - far.exp()) - torch.where(plain <= clipped, plain, 0.0)
        coef = torch.where(w != 0, w * slope, 0.0)
        return {"loss": (w * token_loss).sum(), "token_loss": token_loss, "logp": torch.where(w != 0, logp, 0.0),
                "dlogits": _plain_gradient(s["logits"], targets, m, ls, coef, scale)}
    off, w = s["offsets"], s["weights"]
    at = off[:-1, None] + torch.arange(s["longest"], device=off.device)
    inside = at < off[1:, None]
    each = torch.where(targets >= 0, logp - s["ref_logp"], 0.0)
    seq_ratio = torch.where(inside, each[at.clamp(max=each.shape[0] - 1)], 0.0).sum(1)
    margin = BETA * (seq_ratio[0::2] - seq_ratio[1::2])
    soft = torch.log1p(torch.exp(-margin.abs()))       # -log sigmoid(|margin|)
    loss_up, loss_down = soft + (-margin).clamp(min=0), soft + margin.clamp(min=0)
    pair_loss = (1 - SMOOTH) * loss_up + SMOOTH * loss_down
    sig = 1 / (1 + torch.exp(-margin))
    slope = w * BETA * (SMOOTH * sig - (1 - SMOOTH) * (1 - sig))
    coef = torch.repeat_interleave(torch.stack([slope, -slope], 1).reshape(-1), off.diff(),
                                   output_size=logp.shape[0])
    coef = torch.where(targets >= 0, coef, 0.0)
    return {"loss": (w * pair_loss).sum(), "pair_loss": pair_loss, "seq_ratio": seq_ratio,
            "dlogits": _plain_gradient(s["logits"], targets, m, ls, coef, scale)}


def work(case):
    if case["kind"] == "dropout":
        n, e = case["K"] * case["n"], SIZES[case["dtype"]]
        return {"bytes": 5 * n * e, "flops": 2 * n}
    e, V, n = SIZES[case["dtype"]], case["V"], _rows(case)
    if case["kind"] == "logp":
        return {"bytes": n * V * e * (2 if case["grad"] else 1) + 16 * n, "flops": (8 if case["grad"] else 4) * n * V}
    # rows that count are read, all are written
    read = n * (1 - case["masked"]) if case["kind"] == "policy" else sum(k - k // 4 for k in _lengths(case))
    return {"bytes": (read + n) * V * e + 28 * n, "flops": 8 * read * V}


# -- the same in 64 bits --------------------------------------------------------
def _exact_bits(K, n):
    """The 16-bit numbers of the dropout stream, numpy's unsigned 64-bit arithmetic."""
    def mix(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    gamma = np.uint64(0x9E3779B97F4A7C15)
    out = np.empty((K, n), np.uint16)
    with np.errstate(over="ignore"):
        for k in range(K):
            key = np.array([SEED ^ 0x44524F504F555421], np.uint64)
            for number in (T, k + 1, SITE):
                key = mix(key + gamma * np.uint64(number + 1))
            z = mix(key + gamma * np.arange(1, (n + 3) // 4 + 1, dtype=np.uint64))
            out[k] = z.astype("<u8").view("<u2")[:n]
    return out


def _exact_dropout(case, s):
    q = round(case["p"] * 65536)
    keep = torch.from_numpy(_exact_bits(case["K"], case["n"]) >= q).cuda()
    gain = keep.double().mul_(65536.0 / (65536 - q))
    return {"out": s["x"].double().mul_(gain).add_(s["residual"].double()), "dx": gain.mul_(s["dy"].double())}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "dropout":
        return _exact_dropout(case, s)
    logits, targets, scale = s["logits"], s["targets"], case["scale"]
    n, V = logits.shape
    some = max(1, (1 << 26) // V)      # rows at a time

    def log_softmax(i):
        x = logits[i: i + some].double().requires_grad_()
        lp = torch.log_softmax(x * scale, -1)
        y = targets[i: i + some]
        return x, torch.where(y >= 0, lp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)

    logp = torch.cat([log_softmax(i)[1].detach() for i in range(0, n, some)])
    if case["kind"] == "logp" and not case["grad"]:
        return {"logp": logp}
    if case["kind"] == "logp":
        r, slope = {"logp": logp}, s["dlogp"].double()
    else:
        logp.requires_grad_()
        w = s["weights"].double()
        if case["kind"] == "policy":
            adv = s["advantages"].double()
            ratio = torch.exp(logp - s["old_logp"].double())
            far = s["ref_logp"].double() - logp
            each = KL * (far.exp() - far - 1) - torch.minimum(
                ratio * adv, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
            loss = (w * each).sum()
            r = {"loss": loss.detach(), "token_loss": torch.where(w != 0, each, 0.0).detach(),
                 "logp": torch.where(w != 0, logp, 0.0).detach()}
        else:
            ratio = torch.where(targets >= 0, logp - s["ref_logp"].double(), 0.0)
            seq = torch.stack([part.sum() for part in torch.split(ratio, s["offsets"].diff().tolist())])
            margin = BETA * (seq[0::2] - seq[1::2])
            up, down = (torch.nn.functional.logsigmoid(v) for v in (margin, -margin))
            each = -(1 - SMOOTH) * up - SMOOTH * down
            loss = (w * each).sum()
            r = {"loss": loss.detach(), "pair_loss": each.detach(), "seq_ratio": seq.detach()}
        slope = torch.autograd.grad(loss, logp)[0]
    r["dlogits"] = torch.empty((n, V), dtype=torch.float64, device="cuda")
    for i in range(0, n, some):
        x, lp = log_softmax(i)
        r["dlogits"][i: i + some] = torch.autograd.grad((lp * slope[i: i + some]).sum(), x)[0]
    return r
