"""Operators on both sides of a language model's backward pass, as cases that can be timed and compared.

A case is one call of an operator as a training program makes it, or the two calls of its
directions: log-probabilities of given tokens with the entropy and the top alternatives of each
row (``token_scores``), the gradient of the log-probabilities and the entropy in the logits
(``token_scores_backward``), and the orthogonalised gradients of K workers' weight matrices by
Newton-Schulz products (``orthogonalize``).

``run`` computes them in elementary torch operations in 32 bits, or, where ``own`` is
true, through the library. ``exact`` does so in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
STEPS = 5
QUINTIC = (3.4445, -4.7750, 2.0315)     # a, b, c of X <- a X + b (X X') X + c (X X')^2 X


def _scores(name, n, V, dtype, top, *, given=1, grad=False, scale=1.0, padded=False, masked=0.0):
    return {"name": name, "kind": "scores", "n": n, "V": V, "dtype": dtype, "top": top, "given": given,
            "grad": grad, "scale": scale, "padded": padded, "masked": masked}


def _matrices(name, K, m, n, dtype):
    return {"name": name, "kind": "matrices", "K": K, "m": m, "n": n, "dtype": dtype}


def listed():
    return [
        # one token as it is sampled, with the alternatives that a service shows: the smallest call
        _scores("scores_token", 1, 131_072, "bf16", 20),
        # rollouts scored with their entropy and a few alternatives, an odd vocabulary
        _scores("scores_rollout", 4_096, 50_257, "bf16", 8, scale=1 / 0.7),
        # a teacher's 64 best tokens of each row, kept for distillation; fp32, a padded vocabulary
        _scores("scores_teacher", 512, 128_256, "f32", 64, padded=True),
        # a short batch of a policy with an entropy bonus, both directions
        _scores("entropy_small", 64, 32_000, "bf16", 0, grad=True),
        # the student of that teacher: 16 given tokens a row, a fifth of the rows masked
        _scores("student_odd", 3_001, 50_257, "bf16", 0, given=16, grad=True, masked=0.2),
        # the largest batch with an entropy bonus and the alternatives it logs
        _scores("entropy_large", 8_192, 131_072, "bf16", 5, grad=True, masked=0.1),
        # four workers' gradients of a small model's head
        _matrices("head_small", 4, 1_000, 64, "f32"),
        # eight workers' gradients of a convolution of 512 channels by 512 x 3 x 3, as GMC takes them
        _matrices("conv_f32", 8, 512, 4_608, "f32"),
        # the same workers' last layer, 1,000 classes
        _matrices("classes", 8, 1_000, 4_096, "bf16"),
        # a step's share of small layers, 32 workers
        _matrices("blocks", 32, 256, 1_024, "bf16"),
        # one square layer
        _matrices("square", 1, 4_096, 4_096, "bf16"),
        # the largest: two workers' first layer behind the convolutions
        _matrices("layer_large", 2, 4_096, 25_088, "bf16"),
    ]


def _spread(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
    if rng.random() < 0.55:
        V = _spread(rng, 500, 131_072)
        V -= V % 64 if rng.random() < 0.4 else 0
        most = 1_900_000_000 // SIZES[dtype] // V
        c = _scores("", _spread(rng, 1, min(most, 16_384)), V, dtype, rng.choice([0, 1, 5, 20, 64]),
                    given=rng.choice([0, 1, 1, 4, 17]), scale=rng.choice([1.0, 1.0, 1 / 0.7, 0.5]),
                    padded=rng.random() < 0.3)
        c["grad"] = rng.random() < 0.5
        c["masked"] = rng.choice([0.0, 0.2, 0.5]) if c["given"] else 0.0
    else:
        # products of one step and worker up to those of 4,096 x 25,088, of the wider types a fifth
        most = 1.3e12 if dtype == "bf16" else 2.6e11
        while True:
            m, n = _spread(rng, 16, 8_192), _spread(rng, 16, 25_088)
            if rng.random() < 0.4:
                m, n = max(16, m - m % 64), max(16, n - n % 64)
            each = min(m, n) ** 2 * (3 * max(m, n) + min(m, n))
            if each <= most:
                break
        K = _spread(rng, 1, max(1, min(32, int(2 * most / each), (1 << 28) // (m * n))))
        c = _matrices("", K, m, n, dtype)
    del c["name"]
    return c


# -- inputs -------------------------------------------------------------------
def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    dtype = DTYPES[case["dtype"]]
    if case["kind"] == "matrices":
        # a layer's gradient: a few directions that the batch agrees on, less and less, and the
        # noise of its samples; small numbers, each worker's own
        K, m, n = case["K"], case["m"], case["n"]
        r = min(m, n, 32)
        size = torch.arange(1, r + 1, device="cuda") ** -0.5
        g = torch.matmul(normal(K, m, r) * size, normal(K, r, n))
        return {"g": g.add_(normal(K, m, n), alpha=0.5).mul_(1e-3).to(dtype)}
    n, V = case["n"], case["V"]
    last = V - V // 200 if case["padded"] else V
    # logits of a model: a few units wide, the sampled token usually among the larger ones
    given = case["given"]
    targets = torch.randint(0, last, (n, max(given, 1)), generator=gen, device="cuda")
    x = normal(n, V).mul_(2.5)
    x[torch.arange(n, device="cuda")[:, None], targets] += torch.rand(n, targets.shape[1], generator=gen, device="cuda") * 9
    if case["padded"]:
        x[:, last:] = -math.inf
    s = {"logits": x.to(dtype)}
    if given:
        keep = torch.rand(n, generator=gen, device="cuda") >= case["masked"]
        s["targets"] = torch.where(keep[:, None], targets, -1)
        if given == 1:
            s["targets"] = s["targets"][:, 0].contiguous()
    if case["grad"]:
        # slopes of a loss per token; 16-bit gradients of fp16 are kept in range by a loss scale
        unit = 1.0 if dtype == torch.float16 else 1 / n
        if given:
            s["dlogp"] = normal(*s["targets"].shape) * unit
        s["dentropy"] = -(0.02 + 0.1 * torch.rand(n, generator=gen, device="cuda")) * unit
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    return s


# -- the operators ------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_1905_12948_gb300 import orthogonalize, token_scores, token_scores_backward
    case = s["case"]
    if case["kind"] == "matrices":
        return {"update": orthogonalize(s["g"], steps=STEPS, coefficients=QUINTIC)}
    y = s.get("targets")
    r = token_scores(s["logits"], y, top=case["top"], scale=case["scale"], return_stats=case["grad"])
    out = {"logp": r.logp, "entropy": r.entropy, "top_logp": r.top_logp, "top_index": r.top_index}
    if case["grad"]:
        out["dlogits"] = token_scores_backward(s["logits"], y, r.stats, s.get("dlogp"), s["dentropy"],
                                               scale=case["scale"])
    return {k: v for k, v in out.items() if v is not None}


def _plain_matrices(g):
    x = g.float()
    if x.shape[1] > x.shape[2]:
        x = x.transpose(1, 2)
    size = (x * x).sum((1, 2), keepdim=True).sqrt()
    x = torch.where(size > 0, x / size, 0.0)
    a, b, c = QUINTIC
    for _ in range(STEPS):
        xx = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * xx + c * torch.matmul(xx, xx), x)
    if g.shape[1] > g.shape[2]:
        x = x.transpose(1, 2)
    return x.to(g.dtype).contiguous()


def _plain_top(logits, top):
    """The indices of the `top` largest values of each row, the lower index first where two are equal."""
    bits = (logits.float() + 0.0).view(torch.int32).long()
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))       # ascending with the value
    V = logits.shape[1]
    key = order * (1 << 20) + torch.arange(V - 1, -1, -1, device=logits.device)
    return V - 1 - (torch.topk(key, top, dim=1).values & ((1 << 20) - 1))


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "matrices":
        return {"update": _plain_matrices(s["g"])}
    scale, logits, y = case["scale"], s["logits"], s.get("targets")
    z = logits.float()
    z = (z - z.amax(1, keepdim=True)).mul_(scale)
    e = z.exp()
    total = e.sum(1)
    ls = total.log()
    mean = torch.where(e > 0, e * z, 0.0).sum(1) / total
    counts = torch.ones_like(ls, dtype=torch.bool) if y is None else (y >= 0 if y.dim() == 1 else (y >= 0).any(1))
    entropy = ls - mean
    out = {"entropy": torch.where(counts, entropy, 0.0)}
    if y is not None:
        some = y[:, None] if y.dim() == 1 else y
        logp = z.gather(1, some.clamp(min=0)) - ls[:, None]
        out["logp"] = torch.where(some >= 0, logp, 0.0).view(y.shape)
    if case["top"]:
        best = _plain_top(logits, case["top"])
        out["top_index"] = torch.where(counts[:, None], best, -1)
        out["top_logp"] = torch.where(counts[:, None], z.gather(1, best) - ls[:, None], 0.0)
    if case["grad"]:
        lp = z.sub_(ls[:, None])
        p = e.div_(total[:, None])
        h = torch.where(counts, s["dentropy"], 0.0)[:, None]
        d = torch.where(p > 0, lp + entropy[:, None], 0.0).mul_(-h)
        if y is not None:
            g = torch.where(some >= 0, s["dlogp"].view(some.shape), 0.0)
            d = d.sub_(g.sum(1, keepdim=True)).mul_(p)
            d.scatter_add_(1, some.clamp(min=0), g)
        else:
            d = d.mul_(p)
        out["dlogits"] = d.mul_(scale).to(logits.dtype)
    return out


def work(case):
    e = SIZES[case["dtype"]]
    if case["kind"] == "matrices":
        # X X' and its square are symmetric: half of their products do
        K, m, n = case["K"], min(case["m"], case["n"]), max(case["m"], case["n"])
        return {"bytes": 2 * K * m * n * e, "flops": STEPS * K * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)}
    n, V = case["n"], case["V"]
    read = n * (1 - case["masked"])      # rows that count are read, all gradients are written
    each = 8 * case["given"] + 4 * case["given"] * (1 + case["grad"]) + 12 * case["top"] + 4 + 4 * case["grad"]
    return {"bytes": (read + (n if case["grad"] else 0)) * V * e + n * each,
            "flops": (16 if case["grad"] else 7) * read * V}


# -- the same in 64 bits --------------------------------------------------------
def _exact_matrices(case, s):
    K, m, n = s["g"].shape
    if 2 * STEPS * K * min(m, n) ** 2 * (2 * max(m, n) + min(m, n)) > 6e12:
        return None
    a, b, c = QUINTIC
    out = torch.empty((K, m, n), dtype=torch.float64, device="cuda")
    for k in range(K):
        x = s["g"][k].double()
        x = x / torch.linalg.vector_norm(x)
        if m > n:
            for _ in range(STEPS):
                g = x.T @ x
                x = a * x + x @ (b * g + c * (g @ g))
        else:
            for _ in range(STEPS):
                g = x @ x.T
                x = a * x + (b * g + c * (g @ g)) @ x
        out[k] = x
    return {"update": out}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "matrices":
        return _exact_matrices(case, s)
    logits, y, scale = s["logits"], s.get("targets"), case["scale"]
    n, V = logits.shape
    some = max(1, (1 << 25) // V)      # rows at a time
    parts = []
    for i in range(0, n, some):
        rows = slice(i, i + some)
        x = logits[rows].double().requires_grad_()
        lp = torch.log_softmax(x * scale, 1)
        finite = torch.where(lp == -math.inf, 0.0, lp)
        entropy = -(lp.exp() * finite).sum(1)
        r, loss = {}, 0.0
        scored = torch.ones(x.shape[0], dtype=torch.bool, device="cuda")
        if y is not None:
            t = y[rows].reshape(x.shape[0], -1)
            scored = (t >= 0).any(1)
            logp = torch.where(t >= 0, lp.gather(1, t.clamp(min=0)), 0.0)
            r["logp"] = logp.detach().view(y[rows].shape)
            if case["grad"]:
                loss = (logp * s["dlogp"][rows].reshape(t.shape)).sum()
        entropy = torch.where(scored, entropy, 0.0)
        r["entropy"] = entropy.detach()
        if case["top"]:
            r["top_logp"] = torch.where(scored[:, None], torch.topk(lp.detach(), case["top"], dim=1).values, 0.0)
        if case["grad"]:
            r["dlogits"] = torch.autograd.grad(loss + (entropy * s["dentropy"][rows]).sum(), x)[0]
        parts.append(r)
    out = {k: torch.cat([r[k] for r in parts]) for k in parts[0]}
    if case["top"]:
        out["top_index"] = None
    return out
