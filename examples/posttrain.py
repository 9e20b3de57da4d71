"""Post-training of a small language model by K simulated workers, their gradients
compressed by GMC (Alg. 1) each step.

    python examples/posttrain.py --loss policy
    python examples/posttrain.py --loss preference

The model: an embedding E of 64 prompt tokens, dropout, a head W of `vocab` tokens. Every
worker has its own prompts and its own dropout masks, which follow from (seed, step, worker):

    h = dropout(E[prompt])         dropout, the K workers in one call
    logits = h W^T                 a matrix product of torch
    loss, dlogits                  TokenLoss.policy or TokenLoss.preference
    dW = dlogits^T h               and, through dropout_backward, dE
    GMC.step(K x d gradients)      top-k of each worker's accumulator, one update

policy: a token is sampled from the model itself for every prompt; tokens of a prompt's own
class are rewarded, the advantage is the reward above the batch's mean. Printed: the mean
reward, 1 / classes to begin with. preference: pairs of short answers, the preferred one made
of tokens of the prompt's class. Printed: the loss, log 2 to begin with.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_1905_12948_gb300 import GMC, TokenLoss, dropout, dropout_backward, token_logp

PROMPTS, CLASSES = 64, 8


def parse(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--loss", choices=("policy", "preference"), default="policy")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--rows", type=int, default=256, help="tokens a worker scores each step")
    ap.add_argument("--ratio", type=float, default=0.05, help="share of the gradient that a worker sends")
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--seed", type=int, default=0)
    return ap.parse_args(argv)


def forward(w, prompts, a, t):
    """(E, W, hidden states of the K workers) from the parameters w."""
    E = w[: PROMPTS * a.width].view(PROMPTS, a.width)
    W = w[PROMPTS * a.width:].view(a.vocab, a.width)
    return E, W, dropout(E[prompts], a.dropout, seed=a.seed, t=t)      # (K, rows, width)


def tokens_of(classes, a, gen):
    """A token of each class: token v is of class v mod CLASSES."""
    step = torch.randint(0, a.vocab // CLASSES, classes.shape, generator=gen, device="cuda")
    return step * CLASSES + classes


def policy_worker(loss, logits, prompts, reference, a, gen):
    """One worker's loss: tokens sampled from the model, rewarded by class."""
    y = torch.multinomial(torch.softmax(logits, -1), 1, generator=gen)[:, 0]
    reward = (y % CLASSES == prompts % CLASSES).float()
    old = token_logp(logits, y)                     # the policy that sampled them: this one
    r = loss.policy(logits, y, old, reward - reward.mean(), ref_logp=token_logp(reference, y), kl=0.01)
    return float(reward.mean()), r.dlogits


def preference_worker(loss, logits, targets, offsets, reference):
    r = loss.preference(logits, targets, offsets, beta=0.5, ref_logp=token_logp(reference, targets))
    return float(r.loss), r.dlogits


def train(a):
    torch.manual_seed(a.seed)
    gen = torch.Generator(device="cuda").manual_seed(a.seed)
    d = (PROMPTS + a.vocab) * a.width
    w0 = torch.randn(d, device="cuda") * 0.1
    eta = 20.0 if a.loss == "policy" else 5.0
    gmc = GMC(d, a.workers, beta=0.9, eta=eta, compressor="topk", ratio=a.ratio, seed=a.seed)
    gmc.set_params(w0)
    length = 8                                       # of an answer, in tokens
    pairs = a.rows // (2 * length)
    rows = a.rows if a.loss == "policy" else pairs * 2 * length
    loss = TokenLoss(max_rows=rows, max_pairs=pairs)
    offsets = torch.arange(0, rows + 1, length, device="cuda")
    grads = torch.zeros((a.workers, d), device="cuda")
    history = []
    for t in range(a.steps):
        w = gmc.params()
        if a.loss == "policy":
            prompts = torch.randint(0, PROMPTS, (a.workers, rows), generator=gen, device="cuda")
        else:    # a pair's two answers belong to one prompt
            prompts = torch.randint(0, PROMPTS, (a.workers, pairs), generator=gen, device="cuda")
            prompts = prompts.repeat_interleave(2 * length, 1)
        E, W, h = forward(w, prompts, a, t)
        h0 = w0[: PROMPTS * a.width].view(PROMPTS, a.width)[prompts]
        W0 = w0[PROMPTS * a.width:].view(a.vocab, a.width)
        grads.zero_()
        dh = torch.empty_like(h)
        value = 0.0
        for k in range(a.workers):
            logits, reference = h[k] @ W.T, h0[k] @ W0.T
            if a.loss == "policy":
                v, dlogits = policy_worker(loss, logits, prompts[k], reference, a, gen)
            else:
                own = torch.arange(rows, device="cuda") // length % 2 == 0     # the preferred answers
                targets = torch.where(own, tokens_of(prompts[k] % CLASSES, a, gen),
                                      torch.randint(0, a.vocab, (rows,), generator=gen, device="cuda"))
                v, dlogits = preference_worker(loss, logits, targets, offsets, reference)
            value += v / a.workers
            grads[k, PROMPTS * a.width:] = (dlogits.T @ h[k]).reshape(-1)
            dh[k] = dlogits @ W
        dE = dropout_backward(dh, a.dropout, seed=a.seed, t=t)
        for k in range(a.workers):
            grads[k, : PROMPTS * a.width].view(PROMPTS, a.width).index_add_(0, prompts[k], dE[k])
        gmc.step(grads)
        history.append(value)
        if t % 10 == 0 or t == a.steps - 1:
            print(f"step {t}: {'mean reward' if a.loss == 'policy' else 'loss'} {value:.4f}", flush=True)
    assert gmc.check() == 0
    stats = gmc.stats()
    print(f"relative communication cost {stats['rcc']:.4f}")
    gmc.close()
    loss.close()
    return history


if __name__ == "__main__":
    train(parse())
