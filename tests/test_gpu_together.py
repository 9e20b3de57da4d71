"""Token scores, their gradient, orthogonalised gradients and the compressed step, one after the other."""
import os
import sys

import numpy as np
import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_a_step_of_workers_with_an_entropy_term():
    """K workers with a head W: loss, dlogits, dW, its orthogonalised form in the K x d gradients, GMC.step."""
    import torch

    import oracle
    from paper_1905_12948_gb300 import GMC, orthogonalize, token_scores, token_scores_backward
    K, rows, V, width, c = 3, 40, 333, 48, 0.02
    d, at = V * width + 29, 17
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    w0 = rand(d) * 0.1
    gmc = GMC(d, K, 0.9, 0.05, compressor="topk", ratio=0.02)
    host = oracle.GMC(d, K, 0.9, 0.05, compressor=oracle.TOPK, ratio=0.02)
    gmc.set_params(w0)
    host.set_params(w0.cpu().numpy())
    for step in range(3):
        W = gmc.params()[at: at + V * width].view(V, width)
        grads = rand(K, d) * 1e-3
        around = grads.clone()
        part = grads[:, at: at + V * width].view(K, V, width)
        for k in range(K):
            h, y, adv = rand(rows, width), torch.randint(0, V, (rows,), generator=gen, device="cuda"), rand(rows)
            logits = h @ W.T
            s = token_scores(logits, y, top=4, return_stats=True)
            dl = token_scores_backward(logits, y, s.stats, -adv / rows, torch.full_like(adv, -c / rows))
            z = logits.double().requires_grad_()
            lp = torch.log_softmax(z, 1)
            loss = -(adv.double() * lp[torch.arange(rows), y]).mean() + c * (lp.exp() * lp).sum(1).mean()
            want, = torch.autograd.grad(loss, z)
            bound = ref.gradient_bound(logits.double().cpu().numpy(), y.cpu().numpy()[:, None], (-adv / rows).double().cpu().numpy()[:, None],
                                       np.full(rows, -c / rows), 1.0, "f32")
            assert (np.abs((dl.double() - want).cpu().numpy()) <= bound).all()
            assert torch.equal(s.top_index[:, 0], logits.argmax(1))
            part[k] = dl.T @ h
        raw = part.clone()
        assert orthogonalize(part, out=part).data_ptr() == part.data_ptr()
        want = ref.products(raw)
        own = (ref.rounded(raw, fine=True) - want).flatten(1).norm(dim=1) + (ref.in_float32(raw) - want).flatten(1).norm(dim=1)
        assert ((part.double() - want).flatten(1).norm(dim=1) <= 2 * own + 2.0 ** -24 * want.flatten(1).norm(dim=1)).all()
        assert torch.equal(grads[:, :at], around[:, :at]) and torch.equal(grads[:, at + V * width:], around[:, at + V * width:])
        gmc.step(grads)
        host.step(grads.cpu().numpy())
        assert np.array_equal(gmc.params().cpu().numpy().view(np.uint32), host.w.view(np.uint32))
    assert gmc.check() == 0
    gmc.close()


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_the_example_with_an_entropy_term_and_orthogonal_gradients(loss):
    import posttrain
    h = posttrain.train(posttrain.parse(["--loss", loss, "--steps", "3", "--entropy", "0.01", "--orthogonal"]))
    assert len(h) == 3 and all(np.isfinite(h))


def test_a_step_in_a_graph():
    """Scores, gradient and orthogonalised update captured once and replayed on new inputs."""
    import torch
    from paper_1905_12948_gb300 import orthogonalize, token_scores, token_scores_backward
    rows, V, width = 64, 500, 200
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, y = torch.randn(rows, V, generator=gen, device="cuda"), torch.randint(0, V, (rows,), generator=gen, device="cuda")
    h = torch.randn(rows, width, generator=gen, device="cuda")
    g = torch.full((rows,), -1 / rows, device="cuda")

    def step():
        s = token_scores(x, y, return_stats=True)
        return orthogonalize((token_scores_backward(x, y, s.stats, g, g).T @ h).bfloat16())

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        x.copy_(torch.randn(rows, V, generator=gen, device="cuda"))
        graph.replay()
        got = out.clone()
        assert torch.equal(got, step())


def test_inference_mode_leaves_and_versions():
    import torch
    from paper_1905_12948_gb300 import orthogonalize, token_scores
    with torch.inference_mode():
        x = torch.randn(4, 300, device="cuda")
        assert token_scores(x, top=2).top_index.shape == (4, 2)
        m = torch.randn(2, 30, 40, device="cuda")
        assert orthogonalize(m, out=m).data_ptr() == m.data_ptr()
    leaf = torch.randn(4, 300, device="cuda", requires_grad=True)
    assert not token_scores(leaf, return_stats=True).entropy.requires_grad
    view = torch.randn(3, 30, 40, device="cuda")
    before = view._version
    orthogonalize(view, out=view)
    assert view._version > before


def test_inputs_freed_before_the_call_has_run():
    import torch
    from paper_1905_12948_gb300 import orthogonalize, token_scores, token_scores_backward
    n, V = 64, 4_096
    g = torch.Generator(device="cuda").manual_seed(1)

    def inputs():
        x = torch.rand(n, V, generator=g, device="cuda")
        y = torch.arange(n, device="cuda")
        return dict(x=x, y=y, stats=token_scores(x, y, return_stats=True).stats.clone(), a=torch.rand(n, generator=g, device="cuda"),
                    h=torch.rand(n, generator=g, device="cuda"), m=torch.rand(3, 150, 170, generator=g, device="cuda"))

    def run(i, **stream):
        return [*token_scores(i["x"], i["y"], top=3, **stream)[:4], token_scores_backward(i["x"], i["y"], i["stats"], i["a"], i["h"], **stream),
                orthogonalize(i["m"], **stream)]

    i = inputs()
    want = [t.clone() for t in run(i)]
    places = {t.data_ptr() for t in i.values()}
    sizes = [(t.shape, t.dtype) for t in i.values()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)
    got = run(i, stream=s)
    assert not s.query()
    del i
    others = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in sizes * 3]
    assert not s.query() and not places & {t.data_ptr() for t in others}
    for t in others:
        t.zero_()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
