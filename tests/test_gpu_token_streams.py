"""Inputs of a call on another stream that the caller lets go of before the call has run."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["logp", "backward", "policy", "preference", "dropout"])
def test_inputs_freed_before_the_call_has_run(call):
    import torch
    from paper_1905_12948_gb300 import TokenLoss, dropout, token_logp, token_logp_backward
    n, V = 64, 4_096
    g = torch.Generator(device="cuda").manual_seed(1)
    loss = TokenLoss(n, 1)

    def inputs():
        """One tensor of a size of its own for each argument."""
        rand = lambda *s: torch.rand(*s, generator=g, device="cuda")
        return dict(x=rand(n, V), y=torch.arange(n, device="cuda"), a=-rand(n), b=rand(n), c=rand(n), d=-rand(n),
                    stats=token_logp(rand(n, V), torch.arange(n, device="cuda"), return_stats=True)[1], res=rand(n, V),
                    off=torch.tensor([0, 20, n], device="cuda"))

    def run(i, **stream):
        if call == "logp":
            return [token_logp(i["x"], i["y"], **stream)]
        if call == "backward":
            return [token_logp_backward(i["x"], i["y"], i["stats"], i["a"], **stream)]
        if call == "policy":
            r = loss.policy(i["x"], i["y"], i["a"], i["b"], weights=i["c"], ref_logp=i["d"], kl=0.1, **stream)
        elif call == "preference":
            r = loss.preference(i["x"], i["y"], i["off"], beta=0.1, ref_logp=i["d"], weights=i["c"][:1], **stream)
        else:
            return [dropout(i["x"], 0.3, seed=1, residual=i["res"], **stream)]
        return list(r)

    i = inputs()
    want = [t.clone() for t in run(i)]
    used = {"logp": "xy", "backward": ["x", "y", "stats", "a"], "policy": "xyabcd", "preference": ["x", "y", "off", "c", "d"],
            "dropout": ["x", "res"]}[call]
    places = {i[k].data_ptr() for k in used}
    sizes = [(i[k].shape, i[k].dtype) for k in i]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)      # a fifth of a second
    got = run(i, stream=s)
    assert not s.query()
    del i
    others = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in sizes * 3]
    assert not s.query()      # (nothing above waits: the call has still not run)
    assert not places & {t.data_ptr() for t in others}
    for t in others:
        t.zero_()
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    loss.close()
