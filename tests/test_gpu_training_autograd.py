"""What the trainers' calls write counts as changed in place: a backward pass that would read it afterwards is an error, not a wrong gradient."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


def _row_inputs():
    w = torch.randn(6, 100, device="cuda", requires_grad=True)
    return w, w.exp(), torch.arange(6, device="cuda"), torch.full((6,), -1 / 6, device="cuda")    # exp keeps its result for its gradient


@pytest.mark.parametrize("call", ["loss", "grad"])
def test_logits_that_a_gradient_takes_the_place_of(slaq, call):
    w, x, t, g = _row_inputs()
    if call == "loss":
        _, grad = slaq.token_loss(x, t, g, out=x)
    else:
        r = slaq.token_logprobs(x, t)
        grad = slaq.token_logprobs_grad(x, t, r.norm, g, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        x.backward(grad.clone())


def test_logits_that_are_left_as_they_were_pass_their_gradient_on(slaq):
    w, x, t, g = _row_inputs()
    _, grad = slaq.token_loss(x, t, g)
    x.backward(grad)
    want = torch.autograd.grad(torch.nn.functional.cross_entropy(w.exp(), t), w)[0]
    torch.testing.assert_close(w.grad, want, rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("call", ["row_grad", "losses"])
def test_other_results(slaq, call):
    a = torch.randn(6, device="cuda", dtype=torch.float32 if call == "row_grad" else torch.float64)
    w = torch.ones_like(a, requires_grad=True)
    y = w * a                                     # keeps a
    if call == "row_grad":
        slaq.job_row_grad(torch.tensor([0, 6], device="cuda"), out=a)
    else:
        slaq.job_losses(torch.arange(7, device="cuda"), None, -torch.ones(6, device="cuda"), out=a)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.sum().backward()


@pytest.mark.parametrize("bits", [8, 32])
def test_weights_that_a_step_changes(slaq, bits):
    p = torch.randn(300, device="cuda", requires_grad=True)
    plan = slaq.AdamW([p], [torch.ones(300, device="cuda")], state_bits=bits)
    loss = p.square().sum()
    plan.step()
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()
    p.square().sum().backward()
    torch.testing.assert_close(p.grad, 2 * p.detach())
