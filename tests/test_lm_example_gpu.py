"""The operators of include/def_train.h together, as the language-model example uses them: one worker's gradient against
automatic differentiation in fp32, and the loss over some steps of def_step."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    from paper_2004_05298_b200 import lm_example
    return lm_example


def _reference(E, layout, z, tokens, targets, length):
    """The same model in fp32 with torch's own differentiation."""
    z = z.clone().requires_grad_()
    P = lambda name: layout.view(z, name)                                  # noqa: E731
    norm = lambda v, w: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6) * w   # noqa: E731
    h = P("embed")[tokens]
    n = norm(h, P("pre0"))
    for i in range(layout.blocks):
        m = n.view(-1, length, layout.width)
        m = (m + torch.nn.functional.pad(m, (0, 0, 1, 0))[:, :-1]).reshape(n.shape)
        g, u = (m @ P("gate_up%d" % i).t()).chunk(2, 1)
        h = h + P("gate%d" % i) * norm((torch.sigmoid(g) * g * u) @ P("down%d" % i).t(), P("post%d" % i))
        n = norm(h, P("pre%d" % (i + 1)))
    logp = torch.log_softmax(n @ P("head").t(), 1)
    loss = -logp.gather(1, targets[:, None]).mean()
    loss.backward()
    return loss.detach(), z.grad, logp.detach()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_of_a_worker(E, dtype):
    layout, T, length = E.Layout(131, 72, 200, 2), 96, 32
    z = layout.initial(3)
    tokens, targets = next(E.batches(layout.vocab, 1, T, length, 5))[0]
    run = E.Pass(layout, T, length, dtype)
    grad = torch.full((layout.d,), float("nan"), device="cuda")
    loss = run.forward(z, tokens, targets)
    ids, top = (v.clone() for v in run.alternatives())
    run.backward(z, tokens, targets, grad)
    want_loss, want, logp = _reference(E, layout, z, tokens, targets, length)
    # An activation kept in 8 bits is off by at most half of a 64th of its group's largest magnitude, about 1 % of the
    # group's root mean square; bf16 adds 2^-8.  Two blocks deep and averaged over 96 tokens, a parameter's gradient is
    # off by a few per cent of its norm.
    assert abs(float(loss) - float(want_loss)) <= (2e-2 if dtype == torch.bfloat16 else 1e-4)
    for name in layout.at:
        got, ref = layout.view(grad, name), layout.view(want, name)
        assert float((got - ref).norm() / ref.norm()) < 0.05, name
    if dtype == torch.float32:                                             # the forward pass itself is not compressed
        assert float((top - logp.gather(1, ids)).abs().max()) < 1e-3


def test_training_goes_down(E):
    losses, model, layout = E.train(steps=40, workers=3, ratio=4, vocab=128, width=128, hidden=256, blocks=2, tokens=512, length=32)
    assert all(math.isfinite(v) for v in losses) and bool(torch.isfinite(model).all())
    assert losses[0] > 0.8 * math.log(128) and losses[-1] < 0.6 * losses[0], (losses[0], losses[-1])
