"""The language-model example with its tokens mixed by the recurrence, its feed-forward block fused, and its projections'
gradients orthogonalised: one worker's gradient against automatic differentiation in fp32, and a few steps."""
import math

import pytest
import torch

import block_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    from paper_2004_05298_b200 import lm_example
    return lm_example


def _reference(layout, z, tokens, targets, length):
    """The same model in fp32 with torch's own differentiation, token after token."""
    z = z.clone().requires_grad_()
    P = lambda name: layout.view(z, name)                                  # noqa: E731
    norm = lambda v, w: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6) * w   # noqa: E731
    C = layout.width
    h = P("embed")[tokens]
    n = norm(h, P("pre0"))
    for i in range(layout.blocks):
        if layout.mixer == "recurrence":
            xg = (n @ P("mix%d" % i).t()).view(-1, length, 2 * C)
            state, rows = torch.zeros_like(xg[:, 0, :C]), []
            for t in range(length):
                keep = torch.sigmoid(xg[:, t, C:])
                state = keep * state + (1 - keep) * xg[:, t, :C]
                rows.append(state)
            m = torch.stack(rows, 1).reshape(n.shape)
        else:
            m = n.view(-1, length, C)
            m = (m + torch.nn.functional.pad(m, (0, 0, 1, 0))[:, :-1]).reshape(n.shape)
        g, u = (m @ P("gate_up%d" % i).t()).chunk(2, 1)
        h = h + P("gate%d" % i) * norm((torch.sigmoid(g) * g * u) @ P("down%d" % i).t(), P("post%d" % i))
        n = norm(h, P("pre%d" % (i + 1)))
    loss = -torch.log_softmax(n @ P("head").t(), 1).gather(1, targets[:, None]).mean()
    loss.backward()
    return loss.detach(), z.grad


@pytest.mark.parametrize("mixer,fused", [("recurrence", False), ("recurrence", True), ("shift", True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_of_a_worker(E, dtype, mixer, fused):
    layout, T, length = E.Layout(131, 72, 200, 2, mixer), 96, 32
    z = layout.initial(3)
    tokens, targets = next(E.batches(layout.vocab, 1, T, length, 5))[0]
    run = E.Pass(layout, T, length, dtype, fused=fused)
    grad = torch.full((layout.d,), float("nan"), device="cuda")
    loss = run.forward(z, tokens, targets)
    run.backward(z, tokens, targets, grad)
    want_loss, want = _reference(layout, z, tokens, targets, length)
    # As for the model without these: a value kept in 8 bits is off by about 1 % of its group's root mean square, bf16 adds 2^-8;
    # two blocks deep and averaged over 96 tokens, a parameter's gradient is off by a few per cent of its norm.
    assert abs(float(loss) - float(want_loss)) <= (2e-2 if dtype == torch.bfloat16 else 1e-4)
    for name in layout.at:
        got, ref = layout.view(grad, name), layout.view(want, name)
        assert float((got - ref).norm() / ref.norm()) < 0.05, name


def test_orthogonalised_gradients_of_all_workers(E):
    layout, W = E.Layout(64, 48, 80, 2, "recurrence"), 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    grads = torch.empty(W, layout.d, device="cuda").normal_(0, 1e-3, generator=gen)
    old = grads.clone()
    E.Orthogonal(layout, W, 0.5)(grads)
    names = layout.projections()
    assert len(names) == 6
    for name in layout.at:
        for w in range(W):
            got, was = layout.view(grads[w], name), layout.view(old[w], name)
            if name not in names:
                assert torch.equal(got, was), name
                continue
            rows, cols = was.shape
            want, err = block_ref.orthogonalize(was, scale=0.5 * math.sqrt(max(1.0, rows / cols)))
            assert float((got.double() - want).norm()) <= err + 2.0 ** -24 * float(want.norm())


def test_training_runs_with_everything(E):
    losses, model, _ = E.train(steps=6, workers=2, ratio=4, vocab=96, width=64, hidden=128, blocks=2, tokens=256, length=64, mixer="recurrence", fused=True,
                               orthogonal=0.01)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses) and bool(torch.isfinite(model).all())


def test_a_model_without_blocks_has_nothing_to_orthogonalise(E):
    layout = E.Layout(32, 16, 24, 0)
    grads = torch.randn(2, layout.d, device="cuda")
    old = grads.clone()
    E.Orthogonal(layout, 2, 0.5)(grads)
    assert torch.equal(grads, old)
