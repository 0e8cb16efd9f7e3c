"""The example's training step: the operators and the all-reduce together."""
import importlib.util
import os

import pytest

from helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def T():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    T = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(T)
    return T


@pytest.mark.parametrize("state", [8, 32])
@pytest.mark.parametrize("sparsity", [0.0, 0.9])
def test_the_loss_falls(T, state, sparsity):
    log(f"train {state} {sparsity}")
    losses, trainer = T.train(steps=40, state=state, sparsity=sparsity)
    assert losses[-1] < 0.5 * losses[0]
    for r in trainer.reduced[1:]:
        assert torch.equal(r, trainer.reduced[0])
    if sparsity:
        share = float((trainer.grads[0] == 0).float().mean())
        assert share > 0.8                                        # the bucket that was sent is sparse


def test_a_message_is_the_same_step(T):
    """From the reduced bucket or from its Pici message: the same bits."""
    log("train message")
    a = T.train(steps=5, state=8, message=False)[1]
    b = T.train(steps=5, state=8, message=True)[1]
    assert torch.equal(a.model.params, b.model.params)
    for name in a.states:
        for k in a.states[name]:
            assert torch.equal(a.states[name][k].view(torch.uint8), b.states[name][k].view(torch.uint8)), (name, k)


def test_gradients_of_the_whole_model(T):
    """Against autograd in 64 bits.  The products are fp32 sums of up to 512
    terms; 2^-13 of each tensor's largest gradient leaves 2^11 roundings."""
    log("train gradients")
    model = T.Model(96, 2, 16, 2)
    for name in model.bucket.shapes:                               # away from ones and zeros
        g = torch.Generator(device="cuda").manual_seed(len(name) + ord(name[-1]))
        model.param(name).add_(torch.randn(model.param(name).shape, generator=g, device="cuda") * 0.1)
    x, y = T.batches(model, 1, 512)[0]
    flat = model.bucket.new()
    pred, kept = model.forward(x)
    model.backward(kept, pred - y, flat)
    p = {n: model.param(n).double().requires_grad_() for n in model.bucket.shapes}
    z = x.double()
    for k in range(model.layers + 1):
        h = torch.nn.functional.layer_norm(z, (model.width,), p[f"weight{k}"], p[f"bias{k}"], 1e-5) @ p[f"linear{k}"]
        z = h if k == model.layers else z + h
    (0.5 * (z - y.double()).square().sum()).backward()
    for name, t in p.items():
        err = (model.bucket.view(flat, name).double() - t.grad).abs().max()
        assert float(err) <= 2.0 ** -13 * float(t.grad.abs().max()), name
