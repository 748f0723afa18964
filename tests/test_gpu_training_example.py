"""The example that trains with the operators of the training step and captures its state on the way."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_mlp", os.path.join(ROOT, "examples", "train_mlp.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("rows,hidden,ffn", [(1024, 256, 1024), (333, 200, 520)])
def test_it_learns_and_goes_on_from_its_checkpoint(tmp_path, rows, hidden, ffn):
    losses, again, same = _example().main(["--steps", "30", "--snapshot-at", "12", "--rows", str(rows), "--hidden", str(hidden), "--ffn", str(ffn),
                                           "--dir", str(tmp_path)])
    assert len(losses) == 30 and losses[-1] < 0.8 * losses[0]
    assert same and len(again) == 17
    assert not os.listdir(tmp_path)


def test_its_gradients_are_those_of_torch():
    """Against automatic differentiation in 64 bits, on the parameters as they are in 16 bits.  Two things stand between
    them.  What is kept in 8 bits is off by half a step of 2^-6 of its group's power of two at most, 2^-7 of what is in it;
    an activation's slope moves by less than 1.2 of that; everything that is rounded to bfloat16 on the way (norm, h, dh, dn)
    is off by 2^-9 of itself.  As independent errors over sums of hundreds of terms they stay below 2^-6 of a gradient's norm."""
    import torch
    E = _example()
    block = E.Block(512, 128, 320, seed=3)
    x, target = E.batch(0, 512, 128)
    y = block.forward(x)
    dy = (2 * (y.float() - target)).bfloat16()
    dx = block.backward(dy.clone())
    p = {n: t.double().requires_grad_() for n, t in block.param.items()}
    xd = x.double().requires_grad_()
    n = torch.nn.functional.layer_norm(xd, (128,), p["gamma"], p["beta"], E.EPS)
    h = torch.nn.functional.gelu(n @ p["fc1.w"].t() + p["fc1.b"], approximate="tanh")
    want = xd + h @ p["fc2.w"].t() + p["fc2.b"]
    want.backward(dy.double())
    assert (y.double() - want).norm() < 2.0 ** -7 * want.norm()
    for name, grad in block.grad.items():
        assert (grad.double() - p[name].grad).norm() < 2.0 ** -6 * p[name].grad.norm(), name
    assert (dx.double() - xd.grad).norm() < 2.0 ** -6 * xd.grad.norm()
