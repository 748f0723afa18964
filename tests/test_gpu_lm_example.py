"""The example that trains a small language model with all operators of the step and captures its state on the way."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_lm", os.path.join(ROOT, "examples", "train_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("rows,vocab,hidden,ffn,blocks", [(1024, 1024, 256, 1024, 2), (333, 1001, 200, 520, 1), (70, 64, 96, 100, 0)])
def test_it_goes_on_from_its_checkpoint(tmp_path, rows, vocab, hidden, ffn, blocks):
    sizes = {"--rows": rows, "--vocab": vocab, "--hidden": hidden, "--ffn": ffn, "--blocks": blocks}
    losses, again, same = _example().main(["--steps", "12", "--snapshot-at", "5", "--dir", str(tmp_path)] + [str(x) for kv in sizes.items() for x in kv])
    assert len(losses) == 12 and all(math.isfinite(x) for x in losses)
    assert same and len(again) == 6
    assert not os.listdir(tmp_path)


def test_its_gradients_are_those_of_torch():
    """Against automatic differentiation in 64 bits, on the parameters as they are in 16 bits.  What is rounded to bfloat16 on the way
    forward (x, y, h, u, the logits) is off by 2^-9 of itself at the root of the mean square or less, and so is what is on the way back (dlogits,
    dy, du, dx, dh); what goes into the activation is kept in 8 bits, off by 2^-7 of its group's largest at most.  Some ten
    such roundings, independent of each other, stand before any gradient: below 2^-5 of its norm with room to spare."""
    import torch
    E = _example()
    model = E.Model(512, 384, 128, 320, 2, seed=3)
    tokens, after = E.batch(0, 512, 384)
    dlogprob = torch.where(after == E.NONE, 0.0, -1.0 / (after != E.NONE).sum())
    logprob = model.forward(tokens, after).double().clone()
    model.backward(tokens, after, dlogprob)
    p = {n: t.double().requires_grad_() for n, t in model.param.items()}
    norm = lambda x, gamma: x / torch.sqrt((x * x).mean(1, keepdim=True) + E.EPS) * gamma  # noqa: E731
    x = p["embed"][tokens]
    for b in range(2):
        h = torch.nn.functional.gelu(norm(x, p[f"{b}.before"]) @ p[f"{b}.fc1.w"].t() + p[f"{b}.fc1.b"], approximate="tanh")
        x = x + p[f"{b}.gate"] * norm(h @ p[f"{b}.fc2.w"].t(), p[f"{b}.after"])
    logp = torch.log_softmax(norm(x, p["norm"]) @ p["embed"].t(), 1)
    given = after != E.NONE
    want = torch.where(given, logp.gather(1, torch.where(given, after, 0)[:, None])[:, 0], 0.0)
    (want * dlogprob.double()).sum().backward()
    assert (logprob - want).norm() < 2.0 ** -6 * want.norm()
    for name, grad in model.grad.items():
        assert (grad.double() - p[name].grad).norm() < 2.0 ** -5 * p[name].grad.norm(), name
    model.close()


def test_an_update_of_it_is_adamw():
    """The masters after one step against the formula in 64 bits, on the gradients as they are: off by the step's some 30 roundings of
    2^-24; the working copy by one to 16 bits."""
    import torch

    from oracle import training as T
    E = _example()
    model = E.Model(256, 200, 64, 96, 1, seed=4)
    tokens, after = E.batch(0, 256, 200)
    dlogprob = torch.where(after == E.NONE, 0.0, -1.0 / (after != E.NONE).sum())
    model.forward(tokens, after)
    model.backward(tokens, after, dlogprob)
    before = {n: t.double().cpu().numpy() for n, t in model.master.items()}
    grads = {n: t.double().cpu().numpy() for n, t in model.grad.items()}
    model.update()
    factor = T.adamw_factor(1.0, sum((g ** 2).sum() for g in grads.values()), 1.0)
    for n, p in before.items():
        want, _, _ = T.adamw(p, grads[n], 0 * p, 0 * p, 1, E.RATE, 0.9, 0.99, 1e-8, factor, 0.01 if p.ndim == 2 else 0.0)
        off = abs(model.master[n].double().cpu().numpy() - want)
        assert (off <= 2.0 ** -23 * abs(want) + 32 * 2.0 ** -24 * E.RATE).all(), n
        assert torch.equal(model.param[n], model.master[n].bfloat16()), n
    model.close()
