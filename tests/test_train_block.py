"""The operators together: examples/train_block.py against the same model in 32 bits."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _rms(x, w, eps):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w


def _reference(ex, model, words):
    """Leaves in 32 bits and the normed output of the last block; matrix products without transposed views."""
    leaves = {name: w.float().clone().requires_grad_() for name, w in model.weights.items()}
    total = leaves["embedding"][words]
    normed = _rms(total, leaves["pre0"], ex.EPS)
    for i in range(model.blocks):
        both = normed @ leaves[f"gate_up{i}"].t()
        g, u = both[:, : model.hidden], both[:, model.hidden:]
        y = (torch.nn.functional.silu(g) * u) @ leaves[f"down{i}"].t()
        total = total + leaves[f"scale{i}"] * _rms(y, leaves[f"post{i}"], ex.EPS)
        normed = _rms(total, leaves[f"pre{i + 1}"], ex.EPS)
    return leaves, normed


@pytest.mark.gpu
def test_first_step():
    ex = _example()
    tokens, width, hidden, vocab = 301, 136, 200, 1003
    model = ex.Model(tokens, width, hidden, vocab, 2)
    words, targets = ex.batch(tokens, vocab, 0)
    loss = model.forward(words, targets)
    model.backward(words, targets)
    leaves, normed = _reference(ex, model, words)
    want = torch.nn.functional.cross_entropy(normed @ leaves["head"].t(), targets, ignore_index=ex.IGNORE)
    want.backward()
    # A step rounds twelve tensors a block to 8 significant bits on the way there and back, each 2^-9 of a number at the root of their squares' mean; their errors
    # pass through a norm or a product, which keep their share of the result's norm, and come together by squares: sqrt(2 * 12 + 6) * 2^-9 = 0.011; a norm's weights are sums
    # that cancel, and get four times as much.
    for name, leaf in leaves.items():
        off, size = float((model.grads[name].float() - leaf.grad).norm()), float(leaf.grad.norm())
        assert off <= (0.044 if leaf.dim() == 1 or leaf.shape[0] == 1 else 0.022) * size, (name, off / size)
    assert abs(float(loss) - float(want.detach())) <= 0.011 * float(want.detach())
    norm = float(torch.stack([g.double().square().sum() for g in model.grads.values()]).sum().sqrt())
    before = {name: g.clone() for name, g in model.grads.items()}
    model.update(0.5)
    assert abs(float(model.norm) - norm) <= 2.0 ** -20 * norm
    for name, g in model.grads.items():
        want = before[name].double() * min(1.0, 1.0 / norm)
        assert bool(torch.all((g.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs() + 2.0 ** -133)), name
    model.close()


@pytest.mark.gpu
def test_single_tokens_and_running():
    ex = _example()
    model, losses = ex.train(steps=3, tokens=300, width=64, hidden=72, vocab=500, blocks=1)
    assert all(v == v for v in losses)
    word = torch.tensor(7, device="cuda")
    z = model.one_token(word)
    leaves, normed = _reference(ex, model, word.reshape(1))
    want = (normed @ leaves["head"].t())[0].detach()
    assert float((z.float() - want).norm()) <= 0.022 * float(want.norm())
    model.close()
