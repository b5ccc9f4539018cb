"""The operators together: examples/train_fp8.py against the same training in 32 bits."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_fp8", os.path.join(ROOT, "examples", "train_fp8.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.gpu
def test_first_step_and_training():
    ex = _example()
    tokens, features, hidden, vocab = 700, 520, 328, 3001
    head = ex.Head(tokens, features, hidden, vocab)
    W1, W2 = head.W1.clone().requires_grad_(), head.W2.to(torch.bfloat16).float().requires_grad_()
    x, targets = ex.batch(tokens, features, vocab, 0)
    loss = head.forward(x, targets)
    head.backward(targets)
    xf = x.float().requires_grad_()
    want = torch.nn.functional.cross_entropy((xf @ W1.t()) @ W2.t(), targets, ignore_index=ex.IGNORE)
    want.backward()
    # E4M3 has four significant bits: a product of two roundings each up to 2^-4 of the element, whose sum over hundreds of elements is of that share
    # of the result's norm at most
    for got, ref in ((head.dW1, W1.grad), (head.dW2.float(), W2.grad), (head.dx.float(), xf.grad)):
        assert float((got - ref).norm()) <= 2 * 2.0 ** -4 * float(ref.norm())
    assert abs(float(loss) - float(want.detach())) <= 2 * 2.0 ** -4 * float(want.detach())
    assert bool(torch.all(head.dx[targets == ex.IGNORE] == 0.0))
    head.close()
    head, losses = ex.train(steps=15, tokens=tokens, features=features, hidden=hidden, vocab=vocab)
    assert losses[-1] < 0.5 * losses[0]
    x, targets = ex.batch(1, features, vocab, 99)
    h = head.one_token(x)
    assert float((h.float() - x.float() @ head.W1.t()).norm()) <= 2 * 2.0 ** -4 * float((x.float() @ head.W1.t()).norm())
    head.close()
