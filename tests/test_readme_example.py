"""README.md's example of the low-precision operators runs as it is written, from a context that has no work memory yet."""
import os
import re

import pytest

torch = pytest.importorskip("torch")

from paper_2508_00441_amd import binding as oz, device  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,vocab", [(512, 1024, 1024, 5000), (1, 64, 65536, 300), (2048, 512, 1024, 8192)])
def test_product_and_loss(m, n, k, vocab):
    with open(os.path.join(ROOT, "README.md")) as f:
        example = next(code for code in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "ozaki_gemm_fp8(" in code)
    gen = torch.Generator(device="cuda").manual_seed(1)
    X, weights = torch.randn((m, k), device="cuda", generator=gen).bfloat16(), torch.randn((n, k), device="cuda", generator=gen) / k ** 0.5
    Qw, Sw = torch.empty((n, k), dtype=torch.uint8, device="cuda"), torch.empty((-(-k // 128), -(-n // 128)), device="cuda")
    D, W = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), (torch.randn((vocab, n), device="cuda", generator=gen) / n ** 0.5).bfloat16()
    dD, dW = torch.empty_like(D), torch.empty_like(W)
    targets = torch.randint(0, vocab, (m,), device="cuda", generator=gen)
    loss, lse, dloss = torch.empty((m,), device="cuda"), torch.empty((m,), device="cuda"), torch.full((m,), 1.0 / m, device="cuda")
    context = oz.ozaki_context_create()
    oz.ozaki_context_use(context)
    try:
        oz.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        oz.ozaki_quantise_fp8(n, k, weights, k, oz.TYPE_F32, oz.SCALE_BLOCKS, Qw, k, Sw, Sw.shape[1])
        exec(example, dict(locals(), torch=torch, oz=oz, device=device))
        torch.cuda.synchronize()
    finally:
        oz.ozaki_context_use(None)
        oz.ozaki_context_destroy(context)
    # two roundings to four significant bits of every element, whose sum over k is of that share of the result's norm at most
    want = X.float() @ weights.t().contiguous()
    assert float((D.float() - want).norm()) <= 2 * 2.0 ** -4 * float(want.norm())
    h = D.float().requires_grad_()
    mean = torch.nn.functional.cross_entropy(h @ W.float().t().contiguous(), targets)
    mean.backward()
    assert abs(float(loss.mean()) - float(mean.detach())) <= 1e-4 * (1 + float(mean.detach()))
    # (g and dD are rounded to 8 significant bits, 2^-8 of a term each at most; the sum of g's is of that share of the norm, with room for what cancels)
    assert float((dD.float() - h.grad).norm()) <= 2.0 ** -6 * float(h.grad.norm())
