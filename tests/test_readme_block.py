"""README.md's example of a feed-forward block and its gradient runs as it is written, from a context that has no work memory yet."""
import os
import re

import pytest

torch = pytest.importorskip("torch")

from paper_2508_00441_amd import binding as oz, device  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,hidden", [(1, 264, 1000), (96, 512, 1024), (700, 328, 520)])
def test_block(m, n, hidden):
    with open(os.path.join(ROOT, "README.md")) as f:
        example = next(code for code in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "ozaki_gated_linear(" in code)
    gen = torch.Generator(device="cuda").manual_seed(m)
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=gen)    # noqa: E731
    new = lambda *shape: torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")    # noqa: E731
    names = dict(Wg=rand(hidden, n) / n ** 0.5, Wu=rand(hidden, n) / n ** 0.5, Wd=rand(n, hidden) / hidden ** 0.5, r=rand(m, n), dr=rand(m, n), da2=rand(m, n))
    names = {name: v.bfloat16() for name, v in names.items()} | dict(w1=1 + 0.1 * rand(n), w2=1 + 0.1 * rand(n), dw1=torch.zeros(n, device="cuda"), dw2=torch.zeros(n, device="cuda"))
    names |= dict(a=new(m, n), g=new(m, hidden), u=new(m, hidden), h=new(m, hidden), r2=new(m, n), a2=new(m, n), dr2=new(m, n), dh=new(m, hidden), da=new(m, n), dWd=new(n, hidden),
                  dWg=new(hidden, n), dWu=new(hidden, n))
    leaves = {name: names[name].float().requires_grad_() for name in ("r", "Wg", "Wu", "Wd", "w1", "w2")}
    context = oz.ozaki_context_create()
    oz.ozaki_context_use(context)
    try:
        oz.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        exec(example, dict(names, m=m, n=n, hidden=hidden, oz=oz, device=device, torch=torch))
        torch.cuda.synchronize()
    finally:
        oz.ozaki_context_use(None)
        oz.ozaki_context_destroy(context)
    norm = lambda x, w: x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6) * w    # noqa: E731
    a = norm(leaves["r"], leaves["w1"])
    r2 = leaves["r"] + (torch.nn.functional.silu(a @ leaves["Wg"].t()) * (a @ leaves["Wu"].t())) @ leaves["Wd"].t()
    a2 = norm(r2, leaves["w2"])
    ((a2 * names["da2"].float()).sum() + (r2 * names["dr"].float()).sum()).backward()
    # twelve tensors between the ends are rounded to 8 significant bits, 2^-9 of a number at the root of their squares' mean, and come together by squares: 2^-7; with
    # room for what a single row does not average out, twice that
    for got, want in ((names["r2"], r2), (names["a2"], a2), (names["dr2"], leaves["r"].grad), (names["dWg"], leaves["Wg"].grad), (names["dWu"], leaves["Wu"].grad),
                      (names["dWd"], leaves["Wd"].grad), (names["dw1"], leaves["w1"].grad), (names["dw2"], leaves["w2"].grad)):
        assert float((got.float() - want.detach()).norm()) <= 2.0 ** -6 * float(want.detach().norm())
