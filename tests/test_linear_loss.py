"""ozaki_linear_loss and ozaki_linear_loss_grad against their definitions in 64 bits, within bounds of their 32-bit sums and of the 16 bits of g."""
import pytest

torch = pytest.importorskip("torch")

import low_precision as plain  # noqa: E402
from paper_2508_00441_amd import binding as lib, device  # noqa: E402

SHAPES = [(1, 1, 1), (1, 1000, 64), (3, 5, 8), (7, 513, 100), (16, 2000, 257), (17, 300, 72), (33, 129, 640), (64, 4099, 128), (65, 1000, 33), (200, 3001, 200),
          (257, 255, 1000), (300, 511, 64)]
EXP = 2.0 ** -20                                                    # relative, of an exponential, a logarithm and the sums around them


class Problem:
    def __init__(self, tokens, vocab, k, type, seed, ignored=0.2, spread=2.0, ignore=-100):
        gen = torch.Generator().manual_seed(seed)
        dtype = plain.DTYPES[type]
        self.tokens, self.vocab, self.k, self.type, self.ignore = tokens, vocab, k, type, ignore
        self.h = torch.randn((tokens, k), generator=gen).to(dtype)
        self.w = (torch.randn((vocab, k), generator=gen) * spread / k ** 0.5).to(dtype)
        self.targets = torch.randint(0, vocab, (tokens,), generator=gen)
        self.targets[torch.rand((tokens,), generator=gen) < ignored] = ignore
        self.dloss = torch.randn((tokens,), generator=gen)
        self.upload()

    def upload(self):
        self.H, self.W = plain.padded(self.h, 8, float("nan")).cuda(), plain.padded(self.w, 8, float("nan")).cuda()
        self.T = self.targets.cuda()

    def arguments(self):
        return (self.tokens, self.vocab, self.k, self.H, self.H.shape[1], self.W, self.W.shape[1], lib.TYPES[self.type], self.T, self.ignore)

    def forward(self):
        loss, lse = (torch.full((self.tokens,), float("nan"), device="cuda") for _ in range(2))
        lib.ozaki_linear_loss(*self.arguments(), loss, lse)
        return loss, lse

    def gradient(self, lse, ldh=None, ldw=None, want=("dh", "dw")):
        dtype = plain.DTYPES[self.type]
        dh = torch.full((self.tokens, ldh or self.k), float("nan"), dtype=dtype, device="cuda") if "dh" in want else None
        dw = torch.full((self.vocab, ldw or self.k), float("nan"), dtype=dtype, device="cuda") if "dw" in want else None
        lib.ozaki_linear_loss_grad(*self.arguments(), lse, self.dloss.cuda(), dh, ldh or self.k, dw, ldw or self.k)
        return dh, dw

    def gradient_bounds(self, lse):
        """(the gradient, what the result may be off) of H, and of W."""
        want_h, want_w, g, p, h = plain.loss_gradient(self.h, self.w, self.targets, self.ignore, lse.cpu(), self.dloss)
        u, tiny = plain.ROUNDING[self.type]
        # of g without dloss: its rounding (FP16: also where it runs out of normal numbers, half of 2^-24 below 2^-12), z's and the exponential's errors;
        # dW's other operand is H times the token's share of the largest |dloss|, rounded where the shares differ
        factor = torch.where(self.targets == self.ignore, 0.0, self.dloss.double()).abs().unsqueeze(1)
        dg = u * g.abs() + p * ((plain.logit_error(h, self.w) + EXP).unsqueeze(1) * (1 + u)) + 2.0 ** -22 * g.abs()
        if self.type == "f16":
            dg = dg + 2.0 ** -37 * factor
        shares = torch.unique(factor[factor > 0])
        dgw, least = dg, 0.0
        if len(shares) > 1:
            dgw = dg + u * (1 + u) * g.abs()
            if self.type == "f16":                                  # (half the smallest step of the product of H and the share)
                least = 2.0 ** -25 * float(factor.max()) * torch.where(factor > 0, g.abs() / factor, 0.0).sum(0).unsqueeze(1)
        w, h = self.w.double().abs(), h.abs()
        out = []
        for want, by, other, terms in ((want_h, dg, w, self.vocab + 40), (want_w, dgw.t(), h, self.tokens + 4)):
            size = g.abs() if by is dg else g.abs().t()
            bound = by @ other + 2 * terms * 2.0 ** -24 * ((size + by) @ other) + (0.0 if by is dg else least)
            out.append((want, bound + u * (want.abs() + bound) + tiny))
        return out

    def check_gradient(self, dh, dw, lse):
        for got, (want, bound) in zip((dh, dw), self.gradient_bounds(lse)):
            if got is not None:
                assert bool(torch.all((got[:, : self.k].cpu().double() - want).abs() <= bound))


@pytest.fixture()
def workspace():
    ws = device.Workspace(256 << 20)
    yield ws
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,vocab,k", SHAPES + [(2500, 3000, 136), (3000, 4001, 600), (2900, 4000, 1001)])
def test_loss(tokens, vocab, k, type, workspace):
    x = Problem(tokens, vocab, k, type, tokens + vocab + k)
    loss, lse = x.forward()
    assert lib.ozaki_last_device_status() == 0
    want, want_lse, _ = plain.loss_forward(x.h, x.w, x.targets, x.ignore)
    bound = plain.logit_error(x.h, x.w) + EXP * (1 + want_lse.abs())
    assert bool(torch.all((lse.cpu().double() - want_lse).abs() <= bound))
    assert bool(torch.all((loss.cpu().double() - want).abs() <= 2 * bound + 2.0 ** -23 * want.abs()))
    assert bool(torch.all(loss.cpu()[x.targets == x.ignore] == 0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,vocab,k", SHAPES + [(1500, 6000, 136), (3000, 4001, 600), (2900, 4000, 1001), (700, 9001, 1000),
                                                     (130, 9001, 1000), (65, 33000, 264), (1, 33000, 300), (17, 40001, 72)])
def test_gradient(tokens, vocab, k, type, workspace):
    x = Problem(tokens, vocab, k, type, tokens + vocab + k)
    _, lse = x.forward()
    dh, dw = x.gradient(lse)
    x.check_gradient(dh, dw, lse)
    assert bool(torch.all(dh[(x.T == x.ignore)] == 0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,k", [(77, 2701, 201), (600, 3001, 333)])
def test_few_tokens_that_count_in_pieces(tokens, vocab, k):
    x = Problem(tokens, vocab, k, "bf16", 8, ignored=0.9)
    least = device.Workspace(lib.ozaki_linear_loss_workspace_bytes(tokens, vocab, k, True, True))
    _, lse = x.forward()
    x.check_gradient(*x.gradient(lse), lse)
    least.close()


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("ignored", [0.6, 0.97])
@pytest.mark.parametrize("tokens,vocab,k", [(9, 700, 100), (130, 2000, 201), (700, 9001, 400), (2100, 4500, 264)])
def test_few_tokens_that_count(tokens, vocab, k, ignored, type, workspace):
    x = Problem(tokens, vocab, k, type, 7, ignored=ignored)
    x.H[x.T == x.ignore] = float("nan")
    _, lse = x.forward()
    lse = torch.where(x.T == x.ignore, 0.0, lse)
    dh, dw = x.gradient(lse, ldh=k + 3)
    x.check_gradient(dh, dw, lse)
    assert bool(torch.all(dh[x.T == x.ignore][:, :k] == 0.0)) and bool(torch.isnan(dh[:, k:]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,k", [(1030, 13201, 1100), (513, 22017, 136), (1900, 8705, 600)])
def test_vocabularies_whose_last_tiles_are_few(tokens, vocab, k, workspace):
    test_loss(tokens, vocab, k, "bf16", workspace)
    test_gradient(tokens, vocab, k, "bf16", workspace)


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_gradient_in_pieces_and_one_result_at_a_time(type):
    x = Problem(150, 2900, 200, type, 1)
    least, best = (lib.ozaki_linear_loss_workspace_bytes(x.tokens, x.vocab, x.k, True, m) for m in (True, False))
    assert 0 < least < best
    for size in (best, (least + best) // 2, least):
        ws = device.Workspace(size)
        _, lse = x.forward()
        dh, dw = x.gradient(lse)
        x.check_gradient(dh, dw, lse)
        only_h, only_w = x.gradient(lse, want=("dh",))[0], x.gradient(lse, want=("dw",))[1]
        assert torch.equal(only_h, dh) and torch.equal(only_w, dw)
        ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,k", [(5, 2600, 203), (77, 2701, 201), (301, 3001, 333)])
def test_gradient_in_pieces_of_odd_sizes(tokens, vocab, k):
    x = Problem(tokens, vocab, k, "bf16", 3)
    least = device.Workspace(lib.ozaki_linear_loss_workspace_bytes(tokens, vocab, k, True, True))
    _, lse = x.forward()
    x.check_gradient(*x.gradient(lse), lse)
    least.close()


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_results_inside_larger_ones(type, workspace):
    x = Problem(70, 400, 99, type, 2)
    _, lse = x.forward()
    dh, dw = x.gradient(lse, ldh=103, ldw=117)
    x.check_gradient(dh, dw, lse)
    assert bool(torch.isnan(dh[:, 99:]).all()) and bool(torch.isnan(dw[:, 99:]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("tokens", [20, 300])
def test_what_ignored_tokens_hold_does_not_matter(tokens, type, workspace):
    x = Problem(tokens, 700, 128, type, 3, ignored=0.5)
    gone = x.targets == x.ignore
    x.h[gone] = float("nan")
    x.h[gone.nonzero()[0, 0]] = float("inf")
    x.dloss[gone] = float("nan")
    x.upload()
    loss, lse = x.forward()
    assert bool(torch.all(loss[gone.cuda()] == 0.0)) and bool(torch.isfinite(loss).all())
    dh, dw = x.gradient(lse)
    x.check_gradient(dh, dw, torch.where(gone, 0.0, lse.cpu()))
    assert lib.ozaki_last_device_status() == 0


@pytest.mark.gpu
def test_all_tokens_ignored_and_none_at_all(workspace):
    x = Problem(40, 300, 64, "bf16", 4, ignored=1.1)
    loss, lse = x.forward()
    dh, dw = x.gradient(lse)
    assert bool(torch.all(loss == 0.0)) and bool(torch.all(dh == 0.0)) and bool(torch.all(dw == 0.0))
    dw.fill_(3.0)
    lib.ozaki_linear_loss(0, 300, 64, None, 64, None, 64, lib.TYPE_BF16, None, -100, None, None)
    lib.ozaki_linear_loss_grad(0, 300, 64, None, 64, None, 64, lib.TYPE_BF16, None, -100, None, None, None, 0, dw, 64)
    assert bool(torch.all(dw == 0.0))


@pytest.mark.gpu
def test_targets_outside_the_vocabulary(workspace):
    x = Problem(50, 300, 64, "bf16", 5, ignored=0.0)
    good, lse = x.forward()
    bad = torch.tensor([3, 17, 49])
    x.targets[bad] = torch.tensor([300, -1, 1 << 40])
    x.upload()
    loss, lse = x.forward()
    assert lib.ozaki_last_device_status() == lib.STATUS_TARGET and lib.ozaki_last_device_status() == 0
    fine = torch.ones(50, dtype=torch.bool)
    fine[bad] = False
    assert bool(torch.isnan(loss.cpu()[bad]).all()) and torch.equal(loss.cpu()[fine], good.cpu()[fine])
    dh, dw = x.gradient(lse)
    assert lib.ozaki_last_device_status() == lib.STATUS_TARGET
    x.targets[bad] = x.ignore
    x.check_gradient(dh, dw, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [5, 400])
def test_outputs_far_apart_and_at_infinity(tokens, workspace):
    """Words whose output is minus infinity have no share; a token whose outputs are hundreds apart has a loss of its target's distance."""
    x = Problem(tokens, 900, 64, "bf16", 6, spread=200.0, ignored=0.0)
    x.h[:, 0] = 1.0
    x.w[10:800, 0] = -float("inf")
    x.targets[x.targets >= 10] = 3
    x.upload()
    loss, lse = x.forward()
    want, want_lse, _ = plain.loss_forward(x.h, x.w, x.targets, x.ignore)
    finite = x.w.clone()
    finite[10:800, 0] = 0.0
    bound = plain.logit_error(x.h, finite) + EXP * (1 + want_lse.abs())
    assert bool(torch.all((lse.cpu().double() - want_lse).abs() <= bound))
    assert bool(torch.all((loss.cpu().double() - want).abs() <= 2 * bound + 2.0 ** -23 * want.abs()))


@pytest.mark.gpu
def test_small_upstream_gradients_in_16_bit_floats(workspace):
    """A mean over very many tokens: dloss alone would take g below FP16's smallest number; the result itself is what may underflow."""
    x = Problem(130, 2000, 256, "f16", 7, ignored=0.0)
    x.dloss = torch.full((130,), 1e-5)
    _, lse = x.forward()
    dh, dw = x.gradient(lse)
    x.check_gradient(dh, dw, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_gradient_against_differences(type, workspace):
    """Central differences of the 64-bit loss along random directions, whose own error is of the third derivative's size times the step squared."""
    x = Problem(40, 500, 96, type, 8)
    _, lse = x.forward()
    dh, dw = x.gradient(lse)
    gen = torch.Generator().manual_seed(80)

    def total(h, w):
        return float((plain.loss_forward(h, w, x.targets, x.ignore)[0] * torch.where(x.targets == x.ignore, 0.0, x.dloss.double())).sum())

    for which, got, (_, bound) in zip("hw", (dh, dw), x.gradient_bounds(lse)):
        at = {"h": x.h.double(), "w": x.w.double()}
        for _ in range(3):
            d = torch.randn(at[which].shape, generator=gen, dtype=torch.float64)
            e = 1e-5
            difference = (total(**{**at, which: at[which] + e * d}) - total(**{**at, which: at[which] - e * d})) / (2 * e)
            along = float((got.cpu().double() * d).sum())
            # (the step's own errors: 1e-10 of third derivatives, 1e-16 of a sum of some hundred over 1e-5)
            assert abs(along - difference) <= float((bound * d.abs()).sum()) + 1e-6


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,k", [(1, 3000, 512), (100, 3000, 512), (1500, 5000, 64)])
def test_the_same_bits_every_time_and_in_graphs(tokens, vocab, k, workspace):
    x = Problem(tokens, vocab, k, "bf16", 9)
    dloss = x.dloss.cuda()
    loss, lse = x.forward()
    dh, dw = x.gradient(lse)
    out = [torch.empty_like(t) for t in (loss, lse, dh, dw)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        lib.ozaki_linear_loss(*x.arguments(), out[0], out[1])
        lib.ozaki_linear_loss_grad(*x.arguments(), out[1], dloss, out[2], k, out[3], k)
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, (loss, lse, dh, dw)):
            assert torch.equal(got, want)
        x.H[:, :k].mul_(0.5)                                        # new inputs for the next replay
        loss, lse = x.forward()
        dh, dw = x.gradient(lse)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [9, 70, 300])
def test_offsets_beyond_2_32(tokens, workspace):
    """Weights, and their gradient, whose last words lie beyond 4 GiB."""
    vocab, k, ld = 40000, 100, 1 << 16
    x = Problem(tokens, vocab, k, "bf16", 10)
    wide = torch.full((vocab, ld), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :k] = x.w.cuda()
    x.W = wide
    loss, lse = x.forward()
    want, want_lse, _ = plain.loss_forward(x.h, x.w, x.targets, x.ignore)
    bound = plain.logit_error(x.h, x.w) + EXP * (1 + want_lse.abs())
    assert bool(torch.all((loss.cpu().double() - want).abs() <= 2 * bound + 2.0 ** -23 * want.abs()))
    dh, dw = x.gradient(lse, ldw=ld)
    x.check_gradient(dh, dw, lse)
    assert bool(torch.isnan(dw[:, k:]).all())


P = 1 << 20
FORWARD = dict(tokens=100, vocab=200, k=30, H=P, ldh=32, W=P, ldw=32, type=lib.TYPE_BF16, targets=P, ignore=-100, loss=P, lse=P)
SHARED = [(1, dict(tokens=-1)), (1, dict(tokens=lib.MAX_EXTENT + 1)), (2, dict(vocab=0)), (2, dict(vocab=lib.MAX_EXTENT + 1)), (3, dict(k=0)),
          (3, dict(k=lib.MAX_EXTENT)), (4, dict(H=None)), (4, dict(H=P + 8)), (5, dict(ldh=24)), (5, dict(ldh=36)), (6, dict(W=None)), (6, dict(W=P + 2)),
          (7, dict(ldw=24)), (7, dict(ldw=33)), (8, dict(type=lib.TYPE_F32)), (8, dict(type=3)), (9, dict(targets=None))]


@pytest.mark.parametrize("position,arguments", SHARED + [(11, dict(loss=None)), (12, dict(lse=None))])
def test_refusals_of_the_loss(position, arguments):
    assert lib.ozaki_linear_loss(**{**FORWARD, **arguments}, check=False) == -position


@pytest.mark.parametrize("position,arguments", SHARED + [(11, dict(lse=None)), (12, dict(dloss=None)), (13, dict(dH=None, dW=None)), (13, dict(dH=P + 1)),
                                                         (14, dict(lddh=29)), (15, dict(dW=P + 1)), (16, dict(lddw=29))])
def test_refusals_of_the_gradient(position, arguments):
    a = {n: v for n, v in FORWARD.items() if n != "loss"} | dict(dloss=P, dH=P, lddh=30, dW=P, lddw=30)
    assert lib.ozaki_linear_loss_grad(**{**a, **arguments}, check=False) == -position


@pytest.mark.parametrize("sizes,position", [(dict(tokens=lib.MAX_EXTENT, vocab=lib.MAX_LOGITS // lib.MAX_EXTENT + 1), 2), (dict(k=1 << 62), 3)])
def test_refuses_more_than_a_launch_holds(sizes, position):
    assert lib.ozaki_linear_loss(**{**FORWARD, **sizes}, check=False) == -position
    assert lib.ozaki_linear_loss_workspace_bytes(**{**dict(tokens=100, vocab=200, k=30), **sizes}, grad=False, minimum=False) == 0


def test_without_work_memory():
    assert lib.ozaki_linear_loss_workspace_bytes(0, 200, 30, False, False) == 0 and lib.ozaki_linear_loss_workspace_bytes(100, 200, 30, False, False) > 0
    context = lib.ozaki_context_create()
    lib.ozaki_context_use(context)
    try:
        assert lib.ozaki_linear_loss(**FORWARD, check=False) == lib.STATUS_WORKSPACE
        a = {n: v for n, v in FORWARD.items() if n != "loss"} | dict(dloss=P, dH=P, lddh=30, dW=P, lddw=30)
        assert lib.ozaki_linear_loss_grad(**a, check=False) == lib.STATUS_WORKSPACE
    finally:
        lib.ozaki_context_use(None)
        lib.ozaki_context_destroy(context)


@pytest.mark.gpu
def test_every_cause_is_reported_once(workspace):
    """A target outside the vocabulary and an FP64 product's infinity between two looks at the status: one after the other."""
    x = Problem(50, 300, 64, "bf16", 5, ignored=0.0)
    x.targets[7] = 300
    x.upload()
    A = torch.ones((64, 64), dtype=torch.float64, device="cuda")
    A[3, 5] = float("inf")
    C = torch.empty_like(A)
    product = lambda: lib.ozaki_dgemm(64, 64, 64, A, 64, A, 64, C, 64, lib.SLICE_FP8_E4M3, 4, 0, lib.ACCUM_FP64_HW)  # noqa: E731
    for calls in ((x.forward, product), (product, x.forward)):
        for call in calls:
            call()
        assert [lib.ozaki_last_device_status() for _ in range(3)] == [lib.STATUS_NONFINITE, lib.STATUS_TARGET, lib.STATUS_OK]
    x.forward()
    assert [lib.ozaki_last_device_status() for _ in range(2)] == [lib.STATUS_TARGET, lib.STATUS_OK]
    product()
    assert [lib.ozaki_last_device_status() for _ in range(2)] == [lib.STATUS_NONFINITE, lib.STATUS_OK]


@pytest.mark.parametrize("k", [1, 64, 300, 1000, 4096, 8192])
def test_the_least_work_memory_is_no_more_than_the_recommended(k):
    for tokens in (1, 17, 150, 1000, 4096, 8192, 70000):
        for vocab in (1, 255, 300, 1001, 2900, 8192, 32000, 131072):
            least, best = (lib.ozaki_linear_loss_workspace_bytes(tokens, vocab, k, True, m) for m in (True, False))
            assert 0 < least <= best, (tokens, vocab)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,k", [(40, 300, 1024), (300, 1200, 520), (70, 2600, 1000)])
def test_gradient_with_the_least_work_memory(tokens, vocab, k):
    x = Problem(tokens, vocab, k, "bf16", 21)
    need = lib.ozaki_linear_loss_workspace_bytes(tokens, vocab, k, True, True)
    forward = device.Workspace(lib.ozaki_linear_loss_workspace_bytes(tokens, vocab, k, False, False))
    _, lse = x.forward()
    forward.close()
    least = device.Workspace(need)
    dh, dw = x.gradient(lse)
    x.check_gradient(dh, dw, lse)
    least.close()
    short = torch.empty(need - 256, dtype=torch.uint8, device="cuda")
    lib.ozaki_set_workspace(short, short.numel())
    assert lib.ozaki_linear_loss_grad(*x.arguments(), lse, x.dloss.cuda(), dh, k, dw, k, check=False) == lib.STATUS_WORKSPACE
    lib.ozaki_set_workspace(None, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,vocab", [(5, 900), (70, 900), (400, 9000), (2900, 4000)])
def test_outputs_at_plus_infinity(tokens, vocab, type, workspace):
    """The logarithm of a sum that holds an infinite term is infinite, and so is the loss of any other word; of the word itself it is NaN."""
    x = Problem(tokens, vocab, 64, type, 22, ignored=0.1)
    x.h[:, 0] = torch.where(torch.arange(tokens) % 3 == 0, 1.0, -1.0)
    x.w[:, 0] = 0.0
    x.w[vocab // 2, 0] = float("inf")
    x.w[vocab // 3] = 0.0
    x.w[vocab // 3, 1] = 50.0                                       # large outputs beside it, in other tiles
    x.targets[x.targets == vocab // 2] = 1
    x.targets[0] = vocab // 2
    x.upload()
    loss, lse = x.forward()
    want, want_lse, _ = plain.loss_forward(x.h, x.w, x.targets, x.ignore)
    up = x.h[:, 0] > 0
    finite = x.w.clone()
    finite[vocab // 2, 0] = 0.0
    bound = plain.logit_error(x.h, finite) + EXP * (1 + want_lse.abs())
    assert bool(torch.all(lse.cpu()[up] == float("inf")))
    assert bool(torch.all((lse.cpu().double() - want_lse).abs()[~up] <= bound[~up]))
    counts = x.targets != x.ignore
    counts[0] = False
    assert bool(torch.isnan(loss[0])) and bool(torch.all(loss.cpu()[up & counts] == float("inf"))) and bool(torch.all(loss.cpu()[x.targets == x.ignore] == 0.0))
    assert bool(torch.all((loss.cpu().double() - want).abs()[~up & counts] <= (2 * bound + 2.0 ** -23 * want.abs())[~up & counts]))


@pytest.mark.gpu
@pytest.mark.parametrize("weight", [2.0 ** -10 * 1.37, 2.0 ** -14 * 1.9, 1e-5, 2.0 ** -19 * 1.01])
@pytest.mark.parametrize("tokens,vocab,k", [(14, 60, 96), (200, 600, 96), (1030, 9001, 1000)])
def test_tokens_of_little_weight_in_16_bit_floats(tokens, vocab, k, weight, workspace):
    """Half of the tokens count a small share of the others, and have words of their own: what the gradient of these words is made of is the
    small shares alone.  Down to 2^-19 of the largest weight the elements of H may be off by a rounding to 11 bits or, where they are small,
    by 2^-14."""
    x = Problem(tokens, vocab, k, "f16", 23, ignored=0.1)
    light, own = torch.arange(tokens) % 2 == 1, torch.arange(vocab) >= vocab // 2
    x.h[:, 0] = torch.where(light, 6.0, -6.0)
    x.w[:, 0] = torch.where(own, 6.0, -6.0)                         # outputs of the others' words: lower by 72
    x.targets[light & (x.targets != x.ignore)] = vocab - 1 - torch.arange(int((light & (x.targets != x.ignore)).sum())) % (vocab - vocab // 2)
    x.targets[~light & (x.targets != x.ignore)] %= vocab // 2
    x.dloss = torch.where(light, 64.0 * weight, 64.0)
    x.upload()
    _, lse = x.forward()
    dh, dw = x.gradient(lse)
    want_h, want_w, g, p, h = plain.loss_gradient(x.h, x.w, x.targets, x.ignore, lse.cpu(), x.dloss)
    u, tiny = plain.ROUNDING["f16"]
    factor = torch.where(x.targets == x.ignore, 0.0, x.dloss.double()).unsqueeze(1)
    # g: its rounding, z's and the exponential's errors, and half of FP16's smallest step: g is held times 2^12, for small weights times 2^4 at least
    dg = u * g.abs() + p * ((plain.logit_error(x.h, x.w) + EXP).unsqueeze(1) * (1 + u)) + 2.0 ** -22 * g.abs() + 2.0 ** -29 * factor
    out = dg @ x.w.double().abs()
    out = out + 2 * (vocab + 40) * 2.0 ** -24 * ((g.abs() + dg) @ x.w.double().abs())
    assert bool(torch.all((dh.cpu().double() - want_h).abs() <= out + u * (want_h.abs() + out) + tiny))
    out = dg.t() @ (h.abs() * (1 + u) + 2.0 ** -14) + g.abs().t() @ (u * h.abs() + 2.0 ** -14)
    out = out + 2 * (tokens + 4) * 2.0 ** -24 * ((g.abs() + dg).t() @ (h.abs() + 2.0 ** -14))
    assert bool(torch.all((dw.cpu().double() - want_w).abs() <= out + u * (want_w.abs() + out) + tiny))


@pytest.mark.gpu
@pytest.mark.parametrize("ignored", [0.0, 0.7])
@pytest.mark.parametrize("tokens,vocab,k,type,memory", [(1101, 20001, 1000, "bf16", 0.84), (1030, 30001, 603, "f16", 0.84)])
def test_gradient_in_pieces_by_large_tiles(tokens, vocab, k, type, memory, ignored):
    """Work memory for two or three pieces of the vocabulary that are each large enough for tiles of 256 x 256 in z, dH (in shares) and dW; the
    last piece is shorter and takes other tiles and other numbers of shares."""
    x = Problem(tokens, vocab, k, type, 24, ignored=ignored)
    least, best = (lib.ozaki_linear_loss_workspace_bytes(tokens, vocab, k, True, m) for m in (True, False))
    assert least < memory * best
    ws = device.Workspace(int(memory * best))
    _, lse = x.forward()
    dh, dw = x.gradient(lse)
    x.check_gradient(dh, dw, lse)
    assert bool(torch.all(dh[(x.T == x.ignore)] == 0.0))
    for dh_again, dw_again in (x.gradient(lse), (x.gradient(lse, want=("dh",))[0], x.gradient(lse, want=("dw",))[1])):
        assert torch.equal(dh, dh_again) and torch.equal(dw, dw_again)
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,k", [(20, 3000, 136), (700, 3001, 200), (1500, 9001, 1000), (2900, 4001, 72)])
def test_replays_of_a_graph_follow_the_tokens_that_count(tokens, vocab, k, workspace):
    """What a captured call does is decided on the card: other tokens count in every replay, from none to all."""
    x = Problem(tokens, vocab, k, "bf16", 25)
    all_targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(26))
    dloss = x.dloss.cuda()
    loss, lse = x.forward()
    dh, dw = x.gradient(lse)
    out = [torch.empty_like(t) for t in (loss, lse, dh, dw)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        lib.ozaki_linear_loss(*x.arguments(), out[0], out[1])
        lib.ozaki_linear_loss_grad(*x.arguments(), out[1], dloss, out[2], k, out[3], k)
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    for i, share in enumerate((0.6, 0.0, 0.97, 1.1, 0.3)):
        gen = torch.Generator(device="cuda").manual_seed(i)
        x.T.copy_(torch.where(torch.rand((tokens,), device="cuda", generator=gen) < share, x.ignore, all_targets))
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        loss, lse = x.forward()
        dh, dw = x.gradient(lse)
        for got, want in zip(out, (loss, lse, dh, dw)):
            assert torch.equal(got, want)
        assert bool(torch.all(dh[x.T == x.ignore] == 0.0)) and (share < 1.0 or bool(torch.all(dw == 0.0)))
    x.targets = x.T.cpu()
    x.check_gradient(dh, dw, lse)
