"""ozaki_linear, ozaki_gated_linear and their gradients against their definitions in 64 bits, within bounds of their 32-bit sums and 16-bit roundings."""
import pytest

torch = pytest.importorskip("torch")

import block_operators as plain  # noqa: E402
from low_precision import DTYPES  # noqa: E402
from paper_2508_00441_amd import binding as lib, device  # noqa: E402

ACTIVATIONS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
# few vectors (whole, and the inner dimension in shares), tiles from narrow (the same) to large ones, large ones whose last round is left to smaller ones, along either
# dimension; odd sizes; steps that end inside 16 bytes
SHAPES = [(1, 1, 1), (1, 16, 64), (1, 257, 100), (3, 5, 8), (2, 40, 6200), (16, 100, 6401), (7, 1000, 257), (17, 33, 72), (33, 129, 640), (64, 500, 1000), (65, 1000, 33),
          (100, 300, 4096), (200, 1001, 200), (300, 511, 64), (1000, 4100, 100), (1030, 4104, 264), (2100, 4200, 72), (2310, 4097, 129), (2304, 4352, 256),
          (3000, 2800, 72), (4616, 4090, 40), (2100, 8461, 40), (9, 300, 16400), (700, 1300, 100), (700, 700, 333), (2000, 3201, 136), (1000, 3204, 72), (70, 70000, 40), (500, 2600, 72), (4104, 4096, 40)]
GRAD_SHAPES = [(1, 1, 1), (1, 257, 100), (3, 5, 8), (16, 1000, 136), (17, 33, 72), (40, 3000, 64), (65, 1000, 33), (200, 1001, 200), (300, 511, 64), (513, 264, 1031), (1000, 72, 72),
               (5000, 100, 130), (1030, 2100, 264), (2100, 1100, 4200), (2100, 4200, 300), (4100, 300, 280), (8, 3000, 300), (1030, 8000, 1030), (10000, 600, 1100)]


class Problem:
    def __init__(self, m, n, k, type, act, seed=None, pair=False, bias=True, residual=True):
        gen = torch.Generator(device="cuda").manual_seed(seed or m + n + k)
        rand = lambda *shape: torch.randn(shape, device="cuda", generator=gen)    # noqa: E731
        self.m, self.n, self.k, self.type, self.act, self.dtype = m, n, k, type, act, DTYPES[type]
        self.x = rand(m, k).to(self.dtype)
        self.w = [(2 * rand(n, k) / k ** 0.5).to(self.dtype) for _ in range(2 if pair else 1)]
        self.bias = rand(n).to(self.dtype) if bias and not pair else None
        self.r = rand(m, n).to(self.dtype) if residual and not pair else None
        self.dy = rand(m, n).to(self.dtype)
        self.z = [(2 * rand(m, n)).to(self.dtype) for _ in self.w]
        self.X, self.W = plain.padded(self.x, type), [plain.padded(w, type) for w in self.w]
        self.Z, self.dY = [plain.padded(z, type) for z in self.z], plain.padded(self.dy, type)
        if pair:                                                    # (both at one distance)
            assert self.W[0].shape == self.W[1].shape

    def result(self, rows, columns, more=0):
        return torch.full((rows, columns + more), float("nan"), dtype=self.dtype, device="cuda")

    def forward(self, keep=True, more=0):
        m, n, k, a, t = self.m, self.n, self.k, lib.ACTIVATIONS[self.act], lib.TYPES[self.type]
        Y, Z = self.result(m, n, more), [self.result(m, n, more) if keep else None for _ in self.w]
        ldz = n + more if keep else 0
        if len(self.w) == 2:
            lib.ozaki_gated_linear(m, n, k, self.X, self.X.shape[1], self.W[0], self.W[1], self.W[0].shape[1], t, a, Y, n + more, Z[0], ldz, Z[1], ldz)
        else:
            lib.ozaki_linear(m, n, k, self.X, self.X.shape[1], self.W[0], self.W[0].shape[1], t, self.bias, a, self.r, n, Y, n + more, Z[0], ldz)
        return Y, Z

    def check_forward(self, Y, Z):
        n, wide = self.n, [v.double() for v in [self.x] + self.w]
        if len(self.w) == 2:
            g, dg, u, du, y, dy = plain.gated(*wide, self.act)
            kept = [(g, dg), (u, du)]
        else:
            z, dz, y, dy = plain.linear(*wide, None if self.bias is None else self.bias.double(), self.act, None if self.r is None else self.r.double())
            kept = [(z, dz)]
        assert plain.within(Y[:, :n], y, dy, self.type)
        for got, (want, off) in zip(Z, kept):
            assert got is None or plain.within(got[:, :n], want, off, self.type)
        for got in [Y] + [z for z in Z if z is not None]:
            assert bool(torch.isnan(got[:, n:]).all())

    def gradient(self, want="xwub", more=0):
        m, n, k, a, t = self.m, self.n, self.k, lib.ACTIVATIONS[self.act], lib.TYPES[self.type]
        dX = self.result(m, k, more) if "x" in want else None
        dW = [self.result(n, k, more) if c in want else None for c in ("wu" if len(self.w) == 2 else "w")]
        Z, ldz = self.Z, self.Z[0].shape[1]
        if len(self.w) == 2:
            lib.ozaki_gated_linear_grad(m, n, k, self.X, self.X.shape[1], self.W[0], self.W[1], self.W[0].shape[1], t, a, Z[0], ldz, Z[1], ldz, self.dY, self.dY.shape[1],
                                        dX, k + more, dW[0], dW[1], k + more)
            return dX, dW, None
        dbias = torch.full((n,), float("nan"), device="cuda") if "b" in want else None
        lib.ozaki_linear_grad(m, n, k, self.X, self.X.shape[1], self.W[0], self.W[0].shape[1], t, a, Z[0] if self.act != "none" else None, ldz, self.dY, self.dY.shape[1],
                              dX, k + more, dW[0], k + more, dbias)
        return dX, dW, dbias

    def check_gradient(self, dX, dW, dbias):
        k, x, w, dy, z = self.k, self.x.double(), [v.double() for v in self.w], self.dy.double(), [v.double() for v in self.z]
        if len(self.w) == 2:
            want = plain.gated_grad(x, *w, self.act, *z, dy, self.type)
        else:
            *want, (db, ob) = plain.linear_grad(x, w[0], self.act, z[0], dy, self.type)
            assert dbias is None or plain.within(dbias, db, ob, "f32")
        for got, (value, off) in zip([dX] + dW, want):
            if got is not None:
                assert plain.within(got[:, :k], value, off, self.type)
                assert bool(torch.isnan(got[:, k:]).all())


def _need(x, grad):
    ask = lib.ozaki_gated_linear_workspace_bytes if len(x.w) == 2 else lib.ozaki_linear_workspace_bytes
    return device.Workspace(ask(x.m, x.n, x.k, grad))


@pytest.mark.gpu
@pytest.mark.parametrize("pair", [False, True])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_forward(m, n, k, type, pair):
    act = ACTIVATIONS[(m + n + k) % 5]
    x = Problem(m, n, k, type, act, pair=pair)
    ws = _need(x, False)
    x.check_forward(*x.forward())
    x.check_forward(*x.forward(keep=False, more=3))
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("pair", [False, True])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", GRAD_SHAPES)
def test_gradient(m, n, k, type, pair):
    act = ACTIVATIONS[(m + n + k + pair) % 5]
    x = Problem(m, n, k, type, act, pair=pair)
    ws = _need(x, True)
    x.check_gradient(*x.gradient())
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("pair", [False, True])
@pytest.mark.parametrize("act", ACTIVATIONS)
@pytest.mark.parametrize("m,n,k", [(5, 130, 72), (130, 264, 96)])
def test_every_activation(m, n, k, act, pair):
    for type in ("bf16", "f16"):
        x = Problem(m, n, k, type, act, pair=pair, bias=type == "f16", residual=type == "bf16")
        ws = _need(x, True)
        x.check_forward(*x.forward(more=5))
        x.check_gradient(*x.gradient(more=1))
        ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("pair", [False, True])
def test_results_that_are_not_asked_for(pair):
    x = Problem(100, 136, 200, "bf16", "silu", pair=pair)
    ws = _need(x, True)
    for want in ("x", "w", "xw") + (("u", "xu") if pair else ("b", "xb")):
        x.check_gradient(*x.gradient(want))
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_gradient_against_differences(act):
    """d(sum of c * y) along a direction of each input: the gradient's share against the difference of the forward calls, in FP16 that keeps y's roundings small.
    A central difference over t of a function whose third derivative along the direction is at most 3 is off by t^2 / 2 of the direction's cube, summed with |c|."""
    m, n, k, t = 24, 40, 48, 2.0 ** -4
    x = Problem(m, n, k, "f16", act, pair=True, seed=5)
    ws = _need(x, True)
    Y, Z = x.forward()
    x.Z = [plain.padded(z, "f16") for z in Z]
    dX, dW, _ = x.gradient()
    wide = [v.double() for v in [x.x] + x.w]
    gen = torch.Generator(device="cuda").manual_seed(9)
    for i, grad in enumerate([dX] + dW):
        direction = (torch.randint(0, 3, grad.shape, device="cuda", generator=gen) - 1).double() / 8
        ends = []
        for sign in (1, -1):
            at = list(wide)
            at[i] = at[i] + sign * t * direction
            ends.append(plain.gated(*at, act)[4])
        want = float((x.dy.double() * (ends[0] - ends[1])).sum()) / (2 * t)
        got = float((grad.double() * direction).sum())
        along = (direction @ wide[1].t().contiguous()).abs() + (direction @ wide[2].t().contiguous()).abs() if i == 0 else wide[0] @ direction.t().contiguous()
        u = plain.gated(*wide, act)
        curve = (x.dy.double().abs() * (1 + u[2].abs()) * (1 + along.abs()) ** 3 * 3 * t * t / 2).sum()
        roundings = 2.0 ** -9 * (x.dy.double().abs() * (1 + u[2].abs()) * (1 + along.abs())).sum()
        assert abs(got - want) <= float(curve + roundings)
    ws.close()


def _slope(value, leaves, i, direction):
    """The derivative of value(leaves) along a direction of leaf i by central differences over t and t / 2, and what it may be off: the second one's error is a quarter of the first
    one's, of which their difference is three quarters."""
    out = []
    for t in (2.0 ** -8, 2.0 ** -9):
        ends = [value([v + sign * t * direction if j == i else v for j, v in enumerate(leaves)]) for sign in (1, -1)]
        out.append(float((ends[0] - ends[1]) / (2 * t)))
    return out[1], 2 * abs(out[0] - out[1])


def _directions(grad, gen):
    """Along the gradient's signs the derivative is as large as it can be: everywhere, and on halves of the elements."""
    sign = torch.where(grad >= 0, 0.125, -0.125).double()
    return [sign] + [sign * torch.randint(0, 2, grad.shape, device="cuda", generator=gen) for _ in range(3)]


HALF = 2.0 ** -11                                                   # what rounding to FP16 may change, relative


def _check_slopes(value, leaves, grads, changes):
    """changes[i](direction): for every number that is rounded on its way to gradient i, what a relative change of it comes to in that gradient's slope.  Roundings are at most HALF each
    and independent of one another, with a spread of 0.58 of that: four times the root of the sum of squares is seven times the spread."""
    gen = torch.Generator(device="cuda").manual_seed(21)
    for i, grad in enumerate(grads):
        for direction in _directions(grad, gen):
            want, off = _slope(value, leaves, i, direction)
            along = grad.double() * direction
            terms = ([along] if grad.dtype != torch.float32 else []) + changes[i](direction)
            tolerance = off + 4 * HALF * float(sum(v.square().sum() for v in terms)) ** 0.5 + 2.0 ** -18 * float(along.abs().sum())
            assert tolerance < 0.02 * abs(want), (i, tolerance, want)          # (so that a gradient which is missing, another one's or of the other sign does not pass)
            assert abs(float(along.sum()) - want) <= tolerance, i


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("m,n,k", [(24, 40, 48), (130, 264, 96)])
def test_slopes_of_a_pair(m, n, k, act):
    """The gradient against differences of sum(dy * act(x wg^T) * (x wu^T)) in 64 bits.  g and u are held in FP16, then dg and du are; g's change is act'(g) g of du and act''(g) g, of
    magnitude 1 at most, times dy u of dg."""
    x = Problem(m, n, k, "f16", act, pair=True, seed=5)
    ws = _need(x, True)
    Y, Z = x.forward()
    x.Z = [plain.padded(z, "f16") for z in Z]
    dX, dW, _ = x.gradient()
    ws.close()
    across = lambda v, w: v @ w.t().contiguous()    # noqa: E731
    xs, wg, wu = leaves = [v.double() for v in [x.x] + x.w]
    dy, g, u = x.dy.double(), across(xs, wg), across(xs, wu)
    a, slope, _, _ = plain.activation(g, act)
    dg, du, g_of_dg, g_of_du = dy * u * slope, dy * a, (dy * u).abs(), (dy * slope * g).abs()
    changes = [lambda d: [g_of_dg * across(d, wg).abs() + g_of_du * across(d, wu).abs(), dg * across(d, wg), dg * across(d, wg), du * across(d, wu)],
               lambda d: [v * across(xs, d) for v in (g_of_dg, dg, dg)],
               lambda d: [v * across(xs, d) for v in (g_of_du, du)]]
    _check_slopes(lambda at: (dy * plain.gated(*at, act)[4]).sum(), leaves, [dX] + dW, changes)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("m,n,k", [(24, 40, 48), (130, 264, 96)])
def test_slopes_of_a_layer(m, n, k, act):
    """The same of sum(dy * (act(x w^T + bias) + r)): z is held in FP16, dz is for the two products."""
    x = Problem(m, n, k, "f16", act, seed=6)
    ws = _need(x, True)
    Y, Z = x.forward()
    x.Z = [plain.padded(z, "f16") for z in Z]
    dX, (dW,), dbias = x.gradient()
    ws.close()
    across = lambda v, w: v @ w.t().contiguous()    # noqa: E731
    xs, w, bias = leaves = [x.x.double(), x.w[0].double(), x.bias.double()]
    dy = x.dy.double()
    dz = dy * plain.activation(across(xs, w) + bias, act)[1]
    changes = [lambda d: [v * across(d, w) for v in (dy, dz)], lambda d: [v * across(xs, d) for v in (dy, dz)], lambda d: [dy * d]]
    _check_slopes(lambda at: (dy * plain.linear(*at, act, x.r.double())[2]).sum(), leaves, [dX, dW, dbias], changes)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(5, 264), (70, 264), (70, 261), (1100, 4200)])
def test_residual_in_place(m, n):
    x = Problem(m, n, 96, "bf16", "gelu_tanh")
    ws = _need(x, False)
    Y = x.r.clone()
    lib.ozaki_linear(m, n, x.k, x.X, x.X.shape[1], x.W[0], x.W[0].shape[1], lib.TYPE_BF16, x.bias, lib.ACTIVATION_GELU_TANH, Y, n, Y, n)
    x.check_forward(Y, [None])
    ws.close()


@pytest.mark.gpu
def test_both_weights_in_one_matrix():
    x = Problem(70, 96, 128, "bf16", "silu", pair=True)
    ws = _need(x, False)
    x.W = [torch.cat(x.W)[:96], None]
    x.W[1] = x.W[0].data_ptr() + 96 * 128 * 2
    x.check_forward(*x.forward())
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("pair", [False, True])
def test_large_and_infinite_arguments(pair):
    """Products that are far from zero either way, beyond a 16-bit float's range and not finite: what the formula gives in 32 bits, rounded."""
    m, n, k = 3, 64, 8
    values = torch.tensor([0.0, -0.0, 1e-4, -1e-4, 3.0, -3.0, 11.0, -11.0, 60.0, -60.0, 88.0, -88.0, 110.0, -110.0, 1e4, -1e4, 6e4, -6e4, 1e30, -1e30], dtype=torch.float32)
    for act in ACTIVATIONS:
        x = Problem(m, n, k, "bf16", act, pair=pair, bias=False, residual=False)
        x.x.zero_()
        x.x[:, 0] = 1.0
        for w in x.w:
            w.zero_()
            w[: len(values), 0] = values.cuda()
            w[len(values):, 0] = 1.0
        x.X, x.W = plain.padded(x.x, "bf16"), [plain.padded(w, "bf16") for w in x.w]
        z = x.w[0][:, 0].double().repeat(m, 1)
        x.z = [z.bfloat16() for _ in x.w]
        x.Z = [plain.padded(v, "bf16") for v in x.z]
        ws = _need(x, True)
        if pair:                                                    # (act(g) * u of 1e30 twice is beyond the range)
            x.w[1].clamp_(-1e8, 1e8)
            x.W[1] = plain.padded(x.w[1], "bf16")
        x.check_forward(*x.forward())
        x.w[0].clamp_(-10, 10)                                      # (of the gradient: z is what it is, the products stay in range)
        x.W[0] = plain.padded(x.w[0], "bf16")
        if not pair:
            x.check_gradient(*x.gradient())
        ws.close()
    x = Problem(2, 8, 8, "bf16", "relu", bias=False, residual=False)
    ws = _need(x, False)
    x.X[0, 0] = float("nan")
    x.X[1, 0] = float("inf")
    Y, (Z,) = x.forward()
    assert bool(torch.isnan(Y[0]).all()) and bool(torch.isnan(Z[0]).all())
    z = x.X[1, :8].float() @ x.W[0][:, :8].float().t()
    assert bool(torch.all(Y[1].float() == z.clamp(min=0.0)))
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("m", [3, 40])
@pytest.mark.parametrize("act", ACTIVATIONS)
def test_large_and_infinite_arguments_of_a_pairs_gradient(act, m):
    """What the pair's gradient is formed with far from zero; and numbers that are none or infinite stay in their rows of dX and their columns' rows of dWg and dWu."""
    values = [0.0, -0.0, 1e-4, -1e-4, 3.0, -3.0, 11.0, -11.0, 60.0, -60.0, 88.0, -88.0, 110.0, -110.0, 1e4, -1e4, 6e4, -6e4, 1e30, -1e30]
    n, k = 64, 16
    x = Problem(m, n, k, "bf16", act, pair=True)
    x.z[0][0, : len(values)] = torch.tensor(values, device="cuda").bfloat16()
    x.z[1][0, : len(values)] = 1.0
    x.z[1][1, : len(values)] = torch.tensor(values, device="cuda").bfloat16()
    x.Z = [plain.padded(z, "bf16") for z in x.z]
    ws = _need(x, True)
    finite = x.gradient()
    x.check_gradient(*finite)
    x.Z[0][2, 7], x.Z[1][2, 9] = float("nan"), float("inf")
    got = x.gradient()
    ws.close()
    assert bool(torch.isnan(got[0][2]).all())
    rows, columns = torch.arange(m, device="cuda") != 2, torch.arange(n, device="cuda")
    assert torch.equal(got[0][rows], finite[0][rows])
    # (without an activation dg does not look at g)
    for after, before, kept in zip(got[1], finite[1], (columns != 9 if act == "none" else (columns != 7) & (columns != 9), columns != 7)):
        assert torch.equal(after[kept], before[kept]) and not bool(torch.isfinite(after[~kept]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 40])
def test_numbers_below_fp16s_normal_ones(m):
    """2^-20 and 2^-24 have one significant bit in FP16 and are no normal numbers there; their sums are exact."""
    n, k = 24, 64
    X, W = torch.full((m, k), 2.0 ** -20, dtype=torch.float16, device="cuda"), torch.full((n, k), 0.5, dtype=torch.float16, device="cuda")
    Y, dX, dW = (torch.full(shape, float("nan"), dtype=torch.float16, device="cuda") for shape in ((m, n), (m, k), (n, k)))
    ws = device.Workspace(max(lib.ozaki_linear_workspace_bytes(m, n, k, grad) for grad in (False, True)))
    lib.ozaki_linear(m, n, k, X, k, W, k, lib.TYPE_F16, None, 0, None, 0, Y, n)
    assert bool(torch.all(Y == 2.0 ** -15))
    Z, dY = torch.ones((m, n), dtype=torch.float16, device="cuda"), torch.full((m, n), 2.0 ** -24, dtype=torch.float16, device="cuda")
    lib.ozaki_linear_grad(m, n, k, X, k, W, k, lib.TYPE_F16, lib.ACTIVATION_RELU, Z, n, dY, n, dX, k, dW, k)
    assert bool(torch.all(dX == 12 * 2.0 ** -24)) and bool(torch.all(dW == 0))
    X.fill_(1.0)
    lib.ozaki_linear_grad(m, n, k, X, k, W, k, lib.TYPE_F16, lib.ACTIVATION_RELU, Z, n, dY, n, dX, k, dW, k)
    assert bool(torch.all(dW == m * 2.0 ** -24))
    ws.close()


@pytest.mark.gpu
def test_no_tokens():
    x = Problem(1, 24, 40, "bf16", "silu")
    dW, dbias = x.result(24, 40, 2), torch.full((24,), 7.0, device="cuda")
    lib.ozaki_set_workspace(None, 0)
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    lib.ozaki_linear(0, 24, 40, None, 0, None, 0, lib.TYPE_BF16, None, 0, None, 0, None, 0)
    lib.ozaki_gated_linear(0, 24, 40, None, 0, None, None, 0, lib.TYPE_BF16, 0, None, 0)
    lib.ozaki_linear_grad(0, 24, 40, None, 0, None, 0, lib.TYPE_BF16, 4, None, 0, None, 0, None, 0, dW, 42, dbias)
    assert bool(torch.all(dW[:, :40] == 0)) and bool(torch.isnan(dW[:, 40:]).all()) and bool(torch.all(dbias == 0))
    dW.fill_(float("nan"))
    lib.ozaki_gated_linear_grad(0, 24, 40, None, 0, None, None, 0, lib.TYPE_BF16, 4, None, 0, None, 0, None, 0, None, 0, None, dW, 42)
    assert bool(torch.all(dW[:, :40] == 0)) and bool(torch.isnan(dW[:, 40:]).all())


def test_no_tokens_and_nothing_but_their_gradient():
    """A frozen layer's gradient asks for dX alone, which of no tokens lies at a null address."""
    assert lib.ozaki_linear_grad(0, 24, 40, None, 0, FAKE, 40, lib.TYPE_BF16, 4, None, 0, None, 0, None, 40, None, 0, None, check=False) == 0
    assert lib.ozaki_gated_linear_grad(0, 24, 40, None, 0, FAKE, FAKE, 40, lib.TYPE_BF16, 4, None, 0, None, 0, None, 0, None, 40, None, None, 0, check=False) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(40, 200, 4096), (600, 1031, 328)])
def test_same_bits_every_time_on_another_stream_and_in_a_graph(m, n, k):
    x = Problem(m, n, k, "bf16", "silu", pair=True)
    need = max(lib.ozaki_gated_linear_workspace_bytes(m, n, k, grad) for grad in (False, True))
    ws = device.Workspace(need)
    first = [*x.forward(), *x.gradient()]
    flat = lambda out: [t for o in out if o is not None for t in (o if isinstance(o, list) else [o])]    # noqa: E731
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    context = lib.ozaki_context_create()
    lib.ozaki_context_use(context)
    try:
        with torch.cuda.stream(stream):
            other = device.Workspace(need)
            again = [*x.forward(), *x.gradient()]
        torch.cuda.synchronize()
        for a, b in zip(flat(first), flat(again)):
            assert torch.equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
            held = [*x.forward(), *x.gradient()]
        for step in range(3):
            x.X.copy_(plain.padded((x.x * (1 + step)).to(x.dtype), "bf16"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            lib.ozaki_set_stream(stream.cuda_stream)
            with torch.cuda.stream(stream):
                want = [*x.forward(), *x.gradient()]
            torch.cuda.synchronize()
            for a, b in zip(flat(held), flat(want)):
                assert torch.equal(a, b)
    finally:
        lib.ozaki_context_use(None)
        lib.ozaki_context_destroy(context)
    del other
    ws.close()


@pytest.mark.gpu
def test_too_little_work_memory():
    x = Problem(64, 64, 8192, "bf16", "silu")
    ws = device.Workspace(lib.ozaki_linear_workspace_bytes(64, 64, 8192, False) - 1)
    with pytest.raises(lib.OzakiError) as e:
        x.forward()
    assert e.value.status == lib.STATUS_WORKSPACE
    ws.close()


FAKE = 1 << 20                                                      # (an address that nothing looks at)


def _refused(call, good, changes):
    assert all(at <= len(good) for at, _ in changes)
    for at, value in changes:
        args = list(good)
        args[at - 1] = value
        assert call(*args, check=False) == -at, (call.__name__, at, value)


def test_refusals():
    big, odd = lib.MAX_EXTENT, FAKE + 2
    good = [4, 5, 6, FAKE, 8, FAKE, 8, lib.TYPE_BF16, FAKE, 4, FAKE, 5, FAKE, 5, FAKE, 5]
    _refused(lib.ozaki_linear, good, [(1, -1), (1, big + 1), (2, 0), (2, big + 1), (3, 0), (3, big), (4, None), (4, odd), (5, 5), (5, 9), (5, big), (6, None), (6, odd), (7, 4), (7, 12),
                                      (8, lib.TYPE_F32), (8, 3), (9, FAKE + 1), (10, 5), (10, -1), (11, FAKE + 1), (12, 4), (13, None), (13, FAKE + 1), (14, 4), (15, FAKE + 1), (16, 4)])
    assert lib.ozaki_linear(*([1 << 20, 1 << 20] + good[2:]), check=False) == -2
    good = [4, 5, 6, FAKE, 8, FAKE, FAKE, 8, lib.TYPE_F16, 4, FAKE, 5, FAKE, 5, FAKE, 5]
    _refused(lib.ozaki_gated_linear, good, [(1, -1), (2, 0), (3, 0), (4, None), (4, odd), (5, 5), (6, None), (6, odd), (7, None), (7, odd), (8, 4), (9, lib.TYPE_F32), (10, 5), (11, None),
                                            (11, FAKE + 1), (12, 4), (13, FAKE + 1), (14, 4), (15, None), (15, FAKE + 1), (16, 4)])
    good = [4, 5, 6, FAKE, 8, FAKE, 8, lib.TYPE_BF16, 4, FAKE, 8, FAKE, 8, FAKE, 6, FAKE, 6, FAKE]
    _refused(lib.ozaki_linear_grad, good, [(1, -1), (2, 0), (2, big), (3, 0), (4, None), (5, 9), (6, None), (7, 9), (8, 0), (9, 5), (10, None), (10, odd), (11, 4), (12, None), (12, odd), (13, 9),
                                           (14, FAKE + 1), (15, 5), (16, FAKE + 1), (17, 5), (18, FAKE + 2)])
    assert lib.ozaki_linear_grad(*(good[:13] + [None, 0, None, 0, None]), check=False) == -14
    good = [4, 5, 6, FAKE, 8, FAKE, FAKE, 8, lib.TYPE_BF16, 4, FAKE, 8, FAKE, 8, FAKE, 8, FAKE, 6, FAKE, FAKE, 6]
    _refused(lib.ozaki_gated_linear_grad, good, [(1, -1), (2, 0), (2, big), (3, 0), (4, None), (5, 9), (6, None), (7, None), (8, 9), (9, 0), (10, 5), (11, None), (12, 4), (13, None), (14, 9),
                                                 (15, None), (16, 4), (17, FAKE + 1), (18, 5), (19, FAKE + 1), (20, FAKE + 1), (21, 5)])
    assert lib.ozaki_gated_linear_grad(*(good[:16] + [None, 0, None, None, 0]), check=False) == -17
    lib.ozaki_set_workspace(None, 0)
    assert lib.ozaki_linear_grad(4, 5, 6, FAKE, 8, FAKE, 8, lib.TYPE_BF16, 0, None, 0, FAKE, 8, FAKE, 6, FAKE, 6, FAKE, check=False) == lib.STATUS_WORKSPACE
    assert lib.ozaki_linear_workspace_bytes(0, 4, 4, True) == lib.ozaki_linear_workspace_bytes(4, 4, 0, True) == lib.ozaki_linear_workspace_bytes(4, 0, 4, True) == 0
    assert lib.ozaki_linear_workspace_bytes(64, 64, 65536, False) > 0
    assert lib.ozaki_linear(64, 64, 65536, FAKE, 65536, FAKE, 65536, lib.TYPE_BF16, None, 0, None, 0, FAKE, 64, check=False) == lib.STATUS_WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("pair", [False, True])
def test_beyond_32_bits(pair):
    """Matrices of more than 2^32 bytes and 2^31 elements: the last rows and columns, of the results and of the sums over all tokens."""
    m, n, k = 40000, 60000, 64
    x = Problem(m, 8, k, "bf16", "silu", pair=pair, bias=False, residual=False)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x.n, x.w = n, [(torch.randn((n, k), device="cuda", generator=gen) / 8).bfloat16() for _ in x.w]
    x.W = x.w
    ws = _need(x, False)
    Y, Z = x.forward()
    ws.close()
    rows, columns = torch.tensor([0, 777, m - 300, m - 1], device="cuda"), torch.tensor([0, 1, n - 200, n - 1], device="cuda")
    part = Problem(4, 4, k, "bf16", "silu", pair=pair, bias=False, residual=False)
    part.x, part.w, part.n = x.x[rows], [w[columns] for w in x.w], 4
    part.check_forward(Y[rows][:, columns], [z[rows][:, columns] for z in Z])
    # the gradient, of a dY that is zero but in some rows and columns
    x.Z, x.dY = Z, Y.zero_()
    picked = torch.randn((4, 4), device="cuda", generator=gen).bfloat16()
    x.dY[rows.unsqueeze(1), columns] = picked
    ws = _need(x, True)
    dX, dW, _ = x.gradient("xwu")
    ws.close()
    part.z, part.dy = [z[rows][:, columns] for z in Z], picked
    part.check_gradient(dX[rows], [w[columns] for w in dW], None)
    others = torch.ones((m,), dtype=torch.bool, device="cuda")
    others[rows] = False
    assert bool(torch.all(dX[others] == 0)) and all(int((w != 0).any(1).sum()) == 4 for w in dW)
