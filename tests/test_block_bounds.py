"""The block's operators write what is theirs and nothing else: rows and columns around the results and the memory behind the work memory stay as they were, and
what the work memory held does not matter."""
import random

import pytest

torch = pytest.importorskip("torch")

from low_precision import DTYPES  # noqa: E402
from paper_2508_00441_amd import binding as lib  # noqa: E402

GUARD = 4096


class Memory:
    """Work memory of exactly the size that a call asks for, with bytes behind it that stay."""

    def __init__(self, need, fill):
        self.buf = torch.full((need + GUARD,), fill, dtype=torch.uint8, device="cuda")
        self.buf[need:] = 0x5A
        self.need = need
        lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        lib.ozaki_set_workspace(self.buf if need else None, need)

    def done(self):
        lib.ozaki_set_workspace(None, 0)
        assert bool(torch.all(self.buf[self.need:] == 0x5A))


class Result:
    """rows x columns in the middle of a larger matrix of NaN."""

    def __init__(self, rows, columns, dtype, gen):
        self.rows, self.columns, self.before, self.after = rows, columns, gen.choice([0, 1, 8]), gen.choice([0, 3, 8])
        self.whole = torch.full((rows + 4, self.before + columns + self.after), float("nan"), dtype=dtype, device="cuda")
        self.ld = self.whole.shape[1]
        self.at = self.whole.data_ptr() + (2 * self.ld + self.before) * self.whole.element_size()

    def value(self):
        inside = self.whole[2: 2 + self.rows, self.before: self.before + self.columns]
        mask = torch.ones(self.whole.shape, dtype=torch.bool, device="cuda")
        mask[2: 2 + self.rows, self.before: self.before + self.columns] = False
        assert bool(torch.isnan(self.whole[mask]).all())
        assert not bool(torch.isnan(inside).any())
        return inside.clone()


def _padded(x):
    to = 16 // x.element_size()
    out = torch.full((x.shape[0], -(-x.shape[1] // to) * to), float("nan"), dtype=x.dtype, device="cuda")
    out[:, : x.shape[1]] = x
    return out


def _same(first, second):
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def _sizes(rng, most_m, most_n, most_k):
    size = lambda most: max(1, int(most ** rng.random()))  # noqa: E731
    return size(most_m), size(most_n), size(most_k)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(24))
def test_linear(seed):
    rng = random.Random(seed)
    m, n, k = _sizes(rng, 2600, 4200, 1500) if seed % 3 else _sizes(rng, 90, 3000, 9000)
    type, act, pair = rng.choice(["bf16", "f16"]), rng.randrange(5), seed % 2
    dtype, t = DTYPES[type], lib.TYPES[type]
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + sum(shape))).to(dtype)  # noqa: E731
    X, W = _padded(rand(m, k)), [_padded(rand(n, k) / 16) for _ in range(2)]
    Z, dY, bias, R = [_padded(rand(m, n)), _padded(rand(m, n))], _padded(rand(m, n)), rand(1, n)[0].clone(), rand(m, n)
    ldx, ldw, ldz = X.shape[1], W[0].shape[1], dY.shape[1]
    results = []
    for fill in (0, 0xFF):
        pick = random.Random(seed)
        out = [Result(m, n, dtype, pick) for _ in range(3)]
        out += [Result(m, k, dtype, pick), Result(n, k, dtype, pick)]
        db = torch.full((n + 8,), float("nan"), device="cuda")
        if pair:
            second = Result(n, k, dtype, _Same(out[4]))          # (both at one distance)
            memory = Memory(lib.ozaki_gated_linear_workspace_bytes(m, n, k, False), fill)
            lib.ozaki_gated_linear(m, n, k, X, ldx, W[0], W[1], ldw, t, act, out[0].at, out[0].ld, out[1].at, out[1].ld, out[2].at, out[2].ld)
            memory.done()
            memory = Memory(lib.ozaki_gated_linear_workspace_bytes(m, n, k, True), fill)
            lib.ozaki_gated_linear_grad(m, n, k, X, ldx, W[0], W[1], ldw, t, act, Z[0], ldz, Z[1], ldz, dY, ldz, out[3].at, out[3].ld, out[4].at, second.at, out[4].ld)
            memory.done()
            results.append([o.value() for o in out + [second]])
        else:
            memory = Memory(lib.ozaki_linear_workspace_bytes(m, n, k, False), fill)
            lib.ozaki_linear(m, n, k, X, ldx, W[0], ldw, t, bias, act, R, n, out[0].at, out[0].ld, out[1].at, out[1].ld)
            memory.done()
            memory = Memory(lib.ozaki_linear_workspace_bytes(m, n, k, True), fill)
            lib.ozaki_linear_grad(m, n, k, X, ldx, W[0], ldw, t, act, Z[0], ldz, dY, ldz, out[3].at, out[3].ld, out[4].at, out[4].ld, db.data_ptr() + 16)
            memory.done()
            assert bool(torch.isnan(db[:4]).all()) and bool(torch.isnan(db[4 + n:]).all()) and not bool(torch.isnan(db[4: 4 + n]).any())
            results.append([o.value() for o in out[:2] + out[3:]] + [db[4: 4 + n].clone()])
    _same(*results)


class _Same:
    """The margins of another result, in turn."""

    def __init__(self, other):
        self.margins = [other.before, other.after]

    def choice(self, _):
        return self.margins.pop(0)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(24))
def test_block_norm(seed):
    rng = random.Random(100 + seed)
    rows, k, _ = _sizes(rng, 3000, 16384 if seed % 4 == 0 else 5000, 2)
    type, type_r = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
    post, group = rng.random() < 0.6, rng.choice([0, 1, rows, max(1, rows // 3)])
    t, tr = DTYPES[type], DTYPES[type_r]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=gen)  # noqa: E731
    X, R, dH, dR_out = _padded(rand(rows, k).to(t)), _padded(rand(rows, k).to(tr)), _padded(rand(rows, k).to(t)), _padded(rand(rows, k).to(tr))
    w_post, w_pre, gate = rand(k) if post else None, rand(k), rand(-(-rows // group), k) if group else None
    common = (rows, k, X, X.shape[1], lib.TYPES[type], w_post, gate, group, 0.5, 1e-6)
    results = []
    for fill in (0, 0xFF):
        pick = random.Random(seed)
        R_new, H, dX, dR = (Result(rows, k, d, pick) for d in (tr, t, t, tr))
        dw_post, dw_pre = (torch.full((k + 2,), float("nan"), device="cuda") for _ in range(2))
        dgate = torch.full((-(-rows // group) * k + 2,), float("nan"), device="cuda") if group else None
        memory = Memory(0, fill)
        lib.ozaki_block_norm(*common, R, R.shape[1], lib.TYPES[type_r], R_new.at, R_new.ld, w_pre, H.at, H.ld)
        memory.done()
        memory = Memory(lib.ozaki_block_norm_workspace_bytes(rows, k, group), fill)
        lib.ozaki_block_norm_grad(*common, R, R.shape[1], lib.TYPES[type_r], w_pre, dH, dH.shape[1], dR_out, dR_out.shape[1], dX.at, dX.ld, dR.at, dR.ld,
                                  dw_post.data_ptr() + 4 if post else None, dgate.data_ptr() + 4 if group else None, dw_pre.data_ptr() + 4)
        memory.done()
        sums = [v for v in (dw_post if post else None, dgate, dw_pre) if v is not None]
        for v in sums:
            assert bool(torch.isnan(v[[0, -1]]).all()) and not bool(torch.isnan(v[1:-1]).any())
        results.append([R_new.value(), H.value(), dX.value(), dR.value()] + [v[1:-1].clone() for v in sums])
    _same(*results)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(8))
def test_clipping(seed):
    rng = random.Random(200 + seed)
    count = rng.choice([1, 3, 144, 145, 300])
    sizes = [rng.choice([0, 1, 7, 2048, 2049, 5000, 8192, 8193, 70001]) for _ in range(count)]
    names = [rng.choice(list(DTYPES)) for _ in sizes]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = [torch.randn((n + 1,), device="cuda", generator=gen).to(DTYPES[name])[rng.choice([0, 1]):][:n] for n, name in zip(sizes, names)]
    results = []
    for fill in (0, 0xFF):
        out = [torch.full((n + 4,), float("nan"), dtype=DTYPES[name], device="cuda") for n, name in zip(sizes, names)]
        norm = torch.full((3,), float("nan"), device="cuda")
        memory = Memory(lib.ozaki_gradient_norm_workspace_bytes(count), fill)
        lib.ozaki_clip_gradients(count, x, sizes, [lib.TYPES[name] for name in names], 1.0, 0.7, [o.data_ptr() + 2 * o.element_size() for o in out], norm.data_ptr() + 4)
        memory.done()
        for o, n in zip(out, sizes):
            assert bool(torch.isnan(o[:2]).all()) and bool(torch.isnan(o[2 + n:]).all()) and not bool(torch.isnan(o[2: 2 + n]).any())
        assert bool(torch.isnan(norm[[0, 2]]).all())
        results.append([o[2: 2 + n].clone() for o, n in zip(out, sizes)] + [norm[1:2].clone()])
    _same(*results)


@pytest.mark.gpu
def test_two_contexts_at_once():
    """Calls of two contexts with streams and work memory of their own, taking turns: each has the results that it has alone."""
    m, n, k = 200, 700, 4160
    gen = torch.Generator(device="cuda").manual_seed(5)
    sides = []
    for _ in range(2):
        X, Wg, Wu = (torch.randn((r, k), device="cuda", generator=gen).bfloat16() for r in (m, n, n))
        G, U, dY = (torch.randn((m, 704), device="cuda", generator=gen).bfloat16() for _ in range(3))
        need = max(lib.ozaki_gated_linear_workspace_bytes(m, n, k, g) for g in (False, True))
        sides.append(dict(ws=torch.empty((need,), dtype=torch.uint8, device="cuda"), stream=torch.cuda.Stream(), context=lib.ozaki_context_create(), a=(X, Wg, Wu, G, U, dY)))

    def call(side):
        X, Wg, Wu, G, U, dY = side["a"]
        lib.ozaki_context_use(side["context"])
        lib.ozaki_set_stream(side["stream"].cuda_stream)
        lib.ozaki_set_workspace(side["ws"], side["ws"].numel())
        with torch.cuda.stream(side["stream"]):
            Y, dX, dW = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), torch.empty_like(X), torch.empty((2, n, k), dtype=torch.bfloat16, device="cuda")
        lib.ozaki_gated_linear(m, n, k, X, k, Wg, Wu, k, lib.TYPE_BF16, lib.ACTIVATION_SILU, Y, n)
        lib.ozaki_gated_linear_grad(m, n, k, X, k, Wg, Wu, k, lib.TYPE_BF16, lib.ACTIVATION_SILU, G, 704, U, 704, dY, 704, dX, k, dW[0], dW[1], k)
        return Y, dX, dW

    torch.cuda.synchronize()
    try:
        alone = []
        for side in sides:
            alone.append(call(side))
            torch.cuda.synchronize()
        together = [[call(side) for side in sides] for _ in range(5)]
        torch.cuda.synchronize()
        for turn in together:
            for got, want in zip(turn, alone):
                _same(got, want)
    finally:
        torch.cuda.synchronize()
        lib.ozaki_context_use(None)
        for side in sides:
            lib.ozaki_context_destroy(side["context"])
