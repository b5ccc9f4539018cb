"""ozaki_block_norm and ozaki_block_norm_grad against their definitions in 64 bits, within bounds of their 32-bit elements and sums over rows."""
import itertools

import pytest

torch = pytest.importorskip("torch")

import block_operators as plain  # noqa: E402
from low_precision import DTYPES  # noqa: E402
from paper_2508_00441_amd import binding as lib, device  # noqa: E402

TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]
# every number of threads and pieces a row takes, rows that end inside a piece, one row, fewer and more rows than there are workgroups
SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 512), (70, 513), (33, 1000), (9, 1024), (6, 2048), (11, 1025), (300, 2500), (7, 4096), (900, 4100), (3, 8192), (2, 8200), (5, 16384), (1500, 40), (4200, 100), (301, 9001)]
EPS = 1e-6


class Problem:
    def __init__(self, rows, k, types, post=True, group=None, scale=0.7, seed=None):
        gen = torch.Generator(device="cuda").manual_seed(seed or rows + k)
        rand = lambda *shape: torch.randn(shape, device="cuda", generator=gen)    # noqa: E731
        self.rows, self.k, (self.type, self.type_r), self.group, self.scale = rows, k, types, group, scale
        t, tr = DTYPES[self.type], DTYPES[self.type_r]
        self.x, self.r, self.dh, self.dr_out = rand(rows, k).to(t), (3 * rand(rows, k)).to(tr), rand(rows, k).to(t), rand(rows, k).to(tr)
        self.w_post, self.w_pre = 1 + 0.2 * rand(k) if post else None, 1 + 0.2 * rand(k)
        self.gate = rand(-(-rows // group), k) if group else None
        self.X, self.dH = (plain.padded(v, self.type) for v in (self.x, self.dh))
        self.R, self.dR_out = (plain.padded(v, self.type_r) for v in (self.r, self.dr_out))

    def common(self, x=True):
        return (self.rows, self.k, self.X if x else None, self.X.shape[1], lib.TYPES[self.type], self.w_post if x else None, self.gate if x else None, self.group or 0, self.scale, EPS)

    def result(self, type, more):
        return torch.full((self.rows, self.k + more), float("nan"), dtype=DTYPES[type], device="cuda")

    def forward(self, x=True, r=True, r_out=True, h=True, more=0):
        R_out, H = self.result(self.type_r, more) if r_out and x else None, self.result(self.type, more) if h else None
        lib.ozaki_block_norm(*self.common(x), self.R if r else None, self.R.shape[1], lib.TYPES[self.type_r], R_out, self.k + more, self.w_pre if h else None, H, self.k + more)
        wide = lambda v, there: v.double() if there and v is not None else None    # noqa: E731
        total, off, want, off_h = plain.block_norm(wide(self.x, x), wide(self.r, r), wide(self.w_post, x), wide(self.gate, x), self.group, self.scale, EPS, wide(self.w_pre, h))
        if R_out is not None:
            assert plain.within(R_out[:, : self.k], total, off, self.type_r) and bool(torch.isnan(R_out[:, self.k:]).all())
        if h:
            assert plain.within(H[:, : self.k], want, off_h, self.type) and bool(torch.isnan(H[:, self.k:]).all())
        return R_out, H

    def gradient(self, dh=True, dr_out=True, want=("dx", "dr", "dw_post", "dgate", "dw_pre"), x=True, more=0):
        out = {}
        for name in want:
            if name in ("dx", "dr"):
                out[name] = self.result(self.type if name == "dx" else self.type_r, more)
            elif (name == "dw_post" and self.w_post is not None) or (name == "dw_pre" and dh):
                out[name] = torch.full((self.k,), float("nan"), device="cuda")
            elif name == "dgate" and self.gate is not None:
                out[name] = torch.full_like(self.gate, float("nan"))
        get = out.get
        lib.ozaki_block_norm_grad(*self.common(x), self.R if dh else None, self.R.shape[1], lib.TYPES[self.type_r], self.w_pre if dh else None, self.dH if dh else None, self.dH.shape[1],
                                  self.dR_out if dr_out else None, self.dR_out.shape[1], get("dx"), self.k + more, get("dr"), self.k + more, get("dw_post"), get("dgate"), get("dw_pre"))
        return out

    def check_gradient(self, out, dh=True, dr_out=True):
        wide = lambda v: None if v is None else v.double()    # noqa: E731
        want = plain.block_norm_grad(wide(self.x), wide(self.r), wide(self.w_post), wide(self.gate), self.group, self.scale, EPS, wide(self.w_pre), wide(self.dh) if dh else None,
                                     wide(self.dr_out) if dr_out else None)
        for name, got in out.items():
            value, off = want[name]
            type = self.type if name == "dx" else self.type_r if name == "dr" else "f32"
            width = self.k
            assert plain.within(got[..., :width], value, off, type), name
            assert bool(torch.isnan(got[..., width:]).all()), name


@pytest.fixture()
def workspace():
    ws = device.Workspace(256 << 20)
    yield ws
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,k", SHAPES)
def test_forward(rows, k, types, workspace):
    Problem(rows, k, types, group=max(1, rows // 3)).forward()
    Problem(rows, k, types, post=False).forward(more=1)


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,k", SHAPES)
def test_gradient(rows, k, types):
    for post, group in ((True, max(1, rows // 3)), (False, None)):
        x = Problem(rows, k, types, post=post, group=group)
        ws = device.Workspace(lib.ozaki_block_norm_workspace_bytes(rows, k, group or 0))
        x.check_gradient(x.gradient(more=0 if post else 1))
        ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("group", [1, 2, 3, 7, 50, 299, 300, 1000])
@pytest.mark.parametrize("rows,k", [(300, 72), (2600, 520), (2600, 1100)])
def test_gates(rows, k, group, workspace):
    for post in (True, False):
        x = Problem(rows, k, ("bf16", "f32"), post=post, group=group)
        x.forward()
        x.check_gradient(x.gradient())
        x.check_gradient(x.gradient(want=("dw_post", "dx") if post else ("dgate",)))


# gates that end inside the chunk of a workgroup, beside one another and one after another, and that have one, some and many chunks
@pytest.mark.parametrize("rows,k,group", [(16400, 24, 1), (16400, 24, 5), (16384, 128, 16), (9000, 130, 15), (9000, 130, 17), (5000, 250, 2), (7003, 500, 4), (7003, 500, 7), (40, 100, 1),
                                          (2500, 513, 1), (1100, 2048, 3), (1100, 4100, 1), (600, 9000, 1), (1300, 9000, 4), (3000, 1000, 64), (5000, 90, 1700), (4097, 300, 4096)])
@pytest.mark.parametrize("types", [("bf16", "f32"), ("f32", "f32")])
@pytest.mark.gpu
def test_gates_of_few_and_many_rows(rows, k, group, types, workspace):
    p = Problem(rows, k, types, group=group)
    p.check_gradient(p.gradient())
    for want in (("dgate",), ("dw_post",), ("dx", "dgate"), ("dw_pre", "dw_post")):
        p.check_gradient(p.gradient(want=want))
    p = Problem(rows, k, types, post=False, group=group)
    p.check_gradient(p.gradient(want=("dx", "dgate")))


@pytest.mark.gpu
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("k", [40, 128, 200, 500, 520])
def test_rows_side_by_side_are_rows_of_their_own(k, types, workspace):
    """Each row's results have the bits of a call for it alone, also beside rows that are normed again with a scale, zeros, infinities and NaN."""
    rows = 41
    p = Problem(rows, k, types, group=4)
    for v in (p.X, p.R) if types[0] == "f32" else (p.R,):
        v[1], v[6], v[11], v[18] = v[1] * 1e25, v[6] * 1e-25, 0.0, float("nan")
        v[23, k // 2] = float("inf")
    if types[0] == "f32":
        p.dH[7] *= 1e30

    def call(i, n):
        x, r, dh, dr_out = (v[i : i + n] for v in (p.X, p.R, p.dH, p.dR_out))
        gate = p.gate[i // 4 : (i + n + 3) // 4]
        R_out, H, dR, dX = torch.empty_like(r), torch.empty_like(x), torch.empty_like(r), torch.empty_like(x)
        common = (n, k, x, x.shape[1], lib.TYPES[p.type], p.w_post, gate, 4, p.scale, EPS)
        lib.ozaki_block_norm(*common, r, r.shape[1], lib.TYPES[p.type_r], R_out, k, p.w_pre, H, k)
        lib.ozaki_block_norm_grad(*common, r, r.shape[1], lib.TYPES[p.type_r], p.w_pre, dh, dh.shape[1], dr_out, dr_out.shape[1], dX, k, dR, k, None, None, None)
        bits = torch.int32 if p.type == "f32" else torch.int16
        return [v.reshape(-1)[: n * k].reshape(n, k).view(bits) for v in (R_out, H, dR, dX)]

    together = call(0, rows)
    for i in range(rows):
        for all, one in zip(together, call(i, 1)):
            assert torch.equal(all[i : i + 1], one), i


@pytest.mark.gpu
@pytest.mark.parametrize("post", [True, False])
def test_parts(post, workspace):
    x = Problem(40, 600, ("f16", "f32"), post=post, group=40)
    for parts in itertools.product([True, False], repeat=4):
        given, r, r_out, h = parts
        if (given or r) and ((r_out and given) or h):
            x.forward(x=given, r=r, r_out=r_out, h=h)
    for dh, dr_out in ((True, False), (False, True), (True, True)):
        for want in (("dx",), ("dr",), ("dw_post", "dgate"), ("dw_pre", "dr"), ("dx", "dr", "dw_post", "dgate", "dw_pre")):
            want = [w for w in want if (w != "dw_pre" or dh) and (w != "dw_post" or post)]
            x.check_gradient(x.gradient(dh, dr_out, want), dh, dr_out)
    # a norm alone, without anything in front of it
    x.check_gradient(x.gradient(True, False, ("dr", "dw_pre"), x=False), True, False)


@pytest.mark.gpu
def test_gradient_without_work_memory():
    x = Problem(20, 300, ("bf16", "bf16"))
    lib.ozaki_set_workspace(None, 0)
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    x.check_gradient(x.gradient(want=("dx", "dr")))
    args = x.common() + (x.R, x.R.shape[1], lib.TYPE_BF16, x.w_pre, x.dH, x.dH.shape[1], None, 0, None, 0, None, 0, None, None, torch.zeros(300, device="cuda"))
    assert lib.ozaki_block_norm_grad(*args, check=False) == lib.STATUS_WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k", [(700, 264), (3, 4096), (900, 2056), (300, 16384)])
def test_in_place(rows, k, workspace):
    x = Problem(rows, k, ("bf16", "bf16"), group=rows)
    R_out, H = x.forward()
    out = x.gradient()
    R, X = x.R.clone(), x.X.clone()
    lib.ozaki_block_norm(rows, k, X, k, lib.TYPE_BF16, x.w_post, x.gate, rows, x.scale, EPS, R, k, lib.TYPE_BF16, R, k, x.w_pre, X, k)
    assert torch.equal(R, R_out) and torch.equal(X, H)
    dR, dH = x.dR_out.clone(), x.dH.clone()
    lib.ozaki_block_norm_grad(*x.common(), x.R, k, lib.TYPE_BF16, x.w_pre, dH, k, dR, k, dH, k, dR, k)
    assert torch.equal(dR, out["dr"]) and torch.equal(dH, out["dx"])


@pytest.mark.gpu
@pytest.mark.parametrize("post,group", [(True, 0), (False, 3), (True, 1)])
@pytest.mark.parametrize("rows,k", [(700, 40), (700, 264), (3, 4096), (900, 2056), (300, 16384)])
def test_gradient_in_the_place_of_x(rows, k, post, group, workspace):
    x = Problem(rows, k, ("bf16", "f32"), post=post, group=group or None)
    out = x.gradient()
    x.check_gradient(out)
    X, sums = x.X, {name: torch.full_like(out[name], float("nan")) for name in ("dw_post", "dgate", "dw_pre") if name in out}
    lib.ozaki_block_norm_grad(*x.common(), x.R, x.R.shape[1], lib.TYPE_F32, x.w_pre, x.dH, x.dH.shape[1], x.dR_out, x.dR_out.shape[1], X, X.shape[1], None, 0, sums.get("dw_post"),
                              sums.get("dgate"), sums["dw_pre"])
    assert torch.equal(X[:, :k], out["dx"]) and all(torch.equal(sums[name], out[name]) for name in sums)


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES)
def test_zeros_large_and_small_numbers(types, workspace):
    """Rows of zeros give zeros; rows whose squares leave 32 bits' range, above or below, are normed all the same (eps is nothing beside 2^-40 squared only where it is smaller)."""
    t, tr = (DTYPES[v] for v in types)
    k = 520
    for power in (None, 100, 60, 0, -60) if "f16" not in types else (None, 12, 0, -10):
        x = Problem(4, k, types, seed=3, scale=1.0)
        f = 0.0 if power is None else 2.0 ** power
        x.x, x.r = (x.x.double() * f).to(t), (x.r.double() * f).to(tr)
        x.X, x.R = plain.padded(x.x, types[0]), plain.padded(x.r, types[1])
        R_out, H = x.forward()
        if power is None:
            assert bool(torch.all(H[:, :k] == 0)) and bool(torch.all(R_out[:, :k] == 0))
        if power is None or power <= 0:
            x.check_gradient(x.gradient())
    x = Problem(3, k, types)
    x.X[1, 5] = float("nan")
    R_out = x.result(types[1], 0)
    H = x.result(types[0], 0)
    lib.ozaki_block_norm(*x.common(), x.R, x.R.shape[1], lib.TYPES[types[1]], R_out, k, x.w_pre, H, k)
    assert bool(torch.isnan(H[1]).all()) and not bool(torch.isnan(H[[0, 2]]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("k", [100, 2000, 16384])
def test_means_whose_sums_leave_the_range(k, types, workspace):
    """Gradients of 2^121 and 3 * 2^121: their mean along the row is 2^122, the sum of thousands of them is beyond 2^128."""
    x = Problem(3, k, types, post=False, seed=4)
    d = 2.0 ** 121 * (2 + (-1.0) ** torch.arange(k, device="cuda"))
    x.r[:], x.dh[:], x.w_pre[:] = 1.0, d.to(x.dh.dtype), 1.0
    x.R, x.dH = plain.padded(x.r, types[1]), plain.padded(x.dh, types[0])
    out = x.gradient(True, False, ("dr", "dw_pre"))
    x.check_gradient(out, True, False)
    # the same through the norm behind the block
    x = Problem(3, k, types, seed=4, scale=1.0)
    x.x[:], x.dr_out[:], x.w_post[:] = 1.0, d.to(x.dr_out.dtype), 1.0
    x.X, x.dR_out = plain.padded(x.x, types[0]), plain.padded(x.dr_out, types[1])
    x.check_gradient(x.gradient(False, True, ("dx", "dr")), False, True)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [520, 9000])
def test_gradient_without_a_norm_does_not_look_at_x(k, workspace):
    """Without w_post the gradient of X is scale * gate * dR, whatever X holds."""
    x = Problem(6, k, ("bf16", "bf16"), post=False, group=2)
    want = x.gradient(want=("dx", "dr"))
    x.X[1, 3], x.X[4, k - 1] = float("inf"), float("nan")
    got = x.gradient(want=("dx", "dr"))
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dr"], want["dr"])


@pytest.mark.gpu
def test_gradient_against_differences(workspace):
    """Along a direction, in 32 bits: a central difference over t is off by the third derivative's t^2 / 6, for which the step of half t, a quarter as far off, is the measure."""
    rows, k = 6, 72
    x = Problem(rows, k, ("f32", "f32"), group=2, seed=11)
    total, _, _, _ = plain.block_norm(x.x.double(), x.r.double(), x.w_post.double(), x.gate.double(), 2, x.scale, EPS, x.w_pre.double())
    leaves = {"dx": x.x.double(), "dr": x.r.double(), "dw_post": x.w_post.double(), "dgate": x.gate.double(), "dw_pre": x.w_pre.double()}
    x.R = total.float().contiguous()
    out = x.gradient()
    gen = torch.Generator(device="cuda").manual_seed(1)

    def value(at):
        r, _, h, _ = plain.block_norm(at["dx"], at["dr"], at["dw_post"], at["dgate"], 2, x.scale, EPS, at["dw_pre"])
        return float((h * x.dh.double()).sum() + (r * x.dr_out.double()).sum())

    for name, leaf in leaves.items():
        direction = torch.randn(leaf.shape, dtype=torch.float64, device="cuda", generator=gen)
        slope = []
        for t in (2.0 ** -10, 2.0 ** -11):
            up, down = dict(leaves), dict(leaves)
            up[name], down[name] = leaf + t * direction, leaf - t * direction
            slope.append((value(up) - value(down)) / (2 * t))
        got = float((out[name][..., :k].double() * direction).sum())
        size = float((out[name][..., :k].double() * direction).abs().sum())
        assert abs(got - slope[1]) <= 2 * abs(slope[0] - slope[1]) + 2.0 ** -18 * size, name


@pytest.mark.gpu
@pytest.mark.parametrize("group", [None, 100, 3])
def test_same_bits_every_time_and_in_a_graph(group, workspace):
    x = Problem(2500, 1100, ("bf16", "bf16"), group=group)
    first = x.gradient()
    again = x.gradient()
    assert all(torch.equal(first[name], again[name]) for name in first)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        held = x.gradient()
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    for step in range(3):
        x.dH.mul_(0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = x.gradient()
        torch.cuda.synchronize()
        assert all(torch.equal(held[name], want[name]) for name in want)


FAKE = 1 << 20


def _refused(call, good, changes):
    for at, value in changes:
        args = list(good)
        args[at - 1] = value
        assert call(*args, check=False) == -at, (call.__name__, at, value)


def test_refusals():
    nan, inf = float("nan"), float("inf")
    good = [4, 20, FAKE, 24, lib.TYPE_BF16, FAKE, FAKE, 2, 1.0, EPS, FAKE, 24, lib.TYPE_F32, FAKE, 20, FAKE, FAKE, 20]
    head = [(1, -1), (1, lib.MAX_EXTENT + 1), (2, 0), (2, lib.MAX_NORM + 1), (3, FAKE + 2), (4, 16), (4, 20), (5, 3), (6, FAKE + 2), (7, FAKE + 1), (8, 0), (9, nan), (9, inf), (10, -1.0), (10, nan),
            (10, inf), (13, lib.TYPE_F16)]
    _refused(lib.ozaki_block_norm, good, head + [(11, FAKE + 4), (12, 16), (12, 22), (14, FAKE + 2), (15, 19), (16, None), (16, FAKE + 1), (17, FAKE + 1), (18, 19)])
    nothing = list(good)
    nothing[2] = nothing[5] = nothing[6] = None
    assert lib.ozaki_block_norm(*nothing, check=False) == -14       # (without X there is no sum to store)
    nothing[10] = None
    assert lib.ozaki_block_norm(*nothing, check=False) == -3
    assert lib.ozaki_block_norm(*(good[:2] + [None] + good[3:]), check=False) == -6
    assert lib.ozaki_block_norm(*(good[:13] + [None, 0, None, None, 0]), check=False) == -14
    good = [4, 20, FAKE, 24, lib.TYPE_BF16, FAKE, FAKE, 2, 1.0, EPS, FAKE, 24, lib.TYPE_F32, FAKE, FAKE, 24, FAKE, 24, FAKE, 20, FAKE, 20, FAKE, FAKE, FAKE]
    _refused(lib.ozaki_block_norm_grad, good, head + [(11, None), (11, FAKE + 4), (12, 22), (14, None), (15, FAKE + 2), (16, 20), (17, FAKE + 4), (18, 22), (19, FAKE + 1), (20, 19), (21, FAKE + 2),
                                                      (22, 19), (23, FAKE + 2), (24, FAKE + 1), (25, FAKE + 2)])
    for at, value, answer in ((6, None, -23), (7, None, -24), (15, None, -25)):
        args = list(good)
        args[at - 1] = value
        assert lib.ozaki_block_norm_grad(*args, check=False) == answer
    assert lib.ozaki_block_norm_grad(*(good[:14] + [None, 0, None, 0] + good[18:24] + [None]), check=False) == -15
    assert lib.ozaki_block_norm_grad(*(good[:18] + [None, 0, None, 0, None, None, None]), check=False) == -19
    assert lib.ozaki_block_norm_workspace_bytes(0, 4, 0) == lib.ozaki_block_norm_workspace_bytes(4, 0, 0) == lib.ozaki_block_norm_workspace_bytes(4, lib.MAX_NORM + 1, 0) == 0
    assert lib.ozaki_block_norm(0, 20, None, 0, lib.TYPE_BF16, None, None, 0, 1.0, EPS, None, 0, lib.TYPE_BF16, None, 0, None, None, 0) == 0


@pytest.mark.gpu
def test_no_rows():
    a, b = (torch.full((20,), 7.0, device="cuda") for _ in range(2))
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    lib.ozaki_block_norm_grad(0, 20, None, 0, lib.TYPE_BF16, None, None, 0, 1.0, EPS, None, 0, lib.TYPE_BF16, None, None, 0, None, 0, None, 0, None, 0, a, None, b)
    assert bool(torch.all(a == 0)) and bool(torch.all(b == 0))


def test_no_rows_with_weights():
    """A batch of no rows lies at a null address; the weights and gates that go with every batch are there all the same."""
    norm = (0, 20, None, 0, lib.TYPE_BF16, FAKE, FAKE, 2, 1.0, EPS, None, 0, lib.TYPE_BF16)
    assert lib.ozaki_block_norm(*norm, None, 0, FAKE, None, 0, check=False) == 0
    assert lib.ozaki_block_norm(*norm[:6], None, 0, *norm[8:], None, 0, FAKE, None, 0, check=False) == 0
    assert lib.ozaki_block_norm_grad(*norm, FAKE, None, 0, None, 0, None, 0, None, 0, None, FAKE, None, check=False) == 0
    # what is wrong with any number of rows is refused with none, too
    assert lib.ozaki_block_norm(*norm[:5], FAKE + 2, *norm[6:], None, 0, FAKE, None, 0, check=False) == -6
    assert lib.ozaki_block_norm(*norm[:7], 0, *norm[8:], None, 0, FAKE, None, 0, check=False) == -8


def test_no_rows_and_nothing_but_their_gradients():
    norm = (0, 20, None, 0, lib.TYPE_BF16, None, None, 0, 1.0, EPS, None, 0, lib.TYPE_BF16, FAKE, None, 0, None, 0)
    assert lib.ozaki_block_norm_grad(*norm, None, 20, None, 20, None, None, None, check=False) == 0


@pytest.mark.gpu
def test_no_rows_with_weights_gives_zeros():
    rand = lambda *shape: torch.randn(shape, device="cuda")    # noqa: E731
    x, w_post, w_pre, gate = rand(0, 20).bfloat16(), rand(20), rand(20), rand(3, 20)
    dw_post, dw_pre = (torch.full((20,), 7.0, device="cuda") for _ in range(2))
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    for g, group in ((gate, 2), (None, 0)):
        common = (0, 20, x, 24, lib.TYPE_BF16, w_post, g, group, 1.0, EPS)
        lib.ozaki_block_norm(*common, x, 24, lib.TYPE_BF16, x, 20, w_pre, x, 20)
        lib.ozaki_block_norm_grad(*common, x, 24, lib.TYPE_BF16, w_pre, x, 24, x, 24, x, 20, x, 20, dw_post.fill_(7.0), None, dw_pre.fill_(7.0))
        assert bool(torch.all(dw_post == 0)) and bool(torch.all(dw_pre == 0))


@pytest.mark.gpu
def test_beyond_32_bits(workspace):
    """More than 2^31 elements: the last rows are as they are alone."""
    rows, k = 270000, 8192
    few = Problem(5, k, ("bf16", "bf16"), group=None)
    few.check_gradient(few.gradient(want=("dx", "dr")))
    X, R, dH = (torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    X[-5:], R[-5:], dH[-5:] = few.x, few.r, few.dh
    H = torch.zeros_like(X)
    args = (rows, k, X, k, lib.TYPE_BF16, few.w_post, None, 0, few.scale, EPS)
    dw_pre = torch.zeros((k,), device="cuda")
    lib.ozaki_block_norm_grad(*args, R, k, lib.TYPE_BF16, few.w_pre, dH, k, None, 0, H, k, None, 0, None, None, dw_pre)
    want = few.gradient(True, False, ("dx", "dw_pre"))
    assert torch.equal(H[-5:], want["dx"]) and bool(torch.all(H[:-5] == 0))
    assert bool(torch.all((dw_pre - want["dw_pre"]).abs() <= 2.0 ** -20 * (few.dh.float() * few.r.float()).abs().sum(0)))
    lib.ozaki_block_norm(*args, R, k, lib.TYPE_BF16, R, k, few.w_pre, H, k)
    r, h = few.forward()
    assert torch.equal(H[-5:], h) and torch.equal(R[-5:], r) and bool(torch.all(H[:-5] == 0))
