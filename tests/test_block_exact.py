"""The block's operators on small whole numbers, whose products and sums in 32 bits have no rounding in whatever order they are added: results are equal to the
definition's, so that a row, a column, a share or a step that is left out or taken twice shows however many there are."""
import pytest

torch = pytest.importorskip("torch")

import block_operators as plain  # noqa: E402
from low_precision import DTYPES  # noqa: E402
from paper_2508_00441_amd import binding as lib, device  # noqa: E402


def _whole(gen, most, *shape):
    return torch.randint(-most, most + 1, shape, device="cuda", generator=gen).double()


def _result(rows, columns, type):
    return torch.full((rows, columns), float("nan"), dtype=DTYPES[type], device="cuda")


def _product(x, w):
    return x @ w.t().contiguous()


def _equal(got, want, type):
    assert float(want.abs().max()) < 2 ** 24                         # (every partial sum is a whole number of 24 bits)
    assert torch.equal(got, want.to(DTYPES[type]))


# every kind of tile, with and without shares; steps, rows and columns that end inside one
LINEAR = [(1, 1000, 8200), (16, 100, 6401), (17, 33, 72), (20, 1000, 8192), (48, 1000, 500), (100, 300, 4096), (64, 500, 1000), (100, 5001, 200), (200, 1001, 200), (700, 1300, 100), (1000, 3204, 72),
          (2000, 3201, 136), (2310, 4097, 129), (4616, 4090, 40), (2100, 8461, 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", LINEAR)
def test_linear(m, n, k, type):
    gen, t = torch.Generator(device="cuda").manual_seed(m + n + k), lib.TYPES[type]
    x, w, w2, bias, r = _whole(gen, 1, m, k), _whole(gen, 1, n, k), _whole(gen, 1, n, k), _whole(gen, 4, n), _whole(gen, 4, m, n)
    X, W, W2 = (plain.padded(v, type) for v in (x, w, w2))
    Y, Z, U = (_result(m, n, type) for _ in range(3))
    ws = device.Workspace(lib.ozaki_linear_workspace_bytes(m, n, k, False))
    lib.ozaki_linear(m, n, k, X, X.shape[1], W, W.shape[1], t, bias.to(DTYPES[type]), lib.ACTIVATION_RELU, r.to(DTYPES[type]), n, Y, n, Z, n)
    z = _product(x, w) + bias
    _equal(Z, z, type)
    _equal(Y, z.clamp(min=0) + r, type)
    ws.close()
    ws = device.Workspace(lib.ozaki_gated_linear_workspace_bytes(m, n, k, False))
    Y, Z = _result(m, n, type), _result(m, n, type)
    lib.ozaki_gated_linear(m, n, k, X, X.shape[1], W, W2, W.shape[1], t, lib.ACTIVATION_RELU, Y, n, Z, n, U, n)
    g, u = _product(x, w), _product(x, w2)
    _equal(Z, g, type)
    _equal(U, u, type)
    _equal(Y, g.clamp(min=0) * u, type)
    ws.close()


GRADIENTS = [(1, 257, 100), (3, 5, 8), (16, 1000, 136), (40, 3000, 64), (65, 1000, 33), (300, 511, 64), (333, 1000, 1001), (513, 264, 1031), (720, 1693, 160), (5000, 100, 130), (10000, 600, 40),
             (1030, 2100, 264), (2100, 1100, 4200), (4100, 300, 280), (1030, 8000, 1030), (70001, 40, 24)]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", GRADIENTS)
def test_linear_gradient(m, n, k, type, act):
    gen, t, a = torch.Generator(device="cuda").manual_seed(m + n + k), lib.TYPES[type], lib.ACTIVATIONS[act]
    x, w, w2, z, u, dy = _whole(gen, 1, m, k), _whole(gen, 1, n, k), _whole(gen, 1, n, k), _whole(gen, 2, m, n), _whole(gen, 2, m, n), _whole(gen, 2, m, n)
    X, W, W2, Z, U, dY = (plain.padded(v, type) for v in (x, w, w2, z, u, dy))
    ldx, ldw, ldz = X.shape[1], W.shape[1], Z.shape[1]
    slope = (z > 0).double() if act == "relu" else torch.ones_like(z)
    across = lambda d, v: d.t().contiguous() @ v    # noqa: E731
    ws = device.Workspace(lib.ozaki_linear_workspace_bytes(m, n, k, True))
    dz = dy * slope
    for wanted in ("xwb", "b", "xb", "wb"):
        dX, dW, dbias = _result(m, k, type), _result(n, k, type), torch.full((n,), float("nan"), device="cuda")
        lib.ozaki_linear_grad(m, n, k, X, ldx, W, ldw, t, a, Z, ldz, dY, ldz, dX if "x" in wanted else None, k, dW if "w" in wanted else None, k, dbias)
        _equal(dbias, dz.sum(0), "f32")
        if "x" in wanted:
            _equal(dX, dz @ w, type)
        if "w" in wanted:
            _equal(dW, across(dz, x), type)
    ws.close()
    ws = device.Workspace(lib.ozaki_gated_linear_workspace_bytes(m, n, k, True))
    dX, dW, dW2 = _result(m, k, type), _result(n, k, type), _result(n, k, type)
    lib.ozaki_gated_linear_grad(m, n, k, X, ldx, W, W2, ldw, t, a, Z, ldz, U, ldz, dY, ldz, dX, k, dW, dW2, k)
    dg, du = dy * u * slope, dy * z * slope
    _equal(dX, dg @ w + du @ w2, type)
    _equal(dW, across(dg, x), type)
    _equal(dW2, across(du, x), type)
    ws.close()


# rows side by side, a row to a workgroup, the longest rows; without a gate, with one, with gates that end inside a workgroup's rows and that have one, some and many chunks
NORMS = [(1, 1, 0), (1, 1000, 1), (5, 16384, 2), (33, 1000, 0), (300, 72, 7), (301, 9001, 0), (900, 4100, 900), (1500, 40, 0), (4200, 100, 4200), (2600, 520, 50), (2600, 1100, 299), (16400, 24, 0),
         (16400, 24, 1), (16400, 24, 5), (16384, 128, 16), (9000, 130, 15), (9000, 130, 17), (5000, 250, 2), (7003, 500, 4), (7003, 500, 7), (40, 100, 1), (2500, 513, 1), (1100, 2048, 3), (1100, 4100, 1),
         (600, 9000, 1), (1300, 9000, 4), (3000, 1000, 64), (5000, 90, 1700), (4097, 300, 4096), (100001, 16, 0), (100001, 8, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,k,group", NORMS)
def test_sums_over_rows(rows, k, group, types, post):
    """Rows of 1 and -1 have rho = 1 with eps = 0.  dh of neighbouring columns cancels along the row, so that dr = dr' + dh."""
    gen, (t, tr) = torch.Generator(device="cuda").manual_seed(rows + k), types
    sign = lambda: 2 * torch.randint(0, 2, (rows, k), device="cuda", generator=gen).double() - 1    # noqa: E731
    x, r, dr_out, dh = sign(), sign(), _whole(gen, 2, rows, k), _whole(gen, 2, rows, k)
    dh[:, 1::2] = -(dh * r)[:, 0::2][:, : k // 2] * r[:, 1::2]
    if k % 2:
        dh[:, -1] = 0
    gates = -(-rows // group) if group else 1
    gate, w_post = _whole(gen, 2, gates, k), 2.0 ** _whole(gen, 1, k)
    X, dH, R, dR_out = plain.padded(x, t), plain.padded(dh, t), plain.padded(r, tr), plain.padded(dr_out, tr)
    dr = dr_out + dh
    s = torch.zeros((gates, k), dtype=torch.float64, device="cuda").index_add_(0, torch.arange(rows, device="cuda") // (group or rows), dr * x)
    want = {"dw_pre": (dh * r).sum(0), "dr": dr}
    if post:
        want["dw_post"] = 0.5 * ((gate if group else 1) * s).sum(0)
    if group:
        want["dgate"] = 0.5 * s * (w_post if post else 1)
    ws = device.Workspace(lib.ozaki_block_norm_workspace_bytes(rows, k, group))
    for names in (list(want), ["dw_pre"], ["dgate"], ["dw_post"], ["dw_post", "dgate"]):
        names = [name for name in names if name in want]
        if not names:
            continue
        out = {name: torch.full(want[name].shape, float("nan"), dtype=DTYPES[tr] if name == "dr" else torch.float32, device="cuda") for name in names}
        lib.ozaki_block_norm_grad(rows, k, X, X.shape[1], lib.TYPES[t], w_post.float() if post else None, gate.float() if group else None, group, 0.5, 0.0, R, R.shape[1], lib.TYPES[tr],
                                  torch.ones((k,), device="cuda"), dH, dH.shape[1], dR_out, dR_out.shape[1], None, 0, out.get("dr"), k, out.get("dw_post"), out.get("dgate"), out.get("dw_pre"))
        for name, got in out.items():
            _equal(got, want[name], tr if name == "dr" else "f32")
    ws.close()
