"""ozaki_quantise_fp8: codes and scales equal to the definition's, every one of them."""
import pytest

torch = pytest.importorskip("torch")

import low_precision as plain  # noqa: E402
from paper_2508_00441_amd import binding as lib  # noqa: E402

SHAPES = [(1, 1), (1, 4096), (3, 127), (16, 128), (17, 129), (128, 128), (130, 257), (300, 1000), (129, 2049), (1000, 15)]


def _source(rows, k, type, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, k), generator=gen) * torch.exp(3 * torch.randn((rows, 1), generator=gen))
    if type == "f16":
        x = x.clamp(-60000, 60000)
    return x.to(plain.DTYPES[type])


def _call(x, type, blocks, straight=True, transposed=False, stream=None):
    rows, k = x.shape
    per = 16 // x.element_size()
    X = plain.padded(x, per, float("nan")).cuda()
    shared = plain.BLOCK if blocks else 1
    at = lambda n: -(-n // shared)  # noqa: E731
    Q = torch.full((rows, plain.ceil(k, 16) + 16), 0x55, dtype=torch.uint8, device="cuda") if straight else None
    S = torch.full((-(-k // 128), at(rows) + 3), -1.0, device="cuda") if straight else None
    Qt = torch.full((k, plain.ceil(rows, 16) + 16), 0x55, dtype=torch.uint8, device="cuda") if transposed else None
    St = torch.full((-(-rows // 128), at(k) + 1), -1.0, device="cuda") if transposed else None
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    lib.ozaki_quantise_fp8(rows, k, X, X.shape[1], lib.TYPES[type], lib.SCALE_BLOCKS if blocks else lib.SCALE_VECTORS,
                           Q, Q.shape[1] if straight else 0, S, S.shape[1] if straight else 0,
                           Qt, Qt.shape[1] if transposed else 0, St, St.shape[1] if transposed else 0)
    torch.cuda.synchronize()
    return Q, S, Qt, St


def _same(Q, S, x, blocks):
    q, s = plain.quantised(x.float(), blocks)
    got = Q.cpu()
    values, want = got[:, : x.shape[1]].contiguous().view(torch.float8_e4m3fn).float(), q.float()       # (zeros are equal whatever their sign)
    assert torch.equal(torch.isnan(values), torch.isnan(want)) and torch.equal(values.nan_to_num(0.0), want.nan_to_num(0.0))
    assert bool(torch.all(got[:, x.shape[1]:] == 0x55)), "wrote behind a vector's end"
    sc = S.cpu()
    assert torch.equal(sc[:, : s.shape[1]], s)
    assert bool(torch.all(sc[:, s.shape[1]:] == -1.0))


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("rows,k", SHAPES)
def test_codes_and_scales(rows, k, blocks, type):
    x = _source(rows, k, type, rows * 7 + k)
    for straight, transposed in ((True, False), (False, True), (True, True)):
        Q, S, Qt, St = _call(x, type, blocks, straight, transposed)
        if straight:
            _same(Q, S, x, blocks)
        if transposed:
            _same(Qt, St, x.t().contiguous(), blocks)


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("blocks", [False, True])
def test_zeros_extremes_and_values_that_are_not_finite(blocks, type):
    x = _source(260, 400, type, 5)
    x[:, :128] = 0.0                                                # whole blocks of zeros
    x[5, 130], x[6, 131], x[7, 132] = float("nan"), float("inf"), -float("inf")
    x[140:, 256:] *= 1e-38                                          # scales at their floor
    x[3, 300] = 3e38
    x[200, 5] = -0.0
    Q, S, Qt, St = _call(x, type, blocks, True, True)
    _same(Q, S, x, blocks)
    _same(Qt, St, x.t().contiguous(), blocks)


@pytest.mark.gpu
def test_every_value_and_every_tie_of_the_format():
    codes = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()          # 0 .. 448
    ties = (codes[1:] + codes[:-1]) / 2
    x = torch.cat([codes, -codes, ties, -ties, torch.full((6,), 448.0)]).reshape(1, -1)         # 512: every block ...
    x[0, 0::128] = 448.0                                            # ... with a scale of 1
    Q, S, _, _ = _call(x.contiguous(), "f32", False)
    assert bool(torch.all(S[:, 0] == 1.0))
    _same(Q, S, x, False)


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16", "f32"])
def test_quotients_on_and_next_to_ties(type):
    """Elements a fraction of the block's largest that lies half-way between two codes, and (32 bits) its neighbours."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    ties = ((codes[1:] + codes[:-1]) / 2)
    gen = torch.Generator().manual_seed(11)
    amax = torch.cat([torch.tensor([448.0, 1.75, 7.0, 1.0, 1.5, 3.0 * 2.0 ** -30 if type != "f16" else 3.0]), torch.rand((60,), generator=gen) + 1.0])
    amax = amax.to(plain.DTYPES[type]).double().unsqueeze(1)
    x = (ties * amax / 448.0).to(plain.DTYPES[type])
    if type == "f32":
        x = torch.cat([x, torch.nextafter(x, torch.zeros_like(x)), torch.nextafter(x, torch.full_like(x, 9.0))])
        amax = amax.repeat(3, 1)
    x = torch.cat([x, amax.to(x.dtype), -amax.to(x.dtype)], 1)      # 128: a block each
    for blocks in (False, True):
        Q, S, Qt, St = _call(x, type, blocks, True, True)
        _same(Q, S, x, blocks)
        _same(Qt, St, x.t().contiguous(), blocks)


@pytest.mark.gpu
def test_more_than_2_31_elements():
    rows, k = 1 << 15, (1 << 16) + 128
    X = torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    for r in (0, 1, rows // 2, rows - 2, rows - 1):
        X[r] = torch.randn((k,), device="cuda", generator=gen).to(torch.bfloat16)
    Q, S = torch.empty((rows, k), dtype=torch.uint8, device="cuda"), torch.empty((k // 128, rows), device="cuda")
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    lib.ozaki_quantise_fp8(rows, k, X, k, lib.TYPE_BF16, lib.SCALE_VECTORS, Q, k, S, rows)
    torch.cuda.synchronize()
    for r in (0, 1, 2, rows // 2, rows - 2, rows - 1):
        q, s = plain.quantised(X[r: r + 1].float().cpu(), False)
        assert torch.equal(Q[r: r + 1].view(torch.float8_e4m3fn).float().cpu(), q.float()) and torch.equal(S[:, r: r + 1].cpu(), s)


@pytest.mark.gpu
def test_on_a_stream_of_its_own_and_in_a_graph():
    x = _source(200, 520, "bf16", 9)
    context = lib.ozaki_context_create()
    lib.ozaki_context_use(context)
    try:
        X = plain.padded(x, 8, 0.0).cuda()
        Q, S = torch.zeros((200, 528), dtype=torch.uint8, device="cuda"), torch.zeros((5, 200), device="cuda")
        stream = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
            lib.ozaki_quantise_fp8(200, 520, X, X.shape[1], lib.TYPE_BF16, lib.SCALE_VECTORS, Q, 528, S, 200)
        for seed in (9, 10, 11):
            x = _source(200, 520, "bf16", seed)
            X[:, :520] = x.cuda()
            Q.fill_(0x55)
            graph.replay()
            torch.cuda.synchronize()
            _same(Q, S, x, False)
    finally:
        lib.ozaki_context_use(None)
        lib.ozaki_context_destroy(context)


P = 1 << 20                                                         # an aligned address that nothing is launched with


@pytest.mark.parametrize("position,arguments", [
    (1, dict(rows=-1)), (1, dict(rows=lib.MAX_EXTENT + 1)), (2, dict(k=-1)), (2, dict(k=lib.MAX_EXTENT + 1)), (3, dict(X=None)), (3, dict(X=P + 2)),
    (4, dict(ldx=199)), (4, dict(ldx=204)), (5, dict(type=3)), (5, dict(type=-1)), (6, dict(scaling=2)), (7, dict(Q=None, S=None, Qt=None, St=None)),
    (7, dict(Q=P + 8)), (8, dict(ldq=200)), (8, dict(ldq=192)), (9, dict(S=None)), (9, dict(Q=None)), (10, dict(lds=99)),
    (10, dict(lds=0, scaling=lib.SCALE_BLOCKS)), (11, dict(Qt=P + 4)), (12, dict(ldqt=96)), (12, dict(ldqt=100)), (13, dict(St=None)),
    (13, dict(Qt=None)), (14, dict(ldst=199)), (14, dict(ldst=1, scaling=lib.SCALE_BLOCKS))])
def test_refusals(position, arguments):
    a = dict(rows=100, k=200, X=P, ldx=200, type=lib.TYPE_BF16, scaling=lib.SCALE_VECTORS, Q=P, ldq=208, S=P, lds=100, Qt=P, ldqt=112, St=P, ldst=200)
    assert lib.ozaki_quantise_fp8(**{**a, **arguments}, check=False) == -position
    with pytest.raises(lib.OzakiError):
        lib.ozaki_quantise_fp8(**{**a, **arguments})


def test_refuses_more_than_a_launch_holds():
    a = dict(X=P, ldx=1 << 14, type=lib.TYPE_BF16, scaling=lib.SCALE_VECTORS, Q=P, ldq=1 << 14, S=P, lds=lib.MAX_EXTENT)
    assert lib.ozaki_quantise_fp8(rows=lib.MAX_QUANTISED // (1 << 14) + 1, k=1 << 14, **a, check=False) == -2


def test_nothing_to_do():
    for rows, k in ((0, 100), (100, 0)):
        assert lib.ozaki_quantise_fp8(rows, k, None, 0, lib.TYPE_BF16, lib.SCALE_VECTORS, None, 0, None, 0) == 0
