"""ozaki_gemm_fp8 against the sum of its definition in 64 bits, within the bound of its 32-bit additions."""
import pytest

torch = pytest.importorskip("torch")

import low_precision as plain  # noqa: E402
from paper_2508_00441_amd import binding as lib, device  # noqa: E402

SHAPES = [(1, 1, 1), (1, 64, 128), (1, 1000, 4096), (2, 65, 130), (15, 300, 1000), (16, 512, 8192), (17, 129, 257), (33, 640, 2048), (64, 256, 5000),
          (100, 100, 100), (128, 128, 128), (129, 255, 384), (200, 1000, 1301), (256, 256, 256), (300, 520, 136), (513, 700, 999)]


class Operands:
    def __init__(self, m, n, k, blocks, seed, wide=False):
        gen = torch.Generator().manual_seed(seed)
        a = torch.randn((m, k), generator=gen)
        b = torch.randn((n, k), generator=gen) * 0.05
        if wide:                                                    # scales that differ a great deal from block to block
            a *= torch.exp2(torch.randint(-20, 20, (1, plain.ceil(k, 128) // 128), generator=gen).float()).repeat_interleave(128, 1)[:, :k]
        self.m, self.n, self.k, self.blocks = m, n, k, blocks
        self.qa, self.sa = plain.quantised(a, False)
        self.qb, self.sb = plain.quantised(b, blocks)
        # behind the vectors' ends lie NaN codes
        self.A = plain.padded(self.qa.view(torch.uint8), 16, 0x7F).cuda()
        self.B = plain.padded(self.qb.view(torch.uint8), 16, 0xFF).cuda()
        self.SA = torch.nn.functional.pad(self.sa, (0, 5), value=float("nan")).cuda()
        self.SB = torch.nn.functional.pad(self.sb, (0, 3), value=float("nan")).cuda()

    def exact(self):
        a, b = plain.dequantised(self.qa, self.sa, False).cuda(), plain.dequantised(self.qb, self.sb, self.blocks).cuda()
        cut = plain.cut_products(self.qa, self.sa, False).cuda() @ plain.cut_products(self.qb, self.sb, self.blocks).cuda().t()
        return a @ b.t(), a.abs() @ b.abs().t(), cut

    def multiply(self, D, ldd, type_d, accumulate=0):
        return lib.ozaki_gemm_fp8(self.m, self.n, self.k, self.A, self.A.shape[1], self.SA, self.SA.shape[1], self.B, self.B.shape[1], self.SB,
                                  self.SB.shape[1], lib.SCALE_BLOCKS if self.blocks else lib.SCALE_VECTORS, D, ldd, lib.TYPES[type_d], accumulate)


@pytest.fixture()
def workspace():
    ws = device.Workspace(64 << 20)
    yield ws
    ws.close()


def _check(o, D, type_d, before=None):
    want, magnitudes, cut = o.exact()
    if before is not None:
        want, magnitudes = want + before, magnitudes + before.abs()
    off = (D.double() - want).abs()
    assert bool(torch.all(off <= plain.gemm_bound(o.k, magnitudes, type_d, want, cut))), float(off.max())


@pytest.mark.gpu
@pytest.mark.parametrize("type_d", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products(m, n, k, blocks, type_d, workspace):
    o = Operands(m, n, k, blocks, m + n + k)
    D = torch.full((m, n), float("nan"), dtype=plain.DTYPES[type_d], device="cuda")
    o.multiply(D, n, type_d)
    _check(o, D, type_d)


@pytest.mark.gpu
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("m,n,k", [(2048, 3001, 520), (4100, 2049, 257), (2304, 2304, 1040)])
def test_large_products(m, n, k, blocks, workspace):
    o = Operands(m, n, k, blocks, 1)
    D = torch.full((m, n), float("nan"), dtype=torch.float32, device="cuda")
    o.multiply(D, n, "f32")
    _check(o, D, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("type_d", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("m,n,k", [(3600, 3501, 520), (4100, 3329, 257), (3585, 3584, 1301), (3600, 3600, 100), (3601, 3590, 127), (3600, 3600, 128),
                                   (3584, 3600, 2176), (3600, 3700, 656)])
def test_products_of_many_tiles(m, n, k, blocks, type_d, workspace):
    o = Operands(m, n, k, blocks, 12)
    D = torch.full((m, n), float("nan"), dtype=plain.DTYPES[type_d], device="cuda")
    o.multiply(D, n, type_d)
    _check(o, D, type_d)


@pytest.mark.gpu
@pytest.mark.parametrize("type_d", ["bf16", "f32"])
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("m,n,k", [(1, 64, 65536), (3, 130, 12401), (16, 65, 20000)])
def test_few_vectors_of_many_elements(m, n, k, blocks, type_d, workspace):
    o = Operands(m, n, k, blocks, 14)
    D = torch.full((m, n), float("nan"), dtype=plain.DTYPES[type_d], device="cuda")
    o.multiply(D, n, type_d)
    _check(o, D, type_d)


@pytest.mark.gpu
@pytest.mark.parametrize("type_d", ["bf16", "f16"])
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("m,n,k", [(4353, 3841, 264), (3841, 4353, 401), (4609, 3600, 128)])
def test_products_whose_last_tiles_are_few(m, n, k, blocks, type_d, workspace):
    o = Operands(m, n, k, blocks, 13)
    D = torch.full((m, n), float("nan"), dtype=plain.DTYPES[type_d], device="cuda")
    o.multiply(D, n, type_d)
    _check(o, D, type_d)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 200, 2000), (40, 200, 700), (2400, 2400, 300)])
def test_scales_far_apart(m, n, k, workspace):
    o = Operands(m, n, k, True, 2, wide=True)
    D = torch.empty((m, n), dtype=torch.float32, device="cuda")
    o.multiply(D, n, "f32")
    _check(o, D, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("type_d", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("m,n,k", [(1, 300, 4096), (70, 130, 300), (2400, 2400, 128)])
def test_rows_of_a_larger_result_on_top_of_what_is_there(m, n, k, type_d, workspace):
    o = Operands(m, n, k, True, 3)
    for offset, ldd in ((0, plain.ceil(n, 4) + 4), (1, n + 3)):
        whole = torch.randn((m * ldd + 8,), device="cuda").to(plain.DTYPES[type_d])
        kept = whole.clone()
        view = lambda x: x[offset: offset + m * ldd].view(m, ldd)   # noqa: E731
        o.multiply(whole[offset:], ldd, type_d, 1)
        _check(o, view(whole)[:, :n], type_d, view(kept)[:, :n].double())
        assert torch.equal(view(whole)[:, n:], view(kept)[:, n:]) and torch.equal(whole[offset + m * ldd:], kept[offset + m * ldd:])


@pytest.mark.gpu
def test_no_inner_dimension(workspace):
    D = torch.full((5, 9), 3.0, device="cuda")
    lib.ozaki_gemm_fp8(5, 7, 0, None, 0, None, 0, None, 0, None, 0, lib.SCALE_BLOCKS, D, 9, lib.TYPE_F32, 1)
    assert bool(torch.all(D == 3.0))
    lib.ozaki_gemm_fp8(5, 7, 0, None, 0, None, 0, None, 0, None, 0, lib.SCALE_BLOCKS, D, 9, lib.TYPE_F32, 0)
    assert bool(torch.all(D[:, :7] == 0.0)) and bool(torch.all(D[:, 7:] == 3.0))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 64, 2400])
def test_a_nan_code_spoils_its_row_only(m, workspace):
    n, k = 2304 if m > 64 else 300, 400
    o = Operands(m, n, k, True, 4)
    o.A[m // 2, 17] = 0x7F
    D = torch.empty((m, n), dtype=torch.float32, device="cuda")
    o.multiply(D, n, "f32")
    nan = torch.isnan(D)
    assert bool(nan[m // 2].all()) and int(nan.sum()) == n


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 2000, 4096), (300, 500, 4096), (2400, 2400, 700)])
def test_the_same_bits_every_time_and_in_graphs(m, n, k, workspace):
    o = Operands(m, n, k, True, 5)
    D, E = (torch.empty((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    o.multiply(D, n, "bf16")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        o.multiply(E, n, "bf16")
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        E.fill_(float("nan"))
        o.SA.mul_(2.0)                                              # new inputs for every replay
        D.mul_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(D, E)


@pytest.mark.gpu
def test_two_contexts_on_their_own_streams():
    o = [Operands(8, 600, 6000, True, s) for s in (6, 7)]
    D = [torch.zeros((8, 600), device="cuda") for _ in o]
    contexts, streams, kept = [], [], []
    try:
        for x in o:
            contexts.append(lib.ozaki_context_create())
            streams.append(torch.cuda.Stream())
            lib.ozaki_context_use(contexts[-1])
            need = lib.ozaki_gemm_fp8_workspace_bytes(x.m, x.n, x.k)
            kept.append(torch.empty(max(need, 256), dtype=torch.uint8, device="cuda"))
            torch.cuda.synchronize()
            lib.ozaki_set_stream(streams[-1].cuda_stream)
            lib.ozaki_set_workspace(kept[-1], kept[-1].numel())
        for _ in range(3):
            for c, x, d in zip(contexts, o, D):
                lib.ozaki_context_use(c)
                x.multiply(d, 600, "f32")
        torch.cuda.synchronize()
        for x, d in zip(o, D):
            _check(x, d, "f32")
    finally:
        lib.ozaki_context_use(None)
        for c in contexts:
            lib.ozaki_context_destroy(c)


@pytest.mark.gpu
def test_offsets_beyond_2_32():
    """Vectors whose last ones start beyond 4 GiB, on either side and in the result."""
    k, ld = 130, 1 << 17
    m = (1 << 15) + 300
    gen = torch.Generator(device="cuda").manual_seed(8)
    big = torch.full((m, ld), 0x7F, dtype=torch.uint8, device="cuda")
    q = (torch.randn((m, k), device="cuda", generator=gen) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    big[:, :k] = q.view(torch.uint8)
    small = (torch.randn((40, k), device="cuda", generator=gen) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    B = torch.zeros((40, 144), dtype=torch.uint8, device="cuda")
    B[:, :k] = small.view(torch.uint8)
    ones = torch.ones((2, m), device="cuda")
    want = q.double() @ small.double().t()
    magnitudes = q.double().abs() @ small.double().abs().t()
    cut = plain.cut_products(q, ones, False) @ plain.cut_products(small, ones[:, :40], False).t()
    ws = device.Workspace(max(lib.ozaki_gemm_fp8_workspace_bytes(m, 40, k), lib.ozaki_gemm_fp8_workspace_bytes(40, m, k)))
    ldd = 1 << 17
    D = torch.empty((m, ldd), dtype=torch.bfloat16, device="cuda")
    lib.ozaki_gemm_fp8(m, 40, k, big, ld, ones, m, B, 144, ones, m, lib.SCALE_VECTORS, D, ldd, lib.TYPE_BF16)
    assert bool(torch.all((D[:, :40].double() - want).abs() <= plain.gemm_bound(k, magnitudes, "bf16", want, cut)))
    lib.ozaki_gemm_fp8(40, m, k, B, 144, ones, m, big, ld, ones, m, lib.SCALE_VECTORS, D, ldd, lib.TYPE_BF16)
    assert bool(torch.all((D[:40, :m].double() - want.t()).abs() <= plain.gemm_bound(k, magnitudes.t(), "bf16", want.t(), cut.t())))
    ws.close()


P = 1 << 20


@pytest.mark.parametrize("position,arguments", [
    (1, dict(m=-1)), (1, dict(m=lib.MAX_EXTENT + 1)), (2, dict(n=-1)), (2, dict(n=lib.MAX_EXTENT + 1)), (3, dict(k=-1)), (3, dict(k=lib.MAX_EXTENT + 1)),
    (4, dict(A=None)), (4, dict(A=P + 8)), (5, dict(lda=304)), (5, dict(lda=301)), (5, dict(lda=lib.MAX_EXTENT + 16)), (6, dict(Sa=None)), (7, dict(ldsa=99)),
    (8, dict(B=None)), (8, dict(B=P + 1)), (9, dict(ldb=288)), (10, dict(Sb=None)), (11, dict(ldsb=1)), (11, dict(ldsb=199, scaling_b=lib.SCALE_VECTORS)),
    (12, dict(scaling_b=2)), (13, dict(D=None)), (13, dict(D=P + 1)), (14, dict(ldd=199)), (15, dict(type_d=3)), (16, dict(accumulate=2))])
def test_refusals(position, arguments):
    a = dict(m=100, n=200, k=320, A=P, lda=320, Sa=P, ldsa=100, B=P, ldb=320, Sb=P, ldsb=2, scaling_b=lib.SCALE_BLOCKS, D=P, ldd=200, type_d=lib.TYPE_BF16,
             accumulate=0)
    assert lib.ozaki_gemm_fp8(**{**a, **arguments}, check=False) == -position


def test_without_work_memory():
    m, n, k = 1, 64, 65536
    need = lib.ozaki_gemm_fp8_workspace_bytes(m, n, k)
    assert need > 0 and lib.ozaki_gemm_fp8_workspace_bytes(4096, 4096, 4096) == 0 and lib.ozaki_gemm_fp8_workspace_bytes(-1, 4, 4) == 0
    context = lib.ozaki_context_create()
    lib.ozaki_context_use(context)
    try:
        assert lib.ozaki_gemm_fp8(m, n, k, P, k, P, m, P, k, P, n, lib.SCALE_BLOCKS, P, n, lib.TYPE_BF16, check=False) == lib.STATUS_WORKSPACE
    finally:
        lib.ozaki_context_use(None)
        lib.ozaki_context_destroy(context)


def test_nothing_to_do():
    for m, n in ((0, 100), (100, 0)):
        assert lib.ozaki_gemm_fp8(m, n, 128, None, 0, None, 0, None, 0, None, 0, lib.SCALE_BLOCKS, None, 0, lib.TYPE_BF16) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("m,n,k,type_d", [(300, 500, 4096, t) for t in ("bf16", "f32", "f16")] + [(1, 64, 65536, t) for t in ("bf16", "f32", "f16")] +
                         [(5, 131, 20000, "bf16"), (3600, 3600, 128, "bf16"), (3600, 3700, 656, "f16"), (4353, 3841, 264, "bf16"), (3841, 4353, 401, "f16")])
def test_cut_and_large_products_on_top_of_what_is_there(m, n, k, type_d, blocks, workspace):
    """An inner dimension in shares, tiles of 256 x 256, and those whose last ones are left to smaller tiles: inside larger results, aligned and not."""
    assert (lib.ozaki_gemm_fp8_workspace_bytes(m, n, k) > 0) == (m <= 300)
    o = Operands(m, n, k, blocks, 15)
    for offset, ldd in ((0, plain.ceil(n, 8) + 8), (1, n + 3)):
        whole = torch.randn((m * ldd + 8,), device="cuda").to(plain.DTYPES[type_d])
        kept = whole.clone()
        view = lambda x: x[offset: offset + m * ldd].view(m, ldd)   # noqa: E731
        o.multiply(whole[offset:], ldd, type_d, 1)
        _check(o, view(whole)[:, :n], type_d, view(kept)[:, :n].double())
        assert torch.equal(view(whole)[:, n:], view(kept)[:, n:])
        assert torch.equal(whole[:offset], kept[:offset]) and torch.equal(whole[offset + m * ldd:], kept[offset + m * ldd:])


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(3600, 3700, 400), (4353, 3841, 264)])
def test_large_products_of_scales_far_apart(m, n, k, workspace):
    o = Operands(m, n, k, True, 16, wide=True)
    D = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    o.multiply(D, n, "bf16")
    _check(o, D, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,type_d", [(3600, 3700, 400, "bf16"), (4353, 3841, 264, "f16"), (300, 500, 4096, "bf16"), (1, 64, 65536, "bf16")])
def test_a_nan_code_spoils_its_row_or_column_only(m, n, k, type_d, workspace):
    for side in "AB":
        o = Operands(m, n, k, True, 17)
        D = torch.empty((m, n), dtype=plain.DTYPES[type_d], device="cuda")
        if side == "A":
            o.A[m // 2, 17] = 0x7F
        else:
            o.B[n - 1, k - 1] = 0xFF
        o.multiply(D, n, type_d)
        nan = torch.isnan(D)
        assert bool(nan[m // 2].all() if side == "A" else nan[:, n - 1].all()) and int(nan.sum()) == (n if side == "A" else m)


@pytest.mark.gpu
@pytest.mark.parametrize("blocks", [True, False])
@pytest.mark.parametrize("m,n,k", [(3600, 3700, 400), (4353, 3841, 264), (1, 64, 65536)])
def test_large_and_cut_products_have_the_same_bits_in_graphs(m, n, k, blocks, workspace):
    o = Operands(m, n, k, blocks, 18)
    D, E = (torch.empty((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        o.multiply(E, n, "bf16")
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        E.fill_(float("nan"))
        o.A[:, :k] = torch.roll(o.A[:, :k], 1, 1)                   # new inputs for every replay
        graph.replay()
        torch.cuda.synchronize()
        for _ in range(2):
            D.fill_(float("nan"))
            o.multiply(D, n, "bf16")
            assert torch.equal(D, E)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(300, 500, 4096), (1, 64, 65536)])
def test_two_contexts_with_work_memory_of_their_own(m, n, k):
    """An inner dimension in shares: calls that run at the same time meet in their own context's memory."""
    o = [Operands(m, n, k, True, s) for s in (19, 20)]
    D = [torch.zeros((m, n), device="cuda") for _ in o]
    contexts, kept = [], []
    try:
        for x in o:
            contexts.append(lib.ozaki_context_create())
            lib.ozaki_context_use(contexts[-1])
            need = lib.ozaki_gemm_fp8_workspace_bytes(m, n, k)
            assert need > 256
            kept.append((torch.empty(need, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()))
            torch.cuda.synchronize()
            lib.ozaki_set_stream(kept[-1][1].cuda_stream)
            lib.ozaki_set_workspace(kept[-1][0], need)
        for _ in range(20):
            for c, x, d in zip(contexts, o, D):
                lib.ozaki_context_use(c)
                x.multiply(d, n, "f32")
        torch.cuda.synchronize()
        for x, d in zip(o, D):
            _check(x, d, "f32")
    finally:
        lib.ozaki_context_use(None)
        for c in contexts:
            lib.ozaki_context_destroy(c)


@pytest.mark.gpu
def test_offsets_beyond_2_32_in_large_tiles():
    """Many vectors whose last ones start beyond 4 GiB, on either side and in the result."""
    k, ld, n = 130, 1 << 17, 1300
    m = (1 << 15) + 300
    gen = torch.Generator(device="cuda").manual_seed(9)
    big = torch.full((m, ld), 0x7F, dtype=torch.uint8, device="cuda")
    q = (torch.randn((m, k), device="cuda", generator=gen) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    big[:, :k] = q.view(torch.uint8)
    small = (torch.randn((n, k), device="cuda", generator=gen) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    B = torch.zeros((n, 144), dtype=torch.uint8, device="cuda")
    B[:, :k] = small.view(torch.uint8)
    ones = torch.ones((2, m), device="cuda")
    want = torch.mm(q.double(), small.double().t().contiguous())
    magnitudes = torch.mm(q.double().abs(), small.double().abs().t().contiguous())
    cut = torch.mm(plain.cut_products(q, ones, False), plain.cut_products(small, ones[:, :n], False).t().contiguous())
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    assert lib.ozaki_gemm_fp8_workspace_bytes(m, n, k) == 0
    D = torch.empty((m, ld), dtype=torch.bfloat16, device="cuda")
    lib.ozaki_gemm_fp8(m, n, k, big, ld, ones, m, B, 144, ones, m, lib.SCALE_VECTORS, D, ld, lib.TYPE_BF16)
    assert bool(torch.all((D[:, :n].double() - want).abs() <= plain.gemm_bound(k, magnitudes, "bf16", want, cut)))
    lib.ozaki_gemm_fp8(n, m, k, B, 144, ones, m, big, ld, ones, m, lib.SCALE_VECTORS, D, ld, lib.TYPE_BF16)
    assert bool(torch.all((D[:n, :m].double().t() - want).abs() <= plain.gemm_bound(k, magnitudes, "bf16", want, cut)))
