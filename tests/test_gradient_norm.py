"""ozaki_gradient_norm and ozaki_clip_gradients against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

from low_precision import DTYPES, ROUNDING  # noqa: E402
from paper_2508_00441_amd import binding as lib, device  # noqa: E402

NAMES = list(DTYPES)
#: sixteen squares added one after another and eight such sums, each time half a unit in the last place, of which the root halves what they come to, and its own rounding
OFF = (0.5 * (16 + 3 + 1) + 1) * 2.0 ** -24


def _tensors(sizes, seed=0, spread=1.0, shift=0):
    """Tensors of alternating types; `shift` elements into a larger allocation."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        whole = (spread * torch.randn((n + shift,), device="cuda", generator=gen)).to(DTYPES[NAMES[i % 3]])
        out.append(whole[shift:])
    return out


def _types(tensors):
    return [lib.TYPES[next(name for name in NAMES if DTYPES[name] == x.dtype)] for x in tensors]


def _norm(tensors, scale):
    return abs(scale) * math.sqrt(math.fsum(float(x.double().square().sum()) for x in tensors))


def _clip(tensors, scale, max_norm, out=None, norm=None, given=0):
    out = [torch.full_like(x, float("nan")) for x in tensors] if out is None else out
    norm = torch.full((1,), float("nan"), device="cuda") if norm is None else norm
    lib.ozaki_clip_gradients(len(tensors), tensors, [x.numel() for x in tensors], _types(tensors), scale, max_norm, out, norm, given)
    return out, norm


def _check(tensors, scale, max_norm, out, norm):
    want = _norm(tensors, scale)
    assert abs(float(norm) - want) <= OFF * want
    factor = scale * (min(1.0, max_norm / want) if want > 0 else 1.0)
    for x, y in zip(tensors, out):
        rel, tiny = ROUNDING[NAMES[_types([x])[0]]]
        exact = x.double() * factor
        # the norm, the quotient, its product with the scale, the product with the element
        off = (OFF + 4 * 2.0 ** -24) * exact.abs() + 2.0 ** -149
        assert bool(torch.all((y.double() - exact).abs() <= off + rel * (exact.abs() + off) + tiny))


@pytest.fixture()
def workspace():
    ws = device.Workspace(8 << 20)
    yield ws
    ws.close()


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("sizes", [[1], [3, 1, 2], [32768, 32769, 32767], [100003, 5, 4096, 0, 1000], [7] * 95, [130] * 96, [1001] * 97, [9, 40000] * 150, [3_000_001, 2_000_003, 64]])
def test_norm_and_clip(sizes, shift, workspace):
    x = _tensors(sizes, seed=len(sizes) + shift, shift=shift)
    norm = torch.full((1,), float("nan"), device="cuda")
    for scale, max_norm in ((1.0, 0.5), (1.0, 1e9), (0.25, 2.0), (-0.5, 1.0)):
        lib.ozaki_gradient_norm(len(x), x, [v.numel() for v in x], _types(x), scale, norm)
        out, again = _clip(x, scale, max_norm)
        assert torch.equal(norm, again)
        _check(x, scale, max_norm, out, again)


@pytest.mark.gpu
def test_in_place_and_given(workspace):
    x = _tensors([50000, 33, 1000], seed=4)
    copies = [v.clone() for v in x]
    out, norm = _clip(x, 1.0, 3.0)
    _clip(copies, 1.0, 3.0, out=copies)
    assert all(torch.equal(a, b) for a, b in zip(out, copies))
    # a norm that the caller has, of more than these tensors; without work memory
    lib.ozaki_set_workspace(None, 0)
    other = torch.full((1,), 1000.0, device="cuda")
    out, norm = _clip(x, 1.0, 3.0, norm=other, given=1)
    assert float(norm) == 1000.0
    for a, b in zip(x, out):
        assert torch.equal((a.float() * (torch.tensor(3.0) / torch.tensor(1000.0)).cuda()).to(a.dtype), b)
    # within bounds nothing is written where results go to where the elements are
    same = [v.clone() for v in x]
    _clip(same, 1.0, 3.0, out=same, norm=torch.full((1,), 2.0, device="cuda"), given=1)
    assert all(torch.equal(a, b) for a, b in zip(x, same))


@pytest.mark.gpu
def test_large_small_and_not_finite(workspace):
    big = torch.full((70000,), 2.0 ** 100, device="cuda")
    out, norm = _clip([big], 1.0, 1.0)
    _check([big], 1.0, 1.0, out, norm)
    small = torch.full((70000,), 2.0 ** -120, device="cuda")
    _, norm = _clip([small], 1.0, 1.0)
    assert abs(float(norm) - _norm([small], 1.0)) <= OFF * _norm([small], 1.0)
    zeros = torch.zeros((5000,), device="cuda")
    out, norm = _clip([zeros], 1.0, 0.0)
    assert float(norm) == 0.0 and bool(torch.all(out[0] == 0))
    for bad, check in ((float("inf"), lambda y: bool(torch.all(y[1:] == 0)) and bool(torch.isnan(y[0]))), (float("nan"), lambda y: bool(torch.isnan(y).all()))):
        x = torch.ones((40000,), device="cuda")
        x[0] = bad
        out, norm = _clip([x], 1.0, 1.0)
        assert check(out[0]) and (math.isinf(float(norm)) if math.isinf(bad) else math.isnan(float(norm)))


@pytest.mark.gpu
@pytest.mark.parametrize("element,scale", [(2.0 ** 60, 2.0 ** -110), (2.0 ** 60, -1.5 * 2.0 ** -140), (2.0 ** 100, 2.0 ** -40), (2.0 ** 50, 3.0 * 2.0 ** 60), (2.0 ** -50, 2.0 ** 100),
                                           (2.0 ** -60, 2.0 ** 127), (2.0 ** -100, -1.25 * 2.0 ** 90), (2.0 ** -60, 2.0 ** -50), (1.0, 2.0 ** -120), (1.0, 2.0 ** 110)])
def test_scales_far_from_one(element, scale, workspace):
    """Norms in 32 bits' range of elements whose squares are not, with scales that leave it on the way: 2^60 times 2^-110 as well as 2^-50 times 2^100."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    x = [element * torch.randn((n,), device="cuda", generator=gen) for n in (70001, 3)]
    norm, want = torch.zeros((1,), device="cuda"), _norm(x, scale)
    assert 2.0 ** -126 < want < 2.0 ** 128
    lib.ozaki_gradient_norm(len(x), x, [v.numel() for v in x], _types(x), scale, norm)
    assert abs(float(norm) - want) <= OFF * want


@pytest.mark.gpu
@pytest.mark.parametrize("element,scale", [(1.0, 2.0 ** 127), (2.0 ** 100, 2.0 ** 60), (-(2.0 ** 127), 1.5)])
def test_norms_beyond_32_bits_are_infinite(element, scale, workspace):
    """... of finite elements too, which become zero."""
    x = torch.full((70000,), element, device="cuda")
    (out,), norm = _clip([x], scale, 1.0)
    assert math.isinf(float(norm)) and float(norm) > 0 and bool(torch.all(out == 0))


@pytest.mark.gpu
@pytest.mark.parametrize("element,scale,max_norm", [(2.0 ** 100, 1.0, 2.0 ** -40), (2.0 ** 100, 1.0, 3 * 2.0 ** -60), (2.0 ** 110, 0.75, 2.0 ** -100), (2.0 ** 100, -(2.0 ** -100), 2.0 ** -60),
                                                    (2.0 ** 90, 2.0 ** -90, 2.0 ** -50), (2.0 ** 60, 2.0 ** 50, 2.0 ** -70), (1.0, 1.0, 0.0)])
def test_factors_below_the_normal_numbers(element, scale, max_norm, workspace):
    """max_norm / norm, or its product with the scale, has few bits in 32 bits or none; the results, of a norm of max_norm, have all of theirs."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    x = [(element * torch.randn((n,), device="cuda", generator=gen)).to(dtype) for n, dtype in ((5001, torch.float32), (3, torch.float32), (4099, torch.bfloat16))]
    out, norm = _clip(x, scale, max_norm)
    assert math.isfinite(float(norm))
    _check(x, scale, max_norm, out, norm)
    in_place = [v.clone() for v in x]
    _clip(in_place, scale, max_norm, out=in_place)
    assert all(torch.equal(a, b) for a, b in zip(in_place, out))


@pytest.mark.gpu
def test_nothing(workspace):
    norm = torch.full((1,), 7.0, device="cuda")
    lib.ozaki_gradient_norm(0, None, None, None, 1.0, norm)
    assert float(norm) == 0.0
    norm.fill_(7.0)
    lib.ozaki_clip_gradients(2, [0, 0], [0, 0], [0, 1], 1.0, 1.0, [0, 0], norm)
    assert float(norm) == 0.0


@pytest.mark.gpu
def test_in_a_graph(workspace):
    x = _tensors([200000, 77, 5000] * 40, seed=6)
    sizes, types = [v.numel() for v in x], _types(x)
    out, norm = [torch.zeros_like(v) for v in x], torch.zeros((1,), device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
        lib.ozaki_clip_gradients(len(x), x, sizes, types, 1.0, 1.0, out, norm)
    lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
    for step in range(3):
        for v in x:
            v.mul_(0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, want_norm = _clip(x, 1.0, 1.0)
        torch.cuda.synchronize()
        assert torch.equal(norm, want_norm) and all(torch.equal(a, b) for a, b in zip(out, want))


#: of one tensor and of many: five squares of a thread one after another and three additions of such sums, each half a unit in the last place, of which the root halves what they come to;
#: its own rounding; pairs of numbers from there on (2^-40 is more than all of theirs)
NEAR = (0.5 * (5 + 3) + 1) * 2.0 ** -24 + 2.0 ** -40


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[1], [2047], [2048], [2049], [8191], [8191 + 8192], [4_200_000 - 1], [8192 * 600 - 1], [8_400_001], [7] * 143, [130] * 144, [1001] * 145, [9, 0, 4000] * 96, [3] * 287, [5] * 288,
                                   [2049, 1] * 144 + [77]])
def test_tables_and_chunks(sizes, workspace):
    """Tensors as many as a launch's table holds, one fewer and one more, of one table and of two; chunks that end before, at and behind a piece's end."""
    x = _tensors(sizes, seed=sum(sizes))
    for scale, max_norm in ((1.0, 0.5), (-0.375, 1e9)):
        out, norm = _clip(x, scale, max_norm)
        _check(x, scale, max_norm, out, norm)
        want = _norm(x, scale)
        assert abs(float(norm) - want) <= NEAR * want
        again = [v.clone() for v in x]
        _, norm_again = _clip(again, scale, max_norm, out=again)
        assert torch.equal(norm, norm_again) and all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.gpu
@pytest.mark.parametrize("count", [9215, 9216, 9217, 9500])
def test_thousands_of_tensors(count):
    """64 launches, behind which the second reading goes forwards, and more; whole numbers, whose squares are added without a rounding."""
    ws = device.Workspace(lib.ozaki_gradient_norm_workspace_bytes(count))
    gen = torch.Generator(device="cuda").manual_seed(count)
    whole = torch.randint(-3, 4, (count * 6,), device="cuda", generator=gen).float()
    sizes = [1 + i % 5 for i in range(count)]
    x = [whole[6 * i: 6 * i + n] for i, n in enumerate(sizes)]
    held = torch.full_like(whole, float("nan"))
    out = [held[6 * i: 6 * i + n] for i, n in enumerate(sizes)]
    _, norm = _clip(x, 1.0, 1.0, out=out)
    inside = torch.arange(6, device="cuda").repeat(count) < torch.tensor(sizes, device="cuda").repeat_interleave(6)
    square = float((whole.double() ** 2)[inside].sum())
    assert abs(float(norm) - square ** 0.5) <= 2.0 ** -24 * square ** 0.5
    want = whole * (torch.ones((1,), device="cuda") / norm)
    assert torch.equal(held[inside], want[inside]) and bool(torch.isnan(held[~inside]).all())
    _clip(x, 1.0, 1.0, out=x)
    assert torch.equal(whole[inside], want[inside])
    ws.close()


FAKE = 1 << 20


def test_refusals():
    norm = [2, [FAKE, FAKE], [4, 4], [0, 1], 1.0, FAKE]
    for at, value in ((1, -1), (2, None), (2, [FAKE, None]), (2, [FAKE + 2, FAKE]), (2, [FAKE, FAKE + 1]), (3, None), (3, [4, -1]), (3, [4, 2 ** 38 + 1]), (4, None), (4, [0, 3]), (5, float("nan")),
                      (5, float("inf")), (6, None), (6, FAKE + 2)):
        args = list(norm)
        args[at - 1] = value
        assert lib.ozaki_gradient_norm(*args, check=False) == -at, (at, value)
    clip = [2, [FAKE, FAKE], [4, 4], [0, 1], 1.0, 1.0, [FAKE, FAKE], FAKE, 0]
    for at, value in ((1, -1), (2, [FAKE, None]), (3, [-1, 4]), (4, [3, 0]), (5, float("nan")), (6, float("nan")), (6, -1.0), (7, None), (7, [FAKE, None]), (7, [FAKE + 2, FAKE]), (8, None),
                      (8, FAKE + 1), (9, 2)):
        args = list(clip)
        args[at - 1] = value
        assert lib.ozaki_clip_gradients(*args, check=False) == -at, (at, value)
    lib.ozaki_set_workspace(None, 0)
    assert lib.ozaki_gradient_norm(*norm, check=False) == lib.STATUS_WORKSPACE
    assert lib.ozaki_gradient_norm_workspace_bytes(-1) == 0 and lib.ozaki_gradient_norm_workspace_bytes(0) > 0


def test_more_than_a_call_counts():
    """Chunks and partial sums are counted in 32 bits: 144 tensors of 2^38 elements would be more than 2^32 chunks."""
    lib.ozaki_set_workspace(None, 0)
    most = 2 ** 38
    for count, answer in ((32, lib.STATUS_WORKSPACE), (33, -3), (144, -3)):
        assert lib.ozaki_gradient_norm(count, [FAKE] * count, [most] * count, [1] * count, 1.0, FAKE, check=False) == answer
        assert lib.ozaki_clip_gradients(count, [FAKE] * count, [most] * count, [1] * count, 1.0, 1.0, [FAKE] * count, FAKE, check=False) == answer
    assert lib.ozaki_gradient_norm((1 << 27) + 1, [FAKE], [4], [1], 1.0, FAKE, check=False) == -1
    assert lib.ozaki_gradient_norm_workspace_bytes((1 << 27) + 1) == 0 < lib.ozaki_gradient_norm_workspace_bytes(1 << 27)


@pytest.mark.gpu
def test_beyond_32_bits(workspace):
    x = torch.zeros(((1 << 31) + 70001,), dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.tensor([3.0, -4.0, 12.0])
    x[5] = 84.0
    out, norm = _clip([x], 1.0, 17.0)
    assert float(norm) == 85.0                                      # (5, 12, 13 and 13, 84, 85)
    factor = torch.tensor(17.0) / torch.tensor(85.0)
    assert torch.equal(out[0][-3:].cpu(), (torch.tensor([3.0, -4.0, 12.0]) * factor).bfloat16()) and float(out[0][5]) == float((84.0 * factor).bfloat16())
    assert int((out[0] != 0).sum()) == 4
