"""awe_gemm_w4 at the ends of its range, on the GPU against the definition in 64 bits: infinities, sums that pass FP32's
range although the result does not, and rows of one sign."""
import numpy as np
import pytest
import torch

from paper_2609_24519_amd import awe
from tests import quant_reference as ref
from tests.test_gpu_w4 import T, inputs

pytestmark = pytest.mark.gpu

# rows and outputs that reach every kernel: 1 or 2 x 16 rows by 1 or 2 x 16 outputs, tiles of 64, 128 and 256 outputs
SIZES = [(1, 70), (3, 4200), (40, 90), (40, 4200), (100, 5300), (260, 5300), (300, 14000), (70, 66000)]


def definition(d, K, group, rows):
    """Rows of Y in 64 bits, term by term: an infinity times 0 is NaN, and so is the sum of two of different signs."""
    g = np.arange(K) // group
    u = ref.codes(d["w"], K)
    z = d["zeros"].cpu().numpy().astype(np.int64)[:, g] if d["zeros"] is not None else 8
    x, s = ref.f64(d["x"][rows]), ref.f64(d["scales"])
    edges = np.arange(0, K, group)
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.stack([(np.add.reduceat(r * (u - z), edges, 1) * s).sum(1) for r in x])
    return y * ref.f64(d["x_scales"][rows])[:, None] if d["x_scales"] is not None else y


def check(d, K, group, y, special):
    """The special rows against the definition, infinities and NaN where they belong; the others against their bound."""
    got = awe.matmul_w4(d["x"], d["w"], d["scales"], group, d["zeros"], d["x_scales"], T[y])
    _, bound = ref.w4(d["x"], d["w"], d["scales"], group, d["zeros"], d["x_scales"])
    want = definition(d, K, group, special)
    have = ref.f64(got[special])
    for same in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(same(have), same(want)), same
    fine = np.isfinite(want)
    # computed again in 64 bits, or within the bound of the sums in FP32, which is finite wherever they are
    room = np.where(fine, np.minimum(bound[special], 2.0 ** 120), 0)
    with np.errstate(invalid="ignore"):
        off = np.abs(have - want) - room - ref.HALF[T[y]] * (np.abs(want) + room) - ref.TINY[T[y]] / 2
    assert (off[fine] <= 0).all()
    rest = np.setdiff1d(np.arange(len(d["x"])), special)
    y64, bound = ref.w4(d["x"][rest], d["w"], d["scales"], group, d["zeros"],
                        d["x_scales"][rest] if d["x_scales"] is not None else None)
    ref.close(got[rest], y64, bound, T[y])
    return want


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("x,y,zeros,K,group", [("bf16", "bf16", False, 512, 128), ("f16", "f32", True, 515, 64),
                                               ("bf16", "f32", True, 330, 32)])
def test_infinities_are_the_definitions(M, N, x, y, zeros, K, group):
    d = inputs(M, N, K, group, x, "f32", zeros, seed=M + K)
    inf = float("inf")
    special = sorted({0, M // 2, M - 1, min(M - 1, 17)})
    for i, r in enumerate(special):
        d["x"][r, (7 * r + 3) % K] = inf if i % 2 else -inf
        if i == 2:
            d["x"][r, K - 1] = inf  # beside one of the other sign, at an odd K beside no code
            d["x"][r, 5] = -inf
        if i == 3:
            d["x"][r, K // 2] = float("nan")
    want = check(d, K, group, y, special)
    assert np.isinf(want).any() and np.isnan(want).any()  # (where the code is the zero point)


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("y,zeros,K,group", [("f32", False, 512, 128), ("f32", True, 515, 64), ("bf16", True, 330, 32)])
def test_sums_past_the_range_of_fp32(M, N, y, zeros, K, group):
    # elements of 2^119 to 2^127 whose products with the codes pass FP32's range, and results that do not
    d = inputs(M, N, K, group, "bf16", "f32", zeros, seed=M + K + 1)
    d["scales"] *= 2.0 ** -20
    special = sorted({0, M // 2, M - 1, min(M - 1, 17)})
    g = torch.Generator().manual_seed(M)
    for i, r in enumerate(special):
        d["x"][r] = (torch.randn(K, generator=g) * 2.0 ** (119 + 2 * i)).bfloat16().cuda()
    want = check(d, K, group, y, special)
    assert np.isfinite(want).all()


@pytest.mark.parametrize("M,N", [(1, 70), (40, 4200), (300, 14000)])
def test_scales_that_pass_the_range_before_the_rows_scale(M, N):
    # int8 rows: a group's sum times its scale passes FP32's range, times the row's scale it does not
    K, group = 512, 128
    d = inputs(M, N, K, group, "i8", "f32", True, seed=M)
    d["scales"] *= 2.0 ** 125
    d["x_scales"] *= 2.0 ** -40
    assert np.isfinite(check(d, K, group, "f32", sorted({0, M // 2, M - 1}))).all()


@pytest.mark.parametrize("M,N", SIZES[:6])
@pytest.mark.parametrize("x,y", [("bf16", "f32"), ("f16", "f32"), ("f16", "f16"), ("i8", "f32")])
@pytest.mark.parametrize("zeros,K,group", [(False, 1024, 128), (True, 700, 32)])
def test_rows_of_one_sign(M, N, x, y, zeros, K, group):
    # a large mean, where codes that carry a bias cost most digits
    d = inputs(M, N, K, group, x, "f32", zeros, seed=M + 2)
    d["x"] = (d["x"].float().abs() + 100).clamp(max=127).to(T[x])
    d["scales"] /= 64
    got = awe.matmul_w4(d["x"], d["w"], d["scales"], group, d["zeros"], d["x_scales"], T[y])
    want, bound = ref.w4(d["x"], d["w"], d["scales"], group, d["zeros"], d["x_scales"])
    ref.close(got, want, bound, T[y])


@pytest.mark.parametrize("M,N", [(3, 4200), (260, 5300)])
def test_infinities_under_capture_and_in_strided_rows(M, N):
    # the second computation reads operands as they lie in memory, and runs inside a captured graph
    K, group = 333, 64
    d = inputs(M, N, K, group, "bf16", "f32", True, seed=5)

    def inside(t, lead, extra):
        big = torch.zeros(lead + t.shape[0] * (t.shape[1] + extra), dtype=t.dtype, device="cuda")
        v = big[lead:].view(t.shape[0], t.shape[1] + extra)[:, : t.shape[1]]
        v.copy_(t)
        return v

    for name in ("x", "w", "scales", "zeros"):
        d[name] = inside(d[name], 1, 3)
    awe.matmul_w4(d["x"], d["w"], d["scales"], group, d["zeros"], None, torch.float32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = awe.matmul_w4(d["x"], d["w"], d["scales"], group, d["zeros"], None, torch.float32)
    for k in range(3):
        d["x"][M // 2, 11 * k + 1] = float("inf") if k % 2 else float("-inf")
        d["x"][M - 1] = (torch.randn(K, generator=torch.Generator().manual_seed(k)) * 2.0 ** 112).bfloat16().cuda()
        graph.replay()
        torch.cuda.synchronize()
        check(d, K, group, "f32", [M // 2, M - 1])
        eager = awe.matmul_w4(d["x"], d["w"], d["scales"], group, d["zeros"], None, torch.float32)
        assert torch.equal(torch.nan_to_num(y, nan=1.25), torch.nan_to_num(eager, nan=1.25))


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("x,K,group", [("bf16", 1100, 128), ("f16", 515, 64), ("bf16", 650, 32)])
def test_rows_of_infinities(M, N, x, K, group):
    # whole rows of infinities: their sign where all codes lie on one side of the zero point, times the scale's
    d = inputs(M, N, K, group, x, "f32", False, seed=M + K + 2)
    d["w"][0::5], d["w"][1::5], d["w"][2::5] = 0xff, 0x00, 0x88
    d["scales"][0::10] *= -1
    d["scales"][4::20, 0] = 0
    special = sorted({0, M - 1, M // 2})
    for i, r in enumerate(special):
        d["x"][r] = float("-inf") if i % 2 else float("inf")
        if i == 2:
            d["x"][r, : K // 2] = 1.0  # infinities in the second half alone
    want = check(d, K, group, "f32", special)
    assert np.isposinf(want).any() and np.isneginf(want).any() and np.isnan(want).any()
