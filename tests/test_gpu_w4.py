"""awe_gemm_w4 on the GPU against the definition in 64 bits: types, groups, odd sizes, strides and alignment,
exact cases bit for bit, infinities and NaN, graphs and streams."""
import numpy as np
import pytest
import torch

from paper_2609_24519_amd import awe
from tests import quant_reference as ref

pytestmark = pytest.mark.gpu

T = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8}


def inputs(M, N, K, group, x="bf16", s="f32", zeros=False, x_scales=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(M, K, generator=g)
    d = {"x_scales": None, "zeros": None}
    if x == "i8":
        d["x"] = torch.randint(-128, 128, (M, K), generator=g, dtype=torch.int8)
        if x_scales:
            d["x_scales"] = (0.5 + torch.rand(M, generator=g)) / 64
    else:
        d["x"] = X.to(T[x])
    d["w"] = torch.randint(0, 256, (N, (K + 1) // 2), generator=g, dtype=torch.uint8)
    G = -(-K // group)
    d["scales"] = ((0.25 + torch.rand(N, G, generator=g)) / 16).to(T[s])
    if zeros:
        d["zeros"] = torch.randint(0, 17, (N, G), generator=g, dtype=torch.uint8)
    return {k: v.cuda() if v is not None else None for k, v in d.items()}


def check(d, group, y):
    got = awe.matmul_w4(d["x"], d["w"], d["scales"], group, d["zeros"], d["x_scales"], T[y])
    want, bound = ref.w4(d["x"], d["w"], d["scales"], group, d["zeros"], d["x_scales"])
    ref.close(got, want, bound, T[y])
    return got


@pytest.mark.parametrize("x,s,y,zeros", [("bf16", "bf16", "bf16", False), ("bf16", "f32", "f32", True),
                                         ("f16", "f16", "f16", True), ("f16", "f32", "f32", False),
                                         ("i8", "f32", "bf16", True), ("i8", "f16", "f32", False),
                                         ("i8", "bf16", "f16", True)])
@pytest.mark.parametrize("M,N,K,group", [(1, 1, 1, 32), (1, 256, 256, 32), (3, 17, 33, 32), (2, 70, 511, 64),
                                         (16, 128, 1024, 128), (17, 33, 257, 96), (40, 200, 640, 320),
                                         (64, 64, 2049, 2049), (65, 130, 300, 512), (130, 257, 384, 128),
                                         (300, 129, 1000, 64), (257, 260, 2304, 256), (1, 515, 4100, 128)])
def test_types_and_sizes(M, N, K, group, x, s, y, zeros):
    check(inputs(M, N, K, group, x, s, zeros, seed=M + N + K), group, y)


@pytest.mark.parametrize("x", ["bf16", "f16", "i8"])
@pytest.mark.parametrize("M,N,K,group", [(1, 100, 1000, 32), (5, 64, 2048, 128), (33, 100, 777, 160), (64, 96, 512, 64),
                                         (150, 140, 1111, 128), (256, 256, 1024, 32), (512, 384, 640, 640),
                                         (150, 5000, 1111, 128), (256, 2200, 1024, 32), (100, 5300, 320, 64),
                                         (800, 900, 384, 64), (1000, 650, 300, 512), (700, 790, 1024, 32)])
@pytest.mark.parametrize("zeros", [False, True])
def test_exact_sums(M, N, K, group, x, zeros):
    # small whole numbers and scales that are powers of two: every sum is exact in FP32, in any order
    g = torch.Generator().manual_seed(M * N + K)
    d = inputs(M, N, K, group, "i8", "f32", zeros, x_scales=False, seed=M)
    d["x"] = torch.randint(-4, 5, (M, K), generator=g).to(T[x]).cuda()
    d["scales"] = torch.tensor([0.25, 0.5, 1.0, 2.0])[torch.randint(0, 4, d["scales"].shape, generator=g)].cuda()
    got = awe.matmul_w4(d["x"], d["w"], d["scales"], group, d["zeros"], None, torch.float32)
    want, _ = ref.w4(d["x"], d["w"], d["scales"], group, d["zeros"])
    assert np.abs(want).max() * 4 < 2 ** 22 and np.array_equal(ref.f64(got), want)


@pytest.mark.parametrize("x,zeros", [("bf16", True), ("f16", False), ("i8", True)])
@pytest.mark.parametrize("M,N,K,group", [(3, 4200, 300, 64), (16, 5000, 1100, 128), (40, 4200, 260, 32), (40, 4100, 520, 128),
                                         (65, 16400, 130, 32), (65, 16400, 300, 64), (70, 32900, 300, 128),
                                         (65, 32800, 450, 64), (65, 65600, 257, 128), (66, 65600, 384, 64)])
def test_many_outputs(M, N, K, group, x, zeros):
    # sizes at which workgroups have 32, 128 and 256 outputs, one or two of them per CU
    d = inputs(M, N, K, group, x, "bf16", zeros, seed=N)
    check(d, group, "f32")


@pytest.mark.parametrize("M,N", [(1, 75), (2, 75), (16, 75), (20, 75), (50, 75), (100, 75), (300, 75), (70, 6001), (300, 2005)])
@pytest.mark.parametrize("x", ["bf16", "i8"])
def test_strides_and_alignment(M, N, x):
    # every operand inside a larger buffer at odd offsets, with guards that must stay
    K, group = 333, 64
    G = -(-K // group)
    d = inputs(M, N, K, group, x, "f16", True, seed=M)
    want, bound = ref.w4(d["x"], d["w"], d["scales"], group, d["zeros"], d["x_scales"])

    def inside(t, lead, extra):
        big = torch.zeros(lead + t.shape[0] * (t.shape[1] + extra), dtype=t.dtype, device="cuda")
        v = big[lead:].view(t.shape[0], t.shape[1] + extra)[:, : t.shape[1]]
        v.copy_(t)
        return v

    for lead, extra in ((1, 0), (1, 1), (3, 5), (0, 16)):
        X, W, S, Z = (inside(d[n], lead, extra) for n in ("x", "w", "scales", "zeros"))
        guard = torch.full((lead + M * (N + 3) + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
        Y = guard[lead: lead + M * (N + 3)].view(M, N + 3)
        awe.gemm_w4(M, N, K, X, K + extra, awe._dtype(X.dtype, (awe.BF16, awe.I8)), d["x_scales"], W,
                    W.shape[1] + extra, S, G + extra, awe.F16, Z, G + extra, group, Y, N + 3, awe.BF16)
        ref.close(Y[:, :N], want, bound, torch.bfloat16)
        assert bool((Y[:, N:] == 7).all()) and bool((guard[:lead] == 7).all()) and bool((guard[-8:] == 7).all())


@pytest.mark.parametrize("x", ["bf16", "f16", "i8"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N", [(1, 40), (9, 5000), (33, 4200), (70, 200)])
@pytest.mark.parametrize("lead_x,extra_x,lead_w,extra_w", [(0, 1, 0, 0), (1, 4, 0, 4), (0, 4, 0, 1), (4, 8, 1, 4), (3, 2, 2, 2)])
def test_rows_off_words(M, N, group, x, lead_x, extra_x, lead_w, extra_w):
    # every way in which rows of X and W lie off multiples of 4 bytes; all sums are exact
    K = 1096
    g = torch.Generator().manual_seed(M + group + lead_x)
    d = inputs(M, N, K, group, "i8", "f32", True, x_scales=False, seed=M)
    d["x"] = torch.randint(-4, 5, (M, K), generator=g).to(T[x]).cuda()
    d["scales"] = torch.tensor([0.25, 0.5, 1.0, 2.0])[torch.randint(0, 4, d["scales"].shape, generator=g)].cuda()

    def inside(t, lead, extra):
        big = torch.zeros(lead + t.shape[0] * (t.shape[1] + extra), dtype=t.dtype, device="cuda")
        v = big[lead:].view(t.shape[0], t.shape[1] + extra)[:, : t.shape[1]]
        v.copy_(t)
        return v

    got = awe.matmul_w4(inside(d["x"], lead_x, extra_x), inside(d["w"], lead_w, extra_w), d["scales"], group, d["zeros"],
                        None, torch.float32)
    want, _ = ref.w4(d["x"], d["w"], d["scales"], group, d["zeros"])
    assert np.abs(want).max() * 4 < 2 ** 22 and np.array_equal(ref.f64(got), want)


@pytest.mark.parametrize("M,N", [(3, 40), (40, 700), (70, 7800)])
def test_offsets_past_32_bits(M, N):
    # rows of W and Y so far apart that the last ones lie past 4 GiB
    K, group = 384, 128
    d = inputs(M, N, K, group, "bf16", "f32", True, seed=N)
    ldw = min((1 << 24) - 4, ((5 << 30) // N + 3) // 4 * 4)
    big = torch.empty(N * ldw, dtype=torch.uint8, device="cuda")
    w = big.view(N, ldw)[:, : K // 2]
    w.copy_(d["w"])
    ldy = (5 << 30) // 2 // M
    y = torch.empty(M * ldy, dtype=torch.bfloat16, device="cuda").view(M, ldy)[:, :N]
    awe.gemm_w4(M, N, K, d["x"], K, awe.BF16, None, w, ldw, d["scales"], 3, awe.F32, d["zeros"], 3, group, y, ldy, awe.BF16)
    want, bound = ref.w4(d["x"], d["w"], d["scales"], group, d["zeros"])
    ref.close(y, want, bound, torch.bfloat16)


def test_empty_reduction_writes_zeros():
    for M in (1, 70):
        x, w = torch.zeros(M, 0, dtype=torch.bfloat16, device="cuda"), torch.zeros(9, 0, dtype=torch.uint8, device="cuda")
        y = awe.matmul_w4(x, w, torch.zeros(9, 0, device="cuda"), 32)
        assert y.shape == (M, 9) and bool((y == 0).all())
    d_scales = torch.full((70,), float("inf"), device="cuda")
    y = awe.matmul_w4(x.to(torch.int8), w, torch.zeros(9, 0, device="cuda"), 32, x_scales=d_scales)
    assert bool((y == 0).all())
    assert awe.matmul_w4(x[:0], w, torch.zeros(9, 0, device="cuda"), 32).shape == (0, 9)


@pytest.mark.parametrize("M,N", [(4, 140), (30, 140), (100, 140), (260, 140), (100, 5200), (260, 2200)])
def test_nan_and_infinity_stay_in_their_row(M, N):
    K, group = 512, 128
    d = inputs(M, N, K, group, "bf16", "f32", False, seed=3)
    clean = check(d, group, "bf16")
    d["x"][1, 7] = float("nan")
    d["x"][2, K - 1] = float("inf")
    y = awe.matmul_w4(d["x"], d["w"], d["scales"], group)
    assert bool(torch.isnan(y[1]).all()) and not bool(torch.isfinite(y[2]).any())
    keep = [i for i in range(M) if i not in (1, 2)]
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("x,power", [("bf16", -130), ("f16", -20)])
@pytest.mark.parametrize("M,N", [(3, 80), (40, 80), (100, 80), (100, 5200)])
def test_subnormal_rows(M, N, x, power):
    # elements below the type's smallest normal number count in full
    K, group = 512, 128
    d = inputs(M, N, K, group, x, "f32", True, seed=4)
    d["x"][:] = (d["x"].float() * 2.0 ** power).to(T[x])
    d["scales"] *= 2.0 ** 60
    check(d, group, "f32")


def test_scales_of_zero_and_far_apart():
    # a group whose scale is 0 adds nothing, whatever its neighbours' scales are
    K, group = 512, 128
    for m, N in ((1, 70), (80, 70), (80, 5600)):
        d = inputs(m, N, K, group, "bf16", "f32", True, seed=5)
        d["scales"][:, 1] = 0
        d["scales"][::2, 2] = 2.0 ** 60
        d["scales"][1::3, 0] = 2.0 ** -70
        check(d, group, "f32")


@pytest.mark.parametrize("M,N", [(1, 130), (48, 130), (200, 130), (200, 2500)])
def test_rows_do_not_depend_on_the_others(M, N):
    d = inputs(M, N, 700, 64, "f16", "f32", True, seed=9)
    a = check(d, 64, "f32")
    b = check(d, 64, "f32")
    assert torch.equal(a, b)
    d["x"][: M - 1] = 0
    assert torch.equal(check(d, 64, "f32")[M - 1], a[M - 1])


def test_graph_replays_and_streams():
    cases = [(1, 256, 512, 32, "bf16"), (20, 300, 512, 128, "i8"), (200, 300, 512, 128, "bf16"),
             (200, 2500, 512, 128, "bf16")]
    sets = [(inputs(M, N, K, g, x, seed=i), g) for i, (M, N, K, g, x) in enumerate(cases)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = [awe.matmul_w4(d["x"], d["w"], d["scales"], g, None, d["x_scales"], torch.float32) for d, g in sets]
    for k in range(3):
        for d, _ in sets:
            d["w"].random_(0, 256)
        graph.replay()
        eager = [awe.matmul_w4(d["x"], d["w"], d["scales"], g, None, d["x_scales"], torch.float32) for d, g in sets]
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b), k
