"""Attention over the int8 cache at the ends of its range, on the GPU against 64 bits: large finite scores, and values
whose blocks differ in size by more than a weight's digits."""
import numpy as np
import pytest
import torch

from paper_2609_24519_amd import awe
from tests import quant_reference as ref
from tests.test_gpu_cache import T, WIDE, batch_of, tables, upload

pytestmark = pytest.mark.gpu


def attend(held, table, counts, lengths, q, scale, causal, wide):
    """wide: the rows kernel, otherwise the tokens are split (over workgroups, where there are many)."""
    n, dev, bounds = q.shape[0], q.cuda(), {}
    if wide:
        bounds = dict(rows=WIDE, max_rows=WIDE)
        dev = torch.cat([dev, torch.zeros(WIDE - n, *q.shape[1:], dtype=q.dtype, device="cuda")])
    return awe.attend(upload(held), batch_of(counts, lengths, table, **bounds), dev, scale, causal=causal)[:n]


def reference(held, blocks, length, q, scale, causal, weight):
    """One sequence in 64 bits: (out, bound before the result's own rounding), rows x heads x dim.  weight: what the
    rounding of a weight may be, relative to it.

    R bounds what a token's weight is off by beside that, relative to it: its score's error (as in test_large_scores,
    with two more roundings for the difference from the maximum), four sums of logarithms of size A at most (the
    scales' and the 2^15 of FP16), exp2 (an ulp, 2 U) of the weight and of the factor that takes a step's sum to
    the others', and additions: 32 in a matrix instruction, 64 of waves and parts, and for each step of 64 tokens a
    rescaling (exp2, two products, the addition: 5 U).  It counts in the numerator and in the denominator.  FP16
    holds a weighted token to 2^-40 of the row's largest weighted block, times at most 127.  A weight below 2^-126
    of the largest is no normal number of FP32, and exp2 gives 0 for it: where parts of the tokens meet, such tokens
    may count as nothing."""
    n, heads, D = q.shape
    share = heads // held.heads
    k, v = held.values(blocks, length, "k"), held.values(blocks, length, "v")
    of = np.array([int(blocks[p // held.block]) for p in range(length)])
    out, bound = np.zeros((n, heads, D)), np.zeros((n, heads, D))
    for i in range(n):
        see = min(length, length - n + i + 1) if causal else length
        for h in range(heads if see > 0 else 0):
            K, V, vs = k[h // share, :see], v[h // share, :see], held.vs[of[:see], h // share].astype(np.float64)
            score = K @ q[i, h] * scale
            p = np.exp(score - score.max())
            p /= p.sum()
            out[i, h] = p @ V
            err = (32 + D / 32 + 8) * ref.U * (np.abs(K) @ np.abs(q[i, h]) * abs(scale))
            A = 15 + 2 * np.abs(np.log2(vs[vs > 0])).max(initial=0)
            R = err + (4 * A + 4 + 32 + 64 + 5 * see / 64) * ref.U
            size = (p * (weight + R)) @ np.abs(V) + (p * R).sum() * np.abs(out[i, h])
            size += np.where(p < 2.0 ** -126 * p.max(), p, 0) @ np.abs(V)
            bound[i, h] = 1.01 * (size + see * 2.0 ** -40 * (p * vs).max() * 127)
    return out, bound


ONE = 2.0 ** -11  # weights as one FP16 number
TWO = 2.0 ** -22  # as two, the number and what its rounding left


@pytest.mark.parametrize("new,length,wide", [(1, 200, False), (40, 200, False), (40, 200, True), (1, 5000, False)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("t,ratio", [("bf16", 1e3), ("bf16", 1e9), ("bf16", 1e12), ("bf16", 1e30), ("f16", 1e4)])
def test_large_values_without_weight_cost_the_others_nothing(t, ratio, dim, new, length, wide):
    # blocks of large values whose tokens get no weight (scores of -6000 and less), before and among the others
    block, heads, share = 16, 2, 2
    nb = -(-length // block) + 1
    held = ref.Held(nb, heads, dim, block, seed=dim)
    table = tables([length], block, nb, 2)
    g = torch.Generator().manual_seed(dim + new)
    q = (torch.rand(new, heads * share, dim, generator=g) + 0.5).to(T[t])
    held.k[:] = np.abs(held.k) // 4
    for b in (0, 5):
        held.k[table[0][b]] = -127
        held.ks[table[0][b]] *= 400
        held.vs[table[0][b]] *= np.float32(ratio)
    got = attend(held, table, [new], [length], q, 0.5, True, wide)
    want, bound = reference(held, table[0], length, ref.f64(q), 0.5, True, ONE)
    assert (np.abs(want) < 10).all() and (bound < 0.02).all()
    ref.close(got, want, bound, T[t])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ratio", [1e3, 1e9, 1e12, 1e30])
def test_values_of_later_tokens_do_not_reach_earlier_rows(ratio, dim, wide):
    block, heads, share, length = 16, 1, 2, 200
    held = ref.Held(14, heads, dim, block, seed=dim)
    table = tables([length], block, 14, 3)
    q = torch.randn(length, heads * share, dim, generator=torch.Generator().manual_seed(dim)).bfloat16()
    clean = attend(held, table, [length], [length], q, 0.125, True, wide)
    held.vs[table[0][3]] *= np.float32(ratio)  # tokens 48 .. 63
    held.vs[table[0][8]] *= np.float32(ratio * 1e3)  # tokens 128 .. 143
    got = attend(held, table, [length], [length], q, 0.125, True, wide)
    assert torch.equal(got[:48], clean[:48])
    want, bound = reference(held, table[0], length, ref.f64(q), 0.125, True, ONE)
    ref.close(got, want, bound, torch.bfloat16)


@pytest.mark.parametrize("new,wide", [(1, False), (30, False), (30, True)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_values_from_subnormal_to_large(dim, new, wide):
    # blocks whose scales span FP32's range, zero among them; each row's weights may fall on any of them
    block, heads, length = 16, 1, 256
    held = ref.Held(17, heads, dim, block, seed=dim + 1)
    table = tables([length], block, 17, 4)
    for j, power in enumerate((-140, -100, -60, -30, 0, 30, 60, 100, None, -130, 20, -20, 80, -80, 5, -5)):
        held.vs[table[0][j]] = np.float32(2.0 ** power * 1.3) if power is not None else 0
    g = torch.Generator().manual_seed(dim + new)
    q = torch.zeros(new, 16, dim)
    for h in range(16):  # query head h meets its own block's keys
        held.k[table[0][h]] = 0
        held.k[table[0][h], :, :, h] = 100
        q[:, h, h] = 120 * (0.5 + torch.rand(new, generator=g))
    q = q.bfloat16()
    got = attend(held, table, [new], [length], q, 1.0, False, wide)
    want, bound = reference(held, table[0], length, ref.f64(q), 1.0, False, ONE)
    ref.close(got, want, bound, torch.bfloat16)


@pytest.mark.parametrize("new,length,wide", [(1, 200, False), (1, 9000, False), (20, 200, False), (20, 200, True)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("t,size,scale", [("bf16", s, 0.125) for s in (1e4, 1e6, 1e7, 1e8, 1e9, 1e11, 1e20, 1e36)]
                         + [("f16", 1e3, s) for s in (1e2, 1e5, 1e7, 1e30)])
def test_large_scores(t, size, scale, dim, new, length, wide):
    # A score is off by at most err: sums of D products (32 in a matrix instruction, D / 32 of them) and six
    # roundings (the two factors of a block and column, their product, and the difference from the largest, each
    # half a step).  So only tokens whose score is within 2 err + 120 of the largest have weights above e^-120, and
    # a result lies between the least and the largest of their values, up to the weights' rounding (2^-11, which
    # may fall differently on each value) and its own.
    block, heads, share = 16, 2, 2
    nb = -(-length // block) + 1
    held = ref.Held(nb, heads, dim, block, seed=dim)
    table = tables([length], block, nb, 1)
    g = torch.Generator().manual_seed(new + dim)
    q = (torch.randn(new, heads * share, dim, generator=g) * size).to(T[t])
    got = ref.f64(attend(held, table, [new], [length], q, scale, True, wide))
    assert np.isfinite(got).all()
    K, V = held.values(table[0], length, "k"), held.values(table[0], length, "v")
    x, alone = ref.f64(q), 0
    for i in range(new):
        see = length - new + i + 1
        for h in range(heads * share):
            k, v = K[h // share, :see], V[h // share, :see]
            score = k @ x[i, h] * float(np.float32(scale))
            assert np.abs(score).max() * 1.5 < 3e38
            err = 1.01 * (32 + dim / 32 + 6) * ref.U * (np.abs(k) @ np.abs(x[i, h]) * scale).max()
            near = v[score >= score.max() - 2 * err - 120]
            alone += len(near) == 1
            room = (2.0 ** -11 + 2 * ref.HALF[T[t]]) * np.abs(near).max()
            assert (got[i, h] >= near.min(0) - room).all() and (got[i, h] <= near.max(0) + room).all(), (i, h)
    assert size * scale < 1e6 or alone > 0  # (the bounds mean something)


@pytest.mark.parametrize("new,length,wide", [(1, 200, False), (40, 200, False), (40, 200, True), (1, 5000, False)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_weights_keep_their_digits(t, dim, new, length, wide):
    # each token's values are the last one's with the other sign, and weights differ little, so that results are far
    # smaller than the weighted values and their own rounding hides nothing of the weights'
    block, heads, share = 16, 2, 2
    nb = -(-length // block) + 1
    held = ref.Held(nb, heads, dim, block, seed=dim + 2)
    table = tables([length], block, nb, 5)
    held.v[..., 1::2] = -held.v[..., ::2]
    g = torch.Generator().manual_seed(dim + new)
    q = (torch.randn(new, heads * share, dim, generator=g) * 2).to(T[t])
    scale = 2.0 ** -7
    got = attend(held, table, [new], [length], q, scale, False, wide)
    want, bound = reference(held, table[0], length, ref.f64(q), scale, False, TWO)
    # weights in one FP16 number would not do, for any column (their roundings average out over 5000 tokens)
    k, v = held.values(table[0], length, "k"), held.values(table[0], length, "v")
    for h in range(heads * share if length < 1000 else 0):
        score = k[h // share] @ ref.f64(q)[0, h] * scale
        p = np.exp(score - score.max())
        one = (p * 2 ** 15 * 0.7).astype(np.float16).astype(np.float64) @ v[h // share] / (p.sum() * 2 ** 15 * 0.7)
        half = ref.HALF[T[t]]
        assert (np.abs(one - want[0, h]) > bound[0, h] + half * np.abs(want[0, h])).any()
    ref.close(got, want, bound, T[t])


@pytest.mark.parametrize("new,wide", [(1, False), (40, False), (40, True)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("scale,zero_keys", [(0.0, ()), (0.125, range(7)), (0.125, (6,))])
def test_non_finite_queries_times_zero_are_no_number(scale, zero_keys, bad, new, wide):
    # keys of zero (a block's scale is 0) or a scale of 0 do not make a NaN or an infinity of a query disappear
    held = ref.Held(8, 1, 64, 16, seed=3)
    table = tables([100], 16, 8, 8)
    for j in zero_keys:
        held.ks[table[0][j]] = 0
    q = torch.randn(new, 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16()
    clean = attend(held, table, [new], [100], q, scale, True, wide)
    assert bool(torch.isfinite(clean).all())
    q[new - 1, 1, 5] = bad  # the newest row: it sees the last block, too
    got = attend(held, table, [new], [100], q, scale, True, wide)
    assert bool(torch.isnan(got[new - 1, 1]).all())
    got[new - 1, 1] = clean[new - 1, 1]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dim,t", [(64, "bf16"), (128, "f16"), (256, "bf16")])
def test_rows_do_not_depend_on_the_calls_others(dim, t):
    # the rows kernel: a column's sums do not depend on its tile, nor on what its neighbours are
    held = ref.Held(30, 2, dim, 16, seed=dim)
    lengths, counts = [300, 150], [40, 33]
    table = tables(lengths, 16, 30, 9)
    q = torch.randn(73, 6, dim, generator=torch.Generator().manual_seed(2)).to(T[t])
    got = attend(held, table, counts, lengths, q, 0.1, True, True)
    for first, count, seq, length in ((0, 40, 0, 300), (40, 33, 1, 150), (39, 1, 0, 300), (60, 13, 1, 150)):
        alone = attend(held, table[seq: seq + 1], [count], [length], q[first: first + count], 0.1, True, True)
        assert torch.equal(alone, got[first: first + count]), first
    # one row as a sequence of its own, and neighbours that are large, infinite and NaN
    pair = attend(held, table[[0, 0]], [1, 1], [300, 300], q[[39, 39]], 0.1, True, True)
    assert torch.equal(pair[0], got[39]) and torch.equal(pair[1], got[39])
    odd = q.clone()
    odd[::3] = (odd[::3].float() * 30000).to(T[t])
    odd[1::3, ::2], odd[1::3, 1::2] = float("inf"), float("nan")
    keep = list(range(2, 73, 3))
    assert torch.equal(attend(held, table, counts, lengths, odd, 0.1, True, True)[keep], got[keep])
