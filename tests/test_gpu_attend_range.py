"""Attention over the int8 cache at the ends of its range, on the GPU against 64 bits: large finite scores."""
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
