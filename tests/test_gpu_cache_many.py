"""More sequences in a call than one launch's grid takes: they go over in parts (32,767 for store and load, 65,535 for attention)."""
import numpy as np
import pytest
import torch

from paper_2609_24519_amd import awe
from tests import quant_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sequences,new", [(32768, 1), (70001, 1), (70001, 2)])
def test_sequences_go_over_in_parts(sequences, new):
    # each sequence has `new` tokens, in a block of its own, in no order; the first token of a sequence is all that
    # its first row sees, so that row's result is the token's values
    heads, share, dim, block = 1, 2, 64, 16
    g = torch.Generator().manual_seed(sequences)
    cache = awe.Cache.empty(sequences + 3, heads, dim, block)
    table = torch.randperm(sequences + 3, generator=g)[:sequences].to(torch.int32).view(-1, 1).cuda()
    starts = (torch.arange(sequences + 1, dtype=torch.int32) * new).cuda()
    lengths = torch.full((sequences,), new, dtype=torch.int32, device="cuda")
    b = awe.Batch(starts, lengths, table, sequences * new, new, block)
    k, v = (torch.randn(sequences * new, heads, dim, generator=g).bfloat16().cuda() for _ in "kv")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    awe.store_tokens(cache, b, k, v, flag)
    got_k, got_v = awe.load_tokens(cache, b, torch.float32, flag)
    for got, x in ((got_k, k), (got_v, v)):
        x = x.float().view(sequences, new, heads, dim)
        step = x.abs().amax((1, 3)) / 127  # half a step of the block's scale, and its FP32 roundings
        off = (got.view_as(x) - x).abs().amax((1, 3))
        assert bool((off <= step * (0.5 + 2 * 127 * ref.U) + 4 * 127 * ref.U * step).all())
    q = torch.randn(sequences * new, heads * share, dim, generator=g).bfloat16().cuda()
    out = awe.attend(cache, b, q, 0.125, d_range_flag=flag)
    first = out.view(sequences, new, share, dim)[:, 0].double().cpu().numpy()
    want = got_v.view(sequences, new, 1, dim)[:, 0].double().cpu().numpy()
    # one weight over itself: two FP16 numbers (2^-22), exp2 and logarithms (16 + 4 * 46 U as for any weight), then BF16
    bound = (2.0 ** -22 + 200 * ref.U) * np.abs(want)
    assert (np.abs(first - want) <= bound + ref.HALF[torch.bfloat16] * (np.abs(want) + bound) + 2.0 ** -30).all()
    assert int(flag) == 0
    for i in (0, 32766, 32767, sequences - 1):  # whole rows of some sequences, with their neighbours left out
        one = awe.Batch(starts[i: i + 2] - starts[i], lengths[i: i + 1], table[i: i + 1], new, new, block)
        rows = slice(i * new, (i + 1) * new)
        assert torch.equal(awe.attend(cache, one, q[rows], 0.125), out[rows])


def test_positions_up_to_the_largest():
    # a sequence of nearly 2^30 tokens whose table names five blocks over and over
    heads, share, dim, block, length = 1, 2, 64, 128, (1 << 30) - 5
    held = ref.Held(6, heads, dim, block, seed=1)
    entries = -(-length // block)
    table = (torch.arange(entries, dtype=torch.int32, device="cuda") % 5).view(1, -1)
    table[0, -1] = 5  # the last one gets the new rows
    cache = awe.Cache(*(torch.from_numpy(a.copy()).cuda() for a in (held.k, held.v, held.ks, held.vs)))
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(3, heads, dim, generator=g).bfloat16() for _ in "kv")
    q = torch.randn(3, heads * share, dim, generator=g).bfloat16()
    b = awe.Batch(torch.tensor([0, 3], dtype=torch.int32, device="cuda"),
                  torch.tensor([length], dtype=torch.int32, device="cuda"), table, 3, 3, length)
    awe.store_tokens(cache, b, k.cuda(), v.cuda())
    last = length - (entries - 1) * block  # of the last block
    held.store([5], last, k.float().numpy(), v.float().numpy())
    assert np.array_equal(cache.k.cpu().numpy(), held.k) and np.array_equal(cache.v.cpu().numpy(), held.v)
    out = ref.f64(awe.attend(cache, b, q.cuda(), 0.125))
    times = np.bincount(np.arange(entries - 1) % 5)  # how often each block is seen
    K, V = (np.concatenate([held.values([i], block if i < 5 else last, w)[0] for i in range(6)]) for w in "kv")
    for i in range(3):
        count = np.concatenate([np.repeat(times, block), np.arange(last) < last - 2 + i]).astype(np.float64)
        for h in range(heads * share):
            score = K @ ref.f64(q)[i, h] * 0.125
            p = np.exp(score - score.max()) * count
            want = p @ V / p.sum()
            # as in test_gpu_attend_range.py, with chunks of 2^30 / 4096 tokens: a wave adds a quarter of one, 64 a step
            # (5 U a step: 5 * 1024), and 4096 parts are joined in turn (a quarter of them, 3 U each)
            err = 1.01 * (32 + 2 + 8) * ref.U * (np.abs(K) @ np.abs(ref.f64(q)[i, h]) * 0.125).max()
            bound = (2.0 ** -22 + 2 * (err + (4 * 40 + 100 + 5 * 1024 + 3 * 1024) * ref.U)) * (p @ np.abs(V)) / p.sum()
            off = np.abs(out[i, h] - want) - bound - ref.HALF[torch.bfloat16] * (np.abs(want) + bound)
            assert (off <= 2.0 ** -40).all()
