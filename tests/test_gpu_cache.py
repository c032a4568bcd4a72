"""The int8 cache of keys and values on the GPU: storing bit for bit against the definition in FP32, loading,
attention against 64 bits, ragged and empty sequences, strides, bad tables, graphs, and a run of them together."""
import numpy as np
import pytest
import torch

from paper_2609_24519_amd import awe
from tests import quant_reference as ref

pytestmark = pytest.mark.gpu

T = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def upload(held):
    return awe.Cache(*(torch.from_numpy(a.copy()).cuda() for a in (held.k, held.v, held.ks, held.vs)))


def same_cache(cache, held, scales=True):
    assert np.array_equal(cache.k.cpu().numpy(), held.k) and np.array_equal(cache.v.cpu().numpy(), held.v)
    if scales:
        assert np.array_equal(cache.k_scales.cpu().numpy(), held.ks)
        assert np.array_equal(cache.v_scales.cpu().numpy(), held.vs)


def tables(lengths, block, num_blocks, seed, extra=0):
    """A block table whose sequences own distinct blocks, in no order; entries past a length are garbage."""
    rng = np.random.default_rng(seed)
    wide = max(-(-max(lengths) // block), 1) + extra
    out = rng.integers(-5, num_blocks + 5, (len(lengths), wide)).astype(np.int32)
    ids = list(rng.permutation(num_blocks))
    for b, n in enumerate(lengths):
        for j in range(-(-n // block)):
            out[b, j] = ids.pop()
    return out


def batch_of(counts, lengths, table, first_row=0, rows=None, max_rows=None, max_length=None):
    starts = np.cumsum([first_row] + list(counts)).astype(np.int32)
    return awe.Batch(torch.from_numpy(starts).cuda(), torch.tensor(list(lengths), dtype=torch.int32, device="cuda"),
                     torch.from_numpy(table).cuda(), int(starts[-1]) if rows is None else rows,
                     max(counts) if max_rows is None else max_rows, max(lengths) if max_length is None else max_length)


def flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


SHAPES = [(1, 64, 16, "bf16"), (2, 128, 32, "f16"), (3, 128, 64, "f32"), (2, 256, 128, "bf16"), (8, 128, 16, "bf16")]


# ---- store and load ---------------------------------------------------------------------------
@pytest.mark.parametrize("heads,dim,block,t", SHAPES)
@pytest.mark.parametrize("counts,lengths", [([1], [1]), ([1, 1, 1], [17, 128, 129]), ([5, 0, 40, 1], [5, 30, 47, 200]),
                                            ([16, 33, 127], [16, 97, 131]), ([300, 1], [300, 16])])
def test_store_and_load(counts, lengths, heads, dim, block, t):
    nb = sum(-(-n // block) for n in lengths) + 3
    held = ref.Held(nb, heads, dim, block, seed=heads + sum(lengths))
    table = tables(lengths, block, nb, seed=1)
    cache, f = upload(held), flag()
    g = torch.Generator().manual_seed(sum(counts))
    # tokens of growing size, so that some blocks' scales grow and some keep theirs
    size = 0.2 + 2 * torch.rand(sum(counts), heads, 1, generator=g)
    k, v = ((torch.randn(sum(counts), heads, dim, generator=g) * size).to(T[t]).cuda() for _ in "kv")
    b = batch_of(counts, lengths, table)
    awe.store_tokens(cache, b, k, v, f)
    at = 0
    for i, (n, length) in enumerate(zip(counts, lengths)):
        held.store(table[i], length, *(x[at: at + n].float().cpu().numpy() for x in (k, v)))
        at += n
    same_cache(cache, held)
    # every token of every sequence, and what it stands for
    b = batch_of(lengths, lengths, table)
    got = awe.load_tokens(cache, b, T[t], f)
    for which, x in zip("kv", got):
        want = np.concatenate([np.swapaxes(held.values(table[i], n, which), 0, 1) for i, n in enumerate(lengths)])
        ref.close(x, want, 2.0 ** -24 * np.abs(want), T[t])
    assert int(f) == 0
    # and the rows as they went in, within half a step of their block's scale: x / s' is at most 127 (up to
    # the rounding of s', relative U), its FP32 quotient is off by at most 127 U steps and the clipping to
    # 127 by 127 U more, so half a step becomes 0.5 + 2 * 127 U = 0.5 + 1.6e-5 steps
    at, most = 0, 0.5 + 2 * 127 * ref.U
    for i, (n, length) in enumerate(zip(counts, lengths)):
        for which, x, s in (("k", k, held.ks), ("v", v, held.vs)):
            back = np.swapaxes(held.values(table[i], length, which), 0, 1)[length - n:]
            step = np.stack([s[table[i][p // block]] for p in range(length - n, length)]) if n else np.zeros((0, heads))
            assert (np.abs(back - ref.f64(x[at: at + n])) <= most * step[:, :, None].astype(np.float64)).all()
        at += n


def test_store_token_by_token_matches_definition():
    # a block fills one token at a time; the tokens grow, so that each step puts the older ones on a new scale
    heads, dim, block = 2, 64, 16
    held = ref.Held(4, heads, dim, block, seed=2)
    cache, table = upload(held), np.array([[2, 0, 3]], dtype=np.int32)
    g = torch.Generator().manual_seed(4)
    for p in range(40):
        k, v = (torch.randn(1, heads, dim, generator=g) * (1.1 ** (p % 23)) for _ in "kv")
        awe.store_tokens(cache, batch_of([1], [p + 1], table, max_length=48), k.cuda(), v.cuda())
        held.store(table[0], p + 1, k.numpy(), v.numpy())
        same_cache(cache, held)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_store_zero_tiny_and_non_finite(t):
    heads, dim, block = 2, 64, 16
    held = ref.Held(3, heads, dim, block, seed=3)
    cache, table, f = upload(held), np.array([[1, 2]], dtype=np.int32), flag()
    x = torch.zeros(20, heads, dim)
    x[16:, 0] = torch.tensor([1e-42, -3e-42, 2e-38, 1e-39])[:, None]  # scales below the smallest normal number
    k, v = x.to(T[t]), x.to(T[t]).clone()
    awe.store_tokens(cache, batch_of([20], [20], table), k.cuda(), v.cuda(), f)
    held.store(table[0], 20, k.float().numpy(), v.float().numpy())
    same_cache(cache, held)
    assert int(f) == 0
    k[3, 1, 5], k[17, 0, 0], v[2, 0, 63], v[4, 1, 1] = float("nan"), float("inf"), float("-inf"), 3e38
    awe.store_tokens(cache, batch_of([20], [20], table), k.cuda(), v.cuda(), f)
    held.store(table[0], 20, k.float().numpy(), v.float().numpy())
    same_cache(cache, held)
    assert int(f) != 0


@pytest.mark.parametrize("power", [-140, -126, -40, 0, 120])
def test_store_rounds_quotients_as_the_definition(power):
    # elements at and beside half steps of their scale, from subnormal scales to ones near the largest
    heads, dim, block = 40, 256, 128
    held = ref.Held(2, heads, dim, block, seed=6)
    cache, table = upload(held), np.array([[1, 0]], dtype=np.int32)
    rng = np.random.default_rng(power + 200)
    rows = []
    for _ in "kv":
        most = (rng.uniform(1, 2, (2, heads)) * 2.0 ** power * 127).astype(np.float32)
        x = (rng.integers(-127, 127, (2, block, heads, dim)) + 0.5) * (most / np.float32(127)).astype(np.float64)[:, None, :, None]
        x = x.astype(np.float32)
        to = rng.choice(np.array([-np.inf, 0, np.inf], dtype=np.float32), x.shape)
        x = np.where(to == 0, x, np.nextafter(x, to))
        x = np.clip(x, -most[:, None, :, None], most[:, None, :, None])
        x[:, 5, :, 7] = most  # what sets the scale
        rows.append(x.reshape(2 * block, heads, dim))
    k, v = (torch.from_numpy(x).cuda() for x in rows)
    awe.store_tokens(cache, batch_of([2 * block], [2 * block], table), k, v)
    held.store(table[0], 2 * block, *rows)
    same_cache(cache, held)


def test_store_strides_and_rows_of_no_sequence():
    heads, dim, block, counts, lengths = 3, 64, 16, [4, 9], [20, 9]
    held = ref.Held(6, heads, dim, block, seed=5)
    table = tables(lengths, block, 6, seed=6)
    g = torch.Generator().manual_seed(7)
    big = torch.randn(heads, 30, dim + 3, generator=g).cuda()  # heads outermost, odd offsets
    k, v = big[:, 2:22, 1: dim + 1].transpose(0, 1), torch.randn(1, heads, dim, generator=g).cuda().expand(20, -1, -1)
    b = batch_of(counts, lengths, table, first_row=3, rows=20)  # rows 0..2 and 16..19 belong to no sequence
    cache = upload(held)
    awe.store_tokens(cache, b, k, v)
    at = 3
    for i, (n, length) in enumerate(zip(counts, lengths)):
        held.store(table[i], length, k[at: at + n].cpu().numpy(), v[at: at + n].cpu().numpy())
        at += n
    same_cache(cache, held)
    out = torch.full((2, heads, 20, dim + 5), 9.0, device="cuda")
    o = [x[..., 2: dim + 2].transpose(0, 1) for x in out]
    awe.cache_load(cache, b, o[0], o[0].stride(0), o[0].stride(1), o[1], o[1].stride(0), o[1].stride(1), awe.F32)
    whole = awe.load_tokens(cache, b, torch.float32)
    for x, y in zip(o, whole):
        assert torch.equal(x[3:16], y[3:16]) and bool((x[:3] == 9).all()) and bool((x[16:] == 9).all())
    assert bool((out[..., :2] == 9).all()) and bool((out[..., dim + 2:] == 9).all())


def test_store_bad_tables_and_bounds():
    # sequences outside the host's bounds are left out, tokens of a block out of range too, and the flag says so
    heads, dim, block = 1, 64, 16
    held = ref.Held(8, heads, dim, block, seed=8)
    counts, lengths = [20, 20, 2], [20, 20, 40]
    table = np.array([[0, 1, 0], [2, 99, 0], [-1, 3, 4]], dtype=np.int32)
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(42, heads, dim, generator=g) for _ in "kv")

    def run(b, kept):
        h = ref.Held(8, heads, dim, block, seed=8)
        cache, f = upload(h), flag()
        awe.store_tokens(cache, b, k.cuda(), v.cuda(), f)
        for i in kept:
            r = slice(sum(counts[:i]), sum(counts[: i + 1]))
            h.store(table[i], lengths[i], k[r].numpy(), v[r].numpy())
        same_cache(cache, h)
        return int(f)

    assert run(batch_of(counts, lengths, table), [0, 1, 2]) != 0          # id 99 (id -1 is not written)
    assert run(batch_of(counts, lengths, table, max_rows=19), [2]) != 0   # more rows than the bound
    assert run(batch_of(counts, lengths, table, max_length=39), [0, 1]) != 0  # longer than the bound
    b = batch_of(counts, lengths, table)
    b.lengths[0] = 19                                                      # fewer tokens than rows
    assert run(b, [1, 2]) != 0
    b = batch_of(counts, lengths, table)
    b.starts[1] = -7                                                       # rows that run backwards
    assert run(b, [2]) != 0
    b = batch_of(counts, lengths, table)
    b.starts[3] = 43                                                       # past the tensor
    assert run(b, [0, 1]) != 0


# ---- attention ----------------------------------------------------------------------------------
# rows of the tensors, most of which belong to no sequence: with so many, each wave has columns of its own;
# with the sequences' alone, the tokens are split over the waves
WIDE = 15360


def run_attend(held, table, counts, lengths, share, t, causal, seed=0, scale=None, size=1.0, wide=False, **bounds):
    g = torch.Generator().manual_seed(seed)
    H, n_rows = held.heads * share, sum(counts)
    q = (torch.randn(n_rows, H, held.dim, generator=g) * size).to(T[t])
    scale = held.dim ** -0.5 if scale is None else scale
    q_dev = q.cuda()
    if wide:
        bounds.update(rows=WIDE, max_rows=WIDE)
        q_dev = torch.cat([q_dev, torch.full((WIDE - n_rows, H, held.dim), float("nan"), dtype=T[t], device="cuda")])
    b = batch_of(counts, lengths, table, **bounds)
    f = flag()
    out = torch.full_like(q_dev, 9.0)
    awe.attend(upload(held), b, q_dev, scale, causal=causal, out=out, d_range_flag=f)
    assert bool((out[n_rows:] == 9).all())
    got = out[:n_rows].clone()
    want, bound = [], []
    at = 0
    for i, (n, length) in enumerate(zip(counts, lengths)):
        w, e = ref.attend(held, table[i], length, ref.f64(q[at: at + n]), np.float32(scale), causal)
        want.append(w)
        bound.append(e)
        at += n
    ref.close(got, np.concatenate(want), np.concatenate(bound), T[t])
    return got, q, f


def test_both_ways_are_taken():
    c = awe.CacheStruct(0, 0, 0, 0, 10, 1, 64, 16)
    # a workspace is asked for where tokens are split over workgroups, and only there
    few, many = (awe.BatchStruct(1, 0, 0, 0, 1 << 20, r, r, 60000) for r in (40, WIDE))
    assert awe.cache_attend_workspace_bytes(c, few, 1) > 0 and awe.cache_attend_workspace_bytes(c, many, 1) == 0


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("share,heads,t", [(1, 3, "f16"), (4, 2, "bf16"), (5, 1, "bf16"), (8, 1, "f16"), (17, 1, "bf16")])
def test_attend_single_tokens(share, heads, t, block, dim):
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 0, 128, 129, 300, 513]
    nb = sum(-(-n // block) for n in lengths) + 2
    held = ref.Held(nb, heads, dim, block, seed=dim + block)
    _, _, f = run_attend(held, tables(lengths, block, nb, 3), [1] * len(lengths), lengths, share, t, True)
    assert int(f) == 0


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,block,share,t", [(64, 16, 1, "bf16"), (128, 64, 4, "bf16"), (128, 16, 3, "f16"),
                                               (256, 32, 2, "bf16"), (64, 128, 8, "f16"), (256, 64, 1, "f16")])
def test_attend_prompts(dim, block, share, t, causal, wide):
    counts = [1, 7, 64, 0, 130, 33, 5]
    lengths = [1, 7, 100, 40, 130, 300, 3]  # the last: rows before the first token are empty if causal
    nb = sum(-(-n // block) for n in lengths) + 2
    held = ref.Held(nb, 2, dim, block, seed=dim + block)
    got, _, f = run_attend(held, tables(lengths, block, nb, 4), counts, lengths, share, t, causal, wide=wide)
    if causal:
        assert bool((got[-5:-3] == 0).all()) and bool((got[-3:] != 0).any())
    assert int(f) == 0


@pytest.mark.parametrize("share,new", [(4, 1), (1, 1), (8, 3)])
def test_attend_long_sequences_split(share, new):
    # long enough that its tokens are split over workgroups, beside short ones that are not
    lengths, block = [9000, 1 + new, 4097, 777], 64
    nb = sum(-(-n // block) for n in lengths) + 2
    held = ref.Held(nb, 2, 128, block, seed=11)
    run_attend(held, tables(lengths, block, nb, 5), [new] * 4, lengths, share, "bf16", True)
    # and with a bound far above any length
    run_attend(held, tables(lengths, block, nb, 5, extra=900), [new] * 4, lengths, share, "bf16", True,
               max_length=60000)


@pytest.mark.parametrize("new,wide", [(1, False), (30, False), (30, True)])
def test_attend_shared_and_repeated_blocks(new, wide):
    # sequences with a common beginning, and one whose table names a block twice
    lengths, block = [300, 290, 333, 5000 if not wide else 400], 32
    held = ref.Held(160, 2, 128, block, seed=15)
    table = np.random.default_rng(3).integers(0, 160, (4, 160)).astype(np.int32)
    table[1, :8] = table[0, :8]
    table[2, 5] = table[2, 2]
    table[3, :10] = table[2, :10]
    run_attend(held, table, [new] * 4, lengths, 4, "bf16", True, wide=wide)
    # rows of one sequence as two sequences of the call: the same tokens, the same results
    got, q, _ = run_attend(held, table[:1], [2], [200], 4, "f16", False, wide=wide)
    twice, _, _ = run_attend(held, table[[0, 0]], [1, 1], [200, 200], 4, "f16", False, wide=wide)
    if not wide:  # (a column's sums do not depend on its tile)
        assert torch.equal(got, twice)


@pytest.mark.parametrize("new,wide", [(1, False), (40, False), (40, True)])
def test_attend_blocks_of_very_different_scales(new, wide):
    # one block of large values that gets no weight must not cost the others their digits
    lengths, block = [300], 16
    held = ref.Held(25, 1, 64, block, seed=12)
    table = tables(lengths, block, 25, 6)
    held.vs[table[0][3]] *= 3e4
    held.ks[table[0][3]] *= 0
    held.vs[table[0][5]] = 0
    held.vs[table[0][7]] *= 1e-6
    run_attend(held, table, [new], lengths, 2, "f16", True, scale=0.125, size=8.0, wide=wide)


@pytest.mark.parametrize("new,wide", [(1, False), (40, False), (40, True)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_attend_extreme_queries(new, wide, t):
    # scores of thousands (one token takes all the weight), zero, tiny and large queries, scale 0 and negative
    lengths, block = [200, 200], 16
    held = ref.Held(30, 2, 64, block, seed=13)
    table = tables(lengths, block, 30, 7)
    for size, scale in ((1000.0, 1.0), (0.0, 1.0), (1e-6 if t == "f16" else 1e-30, 1.0), (1.0, 0.0), (1.0, -0.25),
                        (6000.0 if t == "f16" else 1e30, 1e-4 if t == "f16" else 1e-31)):
        run_attend(held, table, [new, new], lengths, 2, t, True, scale=scale, size=size, wide=wide)


@pytest.mark.parametrize("new,wide", [(1, False), (40, False), (40, True)])
def test_attend_non_finite_rows_stay_alone(new, wide):
    lengths, block = [100, 90], 16
    held = ref.Held(20, 1, 64, block, seed=14)
    table = tables(lengths, block, 20, 8)
    clean, q, _ = run_attend(held, table, [new, new], lengths, 2, "bf16", True, wide=wide)
    q[0, 1, 3] = float("nan")
    q[new, 0, 0] = float("inf")
    more = dict(rows=WIDE, max_rows=WIDE) if wide else {}
    q_dev = torch.zeros(WIDE if wide else 2 * new, 2, 64, dtype=torch.bfloat16, device="cuda")
    q_dev[: 2 * new] = q.cuda()
    got = awe.attend(upload(held), batch_of([new, new], lengths, table, **more), q_dev, 0.125)[: 2 * new]
    assert bool(torch.isnan(got[0, 1]).all()) and not bool(torch.isfinite(got[new, 0]).any())
    got[0, 1], got[new, 0] = clean[0, 1], clean[new, 0]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("new,wide", [(1, False), (20, False), (20, True)])
def test_attend_bad_blocks_and_bounds(new, wide):
    lengths, block = [100, 64, 40], 16
    held = ref.Held(20, 2, 64, block, seed=15)
    table = tables(lengths, block, 20, 9)
    table[0, 2], table[1, 0], table[2, :] = 20, -1, 1 << 30
    # the third has no token left: zeros
    _, q, f = run_attend(held, table, [new] * 3, lengths, 2, "bf16", False, wide=wide)
    assert int(f) != 0
    f, n = flag(), WIDE if wide else 3 * new
    q_dev = torch.zeros(n, *q.shape[1:], dtype=q.dtype, device="cuda")
    q_dev[: 3 * new] = q.cuda()
    out = torch.full_like(q_dev, 5.0)
    b = batch_of([new] * 3, lengths, tables(lengths, block, 20, 9), max_length=70, rows=n, max_rows=n)
    awe.attend(upload(held), b, q_dev, 0.125, out=out, d_range_flag=f)
    assert int(f) != 0 and bool((out[:new] == 5).all()) and bool((out[new: 3 * new] != 5).any())
    # and a cache without any block: zeros, and nothing is read
    f = flag()
    none = awe.CacheStruct(0, 0, 0, 0, 0, held.heads, held.dim, block)
    b = batch_of([new] * 3, lengths, tables(lengths, block, 20, 9), rows=n, max_rows=n)
    size = awe.cache_attend_workspace_bytes(none, b, 4)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    awe.cache_attend(none, b, q_dev, 4 * 64, 64, 4, awe.BF16, 0.125, 1, out, 4 * 64, 64, ws, size, f)
    assert int(f) != 0 and bool((out[: 3 * new] == 0).all())


def test_attend_strides_and_rows_of_no_sequence():
    heads, share, dim, block, counts, lengths = 2, 3, 64, 32, [3, 40], [30, 41]
    held = ref.Held(6, heads, dim, block, seed=16)
    table = tables(lengths, block, 6, 10)
    g = torch.Generator().manual_seed(17)
    big = torch.randn(6, 50, dim + 3, generator=g).to(torch.bfloat16).cuda()
    q = big[:, 1:, 1: dim + 1].transpose(0, 1)  # 49 rows, heads outermost, odd offsets
    b = batch_of(counts, lengths, table, first_row=2, rows=49)
    out = torch.full((6, 49, dim + 7), 3.0, dtype=torch.bfloat16, device="cuda")
    o = out[..., 3: dim + 3].transpose(0, 1)
    cache = upload(held)
    awe.attend(cache, b, q, 0.125, out=o)
    want = awe.attend(cache, b, q.contiguous(), 0.125)
    assert torch.equal(o[2:45], want[2:45]) and bool((o[:2] == 3).all()) and bool((o[45:] == 3).all())
    assert bool((out[..., :3] == 3).all()) and bool((out[..., dim + 3:] == 3).all())
    w, e = ref.attend(held, table[1], 41, ref.f64(q[5:45]), np.float32(0.125), True)
    ref.close(o[5:45], w, e, torch.bfloat16)


@pytest.mark.parametrize("counts,lengths,wide", [([1, 1], [300, 5], False), ([1], [5000], False), ([40, 260], [300, 260], True)])
def test_offsets_past_32_bits(counts, lengths, wide):
    # the same tokens in a small cache and in the last blocks of one of 5 GiB each for keys and values
    heads, dim, block, share, far = 8, 256, 128, 2, 20480
    per = [-(-n // block) for n in lengths]
    table = np.zeros((len(lengths), max(per)), dtype=np.int32)
    ids = iter(range(sum(per)))
    for i, n in enumerate(per):
        table[i, :n] = [next(ids) for _ in range(n)]
    g = torch.Generator().manual_seed(8)
    every, rows = sum(lengths), sum(counts)
    k, v = (torch.randn(every, heads, dim, generator=g).bfloat16().cuda() for _ in "kv")
    q = torch.randn(WIDE if wide else rows, heads * share, dim, generator=g).bfloat16().cuda()
    bounds = dict(rows=WIDE, max_rows=WIDE) if wide else {}
    results = []
    for blocks, first in ((sum(per), 0), (far, far - sum(per))):
        cache = awe.Cache.empty(blocks, heads, dim, block)
        at = table + first
        awe.store_tokens(cache, batch_of(lengths, lengths, at), k, v)
        out = torch.zeros_like(q)
        awe.attend(cache, batch_of(counts, lengths, at, **bounds), q, dim ** -0.5, out=out)
        results.append((out, *awe.load_tokens(cache, batch_of(lengths, lengths, at), torch.bfloat16)))
        del cache
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert bool(results[0][0][:rows].any())


def test_attend_workspace_refused_when_small():
    lengths = [9000]
    held = ref.Held(150, 1, 64, 64, seed=18)
    cache, b = upload(held), batch_of([1], lengths, tables(lengths, 64, 150, 11))
    n = awe.cache_attend_workspace_bytes(cache, b, 2)
    if n == 0:
        pytest.skip("nothing is split at this size")
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for w, size in ((None, n), (ws, n - 1)):
        with pytest.raises(awe.AweError) as e:
            awe.cache_attend(cache, b, q, 128, 64, 2, awe.BF16, 1.0, 1, q, 128, 64, w, size)
        assert e.value.status == awe.ERR_WORKSPACE


# ---- together -----------------------------------------------------------------------------------
def test_decoding_steps_captured_and_replayed():
    """A layer as it is served: 4-bit projections of each token to queries, keys and values, the cache, attention
    and a 4-bit projection back, eagerly and as one captured graph replayed step by step."""
    heads, share, dim, block, B, width, steps = 2, 2, 64, 16, 3, 256, 20
    g = torch.Generator().manual_seed(19)
    n_qkv = (heads * share + 2 * heads) * dim
    w_in, w_out = (torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8).cuda()
                   for n, k in ((n_qkv, width), (width, heads * share * dim)))
    s_in, s_out = ((0.5 + torch.rand(w.shape[0], w.shape[1] * 2 // 64, generator=g)).cuda() / 64 for w in (w_in, w_out))
    x = torch.randn(steps, B, width, generator=g).to(torch.bfloat16).cuda()
    table = torch.arange(B * 3, dtype=torch.int32, device="cuda").view(3, B).T.contiguous()
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")

    def program():
        cache = awe.Cache.empty(B * 3, heads, dim, block)
        lengths = torch.tensor([1, 9, 17], dtype=torch.int32, device="cuda")
        for t in (cache.k, cache.v):
            t.zero_()
        for t in (cache.k_scales, cache.v_scales):
            t.fill_(1.0 / 127)
        b, token = awe.Batch(starts, lengths, table, B, 1, 48), torch.zeros(B, width, dtype=torch.bfloat16, device="cuda")

        def step():
            qkv = awe.matmul_w4(token, w_in, s_in, 64).view(B, -1, dim)
            q, k, v = qkv.split([heads * share, heads, heads], 1)
            awe.store_tokens(cache, b, k, v)
            o = awe.attend(cache, b, q, dim ** -0.5)
            return awe.matmul_w4(o.reshape(B, -1), w_out, s_out, 64), o, qkv
        return cache, lengths, token, step

    eager_cache, eager_len, eager_in, eager_step = program()
    cache, lengths, token, step = program()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = step()
    held = ref.Held(B * 3, heads, dim, block, seed=0)
    held.k[:], held.v[:], held.ks[:], held.vs[:] = 0, 0, np.float32(1.0 / 127), np.float32(1.0 / 127)
    for i in range(steps):
        token.copy_(x[i])
        eager_in.copy_(x[i])
        graph.replay()
        want = eager_step()
        torch.cuda.synchronize()
        for a, e in zip(outs, want):
            assert torch.equal(a, e), i
        y, bound = ref.w4(x[i], w_in, s_in, 64)
        ref.close(want[2].view(B, -1), y, bound, torch.bfloat16)
        for s in range(B):
            at = want[2][s: s + 1].float().cpu().numpy()
            n = int(lengths[s])
            held.store(table[s].cpu().numpy(), n, at[:, heads * share: heads * share + heads], at[:, heads * share + heads:])
            o, e = ref.attend(held, table[s].cpu().numpy(), n, at[:, : heads * share].astype(np.float64),
                              np.float32(dim ** -0.5), True)
            ref.close(want[1][s: s + 1], o, e, torch.bfloat16)
        same_cache(cache, held)
        same_cache(eager_cache, held)
        lengths += 1
        eager_len += 1


def test_two_calls_at_once_on_two_streams():
    lengths, block = [5000, 3000], 64
    held = ref.Held(140, 2, 128, block, seed=20)
    table = tables(lengths, block, 140, 12)
    cache = upload(held)
    g = torch.Generator().manual_seed(21)
    q = [torch.randn(2, 8, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
    b = batch_of([1, 1], lengths, table)
    want = [awe.attend(cache, b, x, 0.1) for x in q]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in q], []
    for _ in range(4):
        for s, x in zip(streams, q):
            with torch.cuda.stream(s):
                outs.append(awe.attend(cache, b, x, 0.1))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o, want[i % 2])
