"""Timed cases of the operators of quantised inference: products with 4-bit weights in scaled groups,
and attention over an int8 cache of keys and values, with the cache's writer and reader.

``listed()`` names the cases, ``draw()`` gives further ones of the same ranges; a case is a dict of
plain values.  ``op`` selects the operator:

* ``w4``      Y = X W^T through awe_gemm_w4, W in 4 bits with a scale (and a zero point) per group
* ``store``   awe_cache_store of new tokens, then awe_cache_load of the blocks that they went to
* ``attend``  awe_cache_attend of each sequence's newest tokens over its cached ones

``run`` computes the plain form in 32 bits with elementary torch operations, or, where ``own`` is
set, makes the library's calls.  ``exact`` computes the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "i8": 1}


def listed():
    return [
        # The smallest product in use: one token against a 256 x 256 layer; launch and latency.
        {"name": "w4_token_256", "op": "w4", "M": 1, "N": 256, "K": 256, "x": "f16", "y": "f16", "s": "f16",
         "group": 32, "zeros": False},
        # One token against a layer of 8192 x 8192: the weights' bytes.
        {"name": "w4_token_8192", "op": "w4", "M": 1, "N": 8192, "K": 8192, "x": "bf16", "y": "bf16", "s": "bf16",
         "group": 128, "zeros": False},
        # A decoding batch of 16 tokens quantised to int8, with zero points.
        {"name": "w4_decode16_int8", "op": "w4", "M": 16, "N": 8192, "K": 8192, "x": "i8", "y": "bf16", "s": "f32",
         "group": 128, "zeros": True},
        # Odd sizes: rows unaligned in memory, a short last group, ragged against every tile.
        {"name": "w4_ragged", "op": "w4", "M": 33, "N": 1537, "K": 2049, "x": "f16", "y": "f32", "s": "f32",
         "group": 64, "zeros": True},
        # A prompt of 512 tokens.
        {"name": "w4_prompt512", "op": "w4", "M": 512, "N": 8192, "K": 8192, "x": "bf16", "y": "bf16", "s": "bf16",
         "group": 128, "zeros": False},
        # The largest: 4096 tokens of several prompts.
        {"name": "w4_prompt4096", "op": "w4", "M": 4096, "N": 8192, "K": 8192, "x": "bf16", "y": "bf16", "s": "bf16",
         "group": 128, "zeros": True},
        # A decoding step of 64 sequences writes one token each.
        {"name": "store_decode64", "op": "store", "seqs": 64, "new": 1, "ragged": False, "past": 2000, "heads": 8,
         "dim": 128, "block": 16, "x": "bf16"},
        # Four prompts of different lengths on top of cached prefixes.
        {"name": "store_prompts", "op": "store", "seqs": 4, "new": 2048, "ragged": True, "past": 100, "heads": 8,
         "dim": 128, "block": 64, "x": "bf16"},
        # The smallest attention: three short sequences, one token each; launch and latency.
        {"name": "attend_short", "op": "attend", "seqs": 3, "new": 1, "ragged": True, "past": 40, "heads": 4,
         "share": 1, "dim": 64, "block": 16, "x": "f16", "causal": True},
        # One token of a single long sequence: the cache has to be split over the whole chip.
        {"name": "attend_long", "op": "attend", "seqs": 1, "new": 1, "ragged": False, "past": 65535, "heads": 8,
         "share": 4, "dim": 128, "block": 64, "x": "bf16", "causal": True},
        # A decoding step of 64 sequences of different lengths, eight query heads per stored head.
        {"name": "attend_decode64", "op": "attend", "seqs": 64, "new": 1, "ragged": True, "past": 8192, "heads": 8,
         "share": 8, "dim": 128, "block": 16, "x": "bf16", "causal": True},
        # Prompts: up to 2048 new tokens of four sequences over what is cached and themselves.
        {"name": "attend_prompts", "op": "attend", "seqs": 4, "new": 2048, "ragged": True, "past": 2048, "heads": 8,
         "share": 4, "dim": 128, "block": 64, "x": "bf16", "causal": True},
    ]


def _log(rng, lo, hi):
    """Log-uniform whole number in [lo, hi]; half of those above 64 are multiples of 32."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    if v >= 64 and rng.random() < 0.5:
        v = v // 32 * 32
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["w4", "w4", "w4", "store", "attend", "attend"])
    while True:
        if op == "w4":
            x = rng.choice(["bf16", "f16", "i8"])
            case = {"op": op, "M": _log(rng, 1, 4096), "N": _log(rng, 64, 8192), "K": _log(rng, 64, 16384), "x": x,
                    "y": rng.choice(["bf16", "f16"]) if x == "i8" else x, "s": rng.choice(["f32", "bf16", "f16"]),
                    "group": rng.choice([32, 64, 128, 128, 256, 0]), "zeros": rng.random() < 0.5}
            if case["M"] * case["N"] * case["K"] > 2 ** 36:
                continue
        else:
            new = 1 if rng.random() < 0.6 else _log(rng, 2, 2048)
            case = {"op": op, "seqs": _log(rng, 1, 64) if new < 64 else rng.randint(1, 4), "new": new,
                    "ragged": rng.random() < 0.6, "past": _log(rng, 16, 8192), "heads": rng.choice([1, 2, 4, 8]),
                    "dim": rng.choice([64, 128, 128, 256]), "block": rng.choice([16, 32, 64, 128]),
                    "x": rng.choice(["bf16", "f16"])}
            if op == "attend":
                case["share"] = rng.choice([1, 2, 4, 5, 8])
                case["causal"] = rng.random() < 0.8
                if case["seqs"] * case["heads"] * case["dim"] * (case["past"] + new) > 2 ** 29:
                    continue
                if work(case)["flops"] > 2 ** 37:
                    continue
        return case


# ---- inputs -------------------------------------------------------------------------------
def _lengths(case):
    """(new tokens, all tokens) of each sequence: the given numbers, or spread from them downwards."""
    n, t = [], []
    for b in range(case["seqs"]):
        part = ((b * 37 + 11) % 64 + 1) / 64 if case["ragged"] else 1.0
        new = max(1, math.ceil(case["new"] * part))
        n.append(new)
        t.append(max(1, math.ceil(case["past"] * part)) + new)
    return n, t


def _offsets(counts, dev):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return torch.tensor(at, dtype=torch.int32, device=dev)


def _batch(state, counts, lengths, dev):
    """What a serving program hands on beside the rows: offsets, lengths and the block table."""
    state["starts"] = _offsets(counts, dev)
    state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
    state["rows"], state["max_rows"], state["max_length"] = sum(counts), max(counts), max(lengths)


def _group(case):
    return case["group"] or case["K"]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    if case["op"] == "w4":
        M, N, K, group = case["M"], case["N"], case["K"], _group(case)
        G = -(-K // group)
        x = normal(M, K)
        state = {"op": "w4", "M": M, "N": N, "K": K, "group": group, "y": TYPES[case["y"]], "x_scales": None,
                 "zeros": None}
        if case["x"] == "i8":
            state["x_scales"] = (x.abs().amax(1) / 127).contiguous()
            state["x"] = (x / state["x_scales"][:, None]).round().to(torch.int8)
        else:
            state["x"] = x.to(TYPES[case["x"]])
        state["w"] = torch.randint(0, 256, (N, (K + 1) // 2), generator=g, device=dev, dtype=torch.uint8)
        state["scales"] = ((0.5 + torch.rand(N, G, generator=g, device=dev)) * 0.2 / math.sqrt(K)).to(TYPES[case["s"]])
        if case["zeros"]:
            state["zeros"] = torch.randint(4, 12, (N, G), generator=g, device=dev, dtype=torch.uint8)
        return state

    H, D, blk = case["heads"], case["dim"], case["block"]
    n, t = _lengths(case)
    wide = -(-max(t) // blk)  # blocks of the longest sequence
    used = sum(-(-x // blk) for x in t)
    total = used + used // 8 + 1
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32)  # blocks in no order
    first = _offsets([-(-x // blk) for x in t], dev)
    column = torch.arange(wide, device=dev)
    held = (torch.tensor(t, device=dev)[:, None] + blk - 1) // blk > column[None]
    at = (first[:-1, None] + column[None]).clamp(max=total - 1)
    # stored keys and values of unit size, with the scale of each block's largest
    state = {
        "op": case["op"], "heads": H, "dim": D, "block": blk, "num_blocks": total,
        "table": torch.where(held, order[at.long()], torch.zeros((), dtype=torch.int32, device=dev)).contiguous(),
        "k": torch.randint(-127, 128, (total, H, blk, D), generator=g, device=dev, dtype=torch.int8),
        "v": torch.randint(-127, 128, (total, H, D, blk), generator=g, device=dev, dtype=torch.int8),
        "k_scales": (0.5 + torch.rand(total, H, generator=g, device=dev)) * (1.7 / 127),
        "v_scales": (0.5 + torch.rand(total, H, generator=g, device=dev)) * (1.7 / 127),
    }
    _batch(state, n, t, dev)
    if case["op"] == "store":
        state["new_k"] = normal(sum(n), H, D).to(TYPES[case["x"]])
        state["new_v"] = normal(sum(n), H, D).to(TYPES[case["x"]])
        # the tokens of the blocks that the new ones go to
        state["read"] = {}
        _batch(state["read"], [y - (y - x) // blk * blk for x, y in zip(n, t)], t, dev)
        state["type"] = TYPES[case["x"]]
    else:
        state["q"] = normal(sum(n), H * case["share"], D).to(TYPES[case["x"]])
        state["share"], state["causal"], state["scale"] = case["share"], case["causal"], 1 / math.sqrt(D)
    return state


# ---- one pass -----------------------------------------------------------------------------
def run(state):
    if own:
        return _own(state)
    with torch.no_grad():
        return {"w4": _w4, "store": _store, "attend": _attend}[state["op"]](state)


def _own(state):
    from paper_2609_24519_amd import awe
    if state["op"] == "w4":
        return awe.matmul_w4(state["x"], state["w"], state["scales"], state["group"], zeros=state["zeros"],
                             x_scales=state["x_scales"], out_dtype=state["y"])
    cache = awe.Cache(state["k"], state["v"], state["k_scales"], state["v_scales"])
    batch = _own_batch(awe, state, state["table"])
    if state["op"] == "store":
        awe.store_tokens(cache, batch, state["new_k"], state["new_v"])
        return awe.load_tokens(cache, _own_batch(awe, state["read"], state["table"]), state["type"])
    return awe.attend(cache, batch, state["q"], state["scale"], causal=state["causal"])


def _own_batch(awe, b, table):
    return awe.Batch(b["starts"], b["lengths"], table, b["rows"], b["max_rows"], b["max_length"])


def _w4(s, real=torch.float32):
    K, group = s["K"], s["group"]
    u = torch.stack([s["w"] & 15, s["w"] >> 4], -1).reshape(s["N"], -1)[:, :K].to(real)
    z = s["zeros"].to(real).repeat_interleave(group, 1)[:, :K] if s["zeros"] is not None else 8.0
    w = (u - z) * s["scales"].to(real).repeat_interleave(group, 1)[:, :K]
    y = s["x"].to(real) @ w.T
    if s["x_scales"] is not None:
        y = y * s["x_scales"].to(real)[:, None]
    return y.to(s["y"])


def _tokens(b, dev):
    """(sequence, position) of every row of a batch."""
    starts = b["starts"].long()
    row = torch.arange(b["rows"], device=dev)
    seq = torch.searchsorted(starts[1:].contiguous(), row, right=True)
    return seq, b["lengths"].long()[seq] - (starts[seq + 1] - row)


def _requantised(held, scales, new, block, slot, older, first_block, tokens_last):
    """One of keys and values: the scales that the new rows want, the older tokens of each sequence's
    first block on the new scale, the new rows in 8 bits, written in place."""
    zero = torch.zeros((), device=new.device)
    most = torch.zeros_like(scales)
    most.scatter_reduce_(0, block[:, None].expand(-1, scales.shape[1]), new.abs().amax(-1) / 127, "amax")
    before = torch.where(older[:, None], scales[first_block], zero)
    want_first = torch.maximum(most[first_block], before)
    ratio = torch.where(older[:, None] & (want_first > 0), before / want_first, zero)
    held[first_block] = (held[first_block].float() * ratio[:, :, None, None]).round().clamp(-127, 127).to(torch.int8)
    scales[block] = most[block]
    scales[first_block] = want_first
    want = scales[block][..., None]
    q = torch.where(want > 0, new / want, zero).round().clamp(-127, 127).to(torch.int8)
    if tokens_last:
        held[block, :, :, slot] = q
    else:
        held[block, :, slot] = q


def _store(s):
    blk, table = s["block"], s["table"]
    seq, pos = _tokens(s, table.device)
    block, slot = table[seq, pos // blk].long(), pos % blk
    first = s["lengths"].long() - (s["starts"][1:] - s["starts"][:-1])  # each sequence's first new position
    first_block = table.gather(1, (first // blk)[:, None])[:, 0].long()
    _requantised(s["k"], s["k_scales"], s["new_k"].float(), block, slot, first % blk > 0, first_block, False)
    _requantised(s["v"], s["v_scales"], s["new_v"].float(), block, slot, first % blk > 0, first_block, True)
    seq, pos = _tokens(s["read"], table.device)
    block, slot = table[seq, pos // blk].long(), pos % blk
    k = s["k"][block, :, slot].float() * s["k_scales"][block][..., None]
    v = s["v"][block, :, :, slot].float() * s["v_scales"][block][..., None]
    return k.to(s["type"]), v.to(s["type"])


def _attend(s):
    H, D, blk, share, dev = s["heads"], s["dim"], s["block"], s["share"], s["k"].device
    B, wide = s["table"].shape
    table = s["table"].long()
    k = s["k"][table].float() * s["k_scales"][table][..., None, None]  # B, blocks, heads, block, dim
    v = s["v"][table].float() * s["v_scales"][table][..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(B, H, D, wide * blk)
    v = v.permute(0, 2, 1, 4, 3).reshape(B, H, wide * blk, D)
    seq, pos = _tokens(s, dev)
    row = torch.arange(s["rows"], device=dev) - s["starts"].long()[seq]
    R = s["max_rows"]
    q = torch.zeros(B, R, H, share, D, device=dev)
    q[seq, row] = s["q"].float().view(-1, H, share, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, H, R * share, D)
    score = (torch.matmul(q, k) * s["scale"]).view(B, H, R, share, wide * blk)
    last = s["lengths"].long()[:, None].expand(B, R)
    if s["causal"]:
        last = last - (s["starts"][1:] - s["starts"][:-1]).long()[:, None] + torch.arange(1, R + 1, device=dev)
    keep = torch.arange(wide * blk, device=dev) < last[..., None]
    score = score.masked_fill(~keep[:, None, :, None], float("-inf"))
    most = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(most == float("-inf"), torch.zeros_like(most), most))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, H, R * share, wide * blk), v).view(B, H, R, share, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.permute(0, 2, 1, 3, 4).reshape(B, R, H * share, D)[seq, row].to(s["q"].dtype)


# ---- what a pass cannot do without --------------------------------------------------------
def work(case):
    if case["op"] == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        G = -(-K // _group(case))
        scale = BYTES[case["s"]] + (1 if case["zeros"] else 0)
        return {"bytes": M * K * BYTES[case["x"]] + N * ((K + 1) // 2) + N * G * scale + M * N * BYTES[case["y"]],
                "flops": 2 * M * N * K}
    n, t = _lengths(case)
    H, D, e = case["heads"], case["dim"], BYTES[case["x"]]
    if case["op"] == "store":
        read = sum(y - (y - x) // case["block"] * case["block"] for x, y in zip(n, t))
        # new rows in and their bytes out; the touched blocks' bytes in and their values out
        return {"bytes": 2 * H * D * (sum(n) * (e + 1) + read * (1 + e)), "flops": 2 * H * D * (3 * sum(n) + read)}
    keys = sum(x * y - (x * (x - 1) // 2 if case["causal"] else 0) for x, y in zip(n, t))
    blocks = sum(-(-y // case["block"]) for y in t)
    return {"bytes": 2 * H * D * sum(t) + 8 * H * blocks + 2 * e * sum(n) * H * case["share"] * D,
            "flops": 4 * keys * H * case["share"] * D}


# ---- the definition in 64 bits ------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    real = torch.float64
    if case["op"] == "w4":
        K = case["K"]
        k = torch.arange(K, device=s["w"].device)
        u = (s["w"][:, k // 2].to(torch.int32) >> (4 * (k % 2)).to(torch.int32)) & 15
        g = k // s["group"]
        zero = s["zeros"][:, g].to(real) if s["zeros"] is not None else torch.full_like(u, 8).to(real)
        w = (u.to(real) - zero) * s["scales"].to(real)[:, g]
        y = torch.matmul(s["x"].to(real), w.t().contiguous())
        return y if s["x_scales"] is None else y * s["x_scales"].to(real).unsqueeze(1)
    n, t = _lengths(case)
    blk, H, D = case["block"], case["heads"], case["dim"]
    at, outs = 0, []
    for b in range(case["seqs"]):
        ids = s["table"][b, : -(-t[b] // blk)].long()
        k = s["k"][ids].to(real) * s["k_scales"][ids].to(real)[:, :, None, None]
        v = s["v"][ids].to(real).transpose(2, 3) * s["v_scales"][ids].to(real)[:, :, None, None]
        rows = slice(at, at + n[b])
        at += n[b]
        if case["op"] == "store":
            first = t[b] - n[b]
            touched = ids[first // blk:]
            both = []
            for held, scales, new in ((k, s["k_scales"], s["new_k"]), (v, s["v_scales"], s["new_v"])):
                start = first // blk * blk
                x = torch.zeros(len(touched) * blk, H, D, dtype=real, device=held.device)
                x[first - start: t[b] - start] = new[rows].to(real)
                x = x.view(-1, blk, H, D).transpose(1, 2)  # blocks, heads, block, dim
                want = x.abs().amax((2, 3)) / 127
                if first > start:
                    want[0] = torch.maximum(want[0], scales[touched[0]].to(real))
                values = torch.round(x / want[:, :, None, None])
                if first > start:
                    values[0, :, : first - start] = torch.round(
                        held[first // blk][:, : first - start] / want[0][:, None, None])
                values = (values * want[:, :, None, None]).transpose(1, 2).reshape(-1, H, D)
                both.append(values[: t[b] - start])
            outs.append(both)
            continue
        k = k.transpose(0, 1).reshape(H, -1, D)[:, : t[b]]
        v = v.transpose(0, 1).reshape(H, -1, D)[:, : t[b]]
        q = s["q"][rows].to(real).view(n[b], H, case["share"], D)
        out = torch.zeros(n[b], H, case["share"], D, dtype=real, device=q.device)
        limit = torch.full((n[b],), t[b], device=q.device)
        if case["causal"]:
            limit = torch.arange(t[b] - n[b] + 1, t[b] + 1, device=q.device)
        beyond = torch.arange(t[b], device=q.device)[None, :] >= limit[:, None]
        for h in range(H):
            for j in range(case["share"]):
                score = torch.matmul(q[:, h, j], k[h].t().contiguous()) * s["scale"]
                p = torch.softmax(score.masked_fill(beyond, float("-inf")), -1)
                out[:, h, j] = torch.matmul(p, v[h])
        outs.append(out.reshape(n[b], H * case["share"], D))
    if case["op"] == "store":
        return tuple(torch.cat([o[i] for o in outs]) for i in (0, 1))
    return torch.cat(outs)
