"""Plain implementations in 64 bits (numpy, on the host) of the operators of quantised inference, the
inputs of their tests, and what their roundings may add up to.

U is half a step of FP32 relative to the value.  A sum of terms t in which no term passes through more than
`depth` additions is off by at most depth * U * sum|t| (to first order; 1 % is added for the rest).
"""
import numpy as np
import torch

U = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}  # half a step
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # smallest step


def f64(t):
    return t.detach().cpu().double().numpy()


# ---- 4-bit weights --------------------------------------------------------------------------
def codes(w, K):
    """The codes u[j, k] of packed rows."""
    w = w.cpu().numpy()
    return np.stack([w & 15, w >> 4], -1).reshape(w.shape[0], 2 * w.shape[1])[:, :K].astype(np.int64)


def w4(x, w, scales, group, zeros=None, x_scales=None):
    """(Y, the rounding errors' bound before Y's own) in 64 bits."""
    M, K = x.shape
    g = np.arange(K) // group
    u = codes(w, K)
    z = zeros.cpu().numpy().astype(np.int64)[:, g] if zeros is not None else np.full_like(u, 8)
    s = f64(scales)[:, g]
    sx = f64(x_scales)[:, None] if x_scales is not None else 1.0
    X = f64(x)
    with np.errstate(invalid="ignore", over="ignore"):
        y = (X @ ((u - z) * s).T) * sx
        # The kernels may sum x (16 + u) and subtract (16 + z) sum x: terms of at most x (16 + u) and
        # x (16 + z) with their group's scale.  A term passes through at most 32 additions of one matrix
        # instruction, those of its chunk of at most 256 indices (8), the chunks of its wave or of a lane
        # (K / 64) and the tree or the waves at the end (16), and four roundings of products.
        size = (np.abs(X) @ (np.abs(s) * (32 + u + z)).T) * np.abs(sx)
    return y, 1.01 * (32 + 8 + K / 64 + 16 + 4) * U * size


def close(got, want, bound, dtype):
    """Whether got (dtype) is want within bound and one rounding to dtype; infinities and NaN where want has them."""
    got = f64(got)
    assert got.shape == want.shape
    fine = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) - bound - HALF[dtype] * (np.abs(want) + bound) - TINY[dtype] / 2
    off = np.where(fine, off, -1.0)
    bad = (off > 0) | (~np.isfinite(got) & fine) | (np.isfinite(got) & ~fine)
    assert not bad.any(), "%d of %d off, first at %s: got %s, want %s, bound %s" % (
        bad.sum(), bad.size, np.argwhere(bad)[0], got[tuple(np.argwhere(bad)[0])], want[tuple(np.argwhere(bad)[0])],
        np.broadcast_to(bound, want.shape)[tuple(np.argwhere(bad)[0])])


# ---- the cache --------------------------------------------------------------------------------
class Held:
    """A cache on the host: the same arrays as awe.Cache in numpy."""

    def __init__(self, num_blocks, heads, dim, block, seed):
        rng = np.random.default_rng(seed)
        self.k = rng.integers(-127, 128, (num_blocks, heads, block, dim)).astype(np.int8)
        self.v = rng.integers(-127, 128, (num_blocks, heads, dim, block)).astype(np.int8)
        self.ks = ((0.5 + rng.random((num_blocks, heads))) / 127).astype(np.float32)
        self.vs = ((0.5 + rng.random((num_blocks, heads))) / 127).astype(np.float32)
        self.block, self.heads, self.dim, self.num_blocks = block, heads, dim, num_blocks

    def values(self, blocks, n, which):
        """n tokens of the sequence with these blocks, heads x n x dim in 64 bits; blocks out of range: NaN."""
        out = np.full((self.heads, n, self.dim), np.nan)
        for p in range(0, n, self.block):
            b, m = int(blocks[p // self.block]), min(self.block, n - p)
            if not 0 <= b < self.num_blocks:
                continue
            if which == "k":
                out[:, p: p + m] = self.k[b, :, :m].astype(np.float64) * self.ks[b][:, None, None]
            else:
                out[:, p: p + m] = np.swapaxes(self.v[b, :, :, :m], 1, 2).astype(np.float64) * self.vs[b][:, None, None]
        return out

    def store(self, blocks, length, k, v):
        """One sequence's rows (n x heads x dim float32) as its newest tokens, by the definition in FP32."""
        n = k.shape[0]
        for b in range((length - n) // self.block, -(-length // self.block)):
            if n == 0 or not 0 <= blocks[b] < self.num_blocks:
                continue
            i = int(blocks[b])
            t0, t1 = max(0, length - n - b * self.block), min(self.block, length - b * self.block)
            r0 = b * self.block + t0 - (length - n)
            for x, q, s in ((k, self.k[i], self.ks[i]), (v, np.swapaxes(self.v[i], 1, 2), self.vs[i])):
                for h in range(self.heads):
                    rows = x[r0: r0 + t1 - t0, h].astype(np.float32)
                    rows = np.where(np.isfinite(rows), rows, np.float32(0))
                    old = s[h] if t0 > 0 else np.float32(0)
                    now = max(old, np.float32(np.abs(rows).max()) / np.float32(127))
                    if now > 0 and t0 > 0 and now != old:
                        q[h, :t0] = np.clip(np.rint(q[h, :t0].astype(np.float32) * (old / now)), -127, 127)
                    if now > 0:
                        with np.errstate(over="ignore"):
                            q[h, t0:t1] = np.clip(np.rint(rows / now), -127, 127)
                    else:
                        q[h, t0:t1] = 0
                    s[h] = now


def attend(held, blocks, length, q, scale, causal):
    """One sequence: q rows x heads x dim (64 bits); (out, bound) rows x heads x dim."""
    n, heads, D = q.shape
    share = heads // held.heads
    k, v = held.values(blocks, length, "k"), held.values(blocks, length, "v")
    there = ~np.isnan(k[0, :, 0])
    out, bound = np.zeros((n, heads, D)), np.zeros((n, heads, D))
    for i in range(n):
        last = length - n + i + 1 if causal else length
        use = np.flatnonzero(there[: max(0, last)])
        if not len(use):
            continue
        for h in range(heads):
            K, V = k[h // share][use], v[h // share][use]
            with np.errstate(invalid="ignore", over="ignore"):
                score = K @ q[i, h] * scale
                p = np.exp(score - score.max())
                p /= p.sum()
                out[i, h] = p @ V
                # a score: sums of D products (a matrix instruction's 32, D / 32 of them) and three
                # roundings; exp of scores is off by their error and a few steps of its own; a weight is
                # rounded to FP16 (2^-11) and its sums by depth <= 32 + len / 64 + 64; what FP16 cannot
                # hold below 2^-24 of the row's largest weighted block is 2^-40 of it at most per token
                err = 1.01 * (32 + D / 32 + 3) * U * (np.abs(K) @ np.abs(q[i, h]) * abs(scale)).max()
                rel = 2 * err + 2 * np.abs(score - score.max()).clip(0, 100).max() * U * 4 + 16 * U
                size = p @ np.abs(V)
                bound[i, h] = (2.0 ** -11 + rel + (96 + len(use) / 64) * 2 * U) * size * 1.01 \
                    + np.abs(V).max() * 2.0 ** -38
    return out, bound
