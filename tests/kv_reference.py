"""The 8-bit cache operators in 64 bits on the CPU, token by token from their definitions (test infrastructure)."""
import math

import numpy as np
import torch

M = {"int8": 127.0, "e4m3": 448.0}
TORCH_CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TORCH_TYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


def scale_of(a, fmt):
    """Smallest power of two s = 2^e, e >= -100, with a <= M s."""
    e = -100
    if a > 0:
        e = max(-100, math.frexp(a / M[fmt])[1] - 2)
        while a > math.ldexp(M[fmt], e):
            e += 1
    return math.ldexp(1.0, e)


def nearest(x, fmt):
    """Nearest code value of |x| <= M (float64 array), ties to even."""
    x = np.clip(x, -M[fmt], M[fmt])
    if fmt == "int8":
        return np.rint(x)
    step = np.ldexp(1.0, np.maximum(np.frexp(np.abs(x))[1] - 1, -6) - 3)
    return np.rint(x / step) * step


class Pool:
    """A pool on the CPU: code values (float64) and scales."""

    def __init__(self, pages, heads, block, dim, fmt):
        self.fmt, self.block = fmt, block
        self.codes = {m: np.zeros((pages, heads, block, dim)) for m in "kv"}
        self.scale = {m: np.ones((pages, heads)) for m in "kv"}

    @classmethod
    def of(cls, cache):
        p = cls(cache.pages, cache.kv_heads, cache.block, cache.head_dim,
                "int8" if cache.k.dtype == torch.int8 else "e4m3")
        for m in "kv":
            p.codes[m] = getattr(cache, m).cpu().to(torch.float32).double().numpy()
            p.scale[m] = getattr(cache, m + "_scale").cpu().double().numpy()
        return p

    def rows(self, m, pages, slots, head):
        """Values of slots of one sequence: [len(slots), dim]."""
        pg = np.asarray(pages)[np.asarray(slots, dtype=int) // self.block]
        return self.codes[m][pg, head, np.asarray(slots, dtype=int) % self.block] * self.scale[m][pg, head][:, None]

    def append(self, m, pages, length, new, head):
        """new [n, dim]; the block rule of kv_cache_append."""
        n, blk, fmt = len(new), self.block, self.fmt
        clean = np.where(np.isnan(new), 0.0, new)
        for start in range(length // blk * blk, length + n, blk):
            lo, hi = max(length, start), min(length + n, start + blk)
            if lo >= hi:
                continue
            pg, x = pages[start // blk], clean[lo - length:hi - length]
            finite = np.abs(x[np.isfinite(x)])
            s = scale_of(float(finite.max()) if finite.size else 0.0, fmt)
            if lo > start:
                old = self.scale[m][pg, head]
                s = max(s, old)
                if s > old:
                    self.codes[m][pg, head, :lo - start] = nearest(self.codes[m][pg, head, :lo - start] * old / s, fmt)
            self.codes[m][pg, head, lo - start:hi - start] = nearest(x / s, fmt)
            self.scale[m][pg, head] = s


def attention(pool, pages, q, length, n, heads, kv_heads, causal, scale):
    """q [>= n, heads, dim] float64.  Returns out, lse, per key-head weights, and what the error bounds need:
    sum of p |v|, and a bound on each query's logit magnitude sum |q k|."""
    dim = q.shape[-1]
    out = np.zeros((n, heads, dim))
    lse = np.full((n, heads), -np.inf)
    weights = np.zeros((kv_heads, length))
    spread = np.zeros((n, heads, dim))
    reach = np.zeros((n, heads))
    vmax = np.zeros((n, heads))
    group = heads // kv_heads
    slots = np.arange(length)
    for hk in range(kv_heads):
        if length == 0:
            break
        k, v = pool.rows("k", pages, slots, hk), pool.rows("v", pages, slots, hk)
        for h in range(hk * group, (hk + 1) * group):
            z = q[:n, h] @ k.T * scale
            size = np.abs(q[:n, h]) @ np.abs(k).T * scale
            end = np.full(n, length)
            if causal:
                end = np.clip(length - n + np.arange(n) + 1, 0, length)
            seen = slots[None] < end[:, None]
            some = end > 0
            z = np.where(seen, z, -np.inf)
            top = np.where(some, z.max(1), 0.0)
            p = np.exp(z - top[:, None])
            total = p.sum(1)
            p = np.where(some[:, None], p / np.where(some, total, 1.0)[:, None], 0.0)
            out[:, h] = p @ v
            lse[:, h] = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
            weights[hk] += p.sum(0)
            spread[:, h] = p @ np.abs(v)
            reach[:, h] = np.where(seen, size, 0.0).max(1)
            vmax[:, h] = np.abs(v).max()
    return out, lse, weights, spread, reach, vmax


def survivors(w, budget, first, last):
    """Kept slots of one sequence and head, ascending; w: its weights."""
    n = len(w)
    if n <= budget:
        return list(range(n))
    ends = list(range(first)) + list(range(n - last, n))
    rank = sorted(range(first, n - last), key=lambda j: (bool(np.isnan(w[j])), 0.0 if np.isnan(w[j]) else -w[j], j))
    return sorted(ends + rank[:budget - len(ends)])
