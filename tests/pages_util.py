"""A paged cache and its operators in 64 bits, for tests/test_gpu_pages.py and tests/test_pages_host.py.  Plain loops
over sequences, heads and tokens; shares no code with the library."""
from __future__ import annotations

import math
import random

import numpy as np
import torch

E4M3 = torch.float8_e4m3fn
LEAST, MOST = -117, 120


# ---- e4m3 rows: codes and one exponent

def exponent(row: np.ndarray) -> int:
    """Least k in [LEAST, MOST] with max|x| <= 448 * 2**k over the finite elements (fp64 in, exact)."""
    top = max((abs(float(x)) for x in row if math.isfinite(x)), default=0.0)
    k = LEAST
    while k < MOST and top > math.ldexp(448.0, k):
        k += 1
    return k


def nearest_code(y: float) -> float:
    """The e4m3 value nearest to y, |y| <= 448, ties to the even code."""
    if y == 0.0:
        return 0.0
    _, e = math.frexp(abs(y))                       # |y| = m * 2**e, m in [0.5, 1)
    step = math.ldexp(1.0, max(e - 1, -6) - 3)
    return float(np.round(y / step)) * step         # (np.round: half to even; the division is exact)


def quantised(row: np.ndarray):
    """(values of the codes, exponent) of a row."""
    k = exponent(row)
    most = 240.0 if k == MOST else 448.0
    codes = [nearest_code(max(-most, min(most, math.ldexp(float(x), -k)))) if math.isfinite(x) else math.nan for x in row]
    return np.array(codes), k


def quantised_tensor(x: torch.Tensor):
    """The same for many rows at once, with torch in 64 bits: (codes float8, exponent bytes)."""
    x = x.double()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), 0.0).amax(-1, keepdim=True).numpy()
    m, e = np.frexp(top)
    k = np.clip(np.where(top == 0, LEAST, np.where(m <= 0.875, e - 9, e - 8)), LEAST, MOST)
    most = np.where(k == MOST, 240.0, 448.0)
    y = np.clip(np.ldexp(np.where(finite.numpy(), x.numpy(), 0.0), -k), -most, most)
    _, e = np.frexp(np.abs(y))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    codes = torch.from_numpy(np.where(finite.numpy(), np.round(y / step) * step, np.nan))
    return codes.to(torch.float32).to(E4M3), torch.from_numpy((k + 127).astype(np.uint8)).squeeze(-1)


# ---- a pool, its table and what the sequences hold

class Cache:
    """A pool with `spare` pages of stale rows; sequence s has lens[s] rows.  All on the CPU."""

    def __init__(self, seed, lens, kv_heads, d, page, cache_dtype, dtype, width=None, spare=3, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.kv_heads, self.d, self.page, self.type, self.dtype = list(lens), kv_heads, d, page, cache_dtype, dtype
        used = [-(-n // page) for n in lens]
        self.width = width or max(1, max(used))
        n_page = sum(used) + spare
        order = torch.randperm(n_page, generator=g).tolist()
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = torch.tensor(order[at:at + u], dtype=torch.int32)
            at += u
        self.unused = order[at:]
        self.scales = {"k": None, "v": None}
        self.pool = {}
        for name in ("k", "v"):
            x = (torch.randn(n_page, kv_heads, page, d, generator=g) * scale).to(dtype)
            if cache_dtype == E4M3:
                self.pool[name], self.scales[name] = quantised_tensor(x)
            else:
                self.pool[name] = x

    def rows(self, name, s):
        """[KV heads, lens[s], d] in 64 bits; rows of pages that do not exist are zeros."""
        out = torch.zeros(self.kv_heads, self.lens[s], self.d, dtype=torch.float64)
        for r in range(0, self.lens[s], self.page):
            p = int(self.table[s, r // self.page])
            n = min(self.page, self.lens[s] - r)
            if 0 <= p < self.pool[name].shape[0]:
                x = self.pool[name][p, :, :n].to(torch.float32).double()
                if self.type == E4M3:
                    x = x * torch.ldexp(torch.ones(()).double(), self.scales[name][p, :, :n].int() - 127).unsqueeze(-1)
                out[:, r:r + n] = x
        return out

    def put(self, name, s, r, h, row):
        """Makes row r of head h hold `row` (bf16 or fp32 caches)."""
        self.pool[name][int(self.table[s, r // self.page]), h, r % self.page] = row

    def on(self, dev):
        import paper_2505_19602_amd as skv
        to = lambda t: None if t is None else t.to(dev)
        return skv.Pages(to(self.pool["k"]), to(self.pool["v"]), to(self.table),
                         torch.tensor(self.lens, dtype=torch.int32, device=dev), to(self.scales["k"]), to(self.scales["v"]))


def sees(p, length, causal, window, sinks):
    """Which rows a token at position p sees."""
    j = torch.arange(length)
    ok = torch.ones(length, dtype=torch.bool)
    if causal:
        ok &= j <= p
    if window:
        ok &= (j > p - window) | (j < sinks)
    return ok


def attend(cache, s, q, causal, window, sinks, sm_scale):
    """q [H, n, d] of the last n rows of sequence s -> (out [H, n, d] in 64 bits, how far each element may be off).

    The bound, with u the half step of the arithmetic's type (bf16 2^-8, fp32 2^-24), w the exact weights and
    A = sum_j w_j |v_j|:
      logits: d products summed in fp32, E = d * 2^-24 * sum_c |q_c k_c| * scale, scaled and shifted by at most three
        roundings of magnitudes up to the largest logit, exp2 within 2^-21: a weight is off by at most
        D = E + 3 * 2^-24 * max|logit| + 2^-21, relative, and so is their sum: 2 D A;
      weights rounded to the type before the product, the sum over the rounded ones: u * (A + |out|);
      sums over n keys in fp32: n * 2^-24 * 2 A;   the output's own rounding: u * |out|.
    Products of rounding terms are covered by a factor of 1.01; the least normal number stands for what underflows."""
    q = q.double()
    k, v = cache.rows("k", s), cache.rows("v", s)
    H, n, d = q.shape
    length, group = k.shape[1], H // cache.kv_heads
    out, tol = torch.zeros(H, n, d, dtype=torch.float64), torch.zeros(H, n, d, dtype=torch.float64)
    u = 2.0 ** -8 if cache.dtype == torch.bfloat16 else 2.0 ** -24
    for h in range(H):
        kh, vh = k[h // group], v[h // group]
        for t in range(n):
            ok = sees(length - n + t, length, causal, window, sinks)
            if not ok.any():
                continue
            keys, vals = kh[ok], vh[ok]
            logit = keys @ q[h, t] * sm_scale
            w = torch.softmax(logit, 0)
            out[h, t] = w @ vals
            a = w @ vals.abs()
            e = d * 2.0 ** -24 * float((keys.abs() @ q[h, t].abs()).max()) * sm_scale
            delta = e + 3 * 2.0 ** -24 * float(logit.abs().max()) + 2.0 ** -21
            tol[h, t] = 1.01 * (2 * delta * a + u * (a + out[h, t].abs()) + 2 * len(keys) * 2.0 ** -24 * a
                                + u * out[h, t].abs()) + 2.0 ** -126
    return out, tol


def lengths(rng: random.Random, seqs, most, new, ragged):
    lens, counts = [], []
    for s in range(seqs):
        n = rng.randint(0, new) if ragged and s else new
        lens.append(rng.randint(n, max(n, most)) if ragged and s else max(most, new))
        counts.append(n)
    return lens, counts
