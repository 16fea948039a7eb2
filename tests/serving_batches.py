"""Ragged batches over a paged cache for the tests of the serving operators: seeded, on the host, with the bounds that a
result may be off by.  Slots that nobody's keys are in hold NaN."""
import numpy as np
import torch

from oracle import serving_oracle as S

E4M3_MAX = 448.0
HALF = {torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}   # half a step, relative


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


class Batch:
    """n, k: new and cached tokens of each sequence (k with the new ones).  order: order of the cache's axes in memory."""

    def __init__(self, seed, n, k, Hq, Hkv, d, page, dtype=torch.bfloat16, scales=(1.0, 1.0), order=(0, 1, 2, 3), pad=0,
                 tail=0, extra=2, device="cpu"):
        r = np.random.default_rng(seed)
        self.n, self.k, self.Hq, self.Hkv, self.d, self.page, self.dtype, self.scales = n, k, Hq, Hkv, d, page, dtype, scales
        self.T = sum(n) + tail                                   # (tail: rows behind the last sequence)
        per = [-(-x // page) for x in k]
        self.n_pages = sum(per) + extra
        ids = r.permutation(self.n_pages)
        width = max(per + [1]) + 1
        table = r.integers(-9, 10 ** 6, (len(n), width)).astype(np.int32)   # past a sequence's pages: anything
        at = 0
        for b, c in enumerate(per):
            table[b, :c] = ids[at:at + c]
            at += c
        self.table = table
        self.seq_start = np.concatenate(([0], np.cumsum(n))).astype(np.int32)
        self.kv_len = np.array(k, np.int32)
        used = np.zeros((self.n_pages, page), bool)
        for b, ln in enumerate(k):
            for j in range(ln):
                used[table[b, j // page], j % page] = True
        self.used = used
        self.caches = []
        for s in scales:
            x = r.standard_normal((self.n_pages, page, Hkv, d)).astype(np.float32)
            x[~used] = np.nan
            t = torch.from_numpy(x)
            t = t.to(dtype) if dtype == torch.bfloat16 else (t / s).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)
            buf = torch.empty([t.shape[o] + (pad if o == order[0] else 0) for o in order], dtype=dtype)
            view = buf.narrow(0, 0, t.shape[order[0]]).permute(*[order.index(a) for a in range(4)])
            view.copy_(t)
            self.caches.append(view)
        self.q = bf16(r.standard_normal((self.T, Hq, d)))
        self.new_k, self.new_v = (bf16(r.standard_normal((self.T, Hkv, d))) for _ in range(2))
        self.rng = r

    def values(self, which):
        """What cache `which` stands for."""
        return self.caches[which].float().numpy().astype(np.float64) * self.scales[which]

    def on(self, device):
        """(seq_start, kv_len, pages) there."""
        return tuple(torch.from_numpy(x).to(device) for x in (self.seq_start, self.kv_len, self.table))


def cache_on(view, device):
    """A cache on a device with the same order in memory."""
    order = sorted(range(4), key=lambda a: -view.stride(a))
    return view.permute(*order).contiguous().to(device).permute(*[order.index(a) for a in range(4)])


def attention_bound(o, spread, score, longest, d):
    """How far o may be off, by arithmetic.  With u = 2^-24 and h = 2^-8 (half a step of bf16):
      - a score is a sum of d products in fp32, scaled and taken to base 2: off by at most (d + 8) u score, absolute, which
        moves a probability by that much relative to itself, numerator and denominator;
      - every exponential is off by 2 u (the hardware's) and its rounding to bf16 by h, in the numerator and, as the same
        rounded values are summed, in the denominator;
      - the sums over the keys and the merges of partial ones: longest additions of u each, numerator and denominator;
      - the result's rounding: h |o|.
    The sum of the numerator's terms is spread = sum p |v|."""
    u, h = 2.0 ** -24, 2.0 ** -8
    rel = 2 * (1 + 2 * h) * ((d + 8) * u * score + 2 * u + h + (longest + 64) * u)
    return spread * rel[..., None] + h * np.abs(o) + 1e-30


def check_attention(got, o, spread, score, longest, what):
    got = got.float().cpu().numpy().astype(np.float64)
    bound = attention_bound(o, spread, score, longest, got.shape[-1])
    finite = np.isfinite(o)
    assert np.array_equal(np.isnan(got), np.isnan(o)), f"{what}: NaN where there should be none, or none where there should be"
    assert np.array_equal(got[~finite & ~np.isnan(o)], o[~finite & ~np.isnan(o)]), what
    err = np.abs(got[finite] - o[finite]) / bound[finite]
    print(f"  {what}: largest error {err.max() if err.size else 0:.3f} of its bound", flush=True)
    assert err.size == 0 or err.max() <= 1, what


def check_rounded(got, want, dtype, spread, what, scale=1.0, terms=0):
    """Values rounded once to dtype from fp32 results that are off by terms * 2^-24 * spread; got as stored."""
    got = got.float().cpu().numpy().astype(np.float64)
    want, off = want / scale, np.abs(spread) / scale * terms * 2.0 ** -24
    if dtype == torch.float8_e4m3fn:
        want = np.clip(want, -E4M3_MAX, E4M3_MAX)
    floor = 2.0 ** -10 if dtype == torch.float8_e4m3fn else 0.0           # half of E4M3's smallest step
    bound = np.maximum((np.abs(want) + off) * HALF[dtype], floor) + off
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN"
    ok = ~np.isnan(want)
    err = np.abs(got - want)[ok] - bound[ok]
    assert err.size == 0 or err.max() <= 0, f"{what}: {err.max():.3e} over its bound"
