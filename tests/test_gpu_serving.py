"""The serving operators on the GPU against their definitions in 64 bits: paged append, paged attention, verification of
drafts, at the lengths, masks, strides and arrays where they can go wrong, into outputs filled with NaN."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import serving_oracle as S

sys.path.insert(0, __file__.rsplit("/", 1)[0])
import serving_batches as sb  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F8 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def rf():
    from paper_2603_10026_amd import binding
    binding.load_library()
    return binding


def say(msg):
    print(f"[case] {msg}", flush=True)


def nan_like(t):
    return torch.full(t.shape, float("nan"), dtype=t.dtype, device=DEV)


def attend(rf, bt, causal=True, scale=None, max_q=None, o=None, q=None):
    scale = 1 / math.sqrt(bt.d) if scale is None else scale
    q = bt.q.to(DEV) if q is None else q
    k, v = (sb.cache_on(c, DEV) for c in bt.caches)
    o = nan_like(q) if o is None else o
    rf.rf_paged_attention(q, k, v, *bt.on(DEV), max(bt.n + [0]) if max_q is None else max_q, scale, causal,
                          *bt.scales, o=o)
    torch.cuda.synchronize()
    return o


def expect(bt, causal=True, scale=None):
    scale = 1 / math.sqrt(bt.d) if scale is None else scale
    return S.attention(bt.q.float().numpy(), bt.values(0), bt.values(1), bt.seq_start, bt.kv_len, bt.table, scale, causal)


# n, k, Hq, Hkv, d, page
ATTENTION = [
    ([1], [1], 8, 2, 128, 16), ([1], [15], 4, 4, 64, 16), ([1], [16], 8, 1, 128, 16), ([1], [17], 3, 1, 64, 32),
    ([1] * 5, [1000, 0, 31, 257, 512], 8, 2, 128, 16),                     # one without keys: zeros
    ([1] * 70, [(37 * b) % 300 for b in range(70)], 4, 2, 64, 48),         # more sequences than lanes
    ([1, 1, 1], [4000, 3, 700], 16, 2, 128, 64),                           # one much longer than the others: cut into chunks
    ([5, 1, 3], [900, 640, 3], 8, 2, 128, 32),                             # drafts; a sequence of nothing but new tokens
    ([5] * 4, [333, 1200, 5, 64], 8, 2, 64, 48),
    ([4, 0, 7], [2, 50, 3], 8, 8, 128, 16),                                # fewer keys than tokens: rows that see nothing
    ([17], [100], 1, 1, 64, 16), ([33], [1500], 2, 1, 128, 32), ([40, 1, 0, 9], [40, 900, 77, 300], 12, 4, 64, 80),
    ([130], [130], 4, 1, 128, 64), ([129, 1], [700, 64], 8, 2, 64, 16), ([300, 1, 1], [1100, 500, 2], 4, 2, 128, 16),
    ([1] * 65, [64 * (b % 5) + b for b in range(65)], 8, 2, 128, 16),       # just more sequences than lanes
    ([(3 * b) % 7 for b in range(300)], [(3 * b) % 7 + (97 * b) % 150 for b in range(300)], 4, 4, 64, 16),
    ([1] * 90 + [40], [5] * 89 + [6000, 300], 4, 4, 64, 32),               # one long context among many short ones
    ([1] * 1100, [b % 23 for b in range(1100)], 1, 1, 64, 16),             # more sequences than a workgroup deals at once
    ([1] * 1030 + [20], [3] * 1030 + [2000], 2, 1, 64, 16), ([256], [2300], 8, 8, 64, 128), ([65], [64 * 20 + 1], 6, 2, 128, 48), ([700], [700], 2, 2, 128, 16),
]


@pytest.mark.parametrize("case", range(len(ATTENTION)))
@pytest.mark.parametrize("causal", (True, False))
def test_attention_matches_the_definition(rf, case, causal):
    n, k, Hq, Hkv, d, page = ATTENTION[case]
    say(f"paged attention {n[:6]} {k[:6]} Hq={Hq} Hkv={Hkv} d={d} page={page} causal={causal}")
    bt = sb.Batch(100 + case, n, k, Hq, Hkv, d, page, tail=2)
    o = attend(rf, bt, causal)
    sb.check_attention(o, *expect(bt, causal), max(k), "bf16")
    again = attend(rf, bt, causal)
    assert torch.equal(o.view(torch.int16), again.view(torch.int16))       # the same bits every time


@pytest.mark.parametrize("case", (0, 3, 4, 5, 6, 7, 9, 11, 12, 14, 15, 18, 21, 22))
def test_attention_8_bit_cache(rf, case):
    n, k, Hq, Hkv, d, page = ATTENTION[case]
    say(f"paged attention, 8-bit cache {n[:6]} {k[:6]} Hq={Hq} Hkv={Hkv} d={d} page={page}")
    bt = sb.Batch(200 + case, n, k, Hq, Hkv, d, page, dtype=F8, scales=(0.017, 0.29), tail=1)
    sb.check_attention(attend(rf, bt), *expect(bt), max(k), "fp8")


@pytest.mark.parametrize("dtype", (BF, F8))
@pytest.mark.parametrize("order", ((0, 2, 1, 3), (2, 0, 1, 3), (1, 0, 2, 3)))
def test_attention_strides(rf, order, dtype):
    """Caches with heads outside the slots, heads or slots outermost, and pages of a larger buffer; queries inside a
    projection's output, results between rows of NaN."""
    say(f"paged attention, cache order {order} {dtype}")
    bt = sb.Batch(300, [3, 1, 90], [200, 65, 333], 8, 4, 64, 16, dtype=dtype, order=order, pad=3)
    wide = torch.full((bt.T, 13, 96), float("nan"), dtype=BF, device=DEV)
    q = wide[:, 2:10, 16:80]
    q.copy_(bt.q)
    out = torch.full((bt.T + 1, 8, 2, 64), float("nan"), dtype=BF, device=DEV)
    attend(rf, bt, q=q, o=out[:bt.T, :, 1])
    sb.check_attention(out[:bt.T, :, 1], *expect(bt), 333, "strides")
    assert bool(torch.isnan(out[bt.T]).all()) and bool(torch.isnan(out[:, :, 0]).all())


@pytest.mark.parametrize("scale", (0.0, -0.3, 2.5))
def test_attention_scales(rf, scale):
    say(f"paged attention, scale {scale}")
    bt = sb.Batch(310, [2, 1, 200], [200, 800, 260], 8, 2, 128, 32)
    sb.check_attention(attend(rf, bt, scale=scale), *expect(bt, scale=scale), 800, f"scale {scale}")


@pytest.mark.parametrize("n,k", (([6, 1], [300, 70]), ([1], [2000]), ([150, 3], [180, 40]), ([40], [1400])))
@pytest.mark.parametrize("dtype", (BF, F8))
def test_attention_infinities_and_nan(rf, n, k, dtype):
    """Values that are no numbers in the new tokens' own slots: rows that do not see them are untouched, rows that do
    have them in their column.  (8-bit codes hold no infinity.)"""
    say(f"paged attention, infinities and NaN {n} {k} {dtype}")
    bt = sb.Batch(320, n, k, 8, 2, 64, 16, dtype=dtype)
    for b, (nb, ln) in enumerate(zip(n, k)):
        for back, (col, x) in {nb - 1: (3, math.nan), nb // 2: (5, math.inf), 0: (7, math.nan)}.items():
            j = ln - 1 - back
            bt.caches[1][bt.table[b, j // 16], j % 16, 0, col] = x if dtype == BF else math.nan
    bt.q[0, 4, 2] = math.nan                              # a query of NaN stays in its row
    want = expect(bt)
    assert np.isnan(want[0]).any() and np.isfinite(want[0][:, :, 20]).sum() > 4
    sb.check_attention(attend(rf, bt), *want, max(k), "not finite")


def test_attention_any_max_q_gives_the_same_rows(rf):
    """max_q chooses kernels only."""
    say("paged attention, max_q 0, 1, true, T")
    bt = sb.Batch(330, [1, 60, 1, 9], [900, 1100, 33, 9], 8, 2, 128, 16)
    want = expect(bt)
    for m in (0, 1, 60, bt.T, 1 << 40):
        sb.check_attention(attend(rf, bt, max_q=m), *want, 1100, f"max_q {m}")


def test_attention_bad_pages_and_overlong_sequences_are_nan(rf):
    say("paged attention, pages outside the cache, more keys than the table has room for")
    bt = sb.Batch(340, [1, 1, 1, 2, 80], [100, 40, 50, 64, 90], 4, 2, 64, 16)
    clean = attend(rf, bt)
    width = bt.table.shape[1]
    bt.table[0, 3], bt.table[1, 0] = -1, bt.n_pages       # seen by their sequences' rows
    bt.table[4, 5] = -(2 ** 31)                           # key 80 on: seen by the last tokens of 80 (the first sees 10)
    bt.kv_len[2] = width * 16 + 1
    o = attend(rf, bt)
    assert bool(torch.isnan(o[[0, 1, 2]].float()).all())
    assert torch.equal(o[3:5], clean[3:5])                # another sequence's rows
    assert bool(torch.isnan(o[5 + 70:].float()).all())
    bt.kv_len[:] = 2 ** 31 - 1
    assert bool(torch.isnan(attend(rf, bt).float()).all())
    bt.kv_len[:] = -(2 ** 31)
    assert bool((attend(rf, bt) == 0).all())


@pytest.mark.parametrize("sequences", (3, 9, 200, 1200))
def test_attention_arrays_of_nonsense_stay_inside(rf, sequences):
    """seq_start that descends, leaves the tokens or names them many times over: whatever comes out, rows of no sequence
    are left alone, and so is everything outside."""
    say(f"paged attention and append, seq_start out of range, {sequences} sequences")
    r = np.random.default_rng(351)
    n = [3] * sequences
    bt = sb.Batch(350, n, [400 if b < 3 else 7 for b in range(sequences)], 4, 2, 64, 16, tail=4)
    T, B = bt.T, sequences
    kinds = [np.full(B + 1, T - 1), np.where(np.arange(B + 1) % 2, T, 0), np.arange(B + 1)[::-1], r.integers(-T, 2 * T, B + 1),
             r.integers(-(2 ** 31), 2 ** 31, B + 1), np.full(B + 1, 2 ** 31 - 1), np.full(B + 1, -(2 ** 31))]
    guard = torch.full((T + 64, 4, 64), float("nan"), dtype=BF, device=DEV)
    for i, starts in enumerate(kinds):
        bt.seq_start = starts.astype(np.int32)
        for max_q in (1, T):
            say(f"  kind {i}, max_q {max_q}")
            guard.fill_(float("nan"))
            attend(rf, bt, max_q=max_q, o=guard[32:32 + T])
            assert bool(torch.isnan(guard[:32].float()).all()) and bool(torch.isnan(guard[32 + T:].float()).all())
            if i in (0, 5, 6):
                assert bool(torch.isnan(guard[32:32 + T - 1].float()).all())
        q, nk, nv = (x.to(DEV) for x in (bt.q, bt.new_k, bt.new_v))
        k, v = (sb.cache_on(c, DEV) for c in bt.caches)
        cos, sin = (torch.from_numpy(x).to(DEV) for x in tables(64, 500))
        rf.rf_paged_append(q, nk, nv, k, v, *bt.on(DEV), cos=cos, sin=sin, q_out=guard[32:32 + T])
        torch.cuda.synchronize()
        assert bool(torch.isnan(guard[:32].float()).all()) and bool(torch.isnan(guard[32 + T:].float()).all())


def test_attention_tables_with_room_for_millions_of_keys(rf):
    """Long rows of the page table (keys are then counted in larger units), sequences of ordinary lengths."""
    say("paged attention, a table of 2^24 keys")
    for n, k in (([1, 1, 5], [3000, 40, 700]), ([1, 130], [900, 1500])):
        bt = sb.Batch(370, n, k, 8, 2, 64, 16)
        want = expect(bt)
        wide = np.full((len(n), (1 << 24) // 16), -5, np.int32)
        wide[:, :bt.table.shape[1]] = bt.table
        bt.table = wide
        sb.check_attention(attend(rf, bt), *want, max(k), "wide table")


def test_attention_offsets_past_32_bits(rf):
    """A cache of over 2^32 elements (9 GB each), its pages at both ends."""
    say("paged attention and append, offsets past 32 bits")
    page, Hkv, d = 64, 8, 128
    n_pages = (1 << 32) // (page * Hkv * d) + 40
    k, v = (torch.zeros((n_pages, page, Hkv, d), dtype=BF, device=DEV) for _ in range(2))
    bt = sb.Batch(360, [1, 40], [300, 200], 16, Hkv, d, page, extra=0)
    far = torch.arange(n_pages - bt.n_pages, n_pages)
    far[::2] = torch.arange(0, len(far[::2]))
    for c, x in zip((k, v), bt.caches):
        c[far.to(DEV)] = x.to(DEV)
    starts, lens, pages = bt.on(DEV)
    moved = far.to(DEV)[pages.long().clamp(0, bt.n_pages - 1)].to(torch.int32)
    q = bt.q.to(DEV)
    o = nan_like(q)
    rf.rf_paged_attention(q, k, v, starts, lens, moved, 40, 1 / math.sqrt(d), o=o)
    sb.check_attention(o, *expect(bt), 300, "far pages")
    rf.rf_paged_append(q, bt.new_k.to(DEV), bt.new_v.to(DEV), k, v, starts, lens, moved)
    torch.cuda.synchronize()
    for b, (t0, nb) in enumerate(S.spans(bt.seq_start, bt.T)):
        for i in range(nb):
            j = bt.k[b] - nb + i
            at = int(far[bt.table[b, j // page]])
            assert torch.equal(k[at, j % page].cpu(), bt.new_k[t0 + i]) and torch.equal(v[at, j % page].cpu(), bt.new_v[t0 + i])


# ---- append ---------------------------------------------------------------------------------------

# n, k, Hq, Hkv, d, page, rot, interleaved, norms
APPEND = [
    ([1], [1], 8, 2, 128, 16, 128, False, True), ([1] * 7, [5, 16, 17, 1, 300, 2, 64], 4, 1, 128, 16, 128, True, True),
    ([1] * 130, [1 + (7 * b) % 90 for b in range(130)], 2, 2, 64, 32, 64, False, False),
    ([0, 33, 0, 2, 0], [4, 40, 0, 2, 9], 6, 3, 64, 48, 32, True, True), ([200, 3], [200, 1000], 8, 8, 128, 64, 64, False, True),
    ([3, 4], [1, 9], 5, 1, 128, 16, 96, False, False),                     # tokens without a position
    ([9], [20], 1, 1, 64, 16, 16, False, True), ([9], [20], 3, 1, 64, 16, 48, True, False), ([5], [77], 7, 7, 128, 80, 0, False, True),
    ([5, 1], [77, 12], 7, 7, 64, 16, 0, False, False),
    ([3, 2], [30, 40], 4, 2, 64, 16, 64, False, "q"), ([3, 2], [30, 40], 4, 2, 128, 16, 64, True, "k"),   # one norm alone
    ([600], [600], 16, 2, 64, 16, 64, False, True), ([700], [701], 8, 8, 128, 64, 128, False, True),       # many tokens
]


def tables(rot, rows):
    angle = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def run_append(rf, bt, rot, interleaved, norms, rows=None, in_place=False, strided=False):
    r = np.random.default_rng(5)
    g = [sb.bf16(1 + 0.3 * r.standard_normal(bt.d)) if norms and norms != skip else None for skip in ("k", "q")]
    cs = tables(rot, rows or max(bt.k) + 3) if rot else (None, None)
    k, v = (sb.cache_on(c, DEV) for c in bt.caches)
    if strided:
        both = torch.full((bt.T, (bt.Hq + 2 * bt.Hkv) * bt.d), float("nan"), dtype=BF, device=DEV)
        parts = both.split([bt.Hq * bt.d, bt.Hkv * bt.d, bt.Hkv * bt.d], -1)
        q, nk, nv = (p.unflatten(-1, (-1, bt.d)) for p in parts)
        for to, x in ((q, bt.q), (nk, bt.new_k), (nv, bt.new_v)):
            to.copy_(x)
    else:
        q, nk, nv = (x.to(DEV) for x in (bt.q, bt.new_k, bt.new_v))
    out = q if in_place else nan_like(q)
    dev = lambda x: None if x is None else (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).to(DEV)  # noqa: E731
    rf.rf_paged_append(q, nk, nv, k, v, *bt.on(DEV), q_norm=dev(g[0]), k_norm=dev(g[1]), eps=1e-5, cos=dev(cs[0]),
                       sin=dev(cs[1]), interleaved=interleaved, k_scale=bt.scales[0], v_scale=bt.scales[1], q_out=out)
    torch.cuda.synchronize()
    f = [None if x is None else x.float().numpy() for x in g]
    want = S.append(bt.q.float().numpy(), bt.new_k.float().numpy(), bt.new_v.float().numpy(), f[0], f[1], 1e-5, *cs,
                    interleaved, bt.seq_start, bt.kv_len, bt.table, bt.page)
    return out, k, v, want


def check_append(bt, out, k, v, want, norms, rot, in_place=False):
    """A normalised value is off by (d / 2 + 6) u of itself (a sum of squares, its root, two products), a rotated one by 3
    u more of its two terms, sqrt(2) times the pair's larger at most: `terms` times u times the head's largest value, no more."""
    terms = ((bt.d / 2 + 6) if norms else 0) + (3 if rot else 0)
    terms *= 1.5
    q_want, slots = want
    live = ~np.isnan(q_want) | (np.arange(bt.T) < bt.seq_start[-1])[:, None, None]
    biggest = lambda x: np.broadcast_to(np.nanmax(np.abs(np.where(np.isnan(x), 0, x)), -1, keepdims=True), x.shape)  # noqa: E731
    got = out.clone()
    if not in_place:
        assert bool(torch.isnan(got[int(bt.seq_start[-1]):].float()).all())     # rows of no sequence
    q_live = np.where(live, q_want, 0)
    got[torch.from_numpy(~live).to(DEV)] = 0
    sb.check_rounded(got, q_live, BF, biggest(q_live), "q", terms=terms)
    for which, (cache, was) in enumerate(zip((k, v), bt.caches)):
        cache, expected = cache.cpu(), was.clone()
        for (pg, sl), kv in slots.items():
            if not 0 <= pg < bt.n_pages:
                continue
            x = kv[which][None]
            sb.check_rounded(cache[pg, sl][None], x, bt.dtype, biggest(x), f"slot {pg},{sl}", scale=bt.scales[which],
                             terms=terms + 1 if which == 0 or bt.dtype == F8 else 0)
            expected[pg, sl] = cache[pg, sl]
        same = cache.contiguous().view(torch.uint8) == expected.contiguous().view(torch.uint8)
        assert bool(same.all()), "a slot that no new token has changed"


@pytest.mark.parametrize("case", range(len(APPEND)))
@pytest.mark.parametrize("dtype", (BF, F8))
def test_append_matches_the_definition(rf, case, dtype):
    n, k, Hq, Hkv, d, page, rot, inter, norms = APPEND[case]
    say(f"paged append {n[:6]} {k[:6]} Hq={Hq} Hkv={Hkv} d={d} page={page} rot={rot} interleaved={inter} norms={norms} {dtype}")
    bt = sb.Batch(400 + case, n, k, Hq, Hkv, d, page, dtype=dtype, scales=(1.0, 1.0) if dtype == BF else (0.011, 0.3), tail=2)
    check_append(bt, *run_append(rf, bt, rot, inter, norms), norms, rot)


@pytest.mark.parametrize("order", ((0, 1, 2, 3), (2, 0, 1, 3)))
def test_append_in_place_inside_a_projection(rf, order):
    say(f"paged append in place, strided inputs, cache order {order}")
    bt = sb.Batch(430, [4, 1, 30], [10, 100, 64], 8, 2, 128, 16, order=order, pad=1)
    check_append(bt, *run_append(rf, bt, 128, False, True, in_place=True, strided=True), True, 128, in_place=True)


def test_append_past_the_tables_saturation_and_bad_pages(rf):
    say("paged append: positions past the tables, pages outside the cache, values past the codes")
    bt = sb.Batch(440, [4, 2, 1], [40, 30, 20], 4, 2, 64, 16)
    bt.table[1, 1] = bt.n_pages + 3                       # both tokens of the second sequence: not cached
    out, k, v, want = run_append(rf, bt, 64, False, True, rows=38)   # positions 38, 39 of the first have no angle
    assert np.isnan(want[0][2:4]).all()
    check_append(bt, out, k, v, want, True, 64)
    bt = sb.Batch(441, [3], [3], 1, 1, 64, 16, dtype=F8, scales=(1e-3, 1e-3))
    bt.new_k[1, 0, 5], bt.new_v[2, 0, 7] = math.nan, -math.inf
    out, k, v, want = run_append(rf, bt, 0, False, False)
    check_append(bt, out, k, v, want, False, 0)
    assert float(k.float()[bt.table[0, 0], 0].abs().max()) == 448.0


# ---- verification ---------------------------------------------------------------------------------

def verify_inputs(seed, n, V, dtype, with_draft, sharp=3.0):
    r = np.random.default_rng(seed)
    R = sum(n)
    logits = torch.from_numpy(sharp * r.standard_normal((R, V)))
    p = torch.softmax(logits, -1).to(dtype)
    q = torch.softmax(logits + torch.from_numpy(0.5 * r.standard_normal((R, V))), -1)
    x = torch.multinomial(q, 1, generator=torch.Generator().manual_seed(seed))[:, 0].to(torch.int32) if R else torch.zeros(0, dtype=torch.int32)
    starts = torch.from_numpy(np.concatenate(([0], np.cumsum(n))).astype(np.int32))
    u = torch.from_numpy(r.random(R, np.float32)), torch.from_numpy(r.random(len(n), np.float32))
    return p, q.to(dtype) if with_draft else None, x, *u, starts


def check_verify(rf, args, what, tail=0):
    p, q, x, ua, us, starts = args
    f = lambda t: None if t is None else t.float().numpy()  # noqa: E731
    out, acc, margin = S.verify(f(p), f(q), x.numpy(), f(ua), f(us), starts.numpy())
    # 64-bit sums in another order move a border by V 2^-53 of the whole at most: nothing here may be nearer
    assert margin.min(initial=1) > p.shape[1] * 2.0 ** -52, "inputs on a border"
    dev = [None if t is None else t.to(DEV) for t in args]
    got, a = rf.rf_verify_drafts(*dev, out=torch.full((len(x),), -7, dtype=torch.int32, device=DEV),
                                 accepted=torch.full((len(us),), -7, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert a.cpu().tolist() == acc.tolist(), what
    assert got.cpu().tolist() == out.tolist(), what
    return out, acc


VERIFY = [([1], 1), ([4], 2), ([2, 1, 5], 17), ([3] * 9, 1000), ([9, 1, 2], 4097), ([6] * 4, 32000), ([2, 70, 1], 777),
          ([0, 3, 0, 0, 2], 50001), ([3, 2], 300007), ([130], 64)]


@pytest.mark.parametrize("case", range(len(VERIFY)))
@pytest.mark.parametrize("dtype", (torch.float32, BF))
@pytest.mark.parametrize("with_draft", (True, False))
def test_verify_matches_the_definition(rf, case, dtype, with_draft):
    n, V = VERIFY[case]
    say(f"verify {n[:6]} V={V} {dtype} draft={with_draft}")
    check_verify(rf, verify_inputs(500 + case, n, V, dtype, with_draft), f"{n} {V}")


def test_verify_rows_of_any_alignment_and_behind_the_last_sequence(rf):
    say("verify: pitches and starts of any alignment, rows of no sequence")
    for dtype, V in ((torch.float32, 9001), (BF, 9001)):
        p, q, x, ua, us, starts = verify_inputs(530, [3, 4, 2], V, dtype, True)
        wide = [torch.full((9, V + 5), float("nan"), dtype=dtype) for _ in range(2)]
        wide[0][:, 3:3 + V], wide[1][:, 1:1 + V] = p, q
        want, acc, _ = S.verify(p.float().numpy(), q.float().numpy(), x.numpy(), ua.numpy(), us.numpy()[:2], starts.numpy()[:3])
        got, a = rf.rf_verify_drafts(wide[0].to(DEV)[:, 3:3 + V], wide[1].to(DEV)[:, 1:1 + V], x.to(DEV), ua.to(DEV), us[:2].to(DEV),
                                     starts[:3].to(DEV), out=torch.full((9,), -7, dtype=torch.int32, device=DEV))
        assert got.cpu().tolist() == want.tolist() and a.cpu().tolist() == acc.tolist()
        assert got.cpu().tolist()[7:] == [-7, -7]


def test_verify_borders(rf):
    """Random numbers of 0 and just below 1, equal probabilities, nothing left of the target, tokens outside the
    vocabulary, weights that are no numbers."""
    say("verify: borders")
    V, one = 5000, np.nextafter(np.float32(1), np.float32(0))
    p = torch.zeros((12, V)); q = torch.zeros((12, V))
    p[:, 7], p[:, 4400], q[:, 7], q[:, 4400] = 0.25, 0.75, 0.25, 0.75
    x = torch.full((12,), 7, dtype=torch.int32)
    starts = torch.arange(0, 13, 2, dtype=torch.int32)
    ua = torch.tensor([0.999, 0, 0, 0, float(one), 0, 0.5, 0, 0, 0, 0, 0])
    us = torch.tensor([0.0, float(one), 0.24, 0.26, 0.5, 0.5])
    q[2, 7] = 0.0                                  # p > 0, q = 0: accepted
    q[4] = 1.0                                     # everything the target has is covered: its own probabilities
    q[6, 7], p[6, 7] = 1.0, 0.5                    # u q = p exactly: refused
    x[8] = V                                       # outside: refused
    p[10, 7], q[10, 7], p[10, 3] = 0.1, 0.9, math.nan
    ua[10] = 0.9
    out, acc, _ = S.verify(p.numpy(), q.numpy(), x.numpy(), ua.numpy(), us.numpy(), starts.numpy())
    assert acc.tolist() == [1, 1, 0, 0, 0, 0] and out[10] == -1
    dev = [t.to(DEV) for t in (p, q, x, ua, us, starts)]
    got, a = rf.rf_verify_drafts(*dev)
    assert a.cpu().tolist() == acc.tolist() and got.cpu().tolist() == out.tolist()
    x[8] = -1
    got, a = rf.rf_verify_drafts(p.to(DEV), None, x.to(DEV), *dev[3:])
    out, acc, _ = S.verify(p.numpy(), None, x.numpy(), ua.numpy(), us.numpy(), starts.numpy())
    assert a.cpu().tolist() == acc.tolist() and got.cpu().tolist() == out.tolist()
