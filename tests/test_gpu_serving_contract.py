"""What the header says of a serving step's rows beside the formulas: rows of no sequence may hold anything, and scores of
-inf are as good as no key."""
import math
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, __file__.rsplit("/", 1)[0])
import serving_batches as sb  # noqa: E402
from test_gpu_serving import BF, DEV, F8, attend, expect, rf, run_append, say  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", ([1, 3], [1] * 70, [400, 200]))
@pytest.mark.parametrize("dtype", (BF, F8))
def test_rows_of_no_sequence_may_hold_anything(rf, n, dtype):  # noqa: F811
    """Rows ahead of the first sequence and behind the last one."""
    say(f"rows of no sequence {n[:4]} {dtype}")
    T, bits = sum(n), lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    results = []
    for x in (0.0, math.nan, math.inf):
        bt = sb.Batch(730, n, [a + 20 for a in n], 8, 2, 64, 16, dtype=dtype, scales=(1.0, 1.0) if dtype == BF else (0.02, 0.02), tail=7)
        bt.seq_start = bt.seq_start + 3
        for t in (bt.q, bt.new_k, bt.new_v):
            t[:3] = t[T + 3:] = x
        out, k, v, _ = run_append(rf, bt, 64, False, True)
        o = attend(rf, bt)
        for y in (out, o):
            assert bool(torch.isnan(y[:3].float()).all()) and bool(torch.isnan(y[T + 3:].float()).all())   # as they were
        results.append([bits(y) for y in (out[3:T + 3], k, v, o[3:T + 3])])
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("n,k", (([1, 2, 1], [40, 3000, 700]), ([6], [90]), ([200, 1], [260, 1500]), ([150], [150])))
def test_scores_of_minus_infinity(rf, n, k):  # noqa: F811
    """Some keys of every sequence, the first ones, and all of the last sequence."""
    say(f"scores of -inf {n} {k}")
    bt = sb.Batch(740, n, k, 8, 2, 64, 16)
    bt.q[:, :, 0] = 1.0
    size = expect(bt)[2]                                            # (the finite scores are among these)
    for b, ln in enumerate(k):
        for j in range(ln if b == len(k) - 1 and b > 0 else 20):
            bt.caches[0][bt.table[b, j // 16], j % 16, :, 0] = -math.inf
    with np.errstate(invalid="ignore"):
        o, spread, _ = expect(bt)
    nothing = np.isnan(o).all(-1)
    assert nothing.any() == (len(n) > 1 or n[0] == k[0]) and not nothing.all()
    sb.check_attention(attend(rf, bt), np.where(nothing[..., None], 0, o), np.nan_to_num(spread), size, max(k), "-inf")
