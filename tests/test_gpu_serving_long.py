"""Paged attention of contexts so long that the chunks of a launch take several rounds of the chip, and of sequences whose
keys outlast the page addresses that a wavefront looks up at once."""
import ctypes
import math
import sys

import pytest
import torch

sys.path.insert(0, __file__.rsplit("/", 1)[0])
import serving_batches as sb  # noqa: E402
from test_gpu_serving import BF, DEV, F8, expect, nan_like, rf, say  # noqa: E402,F401
from test_gpu_serving_large import check  # noqa: E402

pytestmark = pytest.mark.gpu

MANY = [2000 + (5501 * b) % 14000 for b in range(24)]
# n, k, Hq, Hkv, d, page, packed rows of a tile
ROUNDS = [
    ([1] * 24, MANY, 8, 8, 64, 16, [16]), ([1] * 24, MANY, 16, 8, 64, 48, [16]),
    ([5] * 24, MANY, 32, 8, 64, 16, [32]), ([1] * 24, MANY, 16, 8, 128, 64, [16]),
    ([1] * 70, [100 + 3 * b for b in range(60)] + [9000 + 900 * b for b in range(10)], 16, 16, 64, 16, [16]),
    ([300] * 3, [16000, 3000, 9000], 32, 8, 64, 16, [128]),
    ([200] + [1] * 20, [12000] + [2000 + 368 * b for b in range(20)], 32, 8, 64, 48, [16, 128]),
]


def shares(n, k, group, Hkv, rows, both):
    """(keys of a workgroup's even share of one round, keys of the longest tile): of the sequences that tiles of so many rows
    take."""
    few = [(a, b) for a, b in zip(n, k) if a * group <= 16]
    mine = few if both and rows == 16 else [x for x in zip(n, k) if x not in few] if both else list(zip(n, k))
    return sum(-(-a * group // rows) * b for a, b in mine) / ((256 if both else 512) // Hkv), max(b for _, b in mine)


@pytest.mark.parametrize("case", range(len(ROUNDS)))
@pytest.mark.parametrize("dtype", (BF, F8))
def test_attention_in_several_rounds(rf, case, dtype):  # noqa: F811
    n, k, Hq, Hkv, d, page, kinds = ROUNDS[case]
    say(f"paged attention in several rounds {n[:4]} {k[:4]} Hq={Hq} Hkv={Hkv} d={d} page={page} {dtype}")
    for rows in kinds:
        even, longest = shares(n, k, Hq // Hkv, Hkv, rows, len(kinds) > 1)
        assert even > 2048 + 64 and longest > even * (1.9 if rows == 128 else 1.15) + 64      # long shares, and a cut
    check(rf, (n, k, Hq, Hkv, d, page), dtype, True)


@pytest.mark.parametrize("n,k,Hq,Hkv,d", (([1], [9001], 8, 2, 64), ([5, 1], [9001, 300], 8, 2, 128), ([40, 1], [9001, 4200], 8, 2, 64),
                                          ([2], [4096 + 16], 4, 4, 128), ([1], [4097], 2, 1, 128)))
@pytest.mark.parametrize("dtype", (BF, F8))
def test_attention_of_long_sequences_in_one_piece(rf, n, k, Hq, Hkv, d, dtype):  # noqa: F811
    """Through the entry point without a workspace: nothing is cut, and a wavefront looks up page addresses three times."""
    say(f"paged attention, uncut {n} {k} Hq={Hq} Hkv={Hkv} d={d} {dtype}")
    bt = sb.Batch(720, n, k, Hq, Hkv, d, 16, dtype=dtype, scales=(1.0, 1.0) if dtype == BF else (0.02, 0.3))
    lib, q, o = rf.load_library(), bt.q.to(DEV), nan_like(bt.q)
    tensors = (q, *(sb.cache_on(c, DEV) for c in bt.caches), *bt.on(DEV))
    desc, od = [rf.tensor_desc(t) for t in tensors], rf.tensor_desc(o)
    code = lib.rf_paged_attention(*[ctypes.byref(x) for x in desc], max(n), 1 / math.sqrt(d), 1, *bt.scales, ctypes.byref(od),
                                  ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert code == rf.RF_OK
    torch.cuda.synchronize()
    sb.check_attention(o, *expect(bt), max(k), "uncut")
