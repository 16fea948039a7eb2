"""Paged attention of long chunks of new tokens, alone and beside decoding requests, at full size, against the
definition in 64 bits on the GPU."""
import math
import sys

import pytest
import torch

sys.path.insert(0, __file__.rsplit("/", 1)[0])
import serving_batches as sb  # noqa: E402
from test_gpu_serving import BF, DEV, F8, rf, say  # noqa: E402,F401

pytestmark = pytest.mark.gpu

# n, k, Hq, Hkv, d, page
LARGE = [
    ([2048], [2100], 32, 8, 128, 64), ([2049], [2049], 32, 4, 128, 16), ([1024, 1024], [1030, 9000], 32, 8, 128, 16),
    ([4100], [5000], 16, 1, 128, 48), ([600] * 4, [601, 3000, 600, 2222], 64, 8, 128, 32), ([2048], [1900], 32, 8, 128, 16),
    ([1500, 1, 1, 1500], [3000, 5000, 7, 1500], 32, 8, 128, 64), ([2500, 3, 2500], [2600, 900, 9000], 16, 8, 64, 16),
]


def check(rf, case, dtype, causal):  # noqa: F811
    n, k, Hq, Hkv, d, page = case
    scales = (1.0, 1.0) if dtype == BF else (0.02, 0.3)
    g = torch.Generator(device=DEV).manual_seed(sum(k) + d)
    per = [-(-x // page) for x in k]
    ids = torch.randperm(sum(per), generator=g, device=DEV)
    table = torch.full((len(k), max(per)), -1, dtype=torch.int32, device=DEV)
    caches = []
    for s in scales:
        x = torch.randn((sum(per), page, Hkv, d), generator=g, device=DEV) / s
        at = 0
        for b, c in enumerate(per):
            table[b, :c] = ids[at:at + c].to(torch.int32)
            at += c
            if k[b] % page:
                x[table[b, c - 1], k[b] % page:] = math.nan            # slots behind the last token
        caches.append(x.clamp(-448, 448).to(dtype) if dtype == F8 else x.to(dtype))
    q = torch.randn((sum(n), Hq, d), generator=g, device=DEV).to(BF)
    if dtype == BF:
        # the last token's value is no number in one column: only rows that see it may show it
        for b, ln in enumerate(k):
            caches[1][table[b, (ln - 1) // page], (ln - 1) % page, 0, 9] = math.inf
    starts = torch.tensor([sum(n[:b]) for b in range(len(n) + 1)], dtype=torch.int32, device=DEV)
    o = rf.rf_paged_attention(q, *caches, starts, torch.tensor(k, dtype=torch.int32, device=DEV), table, max(n), 1 / math.sqrt(d),
                              causal, *scales, o=torch.full_like(q, math.nan))
    t0 = 0
    for b, (nb, ln) in enumerate(zip(n, k)):
        for h in range(Hkv):
            K, V = (c[table[b, :per[b]].long(), :, h].reshape(-1, d)[:ln].double() * s for c, s in zip(caches, scales))
            grp = Hq // Hkv
            Q = q[t0:t0 + nb, h * grp:(h + 1) * grp].double()
            s = (Q.reshape(-1, d) @ K.t() / math.sqrt(d)).view(nb, grp, ln)
            size = (Q.abs().reshape(-1, d) @ K.abs().t()).amax(1).view(nb, grp) / math.sqrt(d)
            if causal:
                s.masked_fill_(torch.ones((nb, ln), dtype=torch.bool, device=DEV).triu(ln - nb + 1)[:, None], -math.inf)
            p = torch.softmax(s, -1).nan_to_num(0.0).view(-1, ln)         # (a row that sees nothing: zeros)
            fine = V.isfinite()
            want = (p @ torch.where(fine, V, 0.0)).view(nb, grp, d)
            spread = (p @ torch.where(fine, V, 0.0).abs()).view(nb, grp, d)
            want = want + torch.where((p @ (~fine).double()).view(nb, grp, d) > 0, math.inf, 0.0)
            sb.check_attention(o[t0:t0 + nb, h * grp:(h + 1) * grp], *(x.cpu().numpy() for x in (want, spread, size)), ln,
                               f"sequence {b} head {h}")
        t0 += nb


@pytest.mark.parametrize("case", range(len(LARGE)))
@pytest.mark.parametrize("dtype", (BF, F8))
def test_attention_of_long_chunks(rf, case, dtype):  # noqa: F811
    say(f"paged attention, long chunks {LARGE[case]} {dtype}")
    check(rf, LARGE[case], dtype, True)


def test_attention_of_long_chunks_without_a_mask(rf):  # noqa: F811
    say("paged attention, long chunks, no mask")
    check(rf, ([2048], [3001], 32, 8, 128, 16), BF, False)
