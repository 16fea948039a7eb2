"""Verification of drafts in its several forms, which have to agree: without draft probabilities and with q = 1 at the
drafted tokens, with a workspace and without one."""
import ctypes
import math
import sys

import numpy as np
import pytest
import torch

from oracle import serving_oracle as S

sys.path.insert(0, __file__.rsplit("/", 1)[0])
from test_gpu_serving import BF, DEV, rf, say  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def verify(rf, args, with_ws):  # noqa: F811
    """(out, accepted) through the C ABI."""
    lib = rf.load_library()
    dev = [None if t is None else t.to(DEV) for t in args]
    R, B = len(args[2]), len(args[4])
    out, acc = (torch.full((x,), -7, dtype=torch.int32, device=DEV) for x in (R, B))
    desc = [None if t is None else rf.tensor_desc(t) for t in (*dev, out, acc)]
    refs = [None if x is None else ctypes.byref(x) for x in desc]
    if with_ws:
        need = lib.rf_verify_drafts_workspace_bytes(B, args[0].shape[1])
        ws = torch.full((need // 4 + 4,), math.nan, device=DEV)
        code = lib.rf_verify_drafts_ws(*refs, ctypes.c_void_p(ws.data_ptr()), need, None)
    else:
        code = lib.rf_verify_drafts(*refs, None)
    assert code == rf.RF_OK
    torch.cuda.synchronize()
    return out.cpu().tolist(), acc.cpu().tolist()


@pytest.mark.parametrize("V", (9, 4500, 9001))
@pytest.mark.parametrize("dtype", (torch.float32, BF))
def test_no_draft_is_probability_one_at_the_drafted_token(rf, V, dtype):  # noqa: F811
    """w = max(0, p - q) with q = 1 at the drafted token: a NaN there is a weight that is no number (no next token), and
    what a target that is not normalised has above 1 stays."""
    say(f"verify without draft probabilities, V={V} {dtype}")
    r = np.random.default_rng(700 + V)
    B, at = 8, 4
    p = torch.softmax(torch.from_numpy(r.standard_normal((2 * B, V))), -1).to(dtype)
    ua = torch.full((2 * B,), 0.999)
    x = torch.full((2 * B,), at, dtype=torch.int32)
    p[::2, at] = 0.01
    p[0, at] = math.nan                       # at the refused token
    p[2, at], ua[2] = 5.0, math.nan           # refused by its random number, 4 above q
    p[4, at], ua[4] = math.inf, math.nan
    p[6, at + 1] = math.nan                   # elsewhere
    x[8], x[10] = V, -1                       # outside
    p[12] = 0.0                               # the drafted token is all that the target has
    p[12, at] = 0.25
    us = torch.from_numpy(r.random(B, np.float32))
    starts = torch.arange(0, 2 * B + 1, 2, dtype=torch.int32)
    q = torch.zeros((2 * B, V), dtype=dtype)
    for i, t in enumerate(x.tolist()):
        if 0 <= t < V:
            q[i, t] = 1.0
    want, accepted, margin = S.verify(p.float().numpy(), q.float().numpy(), x.numpy(), ua.numpy(), us.numpy(), starts.numpy())
    # (64-bit sums in another order move a border by V 2^-53 of the whole at most)
    assert margin.min() > V * 2.0 ** -52, "inputs on a border"
    assert accepted.tolist() == [0] * B and want[0] == want[4] == want[6] == -1 and want[12] == at and (want[[2, 8, 10, 14]] >= 0).all()
    for draft in (None, q):
        for with_ws in (False, True):
            out, acc = verify(rf, (p, draft, x, ua, us, starts), with_ws)
            assert acc == accepted.tolist() and out == want.tolist(), f"draft {draft is not None}, workspace {with_ws}"


@pytest.mark.parametrize("V", (16384, 65536))
@pytest.mark.parametrize("dtype", (torch.float32, BF))
def test_draws_at_a_border_are_the_same_with_and_without_a_workspace(rf, V, dtype):  # noqa: F811
    """Rows whose second half holds the first one's weights in another order, and a draw of one half: which side of the
    border it falls on is up to the rounding of the sums, and has to be the same in both forms."""
    say(f"verify at borders, V={V} {dtype}")
    r = np.random.default_rng(710)
    B = 64
    half = np.exp2(r.uniform(-45, 0, (B, V // 2)))
    p = torch.from_numpy(np.concatenate((half, r.permuted(half, axis=1)), 1)).to(dtype)
    half = p[:, :V // 2].double().numpy()
    assert all(math.fsum(a) == math.fsum(b) for a, b in zip(half, p[:, V // 2:].double().numpy()))
    args = (p, None, torch.zeros(B, dtype=torch.int32), torch.zeros(B), torch.full((B,), 0.5), torch.arange(B + 1, dtype=torch.int32))
    out, acc = verify(rf, args, False)
    got = verify(rf, args, True)
    assert acc == got[1] == [0] * B
    # (either neighbour of the border; weights below the rounding of the sums may lie between)
    for b, t in enumerate(out):
        between = p[b, t + 1:V // 2] if t < V // 2 else p[b, V // 2:t]
        assert math.fsum(between.double().tolist()) <= V * 2.0 ** -52 * half[b].sum()
    assert out == got[0]
