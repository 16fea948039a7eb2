"""The serving operators together, as a program uses them: steps of drafted decoding over one cache, captured graphs that
serve other batches than the captured one, two streams at once, calls without a workspace."""
import ctypes
import math
import sys

import numpy as np
import pytest
import torch

from oracle import serving_oracle as S

sys.path.insert(0, __file__.rsplit("/", 1)[0])
import serving_batches as sb  # noqa: E402
from test_gpu_serving import BF, DEV, F8, attend, expect, nan_like, rf, say, tables, verify_inputs  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", (BF, F8))
def test_steps_of_drafted_decoding(rf, dtype):  # noqa: F811
    """A prompt's chunk, then steps of the last token and three drafts: append, attend, softmax, verify; rejected drafts'
    slots are written over by the next step.  The cache that the operators have built is what the oracle attends to, and
    every output is checked on the way."""
    say(f"serving steps, {dtype}")
    r = np.random.default_rng(9)
    B, Hq, Hkv, d, page, V, n_draft = 3, 8, 2, 64, 16, 503, 3
    width = 12
    table = r.permutation(B * width + 1)[:B * width].reshape(B, width).astype(np.int32)
    scales = (1.0, 1.0) if dtype == BF else (0.02, 0.02)
    kc, vc = (torch.full((B * width + 1, page, Hkv, d), float("nan"), device=DEV).to(dtype) for _ in range(2))
    cos, sin = tables(d, page * width)
    g = [sb.bf16(1 + 0.2 * r.standard_normal(d)) for _ in range(2)]
    lens, n = np.zeros(B, int), [40, 17, 90]
    shadow = [c.float().cpu().numpy().astype(np.float64) for c in (kc, vc)]       # what the cache stands for
    for step in range(4):
        T = sum(n)
        starts, lens = np.concatenate(([0], np.cumsum(n))), lens + np.array(n)
        q, k, v = (sb.bf16(r.standard_normal((T, h, d))) for h in (Hq, Hkv, Hkv))
        args = i32(starts), i32(lens), i32(table)
        turned = rf.rf_paged_append(q.to(DEV), k.to(DEV), v.to(DEV), kc, vc, *args, q_norm=g[0].to(DEV), k_norm=g[1].to(DEV),
                                    cos=torch.from_numpy(cos).to(DEV), sin=torch.from_numpy(sin).to(DEV),
                                    k_scale=scales[0], v_scale=scales[1])
        o = rf.rf_paged_attention(turned, kc, vc, *args, max(n), 1 / math.sqrt(d), k_scale=scales[0], v_scale=scales[1])
        torch.cuda.synchronize()
        f = [x.float().numpy() for x in g]
        want_q, slots = S.append(q.float().numpy(), k.float().numpy(), v.float().numpy(), *f, 1e-6, cos, sin, False,
                                 starts, lens, table, page)
        # a norm, a rotation and a rounding: see check_append() of the append tests
        big = np.abs(want_q).max(-1, keepdims=True)
        sb.check_rounded(turned, want_q, BF, np.broadcast_to(big, want_q.shape), "q", terms=1.5 * (d / 2 + 9))
        for which, cache in enumerate((kc, vc)):
            now = cache.float().cpu().numpy().astype(np.float64) * scales[which]
            for (pg, sl), kv in slots.items():
                x = kv[which]
                big = np.broadcast_to(np.abs(x).max(-1, keepdims=True), x.shape)
                sb.check_rounded(cache[pg, sl], x, dtype, big, "slot", scale=scales[which], terms=1.5 * (d / 2 + 9) + 1)
                shadow[which][pg, sl] = now[pg, sl]
            assert np.array_equal(now, shadow[which], equal_nan=True)               # nothing else has changed
        want = S.attention(turned.float().cpu().numpy(), *shadow, starts, lens, table, 1 / math.sqrt(d), True)
        sb.check_attention(o, *want, lens.max(), f"step {step}")
        # the model's head, as any projection would be; the drafts come from a second, similar one
        rows = torch.cat([torch.arange(e - (1 if step == 0 else n_draft + 1), e) for e in starts[1:]]).to(DEV)
        head = torch.from_numpy(r.standard_normal((Hq * d, V)).astype(np.float32) / 4).to(DEV)
        logits = o[rows].flatten(1).float() @ head
        p = rf.rf_safe_softmax(logits)
        qd = rf.rf_safe_softmax(logits + 0.3 * torch.from_numpy(r.standard_normal(tuple(logits.shape)).astype(np.float32)).to(DEV))
        per = len(rows) // B
        x = torch.multinomial(qd.cpu(), 1, generator=torch.Generator().manual_seed(step))[:, 0].to(torch.int32)
        ua, us = torch.from_numpy(r.random(len(rows), np.float32)), torch.from_numpy(r.random(B, np.float32))
        vs = i32(np.arange(B + 1) * per)
        out, acc = rf.rf_verify_drafts(p, qd, x.to(DEV), ua.to(DEV), us.to(DEV), vs)
        w_out, w_acc, margin = S.verify(p.cpu().numpy(), qd.cpu().numpy(), x.numpy(), ua.numpy(), us.numpy(), vs.cpu().numpy())
        assert margin.min() > V * 2.0 ** -52
        assert out.cpu().tolist() == w_out.tolist() and acc.cpu().tolist() == w_acc.tolist()
        # drafts that were refused leave the sequence: the next step's tokens take their slots
        lens = lens - (per - 1 - w_acc)
        n = [n_draft + 1] * B


def test_a_captured_step_serves_other_batches(rf):  # noqa: F811
    """A graph of append, attention and verification, captured once, replayed over batches of other lengths (a place left
    empty among them) with eager work between the replays: the same bits as eager calls."""
    say("captured serving step")
    B, Hq, Hkv, d, page, width, V = 5, 8, 2, 128, 16, 60, 9000
    r = np.random.default_rng(11)
    n_pages = B * width
    kc, vc = (torch.from_numpy(r.standard_normal((n_pages, page, Hkv, d)).astype(np.float32)).to(DEV).to(BF) for _ in range(2))
    starts, lens = i32(np.arange(B + 1) * 2), i32([900, 10, 2, 333, 512])
    pages = i32(r.permutation(n_pages).reshape(B, width))
    cos, sin = (torch.from_numpy(x).to(DEV) for x in tables(d, page * width))
    q, k, v = (sb.bf16(r.standard_normal((2 * B, h, d))).to(DEV) for h in (Hq, Hkv, Hkv))
    p, qd, x, ua, us, _ = (t.to(DEV) for t in verify_inputs(12, [2] * B, V, torch.float32, True))
    turned, o = torch.empty_like(q), torch.empty_like(q)
    out, acc = torch.empty(2 * B, dtype=torch.int32, device=DEV), torch.empty(B, dtype=torch.int32, device=DEV)

    def step():
        rf.rf_paged_append(q, k, v, kc, vc, starts, lens, pages, cos=cos, sin=sin, q_out=turned)
        rf.rf_paged_attention(turned, kc, vc, starts, lens, pages, 2, 0.09, o=o)
        rf.rf_verify_drafts(p, qd, x, ua, us, starts, out=out, accepted=acc)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        step()
    was = kc.clone(), vc.clone()
    for turn, new in enumerate(([900, 10, 2, 333, 512], [3, 960, 700, 2, 0], [40, 41, 42, 43, 44], [0, 0, 0, 0, 0], [800, 1, 64, 65, 66])):
        say(f"replay {turn}: {new}")
        new = np.array(new)
        lens.copy_(i32(new))
        pages.copy_(i32(np.random.default_rng(turn).permutation(n_pages).reshape(B, width)))
        us.copy_(torch.from_numpy(np.random.default_rng(turn).random(B, np.float32)))
        results = []
        for how in (step, graph.replay):
            kc.copy_(was[0])
            vc.copy_(was[1])
            for t in (turned, o):
                t.fill_(float("nan"))
            out.fill_(-7)
            how()
            torch.cuda.synchronize()
            junk = torch.full((1 << 20,), float("nan"), device=DEV)                # eager work in between
            results.append([t.clone().view(torch.int32 if t.dtype == torch.int32 else torch.int16) for t in (turned, o, kc, vc, out, acc)])
            del junk
        assert all(torch.equal(a, b) for a, b in zip(*results))


def test_two_streams_at_once(rf):  # noqa: F811
    say("two streams")
    batches = [sb.Batch(600 + i, n, k, 8, 2, 128, 16) for i, (n, k) in enumerate((([1] * 4, [3000, 10, 900, 400]), ([200, 1], [900, 800])))]
    want = [attend(rf, b) for b in batches]
    sets = [(b.q.to(DEV), *(sb.cache_on(c, DEV) for c in b.caches), *b.on(DEV), max(b.n)) for b in batches]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(rf.rf_paged_attention(*sets[i], 1 / math.sqrt(128)))
    torch.cuda.synchronize()
    for i in range(2):
        for o in got[i]:
            assert torch.equal(o.view(torch.int16), want[i].view(torch.int16))


@pytest.mark.parametrize("n,k", (([1, 2, 1], [3000, 40, 500]), ([150, 1], [700, 900]), ([7], [2000])))
def test_attention_without_a_workspace(rf, n, k):  # noqa: F811
    """The entry point that takes none, and the one that does with a workspace of NaN that ends in a guard."""
    say(f"paged attention through the C ABI {n} {k}")
    bt = sb.Batch(620, n, k, 8, 2, 64, 16)
    want = expect(bt)
    lib = rf.load_library()
    q, kc, vc, arrays = bt.q.to(DEV), *(sb.cache_on(c, DEV) for c in bt.caches), bt.on(DEV)
    desc = [rf.tensor_desc(t) for t in (q, kc, vc, *arrays)]
    need = lib.rf_paged_attention_workspace_bytes(ctypes.byref(desc[0]), ctypes.byref(desc[1]), ctypes.byref(desc[5]), max(n))
    assert need > 0
    ws = torch.full((need // 4 + 64,), float("nan"), device=DEV)
    for with_ws in (False, True):
        o = nan_like(q)
        od = rf.tensor_desc(o)
        args = [ctypes.byref(x) for x in desc] + [max(n), 1 / math.sqrt(64), 1, 1.0, 1.0, ctypes.byref(od)]
        s = torch.cuda.current_stream().cuda_stream
        code = lib.rf_paged_attention_ws(*args, ctypes.c_void_p(ws.data_ptr()), need, ctypes.c_void_p(s)) if with_ws else \
            lib.rf_paged_attention(*args, ctypes.c_void_p(s))
        assert code == rf.RF_OK
        torch.cuda.synchronize()
        sb.check_attention(o, *want, max(k), f"workspace {with_ws}")
    assert bool(torch.isnan(ws[need // 4:]).all())


def test_verify_without_a_workspace(rf):  # noqa: F811
    say("verify through the C ABI")
    args = verify_inputs(630, [3, 5, 1], 20011, torch.float32, True)
    dev = [t.to(DEV) for t in args]
    want = rf.rf_verify_drafts(*dev)
    lib = rf.load_library()
    out, acc = torch.empty_like(want[0]), torch.empty_like(want[1])
    desc = [rf.tensor_desc(t) for t in (*dev, out, acc)]
    assert lib.rf_verify_drafts(*[ctypes.byref(x) for x in desc], ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == rf.RF_OK
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(acc, want[1])
    need = lib.rf_verify_drafts_workspace_bytes(3, 20011)
    ws = torch.full((need // 4 + 64,), float("nan"), device=DEV)
    assert lib.rf_verify_drafts_ws(*[ctypes.byref(x) for x in desc], ctypes.c_void_p(ws.data_ptr()), need, None) == rf.RF_OK
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and bool(torch.isnan(ws[need // 4:]).all())


def test_calls_on_another_stream_than_the_current_one(rf):  # noqa: F811
    say("an explicit stream")
    bt = sb.Batch(640, [2, 60], [500, 800], 8, 2, 64, 16)
    want = attend(rf, bt)
    q, kc, vc, arrays = bt.q.to(DEV), *(sb.cache_on(c, DEV) for c in bt.caches), bt.on(DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    o = rf.rf_paged_attention(q, kc, vc, *arrays, 60, 1 / math.sqrt(64), stream=s)
    s.synchronize()
    assert torch.equal(o.view(torch.int16)[:bt.seq_start[-1]], want.view(torch.int16)[:bt.seq_start[-1]])
