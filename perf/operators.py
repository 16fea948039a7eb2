"""One step of a serving program with a paged cache and drafted tokens, operator by operator.

``append``: the new tokens' queries and keys are normalised per head and rotated by their
positions, and the keys and values are written into the pages of their sequences.
``attention``: the new tokens of every sequence attend to the sequence's whole cache.
``verify``: drafted tokens are accepted or replaced by comparing the target's and the draft's
probabilities with given random numbers.

Where ``own`` is false ``run`` computes them with elementary torch operations; where it is true it
calls the package.  ``exact`` is the definition in 64 bits, one sequence after the other.

Tokens are packed: sequence b owns rows seq_start[b] .. seq_start[b+1]-1, and after the step its
cache holds kv_len[b] tokens, key j of it in page pages[b, j // page] at slot j % page.
"""
import math

import torch

DEV = "cuda:0"
own = False

EPS = 1e-6
K_SCALE, V_SCALE = 0.017, 0.013          # what one step of an 8-bit cache stands for
MAX_POS = 40960                          # rows of the rotation's tables
SIZE = {"bf16": 2, "f32": 4, "fp8": 1}


def listed():
    return [
        # The cache update of a decode step of 48 requests: latency.
        dict(name="append_decode_t48_h32kv8d128", kind="append", B=48, new=1, mixed=False, k=900, spread=0.9, Hq=32, Hkv=8,
             d=128, rot=128, page=16, cache="bf16", norm=True, interleaved=False),
        # A prefill of several prompts, 8 K tokens in all: queries and keys with norms, halves rotated.
        dict(name="append_prefill_t8k_h32kv8d128", kind="append", B=5, new=1700, mixed=False, k=2500, spread=0.2, Hq=32, Hkv=8,
             d=128, rot=128, page=64, cache="bf16", norm=True, interleaved=False),
        # Narrow heads, half of each rotated in neighbouring pairs, no norms, into an 8-bit cache.
        dict(name="append_fp8_t2k_h16kv16d64", kind="append", B=3, new=701, mixed=False, k=1999, spread=0.5, Hq=16, Hkv=16,
             d=64, rot=32, page=48, cache="fp8", norm=False, interleaved=True),
        # One user, one token, a short context: the smallest call.
        dict(name="attention_decode_b1_k1000", kind="attention", B=1, new=1, mixed=False, k=1000, spread=0.0, Hq=32, Hkv=8,
             d=128, page=16, cache="bf16"),
        # A decode step of a full batch with contexts of very different lengths.
        dict(name="attention_decode_b64_k8192_ragged", kind="attention", B=64, new=1, mixed=False, k=8192, spread=0.95, Hq=32,
             Hkv=8, d=128, page=16, cache="bf16"),
        # Long contexts in an 8-bit cache, the largest in bytes.
        dict(name="attention_decode_fp8_b32_k32768", kind="attention", B=32, new=1, mixed=False, k=32768, spread=0.0, Hq=32,
             Hkv=8, d=128, page=64, cache="fp8"),
        # The last token and four drafted ones of 16 requests.
        dict(name="attention_drafts_b16_n5_k4001", kind="attention", B=16, new=5, mixed=False, k=4001, spread=0.6, Hq=32,
             Hkv=8, d=128, page=32, cache="bf16"),
        # A chunk of a long prompt: 2048 new tokens behind 6 K cached ones, the largest in operations.
        dict(name="attention_chunk_n2048_k8192", kind="attention", B=1, new=2048, mixed=False, k=8192, spread=0.0, Hq=32,
             Hkv=8, d=128, page=64, cache="bf16"),
        # Chunks of 512 tokens of two prompts beside 30 requests that decode; narrow heads, pages that no tile is a multiple of.
        dict(name="attention_mixed_b32_n512_k4096", kind="attention", B=32, new=512, mixed=True, k=4096, spread=0.7, Hq=16,
             Hkv=4, d=64, page=48, cache="bf16"),
        # Three drafted tokens of four requests, a small vocabulary.
        dict(name="verify_b4_n3_v32000", kind="verify", B=4, drafts=3, V=32000, dtype="f32", draft=True),
        # Five drafted tokens of 64 requests, a large vocabulary.
        dict(name="verify_b64_n5_v131072", kind="verify", B=64, drafts=5, V=131072, dtype="f32", draft=True),
        # Drafts without probabilities of their own (a copy of earlier text), bf16, a vocabulary of odd length.
        dict(name="verify_bf16_b128_n4_v50001", kind="verify", B=128, drafts=4, V=50001, dtype="bf16", draft=False),
    ]


def _log(rng, lo, hi):
    """Whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_one(rng):
    kind = rng.choice(["append", "attention", "attention", "verify"])
    if kind == "verify":
        return dict(kind=kind, B=_log(rng, 1, 128), drafts=rng.randint(1, 8), V=_log(rng, 1000, 131072),
                    dtype=rng.choice(["f32", "f32", "bf16"]), draft=rng.random() < 0.7)
    hkv, d = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128, 128])
    case = dict(kind=kind, B=_log(rng, 1, 64), new=1, mixed=False, k=0, spread=round(rng.uniform(0, 0.95), 2),
                Hq=hkv * rng.choice([1, 2, 4, 4, 8]), Hkv=hkv, d=d, page=rng.choice([16, 16, 32, 48, 64, 128]),
                cache=rng.choice(["bf16", "bf16", "fp8"]))
    pick = rng.random()
    if pick > 0.65:
        case.update(new=_log(rng, 9, 2048), mixed=rng.random() < 0.4)
    elif pick > 0.4:
        case.update(new=rng.randint(2, 8))
    case["k"] = _log(rng, max(case["new"], 16), 2500 if kind == "append" else 32768)
    if kind == "append":
        case.update(rot=rng.choice([d, d, d // 2]), norm=rng.random() < 0.6, interleaved=rng.random() < 0.3)
    return case


def draw(rng):
    """One more case of the listed ranges; the bounds keep it below the largest listed one."""
    while True:
        case = _draw_one(rng)
        if case["kind"] == "attention":
            n, k = _lengths(case)
            # (what the plain form, which pads every sequence to the longest, asks for)
            if case["B"] * case["Hq"] * max(n) * max(k) > 5e8 or case["B"] * case["Hkv"] * max(k) * case["d"] > 1.07e9:
                continue
        if case["kind"] == "append" and sum(_lengths(case)[0]) > 8192:
            continue
        w = work(case)
        if w["bytes"] <= 2.1e9 and w["flops"] <= 2.2e11:
            return case


def _lengths(case):
    """New and cached tokens (these with the new ones) of every sequence: spread evenly between the shortest and the
    longest in an order that is not sorted.  `mixed`: one sequence in 16 brings `new` tokens, the others one."""
    n, k = [], []
    for b in range(case["B"]):
        x = (b * 0.6180339887498949) % 1.0
        mine = case["new"] if not case["mixed"] or b % 16 == 0 else 1
        n.append(mine)
        k.append(max(mine, int(round(case["k"] * (1 - case["spread"] * x)))))
    return n, k


def work(case):
    if case["kind"] == "verify":
        # the rows at which the drafts end; the gathered probabilities of the drafts before count for nothing
        rows = case["B"] * case["V"]
        return {"bytes": SIZE[case["dtype"]] * rows * (2 if case["draft"] else 1) + 16 * case["B"] * (case["drafts"] + 1),
                "flops": 4 * rows}
    n, k = _lengths(case)
    t, hq, hkv, d = sum(n), case["Hq"], case["Hkv"], case["d"]
    if case["kind"] == "append":
        read = 2 * t * (hq + 2 * hkv) * d + 4 * t * case["rot"]
        return {"bytes": read + 2 * t * hq * d + 2 * SIZE[case["cache"]] * t * hkv * d, "flops": 10 * t * (hq + hkv) * d}
    pairs = sum(ni * ki - ni * (ni - 1) // 2 for ni, ki in zip(n, k))
    return {"bytes": 2 * SIZE[case["cache"]] * sum(k) * hkv * d + 4 * t * hq * d, "flops": 4 * pairs * hq * d}


def _stored(x, cache, scale):
    """Values as the cache holds them, scaled and rounded to its type."""
    if cache == "bf16":
        return x.to(torch.bfloat16)
    return (x / scale).clamp(-448, 448).to(torch.float8_e4m3fn)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    st = dict(kind=case["kind"])
    if case["kind"] == "verify":
        B, n, V, dtype = case["B"], case["drafts"], case["V"], torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        R = B * (n + 1)
        logits = 4.0 * normal(R, V)
        draft = torch.softmax(logits + 0.7 * normal(R, V), -1)
        target = torch.softmax(logits, -1).to(dtype)
        if case["draft"]:  # the draft model sampled its tokens (the largest of p / exponential) ...
            tokens = (draft / torch.rand((R, V), generator=g, device=DEV).clamp_min(1e-12).log().neg()).argmax(-1)
        else:              # ... or they are copied from somewhere: likely ones, mostly
            tokens = (logits + normal(R, V)).argmax(-1)
        st.update(target=target, draft=draft.to(dtype) if case["draft"] else None, tokens=tokens.to(torch.int32),
                  u_accept=torch.rand(R, generator=g, device=DEV), u_sample=torch.rand(B, generator=g, device=DEV),
                  seq_start=torch.arange(0, R + 1, n + 1, dtype=torch.int32, device=DEV), n=n,
                  out=torch.empty(R, dtype=torch.int32, device=DEV), accepted=torch.empty(B, dtype=torch.int32, device=DEV))
        return st

    n, k = _lengths(case)
    B, T, P, Hq, Hkv, d = case["B"], sum(n), case["page"], case["Hq"], case["Hkv"], case["d"]
    starts = [sum(n[:b]) for b in range(B + 1)]
    per = [-(-x // P) for x in k]
    total = sum(per) + 3                                     # a few pages that nobody owns
    order = torch.randperm(total, generator=g, device=DEV).tolist()
    table = torch.full((B, max(per)), -1, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :per[b]] = torch.tensor(order[at:at + per[b]], dtype=torch.int32)
        at += per[b]
    scales = (1.0, 1.0) if case["cache"] == "bf16" else (K_SCALE, V_SCALE)
    st.update(seq_start=torch.tensor(starts, dtype=torch.int32, device=DEV), kv_len=torch.tensor(k, dtype=torch.int32, device=DEV),
              pages=table.to(DEV), max_q=max(n), max_k=max(k), scales=scales, cache=case["cache"])
    st["k_cache"], st["v_cache"] = (_stored(normal(total, P, Hkv, d), case["cache"], s) for s in scales)
    if case["kind"] == "attention":
        st.update(q=normal(T, Hq, d).to(torch.bfloat16), scale=1.0 / math.sqrt(d))
        st["o"] = torch.empty_like(st["q"])
        return st
    qkv = normal(T, (Hq + 2 * Hkv) * d).to(torch.bfloat16)   # one projection's output
    q, kk, v = qkv.split([Hq * d, Hkv * d, Hkv * d], -1)
    st.update(q=q.unflatten(-1, (Hq, d)), k=kk.unflatten(-1, (Hkv, d)), v=v.unflatten(-1, (Hkv, d)), rot=case["rot"],
              interleaved=case["interleaved"], q_norm=None, k_norm=None)
    if case["norm"]:
        st["q_norm"], st["k_norm"] = ((1 + 0.2 * normal(d)).to(torch.bfloat16) for _ in range(2))
    angle = torch.arange(MAX_POS, dtype=torch.float64, device=DEV)[:, None] * \
        10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
    st.update(cos=angle.cos().float(), sin=angle.sin().float(), q_out=torch.empty((T, Hq, d), dtype=torch.bfloat16, device=DEV))
    return st


# ---- the plain forms ------------------------------------------------------------------------------

def _sequence_of(st, T):
    """The sequence of each packed token and its place in it."""
    t = torch.arange(T, device=DEV)
    b = (t[:, None] >= st["seq_start"][None, 1:]).sum(1)
    return b, t - st["seq_start"][b]


def _rotated(x, st, pos):
    rot, c, s = st["rot"], st["cos"][pos][:, None], st["sin"][pos][:, None]
    if st["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _normed(x, g):
    return x if g is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * g.float()


def _plain_append(st):
    T, P = st["q"].shape[0], st["k_cache"].shape[1]
    b, i = _sequence_of(st, T)
    pos = st["kv_len"][b] - (st["seq_start"][b + 1] - st["seq_start"][b]) + i
    page, slot = st["pages"][b, pos // P].long(), (pos % P).long()
    q = _rotated(_normed(st["q"].float(), st["q_norm"]), st, pos)
    k = _rotated(_normed(st["k"].float(), st["k_norm"]), st, pos)
    st["q_out"].copy_(q)
    st["k_cache"][page, slot] = _stored(k, st["cache"], st["scales"][0])
    st["v_cache"][page, slot] = st["v"] if st["cache"] == "bf16" else _stored(st["v"].float(), st["cache"], st["scales"][1])
    return {"q": st["q_out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _plain_attention(st):
    q, P, L, N = st["q"], st["k_cache"].shape[1], st["max_k"], st["max_q"]
    T, Hq, d = q.shape
    B, Hkv = st["pages"].shape[0], st["k_cache"].shape[2]
    j = torch.arange(L, device=DEV)
    page, slot = st["pages"][:, j // P].long().clamp_min(0), j % P
    k, v = ((st[c][page, slot].float() * s).transpose(1, 2) for c, s in zip(("k_cache", "v_cache"), st["scales"]))
    i = torch.arange(N, device=DEV)
    n = st["seq_start"][1:] - st["seq_start"][:-1]
    rows = q[(st["seq_start"][:-1, None] + i).clamp_max(T - 1)].float()              # [B, N, Hq, d]
    rows = rows.view(B, N, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
    s = torch.matmul(rows, k.transpose(2, 3)) * st["scale"]
    last = (st["kv_len"] - n)[:, None] + i                                           # the last key of query i
    seen = j <= last[:, :, None]
    seen = seen.repeat_interleave(Hq // Hkv, 1)[:, None]
    m = s.masked_fill(~seen, -math.inf).amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(s - m), 0.0)
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    o = torch.where(seen.any(-1, keepdim=True), o, 0.0)
    o = o.view(B, Hkv, N, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, d)
    b, i = _sequence_of(st, T)
    return o[b, i].to(q.dtype)


def _plain_verify(st):
    p, q, x, n, B = st["target"], st["draft"], st["tokens"].long(), st["n"], st["accepted"].shape[0]
    px = p.gather(1, x[:, None])[:, 0].double()
    qx = 1.0 if q is None else q.gather(1, x[:, None])[:, 0].double()
    ok = (st["u_accept"].double() * qx < px).view(B, n + 1)[:, :n]
    a = ok.long().cumprod(1).sum(1)                          # drafts accepted before the first refused one
    row = st["seq_start"][:-1].long() + a
    last = p[row].double()
    if q is None:
        minus = torch.zeros_like(last).scatter_(1, x[row][:, None], last.gather(1, x[row][:, None]))
    else:
        minus = q[row].double()
    rest = (last - torch.where((a < n)[:, None], minus, 0.0)).clamp_min(0)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, last)
    cum = rest.cumsum(1)
    new = (cum <= st["u_sample"].double()[:, None] * cum[:, -1:]).sum(1)
    i = torch.arange(n + 1, device=DEV)
    out = torch.where(i < a[:, None], x.view(B, n + 1), torch.where(i == a[:, None], new[:, None], -1))
    return {"out": out.reshape(-1).to(torch.int32), "accepted": a.to(torch.int32)}


def run(st):
    if not own:
        return {"append": _plain_append, "attention": _plain_attention, "verify": _plain_verify}[st["kind"]](st)
    from paper_2603_10026_amd import binding as rf
    if st["kind"] == "append":
        rf.rf_paged_append(st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["seq_start"], st["kv_len"], st["pages"],
                           q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS, cos=st["cos"], sin=st["sin"],
                           interleaved=st["interleaved"], k_scale=st["scales"][0], v_scale=st["scales"][1], q_out=st["q_out"])
        return {"q": st["q_out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    if st["kind"] == "attention":
        return rf.rf_paged_attention(st["q"], st["k_cache"], st["v_cache"], st["seq_start"], st["kv_len"], st["pages"],
                                     st["max_q"], st["scale"], k_scale=st["scales"][0], v_scale=st["scales"][1], o=st["o"])
    rf.rf_verify_drafts(st["target"], st["draft"], st["tokens"], st["u_accept"], st["u_sample"], st["seq_start"],
                        out=st["out"], accepted=st["accepted"])
    return {"out": st["out"], "accepted": st["accepted"]}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_append(case, st):
    n, k = _lengths(case)
    P, rot = case["page"], case["rot"]
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    out = torch.empty(st["q_out"].shape, dtype=torch.float64, device=DEV)
    freq = torch.tensor([10000.0 ** (-2.0 * f / rot) for f in range(rot // 2)], dtype=torch.float64, device=DEV)
    t = 0
    for b, (nb, kb) in enumerate(zip(n, k)):
        pos = torch.arange(kb - nb, kb, device=DEV)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * freq)[:, None]

        def rotate(x, g):
            x = x.double()
            if g is not None:
                x = x / (x.square().sum(-1, keepdim=True) / case["d"] + EPS).sqrt() * g.double()
            if case["interleaved"]:
                z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * turn
                x = torch.cat((torch.view_as_real(z).flatten(-2), x[..., rot:]), -1)
            else:
                z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
                x = torch.cat((z.real, z.imag, x[..., rot:]), -1)
            return x

        at = st["pages"][b].long()[pos // P] * P + pos % P
        out[t:t + nb] = rotate(st["q"][t:t + nb], st["q_norm"])
        kc.view(-1, *kc.shape[2:])[at] = rotate(st["k"][t:t + nb], st["k_norm"]) / st["scales"][0]
        vc.view(-1, *vc.shape[2:])[at] = st["v"][t:t + nb].double() / st["scales"][1]
        t += nb
    return {"q": out, "k_cache": kc, "v_cache": vc}


def _exact_attention(case, st):
    n, k = _lengths(case)
    P, grp, d = case["page"], case["Hq"] // case["Hkv"], case["d"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    t = 0
    for b, (nb, kb) in enumerate(zip(n, k)):
        ids = st["pages"][b, :-(-kb // P)].long()
        for h in range(case["Hkv"]):
            K = st["k_cache"][ids, :, h].reshape(-1, d)[:kb].double() * st["scales"][0]
            V = st["v_cache"][ids, :, h].reshape(-1, d)[:kb].double() * st["scales"][1]
            Q = st["q"][t:t + nb, h * grp:(h + 1) * grp].double().reshape(nb * grp, d)
            s = (Q @ K.t()).view(nb, grp, kb) / math.sqrt(d)
            if nb > 1:
                s.masked_fill_(torch.ones((nb, kb), dtype=torch.bool, device=DEV).triu(kb - nb + 1)[:, None], -math.inf)
            out[t:t + nb, h * grp:(h + 1) * grp] = (torch.softmax(s, -1).view(nb * grp, kb) @ V).view(nb, grp, d)
        t += nb
    return out


def _exact_verify(case, st):
    n = case["drafts"]
    x, u = st["tokens"].tolist(), st["u_accept"].double().tolist()
    out, accepted = [-1] * len(x), []
    for b, r in enumerate(st["u_sample"].double().tolist()):
        row0, a, rest = b * (n + 1), 0, None
        while rest is None:
            p = st["target"][row0 + a].double()
            if a == n:
                rest = p
                break
            t = x[row0 + a]
            if st["draft"] is None:
                q = torch.zeros_like(p)
                q[t] = 1.0
            else:
                q = st["draft"][row0 + a].double()
            if u[row0 + a] * float(q[t]) < float(p[t]):
                out[row0 + a] = t
                a += 1
            else:
                rest = torch.relu(p - q)
                if not float(rest.sum()) > 0:
                    rest = p
        cum = torch.cumsum(rest, 0)
        out[row0 + a] = int(torch.searchsorted(cum, (r * cum[-1]).reshape(1), right=True))
        accepted.append(a)
    return {"out": torch.tensor(out, dtype=torch.int32), "accepted": torch.tensor(accepted, dtype=torch.int32)}


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "verify": _exact_verify}[case["kind"]](case, st)
