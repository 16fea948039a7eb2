"""What the serving entry points refuse before any launch, and with which code: no GPU needed."""
import ctypes
import sys

import pytest
import torch

from paper_2603_10026_amd import binding as B

sys.path.insert(0, __file__.rsplit("/", 1)[0])
from test_abi import _desc, _r, lib  # noqa: E402,F401

I32, F32, F8, BF = B.RF_I32, B.RF_F32, B.RF_FP8_E4M3, B.RF_BF16
BAD, UNS, ALI, WS = B.RF_ERR_INVALID_ARG, B.RF_ERR_UNSUPPORTED, B.RF_ERR_ALIGNMENT, B.RF_ERR_WORKSPACE


def paged(T=7, Bt=3, Hq=8, Hkv=2, d=128, n_pages=10, page=16, width=4, dtype=BF, **over):
    a = dict(q=_desc([T, Hq, d]), k=_desc([T, Hkv, d]), v=_desc([T, Hkv, d]), qn=_desc([d]), kn=_desc([d]), eps=1e-6,
             cos=_desc([64, d // 2], F32), sin=_desc([64, d // 2], F32), inter=0, starts=_desc([Bt + 1], I32),
             lens=_desc([Bt], I32), pages=_desc([Bt, width], I32), kc=_desc([n_pages, page, Hkv, d], dtype),
             vc=_desc([n_pages, page, Hkv, d], dtype), ks=1.0, vs=1.0, out=_desc([T, Hq, d]), max_q=3, ws=0x10000, bytes=1 << 40)
    a.update(over)
    return {k: _r(x) if isinstance(x, B.RfTensor) else x for k, x in a.items()}


def append(lib, **over):  # noqa: F811
    a = paged(**over)
    return lib.rf_paged_append(a["q"], a["k"], a["v"], a["qn"], a["kn"], a["eps"], a["cos"], a["sin"], a["inter"], a["starts"],
                               a["lens"], a["pages"], a["kc"], a["vc"], a["ks"], a["vs"], a["out"], None)


def attend(lib, with_ws=False, **over):  # noqa: F811
    a = paged(**over)
    args = (a["q"], a["kc"], a["vc"], a["starts"], a["lens"], a["pages"], a["max_q"], 0.1, 1, a["ks"], a["vs"], a["out"])
    if with_ws:
        return lib.rf_paged_attention_ws(*args, ctypes.c_void_p(a["ws"]), a["bytes"], None)
    return lib.rf_paged_attention(*args, None)


PAGED = [
    (dict(q=None), BAD), (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(starts=None), BAD), (dict(lens=None), BAD),
    (dict(pages=None), BAD), (dict(out=None), BAD), (dict(q=_desc([7, 8])), BAD), (dict(q=_desc([7, 8, 128], F32)), UNS),
    (dict(kc=_desc([10, 16, 2, 128], F32), vc=_desc([10, 16, 2, 128], F32)), UNS),           # no fp32 cache
    (dict(vc=_desc([10, 16, 2, 128], F8)), UNS), (dict(vc=_desc([10, 32, 2, 128])), BAD),
    (dict(vc=_desc([10, 16, 2, 128], stride=[8192, 256, 128, 1])), UNS),                     # other strides than the keys'
    (dict(kc=_desc([10, 16, 3, 128]), vc=_desc([10, 16, 3, 128])), BAD),                     # 8 heads over 3
    (dict(q=_desc([7, 0, 128]), out=_desc([7, 0, 128])), BAD), (dict(d=96), UNS), (dict(page=8), UNS), (dict(page=24), UNS),
    (dict(starts=_desc([3], I32)), BAD), (dict(lens=_desc([4], I32)), BAD), (dict(starts=_desc([4], F32)), UNS),
    (dict(lens=_desc([3], I32, stride=[2])), UNS), (dict(pages=_desc([3, 4], F32)), UNS),
    (dict(pages=_desc([3, 4], I32, stride=[8, 2])), UNS), (dict(ks=0.5), BAD), (dict(vs=float("nan")), BAD),
    (dict(dtype=F8, ks=0.0), BAD), (dict(dtype=F8, vs=float("inf")), BAD), (dict(dtype=F8, vs=-1.0), BAD),
    (dict(q=_desc([7, 8, 128], data=0x1008)), ALI), (dict(out=_desc([7, 8, 128], stride=[1028, 128, 1])), ALI),
    (dict(kc=_desc([10, 16, 2, 128], data=0x1008)), ALI), (dict(kc=_desc([10, 16, 2, 128], data=None)), BAD),
    (dict(starts=_desc([4], I32, data=0x1002)), ALI), (dict(pages=_desc([3, 4], I32, data=None)), BAD),
    (dict(q=_desc([7, 8, 128], stride=[1024, 128, 2])), UNS), (dict(out=_desc([6, 8, 128])), BAD),
    (dict(kc=_desc([10, 16, 2, 128], stride=[1 << 32, 1 << 27, 128, 1]), vc=_desc([10, 16, 2, 128], stride=[1 << 32, 1 << 27, 128, 1])), UNS),
    (dict(T=1 << 29), UNS),                                                                  # T * Hq past 2^31
]


@pytest.mark.parametrize("case", range(len(PAGED)))
def test_both_paged_entry_points_refuse(lib, case):  # noqa: F811
    over, code = PAGED[case]
    assert append(lib, **over) == code
    assert attend(lib, **over) == code and attend(lib, with_ws=True, **over) == code


def test_append_refuses(lib):  # noqa: F811
    for over, code in [(dict(k=_desc([7, 8, 128])), BAD), (dict(v=_desc([7, 2, 128], F32)), UNS), (dict(qn=_desc([64])), BAD),
                       (dict(kn=_desc([128], F32)), UNS), (dict(qn=_desc([128], data=0x1004)), ALI), (dict(eps=-1.0), BAD),
                       (dict(eps=float("nan")), BAD), (dict(cos=None), BAD), (dict(sin=None), BAD),
                       (dict(cos=_desc([64, 32], F32)), BAD), (dict(cos=_desc([64, 64]), sin=_desc([64, 64])), UNS),
                       (dict(cos=_desc([64, 12], F32), sin=_desc([64, 12], F32)), UNS),
                       (dict(cos=_desc([64, 72], F32), sin=_desc([64, 72], F32)), BAD),
                       (dict(cos=_desc([0, 64], F32), sin=_desc([0, 64], F32)), BAD),
                       (dict(cos=_desc([64, 64], F32, stride=[128, 2]), sin=_desc([64, 64], F32, stride=[128, 2])), UNS)]:
        assert append(lib, **over) == code, over


def test_attention_refuses(lib):  # noqa: F811
    assert attend(lib, max_q=-1) == BAD
    long = dict(width=200)
    a = paged(**long)
    need = lib.rf_paged_attention_workspace_bytes(a["q"], a["kc"], a["pages"], 3)
    assert 0 < need <= 256 << 20
    for over in (dict(ws=0), dict(ws=0x10008), dict(bytes=need - 1)):
        assert attend(lib, with_ws=True, **long, **over) == WS
    # nothing to cut: no workspace; refused shapes: none either
    a = paged(width=1)
    assert lib.rf_paged_attention_workspace_bytes(a["q"], a["kc"], a["pages"], 3) == 0
    assert lib.rf_paged_attention_workspace_bytes(a["q"], _r(_desc([10, 16, 3, 128])), a["pages"], 3) == 0
    for Hkv in (1, 2, 8, 128, 1024, 4096):
        for mq in (1, 9, 1 << 20):
            a = paged(T=64, Bt=64, Hq=8 * Hkv, Hkv=Hkv, width=10000)
            assert lib.rf_paged_attention_workspace_bytes(a["q"], a["kc"], a["pages"], mq) <= 256 << 20


def test_nothing_to_do_is_ok(lib):  # noqa: F811
    nothing = dict(q=_desc([0, 8, 128], data=None), k=_desc([0, 2, 128], data=None), v=_desc([0, 2, 128], data=None),
                   out=_desc([0, 8, 128], data=None))
    assert append(lib, **nothing) == B.RF_OK and attend(lib, **nothing) == B.RF_OK and attend(lib, with_ws=True, **nothing) == B.RF_OK
    none = dict(lens=_desc([0], I32, data=None), starts=_desc([1], I32), pages=_desc([0, 4], I32, data=None))
    assert append(lib, **none) == B.RF_OK and attend(lib, **none) == B.RF_OK
    assert verify(lib, us=_desc([0], F32, data=None), starts=_desc([1], I32), acc=_desc([0], I32, data=None)) == B.RF_OK


def verify(lib, ws=None, **over):  # noqa: F811
    a = dict(p=_desc([9, 500], F32), q=_desc([9, 500], F32), x=_desc([9], I32), ua=_desc([9], F32), us=_desc([3], F32),
             starts=_desc([4], I32), out=_desc([9], I32), acc=_desc([3], I32))
    a.update(over)
    args = [None if x is None else _r(x) for x in a.values()]
    if ws is None:
        return lib.rf_verify_drafts(*args, None)
    return lib.rf_verify_drafts_ws(*args, ctypes.c_void_p(ws[0]), ws[1], None)


def test_verify_refuses(lib):  # noqa: F811
    for over, code in [(dict(p=None), BAD), (dict(x=None), BAD), (dict(ua=None), BAD), (dict(us=None), BAD), (dict(starts=None), BAD),
                       (dict(out=None), BAD), (dict(acc=None), BAD), (dict(q=_desc([9, 500])), UNS), (dict(q=_desc([9, 499], F32)), BAD),
                       (dict(p=_desc([9, 500], I32)), UNS), (dict(p=_desc([9, 0], F32), q=None), BAD), (dict(x=_desc([8], I32)), BAD),
                       (dict(x=_desc([9], F32)), UNS), (dict(ua=_desc([9], I32)), UNS), (dict(us=_desc([3])), UNS),
                       (dict(starts=_desc([3], I32)), BAD), (dict(out=_desc([9], I32, stride=[2])), UNS),
                       (dict(acc=_desc([3], I32, data=0x1001)), ALI), (dict(p=_desc([9, 500], F32, data=0x1002)), ALI),
                       (dict(q=_desc([9, 500], F32, data=None)), BAD), (dict(p=_desc([9, 500], F32, stride=[1000, 2])), UNS),
                       (dict(p=_desc([9, 1 << 31], F32), q=None), UNS)]:
        assert verify(lib, **over) == code, over
    big = dict(p=_desc([9, 100000], F32), q=None)
    need = lib.rf_verify_drafts_workspace_bytes(3, 100000)
    assert need > 0 and lib.rf_verify_drafts_workspace_bytes(3, 500) == 0 and lib.rf_verify_drafts_workspace_bytes(0, 100000) == 0
    for ws in ((0, need), (0x10008, need), (0x10000, need - 1)):
        assert verify(lib, ws=ws, **big) == WS


def test_cascades_are_described(lib):  # noqa: F811
    MAX, MIN, SUM, ADD, MUL = 0, 1, 2, 0, 1
    for name in ("rf_paged_attention", "rf_paged_attention_ws"):
        assert B.describe_cascade(name) == B.describe_cascade("rf_cascade_attention") == [(MAX, ADD), (SUM, MUL), (SUM, MUL)]
    assert B.describe_cascade("rf_paged_append") == [(SUM, MUL)]
    assert B.describe_cascade("rf_verify_drafts") == [(MIN, ADD), (SUM, MUL), (MIN, ADD)]


def test_the_binding_refuses_tensors_elsewhere():
    """Tensors that are not on the current device: the kernels would follow their pointers."""
    q, kv = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(B.RfError) as e:
        B.rf_paged_attention(q, kv, kv, i, i[:1], i[None], 2, 0.1, stream=0)
    assert e.value.code == BAD
    with pytest.raises(B.RfError):
        B.rf_paged_append(q, q[:, :2], q[:, :2], kv, kv, i, i[:1], i[None], stream=0)
    with pytest.raises(B.RfError):
        B.rf_verify_drafts(torch.zeros(2, 9), None, i, torch.zeros(2), torch.zeros(1), i, stream=0)
    with pytest.raises(TypeError):
        B.rf_paged_attention(q.half(), kv, kv, i, i[:1], i[None], 2, 0.1, stream=0)
    with pytest.raises(ValueError):
        B.rf_paged_attention(q, kv, kv, i, i[:1], i[None], 2, "one", stream=0)


def test_more_workgroups_than_a_launch_has_are_unsupported(lib):  # noqa: F811
    """Refused on the host, like any shape that the kernels do not cover."""
    T, n = 1 << 30, 1 << 23
    tall = dict(T=T, Hq=1, Hkv=1, d=64)
    assert append(lib, **tall, qn=None, kn=None) == UNS
    assert attend(lib, **tall) == UNS and attend(lib, with_ws=True, **tall) == UNS
    a = paged(**tall)
    assert lib.rf_paged_attention_workspace_bytes(a["q"], a["kc"], a["pages"], 3) == 0
    many = dict(us=_desc([n], F32), starts=_desc([n + 1], I32), acc=_desc([n], I32))
    assert verify(lib, **many) == UNS and verify(lib, ws=(0x10000, 1 << 40), **many) == UNS
    assert lib.rf_verify_drafts_workspace_bytes(n, 500) == lib.rf_verify_drafts_workspace_bytes(n, 131072) == 0
    # sums of so many slices do not fit a launch: one launch serves the call
    assert lib.rf_verify_drafts_workspace_bytes(1 << 20, 131072) == 0 < lib.rf_verify_drafts_workspace_bytes(1 << 18, 131072)


def test_workspace_of_paged_attention_is_bounded(lib):  # noqa: F811
    """131 MiB, whatever the batch: heads, tokens, sequences and the longest of them."""
    largest = 0
    for d in (64, 128):
        for group in (1, 3, 8, 16):
            for Hkv in (1, 2, 3, 5, 8, 16, 100, 256, 512):
                for T, Bt in ((1, 1), (8, 8), (64, 64), (300, 2), (4096, 1), (4096, 4), (16384, 100), (100000, 3)):
                    for mq in (1, 9, 600, 1 << 20):
                        a = paged(T=T, Bt=Bt, Hq=group * Hkv, Hkv=Hkv, d=d, n_pages=1 << 20, width=10000)
                        largest = max(largest, lib.rf_paged_attention_workspace_bytes(a["q"], a["kc"], a["pages"], mq))
    assert 128 << 20 < largest <= 131 << 20
