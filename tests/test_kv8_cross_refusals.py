"""What the 8-bit cache's and the cross attention's entry points refuse, before any HIP call, and what they accept
without one.  No GPU needed: the pointers are never followed."""
import ctypes as C
import os

import pytest

PTR, ODD = 1 << 20, (1 << 20) + 2
BF16, F32 = 0, 1


@pytest.fixture(scope="module")
def lib():
    import paper_2411_17178_amd as m
    if not os.path.exists(m.lib_path()):
        from paper_2411_17178_amd import build
        build.build()
    return m.load_library()


def _strides(*s):
    return (C.c_int64 * 3)(*s)


def _store(lib, **kw):
    a = dict(segments=(4, 70), n=2, begin=0, end=2, k=PTR, v=PTR, dt=BF16, strides=None, B=2, H=3, D=64, lens=None, k8=PTR,
             ks=PTR, v8=PTR, vs=PTR)
    a.update(kw)
    seg = (C.c_int32 * max(1, len(a["segments"])))(*a["segments"]) if a["segments"] is not None else None
    return lib.kv8_store(seg, a["n"], a["begin"], a["end"], a["k"], a["v"], a["dt"], a["strides"], a["B"], a["H"], a["D"], a["lens"],
                         a["k8"], a["ks"], a["v8"], a["vs"], None)


@pytest.mark.parametrize("kw,rc", [
    (dict(segments=None), -1), (dict(n=0), -1), (dict(n=33, segments=(1,) * 33), -1), (dict(segments=(4, -1)), -1),
    (dict(segments=(2 ** 31 - 1, 5)), -2), (dict(begin=-1), -1), (dict(end=3), -1), (dict(begin=1, end=1), -1), (dict(begin=2, end=1), -1),
    (dict(B=0), -1), (dict(H=0), -1), (dict(B=1 << 14, H=1 << 12), -2), (dict(D=128), -2), (dict(dt=2), -2), (dict(k=None), -1),
    (dict(v8=None), -1), (dict(ks=None), -1), (dict(k=ODD), -1), (dict(k8=ODD), -1), (dict(vs=ODD), -1), (dict(lens=ODD), -1),
    (dict(strides=_strides(1000, 100, 60)), -1), (dict(strides=_strides(1000, 100, 64)), -1), (dict(strides=_strides(-8, 64, 64)), -1),
    (dict(strides=_strides(1000, 96, 68)), -1), (dict(segments=(2 ** 30, 0), B=1 << 12, H=1 << 12), -2),
    (dict(segments=(0, 0)), 0), (dict(segments=(0, 5), end=1, k=None, v=None, k8=None), 0),
], ids=str)
def test_store_refuses(lib, kw, rc):
    assert _store(lib, **kw) == rc
    if rc:
        assert lib.litevar_last_error()


def test_block_tables(lib):
    import paper_2411_17178_amd as lv
    assert lv.litevar_kv8_blocks([1, 64, 65, 0, 129]) == [0, 1, 2, 4, 4, 7]
    for bad in ([], [1] * 33, [-1], [2 ** 31 - 1, 2 ** 31 - 1]):
        with pytest.raises(lv.LitevarError):
            lv.litevar_kv8_blocks(bad)


def _cross(lib, kv8=False, **kw):
    a = dict(q=PTR, k=PTR, v=PTR, ks=PTR, vs=PTR, o=2 * PTR, B=2, H=4, Hkv=2, q_len=5, kv_len=70, D=64, dt=BF16, qs=None, kvs=None, os=None,
             lens=None, sm=0.125, w=None, bytes=0)
    a.update(kw)
    if kv8:
        return lib.cross_attn_kv8_fwd(a["q"], a["k"], a["ks"], a["v"], a["vs"], a["o"], a["B"], a["H"], a["Hkv"], a["q_len"], a["kv_len"],
                                      a["D"], a["qs"], a["os"], a["lens"], a["sm"], a["w"], a["bytes"], None)
    return lib.cross_attn_fwd(a["q"], a["k"], a["v"], a["o"], a["B"], a["H"], a["Hkv"], a["q_len"], a["kv_len"], a["D"], a["dt"], a["qs"],
                              a["kvs"], a["os"], a["lens"], a["sm"], a["w"], a["bytes"], None)


COMMON = [
    (dict(B=0), -1), (dict(H=0), -1), (dict(Hkv=0), -1), (dict(Hkv=3), -1), (dict(q_len=-1), -1), (dict(kv_len=-1), -1),
    (dict(B=1 << 14, H=1 << 12, Hkv=1), -2), (dict(q_len=1 << 30), -2), (dict(kv_len=2 ** 31 - 1), -2),
    (dict(B=4, H=4096, Hkv=4096, q_len=1 << 23), -2), (dict(D=128), -2), (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1),
    (dict(o=None), -1), (dict(o=PTR), -1), (dict(q=ODD), -1), (dict(k=PTR + 8), -1), (dict(lens=ODD), -1), (dict(sm=0.0), -1),
    (dict(sm=-1.0), -1), (dict(sm=float("nan")), -1), (dict(sm=float("inf")), -1), (dict(sm=-0.0), -1), (dict(sm=1.1e4), -1),
    (dict(qs=_strides(1 << 20, 64, 32)), -1), (dict(os=_strides(1 << 20, 64, 100)), -1), (dict(qs=_strides(1 << 20, -64, 256)), -1),
    (dict(B=1, H=1, Hkv=1, q_len=1, kv_len=100000), -1),                               # needs a workspace
    (dict(B=1, H=1, Hkv=1, q_len=1, kv_len=100000, w=PTR, bytes=100), -1), (dict(B=1, H=1, Hkv=1, q_len=1, kv_len=100000, w=PTR + 8, bytes=1 << 40), -1),
    (dict(q_len=0), 0), (dict(q_len=0, kv_len=0, q=None, k=None, v=None, o=None), 0),
]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("kw,rc", COMMON, ids=str)
def test_cross_attention_refuses(lib, kw, rc, kv8):
    assert _cross(lib, kv8, **kw) == rc
    if rc:
        assert lib.litevar_last_error()


@pytest.mark.parametrize("kv8,kw,rc", [(False, dict(dt=2), -2), (False, dict(kvs=_strides(1 << 20, 64, 100)), -1), (True, dict(ks=None), -1),
                                       (True, dict(vs=ODD), -1), (True, dict(vs=None), -1)], ids=str)
def test_cross_attention_refuses_more(lib, kv8, kw, rc):
    assert _cross(lib, kv8, **kw) == rc


def test_cross_workspace(lib):
    import paper_2411_17178_amd as lv
    assert lv.litevar_cross_attn_workspace_bytes(16, 30, 30, 256, 512) == 0
    assert lv.litevar_cross_attn_workspace_bytes(1, 8, 2, 1, 100000) > 0
    assert lv.litevar_cross_attn_workspace_bytes(1, 1, 1, 0, 0) == 0
    for bad in ((0, 1, 1, 1, 1), (1, 3, 2, 1, 1), (1, 1, 1, -1, 1), (1, 1, 1, 1, -1)):
        with pytest.raises(lv.LitevarError):
            lv.litevar_cross_attn_workspace_bytes(*bad)
    assert lib.litevar_cross_attn_workspace_bytes(1, 1, 1, 1, 1, None) == -1


def test_windowed_attention_on_the_cache_refuses(lib):
    import paper_2411_17178_amd as lv
    plan = lv.litevar_mask_plan_stats((1, 2, 5), 1)            # no device blob: nothing can be launched with it

    def call(handle=C.addressof(plan.handle), q=PTR, k8=PTR, ks=PTR, v8=PTR, vs=PTR, o=2 * PTR):
        return lib.attn_kv8_fwd(handle, q, k8, ks, v8, vs, o, 1, 2, 64, None, None, 0.125, None, 0, PTR, 1 << 30, None)
    assert call() == -5                                        # (the handle's magic is not set)
    for name in ("q", "k8", "ks", "v8", "vs", "o"):
        assert call(**{name: None}) == -1
    assert call(handle=None) == -1
    fake = lv.binding._Plan.from_buffer_copy(plan.handle)      # a handle that passes the checks of the plan itself; it is never launched
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "paper_2411_17178_amd", "csrc", "plan.h")).read()
    fake.magic = int(re.search(r"kMagic\s*=\s*(0x[0-9a-fA-F]+)", text).group(1), 16)
    fake.d_blob = PTR

    def windowed(**kw):
        a = dict(q=PTR, k8=PTR, ks=PTR, v8=PTR, vs=PTR, o=2 * PTR, B=1, H=2, D=64, qs=None, os=None, sm=0.125, share=None, flags=0, w=4 * PTR, bytes=1 << 30)
        a.update(kw)
        return lib.attn_kv8_fwd(C.addressof(fake), a["q"], a["k8"], a["ks"], a["v8"], a["vs"], a["o"], a["B"], a["H"], a["D"], a["qs"], a["os"],
                                a["sm"], a["share"], a["flags"], a["w"], a["bytes"], None)
    for kw, rc in ((dict(B=0), -1), (dict(D=32), -2), (dict(sm=0.0), -1), (dict(flags=4), -1), (dict(flags=1), -1), (dict(q=ODD), -1),
                   (dict(k8=ODD), -1), (dict(ks=ODD), -1), (dict(o=PTR), -1), (dict(qs=_strides(9000, 64, 20)), -1),
                   (dict(os=_strides(9000, 60, 64)), -1)):
        assert windowed(**kw) == rc, kw
