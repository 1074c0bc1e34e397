"""Refusals of the norm-and-rotation and differential-attention calls, before anything is enqueued (CPU only), and
their size queries."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x100000)        # 16-byte aligned, never dereferenced on error paths
MIS = ctypes.c_void_p(0x100008)         # 8-byte aligned only
ODD = ctypes.c_void_p(0x100002)


@pytest.fixture(scope="module")
def sk():
    from paper_2606_20005_amd import streamkl
    return streamkl


def rows(sk, data=0x100000, sb=0, sh=512, sn=64):
    return ctypes.byref(sk._Rows(data, sb, sh, sn))


def norm_call(sk, back=False, **kw):
    a = dict(q=rows(sk), k=rows(sk), B=1, H=4, HK=2, NQ=8, NK=8, d=64, dtype=0, wq=FAKE, wk=FAKE, eps=1e-6, table=FAKE,
             n_pos=8, rot=64, inter=0, qp=None, kp=None, p64=0, qs=0, ks=0, copies=1, yq=FAKE, yk=FAKE)
    b = dict(dyq=FAKE, dyk=FAKE, dyt=0, ws=FAKE, wsb=1 << 30, dxq=FAKE, dxk=FAKE, dwq=FAKE, dwk=FAKE)
    a.update({k: v for k, v in kw.items() if k in a})
    b.update({k: v for k, v in kw.items() if k in b})
    if not back:
        return sk.lib.streamkl_qk_norm_rope_fwd(*a.values(), None)
    a.pop("yq"), a.pop("yk")
    return sk.lib.streamkl_qk_norm_rope_bwd(*a.values(), *b.values(), None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,expect", [
    (dict(B=-1), 1), (dict(NQ=-1), 1), (dict(HK=-2), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(eps=0.0), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(inter=2), 1), (dict(p64=2), 1), (dict(copies=0), 1),
    (dict(d=48), 2), (dict(d=16), 2), (dict(d=288), 2), (dict(rot=24), 2), (dict(rot=80), 1), (dict(rot=-16), 1),
    (dict(table=None), 1), (dict(table=MIS), 1), (dict(n_pos=0), 1), (dict(n_pos=-1), 1), (dict(wq=MIS), 1),
    (dict(qp=ODD), 1), (dict(kp=ctypes.c_void_p(0x100004), p64=1), 1), (dict(NQ=9), 1),
    (dict(NK=1 << 30, B=4), 2), (dict(NK=1 << 29, HK=8), 2),
    (dict(B=0, dwq=None, dwk=None), 0),
    (dict(q=None, k=None, dwq=None, dwk=None), 0), (dict(H=0, HK=0, dwq=None, dwk=None), 0),
])
def test_norm_rope_refusals(sk, back, kw, expect):
    assert norm_call(sk, back, **kw) == expect


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("bad", [dict(data=None), dict(data=0x100008), dict(sb=-8), dict(sh=-8), dict(sn=-8),
                                 dict(sb=4), dict(sh=12), dict(sn=1)])
def test_norm_rope_refuses_rows_it_cannot_read(sk, back, bad):
    assert norm_call(sk, back, q=rows(sk, **bad)) == 1
    assert norm_call(sk, back, k=rows(sk, **bad)) == 1


def test_norm_rope_refuses_outputs(sk):
    for n in ("yq", "yk"):
        assert norm_call(sk, **{n: None}) == 1 and norm_call(sk, **{n: MIS}) == 1
    for n in ("dxq", "dxk", "dyq", "dyk"):
        assert norm_call(sk, True, **{n: None}) == 1 and norm_call(sk, True, **{n: MIS}) == 1
    assert norm_call(sk, True, ws=None) == 1 and norm_call(sk, True, wsb=16) == 1 and norm_call(sk, True, ws=ODD) == 1
    assert norm_call(sk, True, dyt=1) == 1
    assert norm_call(sk, True, q=None, dwq=FAKE) == 1   # a weight gradient of a side that is not there


def test_norm_rope_workspace(sk):
    f = sk.lib.streamkl_qk_norm_rope_bwd_workspace_bytes
    assert f(1, 1, 1, 1, 1, 64) == 2 * 64 * 4
    assert f(0, 4, 4, 10, 10, 64) == 0 and f(-1, 4, 4, 10, 10, 64) == 0 and f(1, 4, 4, 10, 10, 300) == 0
    assert f(16, 32, 8, 16384, 16384, 128) <= 2 * 2048 * 128 * 4   # bounded whatever the extents


def diff_args(sk, **kw):
    a = dict(q1=rows(sk), k1=rows(sk), q2=rows(sk), k2=rows(sk), v=rows(sk), B=1, H=4, HK=2, NQ=8, NK=8, d=64, dv=64,
             scale=0.125, causal=0, lam=FAKE, ql=None, kl=None)
    a.update({k: v for k, v in kw.items() if k in a})
    return a.values()


def diff_call(sk, **kw):
    b = dict(splits=1, ws=None, wsb=0, out=FAKE, out2=None, lse1=None, lse2=None)
    b.update({k: v for k, v in kw.items() if k in b})
    return sk.lib.streamkl_diff_fwd(*diff_args(sk, **kw), *b.values(), None)


def diff_bwd_call(sk, **kw):
    b = dict(dout=FAKE, out=FAKE, out2=FAKE, lse1=FAKE, lse2=FAKE, ws=FAKE, wsb=1 << 40, dq1=FAKE, dk1=FAKE, dq2=FAKE,
             dk2=FAKE, dvv=FAKE, dlam=FAKE, bf16=0)
    b.update({k: v for k, v in kw.items() if k in b})
    return sk.lib.streamkl_diff_bwd(*diff_args(sk, **kw), *b.values(), None)


@pytest.mark.parametrize("call", [diff_call, diff_bwd_call])
@pytest.mark.parametrize("kw,expect", [
    (dict(B=-1), 1), (dict(NQ=-1), 1), (dict(NK=-1), 1), (dict(HK=3), 1), (dict(HK=0), 1), (dict(causal=2), 1),
    (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=1e30), 1),
    (dict(scale=1e-30), 1), (dict(lam=None), 1), (dict(lam=ODD), 1), (dict(ql=ODD), 1), (dict(kl=ODD), 1),
    (dict(d=48), 2), (dict(d=160), 2), (dict(dv=288), 2), (dict(dv=16), 2), (dict(out=None), 1), (dict(out=MIS), 1),
    (dict(out2=MIS), 1), (dict(lse1=ODD), 1), (dict(B=1 << 16, H=1 << 16, HK=1 << 16), 2),
    (dict(NQ=0x7fffffff), 2), (dict(NK=0x7fffffff), 2), (dict(NQ=1 << 30), 2),
])
def test_diff_refusals(sk, call, kw, expect):
    assert call(sk, **kw) == expect


@pytest.mark.parametrize("call", [diff_call, diff_bwd_call])
@pytest.mark.parametrize("name", ["q1", "k1", "q2", "k2", "v"])
@pytest.mark.parametrize("bad,expect", [(dict(data=None), 1), (dict(data=0x100008), 1), (dict(sb=-8), 1), (dict(sh=4), 1),
                                        (dict(sn=65), 1), (dict(sn=1 << 25), 2)])
def test_diff_refuses_rows_it_cannot_read(sk, call, name, bad, expect):
    assert call(sk, **{name: rows(sk, **bad)}) == expect
    assert call(sk, **{name: None}) == 1


def test_diff_refuses_workspaces_and_outputs(sk):
    assert diff_call(sk, splits=0) == 1 and diff_call(sk, splits=257, ws=FAKE, wsb=1 << 40) == 2
    need = sk.diff_workspace_bytes(1, 4, 8, 64, 3)
    assert need == 3 * 4 * 8 * 8 * 66
    assert diff_call(sk, splits=3) == 1 and diff_call(sk, splits=3, ws=FAKE, wsb=need - 1) == 1
    assert diff_call(sk, splits=3, ws=MIS, wsb=need) == 1
    none = dict(dq1=None, dk1=None, dq2=None, dk2=None, dvv=None, dlam=None)
    assert diff_bwd_call(sk, **none) == 1
    assert diff_bwd_call(sk, bf16=2) == 1
    assert diff_bwd_call(sk, ws=None) == 1 and diff_bwd_call(sk, wsb=sk.diff_bwd_workspace_bytes(1, 4, 2, 8, 8, 64, 64, False) - 1) == 1
    for n in ("dout", "lse1", "lse2"):
        assert diff_bwd_call(sk, **{n: None}) == 1
    for n in ("dq1", "dvv", "dlam"):
        assert diff_bwd_call(sk, **{n: ODD}) == 1


@pytest.mark.parametrize("call", [diff_call, diff_bwd_call])
@pytest.mark.parametrize("kw", [
    dict(B=1 << 24, NQ=1), dict(B=1 << 22, NQ=1), dict(B=1 << 13, NQ=1 << 14, NK=0), dict(B=1 << 20, HK=4, NK=513),
])
def test_diff_refuses_grids_past_an_axis(sk, call, kw):
    """2^24 workgroups of 256 threads: more than one axis of a grid holds."""
    assert call(sk, **kw) == 2


def test_diff_refuses_splits_of_very_many_rows(sk):
    assert diff_call(sk, B=1 << 18, NQ=16, splits=2, ws=FAKE, wsb=1 << 50) == 2


def test_diff_empty_extents_launch_nothing(sk):
    none = rows(sk, data=None)
    assert diff_call(sk, B=0, q1=none, k1=none, q2=none, k2=none, v=none, out=None) == 0
    assert diff_call(sk, NQ=0, q1=none, q2=none, out=None) == 0
    assert diff_call(sk, H=0, HK=0, lam=None, q1=none, k1=none, q2=none, k2=none, v=none, out=None) == 0
    assert diff_bwd_call(sk, NQ=0, NK=0, q1=none, q2=none, k1=none, k2=none, v=none, dlam=None, ws=None) == 0


def test_diff_split_count(sk):
    n = sk.diff_split_count
    assert n(2, 16, 16, 4096, 4096, 64, 128) == 1      # fills the chip
    assert n(1, 8, 8, 1, 32768, 128, 128) > 16         # one row a head
    assert n(1, 8, 8, 1, 100, 128, 128) == 1           # four tiles cannot be split into ranges of four
    assert n(1, 1, 1, 1, 1 << 20, 64, 64) <= 256
    assert n(0, 8, 8, 1, 100, 128, 128) == 1 and n(1, 8, 3, 1, 100, 128, 128) == 0 and n(1, 8, 8, 1, 100, 100, 64) == 0
    for B, H, HK, q, k in ((1, 1, 1, 1, 4096), (4, 8, 2, 16, 60000), (1, 2, 1, 500, 500)):
        s = n(B, H, HK, q, k, 64, 64)
        assert 1 <= s <= max(1, (k + 31) // 32 // 4)
