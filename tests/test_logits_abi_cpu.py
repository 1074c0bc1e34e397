"""Refusals of the calls on rows of logits, before anything is enqueued (CPU only), and their size queries."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x100000)   # 16-byte aligned, never dereferenced on error paths
ODD = ctypes.c_void_p(0x100001)
TWO = ctypes.c_void_p(0x100002)
FOUR = ctypes.c_void_p(0x100004)


@pytest.fixture(scope="module")
def sk():
    from paper_2606_20005_amd import streamkl
    return streamkl


def logits(sk, data=0x100000, sb=8000, sn=1000, B=2, N=8, V=1000, dtype=0):
    return ctypes.byref(sk._Logits(data, sb, sn, B, N, V, dtype))


def teacher(sk, ids=0x100000, values=0x100000, K=8, ids64=0, dtype=2, rest=1, scale=1.0):
    return ctypes.byref(sk._TeacherList(ids, values, K, ids64, dtype, rest, scale))


LOGITS = [(dict(B=-1), 1), (dict(N=-1), 1), (dict(V=-1), 1), (dict(V=0), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1),
          (dict(sb=-1), 1), (dict(sn=-1), 1), (dict(data=None), 1), (dict(data=0x100001), 1),
          (dict(data=0x100002, dtype=2), 1), (dict(V=(1 << 22) + 1), 2), (dict(B=1 << 16, N=1 << 16), 2),
          (dict(B=0), 0), (dict(N=0), 0), (dict(B=0, data=None, V=0), 0)]


def logprob_call(sk, x=None, **kw):
    a = dict(tokens=FAKE, tokens64=0, scale=1.0, top=0, ws=FAKE, wsb=1 << 40, logp=FAKE, entropy=FAKE, lse=FAKE, err=FAKE,
             top_logp=None, top_ids=None)
    a.update(kw)
    return sk.lib.streamkl_token_logprobs_fwd(x or logits(sk), *a.values(), None)


def logprob_grad(sk, x=None, **kw):
    a = dict(tokens=FAKE, tokens64=0, scale=1.0, lse=FAKE, err=FAKE, entropy=FAKE, dlogp=FAKE, dentropy=FAKE, dlse=FAKE,
             dx=FAKE, sb=8000, sn=1000)
    a.update(kw)
    return sk.lib.streamkl_token_logprobs_bwd(x or logits(sk), *a.values(), None)


def distill_call(sk, x=None, t=None, **kw):
    a = dict(scale=1.0, direction=0, ws=FAKE, wsb=1 << 40, loss=FAKE, stats=FAKE)
    a.update(kw)
    return sk.lib.streamkl_topk_distill_fwd(x or logits(sk), t or teacher(sk), *a.values(), None)


def distill_grad(sk, x=None, t=None, **kw):
    a = dict(scale=1.0, direction=0, stats=FAKE, dloss=FAKE, factor=1.0, dfactor=FAKE, done=0, dx=FAKE, sb=8000, sn=1000)
    a.update(kw)
    return sk.lib.streamkl_topk_distill_bwd(x or logits(sk), t or teacher(sk), *a.values(), None)


def distill_step(sk, x=None, t=None, **kw):
    a = dict(scale=1.0, direction=0, ws=FAKE, wsb=1 << 40, weight=FAKE, factor=1.0, loss=FAKE, stats=FAKE, dx=FAKE, sb=8000,
             sn=1000)
    a.update(kw)
    return sk.lib.streamkl_topk_distill_step(x or logits(sk), t or teacher(sk), *a.values(), None)


CALLS = [logprob_call, logprob_grad, distill_call, distill_grad, distill_step]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("bad,expect", LOGITS)
def test_logits(sk, call, bad, expect):
    assert call(sk, logits(sk, **bad)) == expect


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf"), 2.0 ** -65, 2.0 ** 65])
def test_scales(sk, call, scale):
    assert call(sk, scale=scale) == 1


@pytest.mark.parametrize("kw,expect", [
    (dict(tokens64=2), 1), (dict(top=-1), 1), (dict(top=129), 2), (dict(tokens=None), 1), (dict(logp=None), 1),
    (dict(tokens=TWO), 1), (dict(tokens=FOUR, tokens64=1), 1), (dict(logp=TWO), 1), (dict(entropy=ODD), 1),
    (dict(lse=TWO), 1), (dict(err=TWO), 1), (dict(top=4), 1), (dict(top=4, top_logp=FAKE), 1),
    (dict(top=4, top_ids=FAKE), 1), (dict(top=4, top_ids=TWO, top_logp=FAKE), 1),
    (dict(tokens=None, logp=None, entropy=None, lse=None, err=None), 1)])
def test_logprob_refusals(sk, kw, expect):
    assert logprob_call(sk, **kw) == expect


def test_more_alternatives_than_tokens(sk):
    assert logprob_call(sk, logits(sk, V=5), top=6, top_ids=FAKE, top_logp=FAKE) == 1


@pytest.mark.parametrize("kw", [dict(ws=None), dict(wsb=16), dict(ws=FOUR)])
def test_workspaces(sk, kw):
    few = logits(sk, B=1, N=2, V=100000)   # rows in parts
    assert sk.lib.streamkl_token_logprobs_workspace_bytes(1, 2, 100000, 0, 4) > 16
    assert sk.lib.streamkl_topk_distill_workspace_bytes(1, 2, 100000, 0, 1) > 16
    assert logprob_call(sk, few, top=4, top_ids=FAKE, top_logp=FAKE, **kw) == 1
    assert distill_call(sk, few, **kw) == 1 and distill_step(sk, few, **kw) == 1


@pytest.mark.parametrize("kw", [dict(lse=None), dict(tokens=None), dict(entropy=None), dict(tokens64=3), dict(lse=TWO),
                                dict(dlogp=TWO), dict(dentropy=ODD), dict(dlse=TWO), dict(err=TWO), dict(tokens=TWO)])
def test_logprob_grad_refusals(sk, kw):
    assert logprob_grad(sk, **kw) == 1


@pytest.mark.parametrize("call", [logprob_grad, distill_grad, distill_step])
@pytest.mark.parametrize("kw,expect", [
    (dict(dx=None), 1), (dict(dx=ODD), 1), (dict(sb=-1), 1), (dict(sn=-1), 1), (dict(sn=999), 1), (dict(sb=999), 1),
    (dict(sb=0), 1), (dict(sn=0), 1), (dict(sb=7999), 1), (dict(sn=1000, sb=1000), 1), (dict(sn=1 << 61), 1),
    (dict(sb=1 << 62), 1), (dict(sb=1000, sn=1999), 1)])
def test_gradient_rows_that_overlap(sk, call, kw, expect):
    assert call(sk, **kw) == expect


@pytest.mark.parametrize("call", [distill_call, distill_grad, distill_step])
@pytest.mark.parametrize("bad,expect", [
    (dict(ids=None), 1), (dict(values=None), 1), (dict(K=0), 1), (dict(K=-1), 1), (dict(K=129), 2), (dict(ids64=2), 1),
    (dict(dtype=3), 1), (dict(rest=2), 1), (dict(scale=0.5), 1), (dict(scale=float("nan"), rest=0), 1),
    (dict(scale=0.0, rest=0), 1), (dict(ids=0x100002), 1), (dict(ids=0x100004, ids64=1), 1), (dict(values=0x100002), 1),
    (dict(values=0x100001, dtype=0), 1)])
def test_teacher_refusals(sk, call, bad, expect):
    assert call(sk, t=teacher(sk, **bad)) == expect


@pytest.mark.parametrize("call", [distill_call, distill_grad, distill_step])
def test_distill_refusals(sk, call):
    assert call(sk, direction=2) == 1 and call(sk, direction=-1) == 1 and call(sk, stats=None) == 1
    assert call(sk, stats=FOUR) == 1
    assert call(sk, t=teacher(sk, rest=0), direction=1) == 2
    if call is not distill_grad:
        assert call(sk, loss=None) == 1 and call(sk, loss=TWO) == 1
    else:
        assert call(sk, dloss=TWO) == 1 and call(sk, dfactor=TWO) == 1 and call(sk, done=2) == 1
        assert call(sk, dfactor=None, done=1) == 1
    if call is distill_step:
        assert call(sk, weight=TWO) == 1


def test_null_structures(sk):
    assert sk.lib.streamkl_token_logprobs_fwd(None, None, 0, 1.0, 0, None, 0, None, None, FAKE, None, None, None, None) == 1
    assert sk.lib.streamkl_topk_distill_fwd(logits(sk), None, 1.0, 0, None, 0, FAKE, FAKE, None) == 1


def test_total_refusals(sk):
    f = sk.lib.streamkl_topk_distill_total
    assert f(FAKE, None, 1.0, -1, FAKE, None) == 1 and f(FAKE, None, 1.0, 5, None, None) == 1
    assert f(None, None, 1.0, 5, FAKE, None) == 1 and f(FAKE, TWO, 1.0, 5, FAKE, None) == 1
    assert f(FAKE, None, 1.0, 5, TWO, None) == 1


def test_workspace_sizes(sk):
    f, g = sk.lib.streamkl_token_logprobs_workspace_bytes, sk.lib.streamkl_topk_distill_workspace_bytes
    assert f(4, 4096, 100000, 0, 64) == 0 and g(4, 4096, 100000, 0, 1) == 0   # a workgroup a row
    assert f(1, 1, 100, 0, 10) == 0
    for bad in ((-1, 1, 10, 0, 1), (1, -1, 10, 0, 1), (1, 1, 0, 0, 0), (1, 1, 10, 5, 1), (1, 1, (1 << 22) + 1, 0, 1),
                (1 << 16, 1 << 16, 100, 0, 1)):
        assert f(*bad) == 0 and g(*bad) == 0
    assert f(1, 1, 10, 0, 11) == 0 and f(1, 1, 1000, 0, 129) == 0 and f(1, 1, 1000, 0, -1) == 0
    for V in (100000, 131072, 270000, 1 << 22):   # parts that the kernels' LDS holds, at most 32 of them
        for rows in (1, 7, 100, 10000):
            for t in (0, 1, 2):
                n = f(rows, 1, V, t, 128)
                parts = n / (rows * (12 + 128 * 8))
                assert n == 0 and V <= 135168 - 16 or 1 < parts < 33
