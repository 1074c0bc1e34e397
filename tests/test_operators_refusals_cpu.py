"""Refusals of the operators' calls that depend on more than one argument (CPU only): nothing is enqueued."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x100000)   # 16-byte aligned, never dereferenced: every call here is refused


@pytest.fixture(scope="module")
def sk():
    from paper_2606_20005_amd import streamkl
    return streamkl


def norm_call(sk, back, nq, nk, n_pos, rot=64, qp=None, kp=None):
    rows = ctypes.byref(sk._Rows(0x100000, 0, 512, 64))
    head = (None if nq is None else rows, None if nk is None else rows, 1, 4, 2, nq or 0, nk or 0, 64, 0, FAKE, FAKE, 1e-6,
            FAKE, n_pos, rot, 0, qp, kp, 0, 0, 0, 1)
    if back:   # without a workspace: refused in any case where a row exists, after the check of the places
        return sk.lib.streamkl_qk_norm_rope_bwd(*head, FAKE, FAKE, 0, None, 0, FAKE, FAKE, FAKE if nq is not None else None,
                                                FAKE if nk is not None else None, None)
    return sk.lib.streamkl_qk_norm_rope_fwd(*head, FAKE, FAKE, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("nq,nk,n_pos,qp,kp", [
    (4, 9, 8, None, None), (4, 9, 8, FAKE, None), (4, 9, 8, None, FAKE), (9, None, 8, None, None),
    (None, 9, 8, None, None), (1, 1 << 20, 4096, None, None)])
def test_default_places_outside_the_table_are_refused(sk, back, nq, nk, n_pos, qp, kp):
    assert norm_call(sk, back, nq, nk, n_pos, qp=qp, kp=kp) == 1


def test_default_places_of_no_rows_and_without_a_rotation(sk):
    """Nothing stands at them: accepted, and nothing is launched."""
    assert norm_call(sk, False, 0, 0, 8) == 0 and norm_call(sk, False, 0, None, 8) == 0
    rows = ctypes.byref(sk._Rows(None, 0, 512, 64))
    for rot in (0, 64):
        assert sk.lib.streamkl_qk_norm_rope_fwd(rows, rows, 0, 4, 2, 100, 100, 64, 0, FAKE, FAKE, 1e-6, FAKE, 8, rot, 0, None,
                                                None, 0, 0, 0, 1, None, None, None) == 0


def test_workspace_of_head_dims_that_are_refused(sk):
    f = sk.lib.streamkl_qk_norm_rope_bwd_workspace_bytes
    for d in (16, 40, 48, 250, 288):
        assert f(2, 4, 2, 10, 10, d) == 0
    assert f(2, 4, 2, 10, 10, 96) > 0
