"""The grade of a matrix's products, as the host sees it (no GPU needed)."""

import ctypes

import pytest


def _mat(lib, grade, dtype=1, m=300, n=400):
    return lib.zo_muon_matrix(0x1000, 0x2000, 0x3000, m, n, n, n, dtype, dtype, grade)


def _need(lib, *args, **kw):
    return lib.LIB.zo_muon_workspace((lib.zo_muon_matrix * 1)(_mat(lib, *args, **kw)), 1)


def test_pairs_take_their_workspace_where_they_are_asked_for(lib):
    assert 0 < _need(lib, lib.ZO_MUON_GRADE_DTYPE) < _need(lib, lib.ZO_MUON_GRADE_F32)
    # fp32 matrices and small ones have them in any case
    for kw in (dict(dtype=0), dict(m=100)):
        assert 0 < _need(lib, lib.ZO_MUON_GRADE_DTYPE, **kw) == _need(lib, lib.ZO_MUON_GRADE_F32, **kw)


@pytest.mark.parametrize("grade", [-1, 2])
def test_an_unknown_grade_is_refused(lib, grade):
    ctx = ctypes.c_void_p(7)
    arr = (lib.zo_muon_matrix * 1)(_mat(lib, grade))
    assert lib.LIB.zo_muon_workspace(arr, 1) == 0
    assert lib.LIB.zo_muon_create(ctypes.byref(ctx), arr, 1, 0x10000, 1 << 40, None) == lib.ZO_ERR_INVALID_ARG
    assert not ctx.value
