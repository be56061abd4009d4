"""Factors of as many columns as an int holds: refused or sized, without an overflow in between.  Host logic, no GPU."""
import ctypes

import pytest

import paper_2401_10187_amd as km

Two, Ptr2 = ctypes.c_int * 2, ctypes.c_void_p * 2
A = [(i + 1) << 44 for i in range(12)]              # nothing is read from these: every call here is refused before
ONE = Two(1, 1)
TYPES = [km.KM_F32, km.KM_BF16]


def size(name, *args):
    out = ctypes.c_size_t(0)
    return getattr(km.lib(), "kronmatmul_%s_workspace_size" % name)(*args, ctypes.byref(out)), out.value


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 1 << 30])
@pytest.mark.parametrize("q", [(2 ** 31 - 1, 1), (2147483633, 1), (2147483632, 1), ((1 << 28) + 1, 7), ((1 << 30) - 1, 2)], ids=str)
def test_more_columns_than_launches_reach(q, m, dtype):
    lib, q, columns = km.lib(), Two(*q), q[0] * q[1]
    assert size("gated_grad", m, ONE, q, dtype)[0] == km.KM_EUNSUPPORTED
    assert size("cross_entropy", m, ONE, q, columns, dtype)[0] == km.KM_EUNSUPPORTED
    assert size("cross_entropy_grad", m, ONE, q, columns, dtype)[0] == km.KM_EUNSUPPORTED
    m = 1                                            # (the addresses are far enough apart for these)
    assert lib.kronmatmul_gated(m, ONE, q, A[0], 1, Ptr2(A[1], A[2]), Ptr2(A[3], A[4]), 0, A[5], dtype, None) == km.KM_EUNSUPPORTED
    assert lib.kronmatmul_gated_grad(m, ONE, q, A[0], columns, A[1], 1, Ptr2(A[2], A[3]), Ptr2(A[4], A[5]), 0, A[6], Ptr2(A[7], A[8]), Ptr2(A[9], A[10]), dtype,
                                     A[11], 1 << 43, None) == km.KM_EUNSUPPORTED
    assert lib.kronmatmul_cross_entropy(m, ONE, q, columns, A[0], 1, Ptr2(A[1], A[2]), A[3], A[4], A[5], dtype, A[6], 1 << 43, None) == km.KM_EUNSUPPORTED
    assert lib.kronmatmul_cross_entropy_grad(m, ONE, q, columns, A[0], A[1], 1, Ptr2(A[2], A[3]), A[4], A[5], A[6], Ptr2(A[7], A[8]), dtype, A[9], 1 << 43,
                                             None) == km.KM_EUNSUPPORTED


@pytest.mark.parametrize("dtype", TYPES)
def test_a_small_vocabulary_of_such_a_factor_is_none(dtype):
    """Only the columns that words are in count."""
    q = Two(2 ** 31 - 1, 1)
    status, need = size("cross_entropy", 5, ONE, q, 1000, dtype)
    assert status == km.KM_OK and 0 < need < 1 << 20
    assert size("cross_entropy_grad", 5, ONE, q, 1000, dtype)[0] == km.KM_OK


@pytest.mark.parametrize("dtype", TYPES)
def test_wrong_arguments_are_still_wrong_first(dtype):
    q = Two(2 ** 31 - 1, 1)
    assert size("cross_entropy", 1, ONE, q, 0, dtype)[0] == km.KM_EINVAL
    assert km.lib().kronmatmul_gated(1, ONE, q, None, 1, Ptr2(A[1], A[2]), Ptr2(A[3], A[4]), 0, A[5], dtype, None) == km.KM_EINVAL
