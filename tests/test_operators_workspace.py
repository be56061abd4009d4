"""The gradients' workspaces: bounded however many tokens there are.  Host logic, no GPU."""
import ctypes

import pytest

import paper_2401_10187_amd as km

Two = ctypes.c_int * 2
SHAPES = [(128, 128, 128, 128), (128, 256, 128, 256), (128, 512, 128, 512), (64, 256, 64, 256), (100, 90, 70, 333), (52, 50, 65, 20), (4, 1024, 4, 4096)]


@pytest.mark.parametrize("dtype", [km.KM_F32, km.KM_BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("name", ["gated_grad", "cross_entropy_grad"])
def test_bounded(name, shape, dtype):
    """What the header says: dX's parts 1 GiB, and for each of the factors' gradients a part from each of at most 256 workgroups, or from each block of columns where
    these are more."""
    p1, q1, p2, q2 = shape
    p, q, out = Two(p1, p2), Two(q1, q2), ctypes.c_size_t(0)
    products = 2 if name == "gated_grad" else 1
    blocks = -(-q1 // 32) * -(-q2 // 32)             # (the smallest blocks of any variant)
    factors = products * 4 * max(256, blocks) * (p1 * q1 + p2 * q2)
    sizes = []
    for m in (1, 100, 8192, 1 << 20, 1 << 30):
        args = (m, p, q, dtype) if products == 2 else (m, p, q, q1 * q2, dtype)
        assert getattr(km.lib(), "kronmatmul_%s_workspace_size" % name)(*args, ctypes.byref(out)) == km.KM_OK
        sizes.append(out.value)
        assert out.value <= (1 << 30) + factors + 5 * 256
    assert sizes[-1] <= sizes[-2] + (32 << 20)       # (the same but for how tokens divide)
