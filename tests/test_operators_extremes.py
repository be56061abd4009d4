"""The gated block where an intermediate product would leave single precision and the result does not."""
import pytest

torch = pytest.importorskip("torch")
import paper_2401_10187_amd as km  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


def column(dtype, *values):
    return torch.tensor([values], device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("t", [3, 1100])
def test_a_closed_gate_closes(act, dtype, t):
    """act(-200) is 0 in single precision (-3e-85), and so are its products with 2e36 and with a gradient of 1e4."""
    one = torch.ones((1, 1), device="cuda", dtype=dtype)
    x = torch.ones((t, 1), device="cuda", dtype=dtype)
    gate, up = (column(dtype, -200.0, -300.0, 1.0, -1000.0), one), (column(dtype, 2e36, -2e36, 3.0, 1e38), one)
    h = km.kron_gated(x, gate, up, act=act).float()
    assert not h[:, [0, 1, 3]].any() and bool((h[:, 2] > 2).all())
    dh = torch.full((t, 4), 1e4, device="cuda", dtype=dtype)
    dh[:, 2] = 0
    for got in (lambda a, b, c: (a, *b, *c))(*km.kron_gated_grad(dh, x, gate, up, act=act)):
        assert not got.any()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_slopes_of_wide_open_and_closed_gates(act, dtype):
    """z = 1e20, whose square is no number in single precision: slope 1; z = -1e20: slope 0.  Values are right to one rounding of the type, or in single
    precision to four."""
    one = torch.ones((1, 1), device="cuda", dtype=dtype)
    x, dh = torch.ones((1, 1), device="cuda", dtype=dtype), torch.ones((1, 4), device="cuda", dtype=dtype)
    gate, up = (column(dtype, 1e20, -1e20, 1e38, -1e38), one), (column(dtype, 1.0, 1.0, 1.0, 1.0), one)
    bound = 2 ** -22 if dtype == torch.float32 else 2 ** -8
    want = gate[0].double().clamp(min=0)
    assert bool(((km.kron_gated(x, gate, up, act=act).double() - want).abs() <= bound * want).all())
    dh[0, 2:] = 0            # (their sum with the others' is no number)
    _, (dg, _), (du, _) = km.kron_gated_grad(dh, x, gate, up, act=act)
    assert dg.float().tolist() == [[1.0, 0.0, 0.0, 0.0]]
    assert bool(((du.double() - dh.double() * want).abs() <= bound * want).all())
