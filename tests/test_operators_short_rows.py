"""Tokens whose rows are shorter than the eight elements that a lane reads at once: every P1 x P2 below 8.  Tolerances as in test_operators.py."""
import pytest

torch = pytest.importorskip("torch")
from test_operators import TYPES, check_cross_entropy, check_gated, close, gated_inputs, gated_reference, FORWARD  # noqa: E402
import paper_2401_10187_amd as km  # noqa: E402

pytestmark = pytest.mark.gpu
SHORT = [(p1, p2) for p1 in range(1, 8) for p2 in range(1, 8) if 2 <= p1 * p2 < 8]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("p", SHORT, ids=str)
def test_short_rows(p, dtype):
    """Few tokens and many, columns that are less than a block and several."""
    for t, q1, q2 in ((40, 5, 9), (700, 40, 70)):
        check_gated((t, p[0], q1, p[1], q2), "silu", dtype)
        check_cross_entropy((t, p[0], q1, p[1], q2), dtype, [q1 * q2 - 3])


@pytest.mark.parametrize("p", SHORT, ids=str)
def test_every_element_counts(p):
    """One element of X at a time: none is left out."""
    n = p[0] * p[1]
    _, gate, up, _ = gated_inputs(n, 1, p[0], 6, p[1], 7, torch.float32)
    x = torch.eye(n, device="cuda") * 3
    close(km.kron_gated(x, gate, up), gated_reference(x, gate, up, "silu")[0], FORWARD[torch.float32])
