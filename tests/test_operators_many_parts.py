"""Gradients whose parts of dX are more than is kept at once: tokens are taken some at a time.  Tolerances as in test_operators.py."""
import pytest

torch = pytest.importorskip("torch")
import paper_2401_10187_amd as km  # noqa: E402
from test_operators import TYPES, check_cross_entropy, check_gated, gated_inputs, gen, loss_inputs, normal  # noqa: E402

pytestmark = pytest.mark.gpu
SHAPE = (128, 130, 128, 70)                         # several blocks of columns of either factor, each token's row 64 KB of fp32


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("t", [3001, 9001])
def test_against_the_definition(t, dtype):
    check_gated((t, *SHAPE), "silu", dtype)
    check_cross_entropy((t, *SHAPE), dtype, [SHAPE[1] * SHAPE[3] - 100])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_rows_are_those_of_smaller_calls_and_bits_stay(dtype):
    t = 8999
    x, gate, up, dh = gated_inputs(31, t, *SHAPE, dtype)
    _, fs, targets, dloss = loss_inputs(32, t, *SHAPE, dtype, 9000)
    targets[1000:5900] = -100                       # (whole slices of a launch without targets)
    lse = km.kron_cross_entropy(x, fs, targets, vocab=9000)[1]
    got = km.kron_gated_grad(dh, x, gate, up)
    lost = km.kron_cross_entropy_grad(dloss, x, fs, targets, lse, vocab=9000)
    for first in range(0, t, 1024):
        some = slice(first, min(t, first + 1024))
        assert torch.equal(km.kron_gated_grad(dh[some], x[some], gate, up)[0], got[0][some])
        part = km.kron_cross_entropy_grad(dloss[some], x[some], fs, targets[some].contiguous(), lse[some], vocab=9000)[0]
        assert torch.equal(part, lost[0][some])
    again = km.kron_gated_grad(dh, x, gate, up)
    assert torch.equal(again[0], got[0]) and all(torch.equal(p, q) for i in (1, 2) for p, q in zip(again[i], got[i]))
    again = km.kron_cross_entropy_grad(dloss, x, fs, targets, lse, vocab=9000)
    assert torch.equal(again[0], lost[0]) and all(torch.equal(p, q) for p, q in zip(again[1], lost[1]))


def test_strided_rows_and_a_graph():
    t = 4000
    x, gate, up, dh = gated_inputs(33, t, *SHAPE, torch.bfloat16)
    g = gen(34)
    wide, dwide = normal(g, t, 16384 + 24, dtype=torch.bfloat16), normal(g, t, 9100 + 7, dtype=torch.bfloat16)
    xs, ds = wide[:, 8:8 + 16384], dwide[:, 3:3 + 9100]
    xs.copy_(x)
    ds.copy_(dh)
    flat = lambda v: [v[0], *v[1], *v[2]]  # noqa: E731
    want = [v.clone() for v in flat(km.kron_gated_grad(dh, x, gate, up))]
    assert all(torch.equal(p, q) for p, q in zip(flat(km.kron_gated_grad(ds, xs, gate, up)), want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = flat(km.kron_gated_grad(ds, xs, gate, up))
    for _ in range(3):
        for v in held:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want))
        assert all(torch.equal(p, q) for p, q in zip(flat(km.kron_gated_grad(dh, x, gate, up)), want))
