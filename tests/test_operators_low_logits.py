"""The loss where all logits are low.  A softmax does not change when logits are shifted, and what is beyond the factors' columns has no part in it,
whatever e^-lse is.

Tolerances, derived before the first run: those of test_operators.py, and what single precision leaves of logits of some -110: e = 8 * 2^-24 |lse|, as in
test_operators_confident.py.  Here it is taken as common to a token's words, which all change by e p: the gradients change by e times those of dZ = p."""
import pytest

torch = pytest.importorskip("torch")
import paper_2401_10187_amd as km  # noqa: E402
from test_operators import BACKWARD, LOSS, TYPES, bf16, close, gen, kron, loss_reference, normal, product_grads  # noqa: E402

pytestmark = pytest.mark.gpu

# (tokens, P1, Q1, P2, Q2): columns q1 that end inside a block of rows beside columns q2 that are whole blocks, and other ends
SHAPES = [(9, 64, 200, 64, 256), (9, 64, 40, 64, 128), (5, 33, 17, 31, 64), (5, 100, 90, 128, 128), (3, 20, 300, 40, 512), (70, 16, 8, 24, 256), (4, 8, 33, 9, 70)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_low_logits(shape, dtype):
    t, p1, q1, p2, q2 = shape
    g = gen(sum(shape))

    def near(n, *s):
        return (n * (1 + 0.1 * normal(g, *s))).to(dtype)
    x, fs, dloss = near(1.0, t, p1 * p2), (near(-120 / p1, p1, q1), near(1 / p2, p2, q2)), normal(g, t)
    targets = torch.randint(0, q1 * q2, (t,), device="cuda", generator=g)
    want_loss, want_lse, want = loss_reference(x, fs, targets, q1 * q2, dloss)
    assert float(want_lse.max()) < -95
    loss, lse = km.kron_cross_entropy(x, fs, targets)
    close(lse, want_lse, LOSS, "lse")
    assert float((loss.double() - want_loss).abs().max()) <= LOSS * (float(want_lse.abs().max()) + 20)
    dx, df = km.kron_cross_entropy_grad(dloss, x, fs, targets, lse)
    p = torch.exp(kron(x.double(), *(f.double() for f in fs)) - want_lse[:, None])
    dz = p.clone()
    dz[torch.arange(t, device="cuda"), targets] -= 1
    rounded, common = [bf16(v) for v in product_grads(x, *fs, dz, dloss)], product_grads(x, *fs, p, dloss.abs())
    e = 8 * 2 ** -24 * float(want_lse.abs().max())
    for name, got, ref, r, c in zip(("dx", "df1", "df2"), (dx, *df), want, rounded, common):
        assert bool(torch.isfinite(got).all()), name
        off, norm = float((got.double() - ref).norm()), float(ref.norm())
        bound = BACKWARD[dtype] * norm if dtype == torch.float32 else 1.5 * float((r - ref).norm()) + 1e-5 * norm
        assert off <= bound + e * float(c.norm()), "%s: %.3g of the norm, %.3g allowed" % (name, off / norm, bound / norm)
