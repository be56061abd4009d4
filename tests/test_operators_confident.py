"""The loss's gradients for tokens whose target is likely: what is left of p - 1 has to be as good as any other gradient.

Tolerances, derived before the first run.  bf16: the three stated roundings (dZ = p - 1 at the target, rounded once; U and dU; the result), computed for each case
in 64 bits, and 1.5 times what they leave, as in test_operators.py.  To that comes what single precision leaves of the logits: the forward pass's sum and the
gradient's exponentials each round a logit less its reference some six times, by 2^-24 of at most |lse| a time: e = 8 * 2^-24 |lse|
in the root mean square over few tokens, generously.  It changes p at the target by e p, and the gradients by what a dZ of e at each token's target gives
(the tokens' parts taken as independent)."""
import pytest

torch = pytest.importorskip("torch")
import paper_2401_10187_amd as km  # noqa: E402
from test_operators import BACKWARD, TYPES, bf16, gen, kron, loss_reference, normal, product_grads  # noqa: E402

pytestmark = pytest.mark.gpu


def confident(seed, t, p1, q1, p2, q2, vocab, dtype, p):
    """Inputs whose targets have a probability of about p: each token is moved along its target's column of the product."""
    g = gen(seed)
    fs = (normal(g, p1, q1, dtype=dtype, scale=p1 ** -0.5), normal(g, p2, q2, dtype=dtype, scale=p2 ** -0.5))
    f1, f2 = (f.double() for f in fs)
    targets = torch.randint(0, vocab, (t,), device="cuda", generator=g)
    targets[0], targets[1] = vocab - 1, 0
    x = 0.7 * normal(g, t, p1 * p2).double()
    along = (f1[:, targets // q2].t()[:, :, None] * f2[:, targets % q2].t()[:, None, :]).flatten(1)
    along = along / along.square().sum(1, keepdim=True)
    base, step = kron(x, f1, f2)[:, :vocab], kron(along, f1, f2)[:, :vocab]
    low, high = torch.full((t, 1), -20.0, device="cuda", dtype=torch.float64), torch.full((t, 1), 60.0, device="cuda", dtype=torch.float64)
    for _ in range(50):
        middle = (low + high) / 2
        z = base + middle * step
        less = torch.softmax(z, 1).gather(1, targets[:, None]) < p
        low, high = torch.where(less, middle, low), torch.where(less, high, middle)
    x = (x + high * along).to(dtype).contiguous()
    got = torch.softmax(kron(x.double(), f1, f2)[:, :vocab], 1).gather(1, targets[:, None])[:, 0]
    assert bool((((1 - got) / (1 - p) - 1).abs() < 0.5).all())      # (rounding X moves a logit a little)
    return x, fs, targets, normal(g, t)


# whole blocks of columns; ends inside blocks; targets in several blocks of columns of either factor; factors of 128
CASES = [(32, 64, 64, 64, 64, 4096), (20, 33, 40, 20, 30, 1150), (24, 64, 300, 40, 513, 153000), (9, 128, 130, 128, 70, 9100)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("p", [0.6, 0.9, 0.99, 0.999, 0.9999])
@pytest.mark.parametrize("shape", CASES, ids=str)
def test_what_is_left_of_likely_targets(shape, p, dtype):
    t, p1, q1, p2, q2, vocab = shape
    x, fs, targets, dloss = confident(t + p1, *shape, dtype, p)
    f1, f2 = (f.double() for f in fs)
    _, want_lse, want = loss_reference(x, fs, targets, vocab, dloss)
    lse = km.kron_cross_entropy(x, fs, targets, vocab=vocab)[1]
    dx, df = km.kron_cross_entropy_grad(dloss, x, fs, targets, lse, vocab=vocab)

    dz = torch.exp(kron(x.double(), f1, f2) - want_lse[:, None])
    dz[:, vocab:] = 0
    dz[torch.arange(t, device="cuda"), targets] -= 1
    rounded = [bf16(v) for v in product_grads(x, *fs, dz, dloss)]

    e = 8 * 2 ** -24 * want_lse.abs().max() * dloss.double().abs()
    a, b, xm = f1[:, targets // q2].norm(dim=0), f2[:, targets % q2].norm(dim=0), x.double().view(t, p1, p2)
    u = (xm @ f2).gather(2, (targets % q2)[:, None, None].expand(t, p1, 1))[:, :, 0].norm(dim=1)
    v = (xm.transpose(1, 2) @ f1).gather(2, (targets // q2)[:, None, None].expand(t, p2, 1))[:, :, 0].norm(dim=1)
    left = [float((e * w).norm()) for w in (a * b, u, v)]
    for name, got, ref, r, more in zip(("dx", "df1", "df2"), (dx, *df), want, rounded, left):
        off, norm = float((got.double() - ref).norm()), float(ref.norm())
        bound = BACKWARD[dtype] * norm if dtype == torch.float32 else 1.5 * float((r - ref).norm()) + 1e-5 * norm
        assert off <= bound + more, "%s: %.3g of the norm, %.3g allowed" % (name, off / norm, (bound + more) / norm)
