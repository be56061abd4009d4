"""Rows, tokens and columns beyond one launch: HIP takes fewer than 2^32 work-items.  Every row is one of 64, whose results are known from a small call."""
import pytest

torch = pytest.importorskip("torch")
import paper_2401_10187_amd as km  # noqa: E402

pytestmark = pytest.mark.gpu


def enough(gib):
    free = torch.cuda.mem_get_info()[0]
    if free < gib << 30:
        pytest.skip("needs %d GiB of device memory, %d are free" % (gib, free >> 30))


def repeated(base, rows):
    """`rows` rows, row i being row i % 64 of `base`."""
    out = torch.empty((rows, *base.shape[1:]), dtype=base.dtype, device="cuda")
    whole = rows // 64 * 64
    out[:whole].view(-1, *base.shape).copy_(base.expand(whole // 64, *base.shape))
    out[whole:] = base[:rows - whole]
    return out


def repeats(got, base):
    whole = len(got) // 64 * 64
    return bool((got[:whole].view(-1, *base.shape) == base).all()) and torch.equal(got[whole:], base[:len(got) - whole])


# four rows to a workgroup of 256; one
@pytest.mark.parametrize("rows,width", [((1 << 26) + 5, 8), ((1 << 24) + 3, 129)])
def test_layer_norm(rows, width):
    enough(40)
    g = torch.Generator(device="cuda").manual_seed(1)
    base = torch.randn((64, width), generator=g, device="cuda").bfloat16()
    w, b = torch.randn((2, width), generator=g, device="cuda").bfloat16().unbind()
    w, b = w.clone(), b.clone()
    want = km.layer_norm(base, w, b)
    x = repeated(base, rows)
    got = km.layer_norm(x, w, b)
    assert all(repeats(p, q) for p, q in zip(got, want))
    dwant = km.layer_norm_grad(base, base, w, *want[1:])[0]
    assert repeats(km.layer_norm_grad(x, x, w, *got[1:])[0], dwant)


def test_loss():
    enough(40)
    g = torch.Generator(device="cuda").manual_seed(2)
    base = torch.randn((64, 1), generator=g, device="cuda").bfloat16()
    fs = [torch.randn((1, 3), generator=g, device="cuda").bfloat16(), torch.randn((1, 2), generator=g, device="cuda").bfloat16()]
    targets = torch.randint(-1, 6, (64,), generator=g, device="cuda")
    # (a call of as many tokens as have the same kernel: few tokens add up in another order)
    want = [v[:64] for v in km.kron_cross_entropy(base.repeat(64, 1), fs, targets.repeat(64))]
    rows = (1 << 28) + 33
    got = km.kron_cross_entropy(repeated(base, rows), fs, repeated(targets, rows))
    assert all(repeats(p, q) for p, q in zip(got, want))


def test_gradient_of_a_factor_far_wider_than_its_vocabulary():
    """2^30 elements and 17 parts of them, all but the vocabulary's zeros."""
    enough(120)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((17, 16), generator=g, device="cuda").bfloat16()
    near, second = torch.randn((16, 50), generator=g, device="cuda").bfloat16(), torch.ones((1, 1), device="cuda").bfloat16()
    targets, dloss = torch.randint(0, 50, (17,), generator=g, device="cuda"), torch.randn(17, generator=g, device="cuda")
    far = torch.zeros((16, (1 << 26) + 3), dtype=torch.bfloat16, device="cuda")
    far[:, :50] = near
    loss, lse = km.kron_cross_entropy(x, (near, second), targets)
    got = km.kron_cross_entropy(x, (far, second), targets, vocab=50)
    assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
    want, (d1, d2) = km.kron_cross_entropy_grad(dloss, x, (near, second), targets, lse)
    dx, (e1, e2) = km.kron_cross_entropy_grad(dloss, x, (far, second), targets, lse, vocab=50)
    assert torch.equal(dx, want) and torch.equal(e2, d2) and torch.equal(e1[:, :50], d1)
    assert not e1[:, 50:].any()
    del e1, far
    torch.cuda.empty_cache()


@pytest.mark.parametrize("width", [1 << 30, (1 << 30) - 1], ids=["aligned", "odd"])
def test_statistics_of_the_longest_row(width):
    """Sums of 2^30 squares: in single precision, a thread's 4 million of them one after the other would lose the small ones (2e-3 of rstd)."""
    enough(30)
    x = torch.empty((1, width), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    total = square = 0.0
    for some in x[0].split(1 << 27):
        total += float(some.double().sum())
        square += float(some.double().square().sum())
    mean = total / width
    _, got, rstd = km.layer_norm(x, torch.ones(width, dtype=torch.bfloat16, device="cuda"))
    # sums of blocks, each good to some 2^-24 a step: a thread adds 256 to 2048 elements, then up to 16384 of these sums
    assert abs(float(got) - mean) <= 1e-5
    assert abs(float(rstd) * (square / width - mean * mean + 1e-5) ** 0.5 - 1) <= 1e-5


def test_gradients_of_the_longest_row():
    """2^30 elements, two rows: the sums over them are right to the last column."""
    enough(60)
    h = 1 << 30
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.empty((2, h), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    w = torch.ones(h, dtype=torch.bfloat16, device="cuda")
    _, mean, rstd = km.layer_norm(x, w)
    assert float(mean.abs().max()) < 1e-3 and float((rstd - 1).abs().max()) < 1e-3
    _, dw, db = km.layer_norm_grad(dy, x, w, mean, rstd)
    for first in range(0, h, h // 8):
        some = slice(first, first + h // 8)
        assert torch.equal(db[some], (dy[0, some].float() + dy[1, some].float()).bfloat16())
        xhat = (x[:, some].float() - mean[:, None]) * rstd[:, None]
        # (one rounding to bf16 of a sum of two products in single precision)
        terms = dy[:, some].float() * xhat
        assert bool(((dw[some].float() - terms.sum(0)).abs() <= 2 ** -8 * terms.sum(0).abs() + 2 ** -22 * terms.abs().sum(0)).all())
        del xhat, terms
    del x, dy, w, dw, db
    torch.cuda.empty_cache()
