"""What a vocabulary may be given as: any whole number."""
import pytest

torch = pytest.importorskip("torch")
import numpy as np  # noqa: E402

import paper_2401_10187_amd as km  # noqa: E402

pytestmark = pytest.mark.gpu


def test_whole_numbers_only():
    x, fs = torch.ones((2, 6), device="cuda"), (torch.ones((2, 3), device="cuda"), torch.ones((3, 4), device="cuda"))
    targets, dloss = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.ones(2, device="cuda")
    loss, lse = km.kron_cross_entropy(x, fs, targets, vocab=5)
    assert torch.equal(km.kron_cross_entropy(x, fs, targets, vocab=np.int64(5))[0], loss)
    for wrong in (5.7, 5.0, "5"):
        with pytest.raises(TypeError):
            km.kron_cross_entropy(x, fs, targets, vocab=wrong)
        with pytest.raises(TypeError):
            km.kron_cross_entropy_grad(dloss, x, fs, targets, lse, vocab=wrong)
    for wrong in (0, -1, 13, 2 ** 70):
        with pytest.raises(ValueError):
            km.kron_cross_entropy(x, fs, targets, vocab=wrong)
