"""Calls of the 8-bit product, the norm and the clipping that lie off the ordinary path, on the GPU."""
import numpy as np
import pytest

import block_reference as ref
from test_gpu_learner import _learner, _np, _torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_a_lazy_copy_becomes_a_tensors_own_before_its_gradient_is_scaled():
    torch, L = _torch(), _learner()
    a = torch.full((1000,), 2.0, device="cuda")
    b = a._lazy_clone()
    norm = L.clip_gradients([b], 1.0)
    want = 2.0 * 1.0 / np.sqrt(4000.0)
    assert abs(norm.item() - np.sqrt(4000.0)) <= 6 * U * np.sqrt(4000.0)
    assert (a == 2).all() and (np.abs(_np(b) - want) <= 8 * U * want).all()
    zeros = torch.zeros(1000, device="cuda")
    out, read = zeros._lazy_clone(), a._lazy_clone()
    L.clip_gradients([read], 1.0, out=[out])
    assert (zeros == 0).all() and (a == 2).all() and (read == 2).all() and (np.abs(_np(out) - want) <= 8 * U * want).all()
    # the same tensor read and written
    both = a._lazy_clone()
    L.clip_gradients([both], 1.0, out=[both])
    assert (a == 2).all() and torch.equal(both, out)
    # what is read is written elsewhere in the list, and the other way around
    x, z = torch.full((100,), 3.0, device="cuda"), torch.full((100,), 4.0, device="cuda")
    y = x._lazy_clone()
    L.clip_gradients([x, z], 1.0, out=[x, y])
    norm = np.sqrt(2500.0)
    assert (np.abs(_np(x) - 3 / norm) <= 8 * U * 3 / norm).all() and (np.abs(_np(y) - 4 / norm) <= 8 * U * 4 / norm).all() and (z == 4).all()
