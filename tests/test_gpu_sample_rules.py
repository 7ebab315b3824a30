"""token_sample where it changes its way through a row: by slices or by a workgroup."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device
from test_gpu_sample import BF16, F32, check, dev_of, logits

pytestmark = pytest.mark.gpu


def used(V, **kw):
    """Whether a call of four rows leaves something in its workspace, as the slices do."""
    x, u = logits(V, 4, V)
    ws = api.new_workspace(api.token_sample_workspace_bytes(4, V, F32), device())
    full = {n: torch.full((4,), a, dtype=torch.int32 if n == "top_k" else F32, device=device()) for n, a in kw.items()}
    api.token_sample(dev_of(x), dev_of(u), workspace=ws, **full)
    torch.cuda.synchronize()
    return bool(ws.any())


def test_top_k_without_top_p_goes_by_a_workgroup_per_row():
    for V in (40001, 131072):
        assert not used(V, top_k=50) and not used(V, top_k=500, min_p=0.1, temperature=0.7)
        assert used(V) and used(V, top_p=0.9) and used(V, top_k=50, top_p=0.9) and used(V, min_p=0.1)
    assert used(131073, top_k=20)
    assert not used(32768, top_p=0.9)


@pytest.mark.parametrize("V", [40001, 131072, 131073, 200001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_around_the_k_that_slices_take(V, dtype):
    x, u = logits(V, 8, V, dtype=dtype)
    ks = np.array([1, 40, 47, 48, 49, 50, 192, 193], np.int32)
    cold = np.array([1, 0, 0.7, 0, 0, -1, np.inf, np.nan], np.float32)
    for kw in (dict(), dict(top_p=0.9), dict(top_p=0.9, min_p=0.05), dict(min_p=0.05)):
        check(x, u, "k around 48", top_k=ks, **kw)
        check(x, u, "k around 48, T of all kinds", top_k=ks, temperature=cold, **kw)
    ties = x.copy()
    ties[:, ::7] = x[:, 5:6]
    check(ties, u, "ties", top_k=ks, top_p=0.8)
    check(ties, u, "ties", top_k=ks)
