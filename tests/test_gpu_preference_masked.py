"""Gradients of the preference loss behind the mask are zeros, whatever stands there."""
import numpy as np
import pytest

from tests.harness import ensure_built
from tests.test_gpu_losses import _mask, _place

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bg():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    ensure_built()
    import paper_2510_11683_gb300 as bg
    return bg


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "ipo"])
@pytest.mark.parametrize("mask", ["random", "prefix", "empty"])
@pytest.mark.parametrize("K,Tc,Tr,layout", [
    (6, 64, 64, "rows"), (5, 31, 200, "rows"), (4, 1000, 77, "sliced"), (7, 2048, 2048, "rows"),
    (3, 6000, 4097, "rows"), (2, 40003, 16, "rows"), (9, 16, 16, "transposed"),
])
def test_no_gradient_behind_the_mask(bg, K, Tc, Tr, layout, mask, kind):
    import torch
    beta, scale = 0.3, 2.0
    t = {}
    for s, T in (("c", Tc), ("r", Tr)):
        rng = np.random.default_rng(K + T + (s == "c"))
        lp = -rng.random((K, T)).astype(np.float32) / T
        m = _mask(rng, K, T, mask)
        lp[~m] = rng.choice([np.nan, np.inf, -np.inf, -3.4e38], int((~m).sum()))
        t[s] = (_place(lp, layout), _place(m, layout), _place(np.full((K, T), 7, np.float32), layout), m)
    ws, out = bg.alloc_train_workspace(), torch.empty(5, device="cuda")
    for average in (False, True):
        for s in "cr":
            t[s][2].fill_(7.0)
        bg.preference_loss(t["c"][0], t["r"][0], out, t["c"][2], t["r"][2], ws, kind=kind, beta=beta,
                           scale=scale, mask_chosen=t["c"][1], mask_rejected=t["r"][1],
                           average=average)
        for s, sign in (("c", -1), ("r", 1)):
            g, m = t[s][2].cpu().numpy(), t[s][3]
            assert np.all(g[~m] == 0)
            # scores are near 0: every pair's margin is on the same side of each loss's zero
            assert np.all(np.sign(g[m]) == sign)
    assert bg.get_device_error(ws) == (0, 0)
