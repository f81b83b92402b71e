"""Which tokens a call selects: response lengths alone select what the mask of those lengths
does, bit for bit."""
import numpy as np
import pytest

from tests.harness import ensure_built
from tests.test_gpu_token_logp import _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bg():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    ensure_built()
    import paper_2510_11683_gb300 as bg
    return bg


@pytest.mark.parametrize("B,P,R", [(5, 2, 70), (1, 0, 1), (7, 3, 33), (9, 0, 1000), (40, 1, 419)])
def test_lengths_alone_select_as_their_mask_does(bg, B, P, R):
    import torch
    H, V = 64, 300
    X, W, Y, g = _inputs(B, P, R, H, V, B + R)
    rng = np.random.default_rng(R)
    n = rng.integers(0, R + 1, B)
    n[:5] = [R, 0, 1, R // 2, R - 1][:B]
    lens = torch.from_numpy(n.astype(np.int32)).cuda()
    mask = torch.arange(R, device="cuda") < lens[:, None]
    got = []
    for prob, m in ((bg.problem(B, P, R, H, V, 1, 1), mask),
                    (bg.problem(B, P, R, H, V, 1, 1, resp_len=lens), None)):
        ws, logp = bg.alloc_workspace(prob), torch.full((B, R), 7.0, device="cuda")
        dX = torch.full((B, R, H), 7.0, dtype=torch.bfloat16, device="cuda")
        dW = torch.full((V, H), 7.0, dtype=torch.bfloat16, device="cuda")
        bg.token_logp_fwd(prob, X, W, Y, ws, logp, mask=m)
        bg.token_logp_bwd(prob, W, g, ws, dX, dW)
        assert bg.get_device_error(ws) == (0, 0)
        got.append((logp, dX, dW))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(got[1][0] != 0, mask)
    assert not got[1][1][~mask].any()
