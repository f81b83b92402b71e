"""The policy loss on Monte Carlo samples, taken back to the hidden states and the head: the loss
takes l stored as [n_t, B] as its transpose, writes dL/dl through the same view, and row j of that
is what elbo_bwd_accumulate takes for sample j."""
import numpy as np
import pytest

from oracle import bgpo_oracle as O
from oracle import policy_oracle as PO
from synth import CONFIGS, make_inputs
from tests.harness import ensure_built, normwise, oracle_advantages, to64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["tiny", "ragged"])
@pytest.mark.parametrize("ratio", ["token", "sequence"])
def test_gradients_of_a_loss_on_samples(name, ratio):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    ensure_built()
    import paper_2510_11683_gb300 as bg
    wl = CONFIGS[name]
    inp = make_inputs(wl, device="cuda")
    X, W, Y = inp["X"], inp["W"], inp["Y"]
    B, n_t = wl.B, wl.n_t
    prob = bg.problem_from(wl)
    ws, tws = bg.alloc_workspace(prob), bg.alloc_train_workspace()
    A64 = oracle_advantages(wl, {k: (v.cpu() if v is not None else None) for k, v in inp.items()})
    A = torch.from_numpy(A64.astype(np.float32)).cuda()
    ell, dell = (torch.empty(n_t, B, device="cuda") for _ in range(2))
    tmp, out = torch.empty(B, device="cuda"), torch.empty(6, device="cuda")
    for j in range(n_t):
        bg.sample_mask(prob, j, ws)
        bg.elbo_fwd(prob, j, X, W, Y, ws, ell[j])
    noise = inp["eps"].T.contiguous()
    old, ref = ell + noise, ell - 0.5 * noise
    kw = dict(beta=0.04, ratio=ratio, norm="rows", clip_low=0.2, clip_high=0.28)
    bg.policy_loss(ell.T, old.T, A, out, dell.T, tws, logp_ref=ref.T, **kw)
    dX = torch.zeros(B, wl.R, wl.H, device="cuda")
    dW = torch.zeros(wl.V, wl.H, device="cuda")
    for j in range(n_t):
        bg.sample_mask(prob, j, ws)
        bg.elbo_fwd(prob, j, X, W, Y, ws, tmp)
        bg.elbo_bwd_accumulate(prob, j, X, W, Y, dell[j], ws, dX, dW)
    assert bg.get_device_error(ws) == (0, 0) and bg.get_device_error(tws) == (0, 0)
    # dL/dl on the kernel's own l, then the gradients of sum dL/dl l in 64 bits
    want, grad, size = PO.policy_loss(to64(ell).T, to64(old).T, to64(A), ref=to64(ref).T, **kw)
    # (ratios are of differences of l: the rounding of l's own size, as in the losses' tests)
    e = 2.0 ** -24
    d = np.abs(to64(ell) - to64(old)).max()
    assert np.all(np.abs(to64(dell).T - grad) <= (24 + (n_t + 4) * d) * e * size.max())
    ts, masks = O.sample_masks(wl.seed, B, wl.R, n_t, wl.t_mode)
    gX, gW = np.zeros((B, wl.R, wl.H)), np.zeros((wl.V, wl.H))
    for j in range(n_t):
        x, w = O.elbo_term_grads(to64(X), to64(W), to64(Y), wl.P, masks[j], ts[j], grad[:, j])
        gX += x
        gW += w
    assert normwise(to64(dW), gW) <= 2e-2 and normwise(to64(dX), gX) <= 2e-2
