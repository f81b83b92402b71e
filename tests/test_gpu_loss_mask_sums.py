"""What the policy loss reports of small ratios behind a scattered mask, against the fp64 oracle.

A token that does not count must leave no trace in the sums, not even a rounding: terms of one
sign keep their relative precision however small the ratios are. Bound, with e = 2^-24: a log
ratio d is rounded once (|d| e of the ratio), expf is off by 2 units (4 e), products with the
weight and the advantage take 6 roundings, and a sum of terms of one sign is off by e for each of
the additions a term goes through: 7 in a thread's eight, a running sum of at most 16 here, 5
across a warp, 5 across its block and 16 across blocks. Under 64 e and |d| e; a row's mean log ratio is itself such
a sum, 24 e |d| with its division.
"""
import numpy as np
import pytest

from oracle import policy_oracle as O
from tests.harness import ensure_built

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.fixture(scope="module")
def bg():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    ensure_built()
    import paper_2510_11683_gb300 as bg
    return bg


def _place(x, layout):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    if layout == "transposed":
        return t.T.contiguous().T
    if layout == "shifted":                    # rows between boundaries of eight
        flat = torch.zeros(t.numel() + 3, dtype=t.dtype, device="cuda")[3:]
        return flat.view(t.shape).copy_(t)
    return t


@pytest.mark.parametrize("layout", ["plain", "shifted", "transposed"])
@pytest.mark.parametrize("N,T", [(3, 8), (40, 64), (7, 256), (5, 1024), (3, 6000), (1, 40000)])
@pytest.mark.parametrize("ratio", [1e-3, 1e-5, 1e-7, 1e-20])
def test_small_ratios_behind_a_scattered_mask(bg, ratio, N, T, layout):
    import torch
    rng = np.random.default_rng(N + T)
    d = np.log(ratio) + 0.1 * rng.standard_normal((N, T))
    old = (-rng.random((N, T)) - 0.1).astype(np.float32)
    lp = (old + d).astype(np.float32)
    # one token in eight counts, behind the others
    mask = np.zeros((N, T), bool)
    at = np.arange(0, T, 8)
    for b in range(N):
        mask[b, np.minimum(at + rng.integers(0, 8, len(at)), T - 1)] = True
    A = (0.5 + rng.random((N, T))).astype(np.float32)       # unclipped: the term is -r A
    size = np.abs(lp.astype(np.float64) - old).max()
    t = [_place(x, layout) for x in (lp, old, A, mask)]
    row = torch.from_numpy(A[:, 0].copy()).cuda()
    ws, out = bg.alloc_train_workspace(), torch.empty(6, device="cuda")
    for adv, adv64 in ((row, A[:, 0]), (t[2], A)):
        for norm in ("rows", "tokens", "sum"):
            for kind in ("token",) if adv is t[2] else ("token", "sequence"):
                tol = (64 + (24 if kind == "sequence" else 1) * size) * E
                dlogp = _place(np.full((N, T), 9, np.float32), layout)
                bg.policy_loss(t[0], t[1], adv, out, dlogp, ws, mask=t[3], norm=norm, ratio=kind)
                want, grad, _ = O.policy_loss(lp, old, adv64, mask=mask, norm=norm, ratio=kind)
                got = out.double().cpu().numpy()
                assert want[1] < 0 and want[5] > 0
                for i in (0, 1, 5):
                    assert abs(got[i] - want[i]) <= tol * abs(want[i]), (i, norm, kind)
                g = dlogp.double().cpu().numpy()
                assert np.all(np.abs(g - grad) <= tol * np.abs(grad))
    assert bg.get_device_error(ws) == (0, 0)


@pytest.mark.parametrize("N,T", [(6, 64), (3, 3000)])
def test_large_values_beside_small_ones(bg, N, T):
    # clipped below: the term is the bound, and the mean ratio is that of the tokens that count
    import torch
    rng = np.random.default_rng(T)
    old = (-rng.random((N, T)) - 0.1).astype(np.float32)
    lp = (old - 12).astype(np.float32)
    mask = rng.random((N, T)) < 0.1
    mask[:, 0] = True
    lp[~mask] = 80.0
    A = np.full(N, -1.5, np.float32)
    t = [torch.from_numpy(x).cuda() for x in (lp, old, A, mask)]
    ws, out, dl = bg.alloc_train_workspace(), torch.empty(6, device="cuda"), torch.empty_like(t[0])
    bg.policy_loss(t[0], t[1], t[2], out, dl, ws, mask=t[3])
    want, grad, _ = O.policy_loss(lp, old, A, mask=mask)
    got = out.double().cpu().numpy()
    assert want[3] == 1 and got[3] == 1 and got[4] == 0 and not dl.any()
    for i in (0, 1, 5):
        assert abs(got[i] - want[i]) <= 80 * E * abs(want[i])
