"""Sums over very many tokens or pairs: what the losses report, against fp64.

Views that repeat one row (stride 0) make batches of 10^10 tokens out of little memory. All
terms of a sum have one sign, so that its error shows relative to it. Bound, with e = 2^-24: a
term takes |d| e from its log ratio's rounding, 4 e from expf and at most 12 e from its other
operations (the KL term's series: 10 products and sums); the sum adds 7 e in a thread's eight, 2 e
for the running sum (which carries what its roundings leave out), 5 e across a warp, 5 e across
its block and 8 e across blocks. Under 48 e and |d| e, whatever the number of tokens.
"""
import numpy as np
import pytest

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


def _row(x, N):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().view(1, -1).expand(N, -1)


def _close(got, want, d):
    assert abs(got - want) <= (48 + abs(d)) * E * abs(want), (got / want - 1) / E


@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("same", [True, False])
def test_tokens_of_a_large_batch(bg, same, per_token):
    import torch
    N, T = 1 << 20, 16384
    rng = np.random.default_rng(5)
    old = -1 - rng.random(T).astype(np.float32)
    d = np.full(T, 0.1) if same else 0.1 + 0.05 * rng.random(T)
    if same:
        old[:] = -1.25
    lp = (old + d).astype(np.float32)
    ref = (lp + (0.3 if same else 0.3 + 0.3 * rng.random(T))).astype(np.float32)
    d = lp.astype(np.float64) - old
    k = ref.astype(np.float64) - lp
    A = np.float32(1.3)
    adv = torch.full((1,), float(A), device="cuda").expand(N)
    if per_token:
        adv = _row(np.full(T, A), N)
    ws, out = bg.alloc_train_workspace(), torch.empty(6, device="cuda")
    bg.policy_loss(_row(lp, N), _row(old, N), adv, out, None, ws, logp_ref=_row(ref, N), beta=0.0,
                   norm="sum")
    got = out.double().cpu().numpy()
    want_pg = -N * float(A) * np.exp(d).sum()
    _close(got[0], want_pg, d.max())
    _close(got[1], want_pg, d.max())
    _close(got[2], N * (np.expm1(k) - k).sum(), 4 * np.abs(k).max())
    _close(got[5], np.exp(d).mean(), d.max())
    assert bg.get_device_error(ws) == (0, 0)


@pytest.mark.parametrize("N,T", [(1 << 26, 256), (1 << 22, 4096), (1 << 19, 20000)])
def test_sequence_ratios_of_a_large_batch(bg, N, T):
    import torch
    old = np.full(T, -1.25, np.float32)
    lp = np.full(T, -1.1, np.float32)
    ref = np.full(T, -0.75, np.float32)
    d, k = float(lp[0]) - float(old[0]), float(ref[0]) - float(lp[0])
    adv = torch.full((1,), 0.7, device="cuda").expand(N)
    ws, out = bg.alloc_train_workspace(), torch.empty(6, device="cuda")
    bg.policy_loss(_row(lp, N), _row(old, N), adv, out, None, ws, logp_ref=_row(ref, N), beta=0.5,
                   ratio="sequence", norm="sum")
    got = out.double().cpu().numpy()
    n = float(N) * T
    pg, kl = -n * float(np.float32(0.7)) * np.exp(d), n * (np.expm1(k) - k)
    # (a row's ratio: e of its mean log ratio, a sum of T with 7 + 5 + 5 + 3 additions a term)
    assert abs(got[1] / pg - 1) <= (48 + 24 * d) * E
    assert abs(got[5] / np.exp(d) - 1) <= (48 + 24 * d) * E
    _close(got[2], kl, 4 * k)
    assert abs(got[0] - (pg + 0.5 * kl)) <= 80 * E * (abs(pg) + 0.5 * kl)
    assert bg.get_device_error(ws) == (0, 0)


@pytest.mark.parametrize("T,repeated", [((1 << 27) - 3, False), (1 << 28, True)])
def test_a_row_of_very_many_tokens(bg, T, repeated):
    # its log ratios are summed over the row; repeated: one value at stride 0
    import torch
    arrays = []
    for x in (-0.55, -1.25, -1.0):
        t = torch.full((1, 1 if repeated else T), x, device="cuda")
        arrays.append(t.expand(1, T))
    lp, old, ref = arrays
    f = [float(a[0, 0]) for a in arrays]
    d, k = f[0] - f[1], f[2] - f[0]
    ws, out = bg.alloc_train_workspace(), torch.empty(6, device="cuda")
    A = torch.full((1,), -1.0, device="cuda")               # ratios above 1: not clipped
    bg.policy_loss(lp, old, A, out, None, ws, logp_ref=ref, beta=0.1, ratio="sequence", norm="rows")
    got = out.double().cpu().numpy()
    assert got[3] == 0 and got[4] == 0
    assert abs(got[5] / np.exp(d) - 1) <= (48 + 24 * d) * E
    assert abs(got[1] / np.exp(d) - 1) <= (56 + 24 * d) * E
    assert abs(got[2] / (np.expm1(k) - k) - 1) <= (56 + 4 * abs(k)) * E
    # a pair of it and a short row
    short = torch.full((1, 8), -0.5, device="cuda")
    out5, h = torch.empty(5, device="cuda"), torch.empty(1, device="cuda")
    bg.preference_loss(lp, short, out5, None, None, ws, ref_chosen=old, ref_rejected=torch.zeros_like(short),
                       beta=1.0, margins=h)
    got = out5.double().cpu().numpy()
    assert abs(got[3] / (T * d) - 1) <= 48 * E and abs(float(h) / (T * d + 4) - 1) <= 48 * E
    assert got[4] == -4
    assert bg.get_device_error(ws) == (0, 0)


@pytest.mark.parametrize("K,T", [(1 << 26, 8), (1 << 23, 300)])
def test_very_many_pairs(bg, K, T):
    import torch
    beta = 0.1
    c, r = _row(np.full(T, -0.45), K), _row(np.full(T, -0.5 - 0.2 / T), K)
    ws, out = bg.alloc_train_workspace(), torch.empty(5, device="cuda")
    bg.preference_loss(c, r, out, None, None, ws, beta=beta)
    got = out.double().cpu().numpy()
    b = float(np.float32(beta))
    sc, sr = T * float(c[0, 0]), T * float(r[0, 0])
    h = b * (sc - sr)
    cancel = 30 * E * b * (abs(sc) + abs(sr))
    assert got[1] == 1
    assert abs(got[0] - np.logaddexp(0, -h)) <= 48 * E * np.logaddexp(0, -h) + cancel
    assert abs(got[2] - h) <= 48 * E * h + cancel
    assert abs(got[3] / (b * sc) - 1) <= 48 * E and abs(got[4] / (b * sr) - 1) <= 48 * E
    assert bg.get_device_error(ws) == (0, 0)
