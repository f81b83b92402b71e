"""Gradients whose memory was swapped between the calls on a GradSet: norm and clipping are of
what the tensors then hold."""
import pytest

from tests.harness import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bg():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    ensure_built()
    import paper_2510_11683_gb300 as bg
    return bg


@pytest.mark.parametrize("inplace", [False, True])
def test_norm_and_clip_follow_their_tensors(bg, inplace):
    import torch
    xs = [torch.full((n,), 1.0, device="cuda") for n in (900, 16, 5000)]
    outs = None if inplace else [torch.empty_like(x) for x in xs]
    norm, ws = torch.empty(1, device="cuda"), bg.alloc_train_workspace()
    gs = bg.grad_set(xs, outs)

    def check(want):
        # (sums of few small squares: exact)
        kept = [x.clone() for x in xs]
        bg.grad_norm(gs, norm, ws)
        assert float(norm) == want
        bg.grad_clip(gs, norm, 1e9)
        for x, o, k in zip(xs, outs or xs, kept):
            assert torch.equal(o.float(), k.float()) and torch.equal(x, k)
        bg.grad_clip(gs, norm, want / 2, ws)
        for o, k in zip(outs or xs, kept):
            assert torch.allclose(o.float(), k.float() / 2, rtol=2.0 ** -7, atol=0)

    xs[1].zero_()
    xs[2].zero_()
    check(30.0)
    # other memory, of another type
    xs[0].data = torch.zeros(900, device="cuda")
    xs[0].data[:1] = 3.0
    y = torch.zeros(5000, dtype=torch.bfloat16, device="cuda")
    y[4999] = 4.0
    xs[2].data = y
    if not inplace:
        outs[1].data = torch.empty(16, dtype=torch.float16, device="cuda")
    check(5.0)
    # the old memory may go to other tensors
    xs[0].data = torch.zeros(900, device="cuda")
    xs[1].data = torch.full((16,), 2.0, device="cuda")
    xs[2].data = torch.zeros(5000, dtype=torch.bfloat16, device="cuda")
    junk = [torch.full((900,), 7.0, device="cuda") for _ in range(8)]
    check(8.0)
    assert all(torch.equal(j, torch.full_like(j, 7.0)) for j in junk)
    assert bg.get_device_error(ws) == (0, 0)
