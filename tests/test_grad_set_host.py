"""A GradSet takes its tensors as they are at each call: with CPU tensors and a stand-in for the
library, what the calls would pass."""
import ctypes

import pytest
import torch


class _Library:
    """Keeps the table of the last call."""

    def _take(self, address, count):
        from paper_2510_11683_gb300 import _lib
        t = (_lib.Grad * count).from_address(address)
        self.table = [(g.data or 0, g.out or 0, g.n, g.type, g.out_type) for g in t]
        return 0

    def bgpo_grad_norm(self, address, count, *_):
        return self._take(address, count)

    def bgpo_grad_clip(self, address, count, *_):
        return self._take(address, count)


@pytest.fixture
def bg(monkeypatch):
    import paper_2510_11683_gb300 as bg
    from paper_2510_11683_gb300 import _lib, train

    def ptr(t, dtype=None, name="tensor", cur=None):
        if t is None:
            return None
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t.data_ptr()

    library = _Library()
    monkeypatch.setattr(train, "_ptr", ptr)
    monkeypatch.setattr(train, "_current_device", lambda: -1)
    monkeypatch.setattr(train, "_stream", lambda stream, cur: None)
    monkeypatch.setattr(_lib, "lib", lambda: library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)     # of a CPU tensor
    bg.library = library
    return bg


def _rows(xs, outs):
    types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return [(x.data_ptr(), o.data_ptr(), x.numel(), types[x.dtype], types[o.dtype])
            for x, o in zip(xs, outs)]


def _calls(bg, gs, norm, ws):
    """What a norm call passed (without outputs) and the table of a clip call."""
    bg.grad_norm(gs, norm, ws)
    first = [(r[0], *r[2:4]) for r in bg.library.table]
    bg.grad_clip(gs, norm, 1.0)
    return first, bg.library.table


@pytest.mark.parametrize("inplace", [False, True])
def test_tensors_whose_memory_was_swapped(bg, inplace):
    xs = [torch.zeros(1000), torch.zeros(77, dtype=torch.bfloat16), torch.zeros(5)]
    outs = xs if inplace else [torch.zeros(x.numel()) for x in xs]
    norm, ws = torch.zeros(1), torch.zeros(8, dtype=torch.uint8)
    gs = bg.grad_set(xs, None if inplace else outs)

    def agree():
        first, table = _calls(bg, gs, norm, ws)
        want = _rows(xs, outs)
        assert table == want and first == [(r[0], *r[2:4]) for r in want]

    agree()
    keep = xs[0].data
    xs[0].data = torch.ones(1000)                       # other memory
    agree()
    xs[1].data = torch.ones(77)                         # of another type
    agree()
    xs[2].set_(keep[:5])                                # within another tensor's
    agree()
    xs[0].resize_(4)                                    # the same memory, fewer elements
    if inplace:
        agree()
        xs[0].resize_(1 << 20)
        agree()
    else:
        with pytest.raises(ValueError, match="4 elements"):
            bg.grad_norm(gs, norm, ws)
        outs[0].resize_(4)
        agree()
        outs[2].data = torch.ones(5, dtype=torch.float16)
        agree()


def test_swapped_memory_is_checked_as_at_first(bg):
    x = torch.zeros(6, 4)
    gs = bg.grad_set([x])
    x.data = torch.zeros(4, 6).T
    with pytest.raises(ValueError, match="contiguous"):
        bg.grad_norm(gs, torch.zeros(1), torch.zeros(8, dtype=torch.uint8))
    x.data = torch.zeros(4, 6, dtype=torch.float64)
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        bg.grad_clip(gs, torch.zeros(1), 1.0)
    y = torch.ones(24)
    x.data = y                                          # and usable again
    bg.grad_clip(gs, torch.zeros(1), 1.0)
    assert bg.library.table == _rows([y], [y])


def test_memory_in_the_table_stays_allocated(bg):
    # the old memory goes to nobody else before the set has seen the change
    x = torch.zeros(1 << 16)
    gs = bg.grad_set([x])
    old = x.data_ptr()
    x.data = torch.zeros(8)
    others = [torch.empty(1 << 16) for _ in range(64)]
    assert old not in [o.data_ptr() for o in others]
    assert ctypes.c_float.from_address(old).value == 0
    assert gs.count == 1
