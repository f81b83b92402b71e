"""Binding of the token-level policy step (include/bgpo_train.h).

    token_logp_fwd(prob, X, W, Y, ws, logp, mask=m)            # log p of the response tokens
    policy_loss(logp, logp_old, A, out, dlogp, tws, ...)       # or preference_loss(...)
    token_logp_bwd(prob, W, dlogp, ws, dX, dW)                 # bf16 gradients
    grad_norm(grads, norm, tws); grad_clip(grads, norm, max_norm, tws)

As in the rest of the binding the caller owns every buffer and outputs are written in
place. The losses take strided views: any [N, T] tensor, transposed or sliced, e.g.
``ell.T`` for l stored as [n_t, B]."""
import ctypes

from . import _lib
from . import _current_device, _ptr, _refuse, _stream, _torch

RATIOS = {"token": 0, "sequence": 1}                  # BGPO_RATIO_*
NORMS = {"rows": 0, "tokens": 1, "sum": 2}            # BGPO_NORM_*
PREFERENCES = {"sigmoid": 0, "hinge": 1, "ipo": 2}    # BGPO_PREF_*


def token_logp_fwd(prob, X, W, Y, ws, logp, mask=None, stream=None):
    """logp (float32 [B, R]) = log-probabilities of the targets Y [B, R] at the selected
    response positions, 0 elsewhere: those of mask (bool or uint8 [B, R]; None: all) within
    the problem's resp_len. ws: alloc_workspace(prob), without pair_dw."""
    torch, cur = _torch(), _current_device()
    if isinstance(mask, torch.Tensor) and mask.dtype is torch.bool:
        mask = mask.view(torch.uint8)
    n = prob.B * prob.R
    st = _lib.lib().bgpo_token_logp_fwd(
        ctypes.byref(prob), _count(mask, n, torch.uint8, "mask", cur),
        _count(X, prob.B * (prob.P + prob.R) * prob.H, torch.bfloat16, "X", cur),
        _count(W, prob.V * prob.H, torch.bfloat16, "W", cur),
        _count(Y, n, torch.int32, "Y", cur), _ptr(ws, torch.uint8, "ws", cur), ws.numel(),
        _count(logp, n, torch.float32, "logp", cur), _stream(stream, cur))
    _lib.check("bgpo_token_logp_fwd", st)


def token_logp_bwd(prob, W, dlogp, ws, dX, dW, stream=None):
    """dX (bfloat16 [B, R, H]) and dW (bfloat16 [V, H]) = gradients of sum dlogp logp over the
    tokens that the preceding token_logp_fwd on ws selected; dX is 0 elsewhere. Both are
    written whole. Beyond 128 tokens dL/dz is rounded to bf16 between the products."""
    torch, cur = _torch(), _current_device()
    n = prob.B * prob.R
    st = _lib.lib().bgpo_token_logp_bwd(
        ctypes.byref(prob), _count(W, prob.V * prob.H, torch.bfloat16, "W", cur),
        _count(dlogp, n, torch.float32, "dlogp", cur), _ptr(ws, torch.uint8, "ws", cur),
        ws.numel(), _count(dX, n * prob.H, torch.bfloat16, "dX", cur),
        _count(dW, prob.V * prob.H, torch.bfloat16, "dW", cur), _stream(stream, cur))
    _lib.check("bgpo_token_logp_bwd", st)


def _count(t, n, dtype, name, cur):
    """Address of a contiguous CUDA tensor of n values of dtype (None for None)."""
    p = _ptr(t, dtype, name, cur)
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} must hold {n} values, got {t.numel()}")
    return p


def alloc_train_workspace(device="cuda"):
    """A cleared uint8 workspace of the losses and of grad_norm / grad_clip."""
    torch = _torch()
    ws = torch.empty(_lib.lib().bgpo_train_workspace_bytes(), dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):
        clear_train_workspace(ws)
    return ws


def clear_train_workspace(ws, stream=None):
    torch, cur = _torch(), _current_device()
    st = _lib.lib().bgpo_train_workspace_clear(_ptr(ws, torch.uint8, "ws", cur), ws.numel(),
                                               _stream(stream, cur))
    _lib.check("bgpo_train_workspace_clear", st)


def _choice(table, value, name):
    code = table.get(value)
    if code is None:
        raise ValueError(f"{name} must be one of {sorted(table)}, got {value!r}")
    return code


def _view(t, shape, dtypes, name, cur):
    """Address and strides of a CUDA tensor of `shape` and of one of `dtypes` on the current
    device; three zeros for None."""
    if t is None:
        return 0, 0, 0
    if isinstance(t, _TENSOR) and t.get_device() == cur >= 0 and t.dtype in dtypes:
        if t.shape == shape:
            return (t.data_ptr(), *t.stride())
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if cur < 0 and isinstance(t, _TENSOR) and t.is_cuda:
        # a tensor that native code made before torch.cuda was initialised
        return _view(t, shape, dtypes, name, _torch().cuda.current_device())
    _refuse(t, dtypes[0], name)


_TENSOR = None       # torch.Tensor and the types of the losses' arrays, after _pair_shape
_F32 = _MASK = ()


def _pair_shape(t, name):
    global _TENSOR, _F32, _MASK
    if _TENSOR is None:
        torch = _torch()
        _F32, _MASK = (torch.float32,), (torch.bool, torch.uint8)
        _TENSOR = torch.Tensor
    if not isinstance(t, _TENSOR):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, got {t.dim()}")
    return t.shape


def _trace(trace):
    return getattr(trace, "handle", trace)


def policy_loss(logp, logp_old, A, out, dlogp, ws, logp_ref=None, mask=None, clip_low=0.2,
                clip_high=0.2, beta=0.0, scale=1.0, ratio="token", norm="rows", trace=None,
                stream=None):
    """Clipped policy loss with a KL term over [N, T] log-probabilities, and its gradient.

    logp, logp_old, logp_ref (optional), dlogp (None: the loss alone): float32 [N, T];
    A: float32 [N] or [N, T]; mask: bool or uint8 [N, T], True where a token counts; out:
    float32 [6] = loss, policy term, KL term, share clipped below and above, mean ratio. What
    stands at masked-out tokens is never used (but has to be readable); their dlogp is 0.
    ratio: "token", or "sequence" (one ratio a row, from its mean log ratio). norm: "rows"
    (mean over rows of their tokens' mean), "tokens" (mean over tokens), "sum"."""
    shape = _pair_shape(logp, "logp")
    ratio, norm = _choice(RATIOS, ratio, "ratio"), _choice(NORMS, norm, "norm")
    cur = _current_device()
    N, T = shape
    if isinstance(A, _TENSOR) and A.dim() == 1:      # one advantage a row
        adv = (*_view(A, shape[:1], _F32, "A", cur), 0)
    else:
        adv = _view(A, shape, _F32, "A", cur)
    a = _lib.POLICY_LOSS_ARGS.pack(
        N, T, ratio, norm, clip_low, clip_high, beta, scale,
        *_view(logp, shape, _F32, "logp", cur), *_view(logp_old, shape, _F32, "logp_old", cur),
        *_view(logp_ref, shape, _F32, "logp_ref", cur), *adv,
        *_view(mask, shape, _MASK, "mask", cur), *_view(dlogp, shape, _F32, "dlogp", cur),
        _sized(out, 6, "out", cur) or 0, _trace(trace) or 0)
    st = _lib.lib().bgpo_policy_loss(a, _ptr(ws, _MASK[1], "ws", cur), ws.numel(),
                                     _stream(stream, cur))
    _lib.check("bgpo_policy_loss", st)


def _sized(t, n, name, cur):
    """Address of a contiguous float32 CUDA tensor of n values."""
    return _count(t, n, _torch().float32, name, cur)


def preference_loss(chosen, rejected, out, d_chosen, d_rejected, ws, ref_chosen=None,
                    ref_rejected=None, mask_chosen=None, mask_rejected=None, beta=0.1, margin=0.0,
                    smoothing=0.0, kind="sigmoid", average=False, scale=1.0, margins=None,
                    trace=None, stream=None):
    """Preference loss on paired log ratios, and its gradient: pair k is row k of `chosen`
    [K, T_chosen] and row k of `rejected` [K, T_rejected] (float32, like their references
    and gradients; masks bool or uint8).

    h = beta (S_chosen - S_rejected) - margin with S a row's sum (average: mean) of
    logp - ref; kind: "sigmoid" (with label smoothing), "hinge", "ipo". out: float32 [5] =
    loss, share of pairs with h > 0, means of h, beta S_chosen, beta S_rejected. margins:
    float32 [K] or None: h. d_chosen and d_rejected may both be None (the loss alone)."""
    c, r = _pair_shape(chosen, "chosen"), _pair_shape(rejected, "rejected")
    if c[0] != r[0]:
        raise ValueError(f"chosen and rejected must have equally many rows, got {c[0]} and {r[0]}")
    kind = _choice(PREFERENCES, kind, "kind")
    cur = _current_device()
    a = _lib.PREFERENCE_LOSS_ARGS.pack(
        c[0], c[1], r[1], kind, bool(average), beta, margin, smoothing, scale,
        *_view(chosen, c, _F32, "chosen", cur), *_view(ref_chosen, c, _F32, "ref_chosen", cur),
        *_view(mask_chosen, c, _MASK, "mask_chosen", cur),
        *_view(d_chosen, c, _F32, "d_chosen", cur),
        *_view(rejected, r, _F32, "rejected", cur),
        *_view(ref_rejected, r, _F32, "ref_rejected", cur),
        *_view(mask_rejected, r, _MASK, "mask_rejected", cur),
        *_view(d_rejected, r, _F32, "d_rejected", cur),
        _sized(margins, c[0], "margins", cur) or 0, _sized(out, 5, "out", cur) or 0,
        _trace(trace) or 0)
    st = _lib.lib().bgpo_preference_loss(a, _ptr(ws, _MASK[1], "ws", cur), ws.numel(),
                                         _stream(stream, cur))
    _lib.check("bgpo_preference_loss", st)


class GradSet:
    """A list of gradients for grad_norm and grad_clip: what a program keeps while its gradient
    tensors live (it holds references to them). Each call takes the tensors as they then are:
    one that was given other memory (``x.data = y``, ``set_``, ``resize_``) is laid out anew.
    A tensor object that replaces another, such as a ``.grad`` that is allocated again, needs a
    new set."""

    def __init__(self, grads, into, cur):
        self.grads, self.into = grads, into
        self._lay_out(cur)

    def _lay_out(self, cur):
        grads, into = self.grads, self.into
        for name, ts in (("gradient", grads), ("output", into)):
            for t in ts:
                _ptr(t, None, name, cur)
        for x, o in zip(grads, into):
            if x.numel() != o.numel():
                raise ValueError(f"an output must have its gradient's {x.numel()} elements, "
                                 f"got {o.numel()}")
        table = (_lib.Grad * max(len(grads), 1))()
        for i, (x, o) in enumerate(zip(grads, into)):
            table[i] = _lib.Grad(x.data_ptr() or None, o.data_ptr() or None, x.numel(),
                                 _grad_type(x, "gradient"), _grad_type(o, "output"))
        self.count = len(grads)
        self.device = grads[0].get_device() if grads else cur
        self.table = table
        self.address = ctypes.addressof(self.table)
        # the memory in the table stays allocated, so that its addresses name nothing else
        self._memory = [t.detach() for ts in (grads, into) for t in ts]
        self._places = _places(grads), _places(into)

    def follow(self, cur, outputs):
        """Lays the set out anew where a gradient (or output) lies elsewhere than it did. (Asking
        takes 0.15 us a tensor: 8 us a call for 60 gradients, as much again for outputs.)"""
        if (_places(self.grads) != self._places[0]
                or outputs and self.into is not self.grads
                and _places(self.into) != self._places[1]):
            self._lay_out(cur)


def _places(ts):
    Tensor = _torch().Tensor
    return list(map(Tensor.data_ptr, ts)), list(map(Tensor.numel, ts))


def _grad_type(t, name):
    torch = _torch()
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def grad_set(grads, into=None):
    """GradSet over contiguous CUDA tensors (float32, bfloat16, float16; of any sizes, zero
    included), each listed once. into: a tensor of the same size for each clipped gradient, of
    any of the types (None: the gradients are clipped in place)."""
    torch, cur = _torch(), _current_device()
    grads = list(grads)
    into = grads if into is None else list(into)
    if len(into) != len(grads):
        raise ValueError(f"into must hold {len(grads)} tensors, got {len(into)}")
    return GradSet(grads, into, cur)


def _check_set(gs, cur, outputs):
    if not isinstance(gs, GradSet):
        raise TypeError("grads must be a GradSet (grad_set)")
    gs.follow(cur, outputs)
    if gs.count and gs.device != (cur if cur >= 0 else _torch().cuda.current_device()):
        raise ValueError(f"the gradients are on cuda:{gs.device}, which is not the current device")


def grad_norm(grads, norm, ws, trace=None, stream=None):
    """norm (float32 [1]) = the Euclidean norm of all gradients of a GradSet. A norm that is
    not finite is also reported in the workspace's error word."""
    torch, cur = _torch(), _current_device()
    _check_set(grads, cur, False)
    st = _lib.lib().bgpo_grad_norm(grads.address, grads.count, _sized(norm, 1, "norm", cur),
                                   _trace(trace), _ptr(ws, torch.uint8, "ws", cur), ws.numel(),
                                   _stream(stream, cur))
    _lib.check("bgpo_grad_norm", st)


def grad_clip(grads, norm, max_norm, ws=None, trace=None, stream=None):
    """Every output of a GradSet = min(1, max_norm / (norm + 1e-6)) times its gradient; norm:
    float32 [1] on the device (grad_norm's). A norm that is not finite scales by 1 and is
    reported in the error word of ws, where one is given."""
    torch, cur = _torch(), _current_device()
    _check_set(grads, cur, True)
    st = _lib.lib().bgpo_grad_clip(grads.address, grads.count, _sized(norm, 1, "norm", cur),
                                   max_norm, _trace(trace), _ptr(ws, torch.uint8, "ws", cur),
                                   0 if ws is None else ws.numel(), _stream(stream, cur))
    _lib.check("bgpo_grad_clip", st)
