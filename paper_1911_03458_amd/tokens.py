"""The operators along a sequence of tokens (include/merit_tokens.h): short causal convolution, selective state space
scan, group norm with an activation.  `binding` re-exports everything here.

Argument marshalling only, as in `binding`: torch device tensors in, new tensors out, on the current stream.  An operand may
be a slice or a broadcast view as long as a token's channels lie side by side (a projection's half, an expanded batch);
parameters and states are contiguous.  Scratch memory comes from PyTorch's allocator, in the stream of the call.  Calls
go through the native module where it can be used and through ctypes otherwise.
"""
from __future__ import annotations

import ctypes

MERIT_BF16 = 3
MERIT_ACT_NONE, MERIT_ACT_RELU, MERIT_ACT_SILU = range(3)
MERIT_PASS_FORWARD, MERIT_PASS_BACKWARD, MERIT_PASS_STEP = range(3)
MERIT_CONV_MAX_TAPS = 8
MERIT_SCAN_MAX_STATES = 64
MERIT_SCAN_TILE = 16

# type of an operand: the plan's, the plan's or fp32, fp32, int32
_T, _P, _F32, _I32 = range(4)


class merit_view(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64 * 2), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


def _binding():
    from . import binding
    return binding


_ENTRIES = ("merit_group_norm", "merit_group_norm_backward", "merit_causal_conv", "merit_causal_conv_backward",
            "merit_causal_conv_step", "merit_scan", "merit_scan_backward", "merit_scan_step")


def _declare(L):
    """Argument types of the entry points (binding.lib() calls this once)."""
    P, i64, c_int, PP = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.POINTER(ctypes.c_void_p)
    L.merit_plan_group_norm.argtypes = [c_int] + [i64] * 4 + [ctypes.c_double, c_int, PP]
    L.merit_plan_causal_conv.argtypes = [c_int] + [i64] * 4 + [c_int, PP]
    L.merit_plan_scan.argtypes = [c_int] + [i64] * 5 + [c_int, PP]
    L.merit_token_plan_destroy.argtypes = [P]
    L.merit_token_plan_workspace.argtypes = [P, c_int, ctypes.POINTER(i64)]
    L.merit_token_plan_kernel.argtypes = [P, c_int, ctypes.POINTER(ctypes.c_char_p)]
    for name in _ENTRIES:
        getattr(L, name).argtypes = [P, P, P, i64, P]
    for name in _ENTRIES + ("merit_plan_group_norm", "merit_plan_causal_conv", "merit_plan_scan", "merit_token_plan_destroy",
                            "merit_token_plan_workspace", "merit_token_plan_kernel"):
        getattr(L, name).restype = c_int


class TokenPlan:
    """Owner of one merit_token_plan handle, and the operands of its calls.

    operands: {entry point: (pass, [(name, type, shape, leading strides, 'in' | 'opt' | 'out' | 'out?'), ...])} in the
    order of the call's argument struct."""

    def __init__(self, handle, dtype, operands):
        self._h, self.dtype, self._operands = handle, dtype, operands
        self._specs, self._bytes = {}, {}

    @property
    def handle(self):
        if not self._h:
            raise ValueError("plan already destroyed")
        return self._h

    def destroy(self):
        if self._h:
            self._specs = {}
            _binding().lib().merit_token_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def workspace(self, which: int) -> int:
        """Bytes of scratch memory that a pass needs."""
        if which not in self._bytes:
            b, n = _binding(), ctypes.c_int64(0)
            b._check(b.lib().merit_token_plan_workspace(self.handle, which, ctypes.byref(n)), "merit_token_plan_workspace")
            self._bytes[which] = int(n.value)
        return self._bytes[which]

    def kernel(self, which: int = MERIT_PASS_FORWARD) -> str:
        b, s = _binding(), ctypes.c_char_p()
        b._check(b.lib().merit_token_plan_kernel(self.handle, which, ctypes.byref(s)), "merit_token_plan_kernel")
        return s.value.decode()

    def torch_dtype(self):
        import torch
        return {MERIT_BF16: torch.bfloat16, 1: torch.float16, 2: torch.float32}[self.dtype]

    def operands(self, where):
        try:
            return self._operands[where]
        except KeyError:
            raise _binding().MeritError(2, where) from None      # a plan of another operator

    def _spec(self, where):
        """What the native call takes in place of this object; None without the module."""
        b = _binding()
        which, ops = self.operands(where)
        spec = None
        if b._native() and where in b._calls.TOKEN_OPS:
            spec = b._calls.token_spec(b._calls.TOKEN_OPS[where], self.handle.value, self.dtype, self.workspace(which),
                                       tuple((kind, shape, lead, "in opt out out?".split().index(role))
                                             for _, kind, shape, lead, role in ops))
        self._specs[where] = spec
        return spec


def _code(t):
    import torch
    return {torch.float16: 1, torch.float32: 2, torch.bfloat16: MERIT_BF16}.get(t.dtype, -1)


def _view(plan, op, t, device):
    """One operand as a merit_view, or the reason why it cannot be one."""
    import torch
    name, kind, shape, lead, _ = op
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a device tensor")
    want = {_T: (plan.torch_dtype(),), _P: (plan.torch_dtype(), torch.float32), _F32: (torch.float32,), _I32: (torch.int32,)}[kind]
    if t.dtype not in want:
        raise TypeError(f"{name}: expected {' or '.join(str(d) for d in want)}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, other operands are on {device}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    dense = 1
    for i in range(len(shape) - 1, lead - 1, -1):
        if shape[i] > 1 and t.stride(i) != dense and t.numel():
            raise ValueError(f"{name}: dimension {i} must be dense (stride {dense}, got {t.stride(i)})")
        dense *= shape[i]
    strides = [t.stride(i) if i < lead else 0 for i in range(2)]
    return merit_view(t.data_ptr() or None, (ctypes.c_int64 * 2)(*strides), max(_code(t), 0), 0)


def _general(plan, where, args, want, stream):
    """The call through ctypes.  args: the operands in order, None where absent; want: for each output left None
    whether to make it."""
    import torch
    b = _binding()
    which, ops = plan.operands(where)
    for (name, _, _, _, role), t in zip(ops, args):
        if role == "in" and t is None:
            raise TypeError(f"{name}: expected a device tensor")
    first = next(t for t in args if t is not None)
    if not isinstance(first, torch.Tensor) or not first.is_cuda:
        raise TypeError(f"{ops[0][0]}: expected a device tensor")
    device = first.device
    with torch.cuda.device(device):
        if stream is None:
            stream = torch.cuda.current_stream()
        elif isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
        with torch.cuda.stream(stream):
            args, made, types = list(args), [], {_T: plan.torch_dtype(), _F32: torch.float32}
            views = (merit_view * len(ops))()
            for i, op in enumerate(ops):
                if args[i] is None and op[4] in ("out", "out?") and want[i]:
                    args[i] = torch.empty(op[2], dtype=types[op[1]], device=device)
                if op[4] in ("out", "out?"):
                    made.append(args[i])
                if args[i] is not None:
                    views[i] = _view(plan, op, args[i], device)
            n = plan.workspace(which)
            scratch = torch.empty(n, dtype=torch.uint8, device=device) if n else None
            b._check(getattr(b.lib(), where)(plan.handle, ctypes.byref(views), scratch.data_ptr() if n else None, n,
                                             ctypes.c_void_p(stream.cuda_stream)), where)
    return tuple(made)


def _call(plan, where, args, want, stream):
    """The outputs, in order (None: neither given nor wanted).  want: bit i for operand i."""
    if stream is None:
        spec = plan._specs.get(where, 0)
        if spec == 0:
            spec = plan._spec(where)
        if spec is not None and plan._h:
            r = _binding()._calls.token_call(spec, want, *args)
            if r.__class__ is tuple:
                return r
            if r is not None:
                raise _binding().MeritError(r, where)
    return _general(plan, where, args, [want >> i & 1 for i in range(len(args))], stream)


def _bits(*flags):
    return sum(1 << i for i, f in enumerate(flags) if f)


# --------------------------------------------------------------------------
# group norm
# --------------------------------------------------------------------------
def merit_plan_group_norm(dtype, N, S, C, groups, eps=1e-5, act=MERIT_ACT_NONE) -> TokenPlan:
    """x[N, S, C]: the S positions x C / groups channels of a group share mean and variance (S = 1: a token by itself)."""
    b, h = _binding(), ctypes.c_void_p()
    b._check(b.lib().merit_plan_group_norm(dtype, N, S, C, groups, float(eps), act, ctypes.byref(h)), "merit_plan_group_norm")
    x, stat, c = (N, S, C), (N, groups), (C,)
    return TokenPlan(h, dtype, {
        "merit_group_norm": (0, [("x", _T, x, 2, "in"), ("weight", _P, c, 0, "opt"), ("bias", _P, c, 0, "opt"),
                                 ("y", _T, x, 2, "out"), ("mean", _F32, stat, 0, "out?"), ("rstd", _F32, stat, 0, "out?")]),
        "merit_group_norm_backward": (1, [("dy", _T, x, 2, "in"), ("x", _T, x, 2, "in"), ("mean", _F32, stat, 0, "in"),
                                          ("rstd", _F32, stat, 0, "in"), ("weight", _P, c, 0, "opt"),
                                          ("bias", _P, c, 0, "opt"), ("dx", _T, x, 2, "out"),
                                          ("dweight", _F32, c, 0, "out?"), ("dbias", _F32, c, 0, "out?")])})


def merit_group_norm(plan, x, weight=None, bias=None, *, stats=False, y=None, stream=None):
    """y = act((x - mean) rstd weight + bias); with stats: (y, mean, rstd), which the backward pass takes."""
    r = _call(plan, "merit_group_norm", (x, weight, bias, y, None, None), 0x38 if stats else 0x08, stream)
    return r if stats else r[0]


def merit_group_norm_backward(plan, dy, x, mean, rstd, weight=None, bias=None, *, dx=None, stream=None):
    """(dx, dweight, dbias), the latter two in fp32."""
    return _call(plan, "merit_group_norm_backward", (dy, x, mean, rstd, weight, bias, dx, None, None), 0x1C0, stream)


# --------------------------------------------------------------------------
# short causal convolution
# --------------------------------------------------------------------------
def merit_plan_causal_conv(dtype, B, L, D, K, act=MERIT_ACT_NONE) -> TokenPlan:
    """x[B, L, D], K taps per channel, over the token itself and the K - 1 before it."""
    b, h = _binding(), ctypes.c_void_p()
    b._check(b.lib().merit_plan_causal_conv(dtype, B, L, D, K, act, ctypes.byref(h)), "merit_plan_causal_conv")
    x, kept, w, d, one = (B, L, D), (B, K - 1, D), (D, K), (D,), (B, D)
    return TokenPlan(h, dtype, {
        "merit_causal_conv": (0, [("x", _T, x, 2, "in"), ("weight", _P, w, 0, "in"), ("bias", _P, d, 0, "opt"),
                                  ("init", _T, kept, 2, "opt"), ("lens", _I32, (B,), 0, "opt"), ("y", _T, x, 2, "out"),
                                  ("final", _T, kept, 2, "out?")]),
        "merit_causal_conv_backward": (1, [("dy", _T, x, 2, "in"), ("x", _T, x, 2, "in"), ("weight", _P, w, 0, "in"),
                                           ("bias", _P, d, 0, "opt"), ("init", _T, kept, 2, "opt"),
                                           ("lens", _I32, (B,), 0, "opt"), ("dfinal", _T, kept, 2, "opt"),
                                           ("dx", _T, x, 2, "out"), ("dweight", _F32, w, 0, "out?"),
                                           ("dbias", _F32, d, 0, "out?"), ("dinit", _T, kept, 2, "out?")]),
        "merit_causal_conv_step": (2, [("kept", _T, kept, 2, "in"), ("x", _T, one, 1, "in"), ("weight", _P, w, 0, "in"),
                                       ("bias", _P, d, 0, "opt"), ("y", _T, one, 1, "out"),
                                       ("kept_out", _T, kept, 2, "out")])})


def merit_causal_conv(plan, x, weight, bias=None, *, init=None, lens=None, final=False, y=None, stream=None):
    """act(bias + sum over a of weight[:, a] x[t - (K-1) + a]).  init: the K - 1 tokens before the first (else zeros);
    lens: int32 lengths of the sequences; final (True, or a tensor, which may be init): also the last K - 1 tokens."""
    given = None if isinstance(final, bool) else final
    r = _call(plan, "merit_causal_conv", (x, weight, bias, init, lens, y, given), 0x60 if final is True else 0x20, stream)
    return r[0] if final is False else r


def merit_causal_conv_backward(plan, dy, x, weight, bias=None, *, init=None, lens=None, dfinal=None, dinit=False, dx=None,
                               stream=None):
    """(dx, dweight, dbias), the latter two in fp32; with dinit: and the gradient of init."""
    r = _call(plan, "merit_causal_conv_backward", (dy, x, weight, bias, init, lens, dfinal, dx, None, None, None),
              0x780 if dinit else 0x380, stream)
    return r if dinit else r[:3]


def merit_causal_conv_step(plan, kept, x, weight, bias=None, *, kept_out=None, y=None, stream=None):
    """One token x[B, D] more, kept[B, K-1, D] before it: (y[B, D], the tokens kept now); kept_out may be kept."""
    return _call(plan, "merit_causal_conv_step", (kept, x, weight, bias, y, kept_out), 0x30, stream)


# --------------------------------------------------------------------------
# selective state space scan
# --------------------------------------------------------------------------
def merit_plan_scan(dtype, B, L, D, N, groups=1, softplus=True) -> TokenPlan:
    """x[B, L, D] with N states a channel; B, C [B, L, groups, N]."""
    b, h = _binding(), ctypes.c_void_p()
    b._check(b.lib().merit_plan_scan(dtype, B, L, D, N, groups, int(bool(softplus)), ctypes.byref(h)), "merit_plan_scan")
    x, bc, A, d, state = (B, L, D), (B, L, groups, N), (D, N), (D,), (B, D, N)
    kept = (B, -(-L // MERIT_SCAN_TILE), D, N)
    one, bc1 = (B, D), (B, groups, N)
    return TokenPlan(h, dtype, {
        "merit_scan": (0, [("x", _T, x, 2, "in"), ("dt", _T, x, 2, "in"), ("A", _F32, A, 0, "in"), ("B", _T, bc, 2, "in"),
                           ("C", _T, bc, 2, "in"), ("skip", _F32, d, 0, "opt"), ("z", _T, x, 2, "opt"),
                           ("dt_bias", _F32, d, 0, "opt"), ("h0", _F32, state, 0, "opt"), ("lens", _I32, (B,), 0, "opt"),
                           ("y", _T, x, 2, "out"), ("h_last", _F32, state, 0, "out?"), ("states", _F32, kept, 0, "out?")]),
        "merit_scan_backward": (1, [("dy", _T, x, 2, "in"), ("x", _T, x, 2, "in"), ("dt", _T, x, 2, "in"),
                                    ("A", _F32, A, 0, "in"), ("B", _T, bc, 2, "in"), ("C", _T, bc, 2, "in"),
                                    ("states", _F32, kept, 0, "in"), ("skip", _F32, d, 0, "opt"), ("z", _T, x, 2, "opt"),
                                    ("dt_bias", _F32, d, 0, "opt"), ("lens", _I32, (B,), 0, "opt"),
                                    ("dh_last", _F32, state, 0, "opt"), ("dx", _T, x, 2, "out"), ("ddt", _T, x, 2, "out"),
                                    ("dB", _T, bc, 2, "out"), ("dC", _T, bc, 2, "out"), ("dz", _T, x, 2, "out?"),
                                    ("dA", _F32, A, 0, "out"), ("dskip", _F32, d, 0, "out?"),
                                    ("ddt_bias", _F32, d, 0, "out?"), ("dh0", _F32, state, 0, "out?")]),
        "merit_scan_step": (2, [("h", _F32, state, 0, "in"), ("x", _T, one, 1, "in"), ("dt", _T, one, 1, "in"),
                                ("A", _F32, A, 0, "in"), ("B", _T, bc1, 1, "in"), ("C", _T, bc1, 1, "in"),
                                ("skip", _F32, d, 0, "opt"), ("z", _T, one, 1, "opt"), ("dt_bias", _F32, d, 0, "opt"),
                                ("y", _T, one, 1, "out"), ("h_out", _F32, state, 0, "out")])})


def merit_scan(plan, x, dt, A, B, C, *, skip=None, z=None, dt_bias=None, h0=None, lens=None, final=False, states=False,
               y=None, stream=None):
    """y[, the state behind the last token][, the kept states, which the backward pass takes]."""
    r = _call(plan, "merit_scan", (x, dt, A, B, C, skip, z, dt_bias, h0, lens, y, None, None),
              0x400 | bool(final) << 11 | bool(states) << 12, stream)
    return r[0] if not (final or states) else tuple(t for t, on in zip(r, (True, final, states)) if on)


def merit_scan_backward(plan, dy, x, dt, A, B, C, states, *, skip=None, z=None, dt_bias=None, lens=None, dh_last=None,
                        dh0=False, stream=None):
    """{'dx', 'ddt', 'dB', 'dC', 'dz', 'dA', 'dskip', 'ddt_bias', 'dh0'}: None for an operand that is absent; dA, dskip,
    ddt_bias and dh0 in fp32."""
    want = 0x3F << 12 & ~(1 << 16) | (z is not None) << 16 | (skip is not None) << 18 | (dt_bias is not None) << 19 | bool(dh0) << 20
    r = _call(plan, "merit_scan_backward", (dy, x, dt, A, B, C, states, skip, z, dt_bias, lens, dh_last) + (None,) * 9, want, stream)
    return dict(zip(("dx", "ddt", "dB", "dC", "dz", "dA", "dskip", "ddt_bias", "dh0"), r))


def merit_scan_step(plan, h, x, dt, A, B, C, *, skip=None, z=None, dt_bias=None, h_out=None, y=None, stream=None):
    """One token x[B, D] more from the state h[B, D, N]: (y[B, D], the state now); h_out may be h."""
    return _call(plan, "merit_scan_step", (h, x, dt, A, B, C, skip, z, dt_bias, y, h_out), 0x600, stream)
