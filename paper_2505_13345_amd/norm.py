"""The norms around a block with its gate, residual scale and residual sum: device buffers and calls, forward and backward.

    out = x_scale * x + y_scale * gate * N_post(y);   h = N_pre(out)

``y`` is the block's output (``OccultLayer.forward``'s), ``x`` the residual stream in front of it, ``h`` the input of
the next block.  Memory plumbing only, like layer.py: buffers are allocated once (the backward pass's [T, d] and its workspace on
first use), a call is one call into the C library on the current stream, and nothing here synchronises or computes.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B

_NORMS = {None: B.OCCULT_NORM_NONE, "rms": B.OCCULT_NORM_RMS, "layer": B.OCCULT_NORM_LAYER}
_GATES = {None: B.OCCULT_GATE_NONE, "channel": B.OCCULT_GATE_CHANNEL, "token": B.OCCULT_GATE_TOKEN, "element": B.OCCULT_GATE_ELEMENT}


class BlockNorm:
    """post, pre: "rms", "layer" or None (no norm there); gate: "channel" ([d]), "token" ([T]), "element" ([T, d]) or None.
    Parameters are passed to the calls: weights and biases [d] and the gate in the layer's type, each may be left out
    (factor 1, summand 0; a gate that the kind asks for has to be there).  One object may serve several blocks, threads and
    streams with forward() calls that bring their own out and h; backward() calls share its buffers and workspace, and so
    have to be in one order: one stream, or streams and graphs that wait for each other."""

    def __init__(self, T, d, dtype="bf16", post=None, pre="rms", gate=None, x_scale=1.0, y_scale=1.0, post_eps=1e-6, pre_eps=1e-6,
                 weight_offset=0.0, device="cuda:0"):
        self._lib = B.load_library()          # fail early and loudly if the HIP library is missing
        for name, kind, known in (("post", post, _NORMS), ("pre", pre, _NORMS), ("gate", gate, _GATES)):
            if kind not in known:
                raise ValueError(f"occult: {name} is {kind!r}, known are {sorted(k for k in known if k)} and None")
        self.T, self.d = T, d
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.cfg = B.make_cfg(T, d, d, 1, 0, 1, 1, dtype)
        self.post, self.pre, self.gate = post, pre, gate
        self._fixed = (_NORMS[post], _NORMS[pre], _GATES[gate], x_scale, y_scale, post_eps, pre_eps, weight_offset)
        self._gate_len = {None: 0, "channel": d, "token": T, "element": T * d}[gate]
        B.occult_block_norm_backward_ws_bytes(self.cfg, B.make_block_norm(_NORMS[post], _NORMS[pre], 0, *self._fixed[3:]))  # checks both
        self._desc = bytes(B.make_block_norm(*self._fixed))   # what every call's own description starts from
        self.out = torch.zeros((T, d), dtype=self.tdtype, device=self.device)
        self.h = torch.zeros((T, d), dtype=self.tdtype, device=self.device)
        self.ws = self.dx = self.dy = self.dgate = None
        # Sums over tokens, which a backward call may add to: zeros from here on, as a fill inside that call would become part of a
        # graph that is captured from it and clear them with every replay.
        self.dpost_weight, self.dpost_bias, self.dpre_weight, self.dpre_bias, channel = torch.zeros(
            (5, d), dtype=torch.float32, device=self.device)
        if gate == "channel":
            self.dgate = channel

    def _at(self, t, name, numel):
        """Device address of a caller's tensor (None passes through), with binding's checks of it in one place: on small batches
        the host's work is as long as the GPU's."""
        if t is None:
            return None
        if t.get_device() != self.device.index:
            raise ValueError(f"occult: {name} is on {t.device}, the buffers are on {self.device}")
        if t.dtype != self.tdtype or t.numel() < numel or not t.is_contiguous():
            B.expect(t, name, self.tdtype, numel)   # says what is wrong
            B._ptr(t)
        return t.data_ptr()

    def _describe(self, gate, post_weight, post_bias, pre_weight, pre_bias):
        if torch.cuda.current_device() != self.device.index:   # the library launches on the current device's stream
            raise ValueError(f"occult: the current device is cuda:{torch.cuda.current_device()}, the buffers are on {self.device}")
        # of this call alone: the library reads it while other threads may call this object
        desc, d = B.occult_block_norm_t.from_buffer_copy(self._desc), self.d
        desc.post_weight = self._at(post_weight, "post_weight", d)
        desc.post_bias = self._at(post_bias, "post_bias", d)
        desc.pre_weight = self._at(pre_weight, "pre_weight", d)
        desc.pre_bias = self._at(pre_bias, "pre_bias", d)
        desc.gate = self._at(gate, "gate", self._gate_len)
        return desc

    def forward(self, x, y=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None, out=None, h=None):
        """x, y [T, d] -> out [T, d], h [T, d] (None without a pre norm); without y the pre norm alone: out is x.
        Results go to this object's buffers unless others are given (out may be x, the residual stream in place)."""
        desc = self._describe(gate, post_weight, post_bias, pre_weight, pre_bias)
        n = self.T * self.d
        out = None if y is None else self.out if out is None else out
        h = None if self.pre is None else self.h if h is None else h
        B._check(self._lib.occult_block_norm(ctypes.byref(self.cfg), ctypes.byref(desc), self._at(x, "x", n), self._at(y, "y", n),
                                             self._at(out, "out", n), self._at(h, "h", n),
                                             B._stream_of(self.device.index)))
        return (x if y is None else out), h

    def _buf(self, name, shape, dtype):
        """A buffer that every call with it overwrites, allocated on first use."""
        t = getattr(self, name)
        if t is None:
            t = torch.empty(shape, dtype=dtype, device=self.device)
            setattr(self, name, t)
        return t

    def backward(self, out, dout, dh=None, y=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None,
                 accumulate=False, want_dy=None):
        """out and y as the forward pass had them, dout the gradient of out from where it is read beside h (None = none), dh that
        of h.  Without y and want_dy: the pre norm alone (out = x; x_scale has no part in its dx).  Where there was a y, with
        neither post norm nor gate, it may still be left out: want_dy then says whether dy is wanted -> dict of dx, dy, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias: each None where there is
        nothing of that name; sums over tokens are f32 (accumulate: added to what the last call left)."""
        desc = self._describe(gate, post_weight, post_bias, pre_weight, pre_bias)
        T, d, f32 = self.T, self.d, torch.float32
        n = T * d
        rows = [self._at(t, name, n) for t, name in ((y, "y"), (out, "out"), (dout, "dout"), (dh, "dh"))]
        if y is None and want_dy is not None and not want_dy:
            rows[0] = rows[1] or rows[2]   # there was a y, which the call need not read
        want_dy = y is not None if want_dy is None else want_dy
        g = {"dx": self._buf("dx", (T, d), self.tdtype), "dy": self._buf("dy", (T, d), self.tdtype) if want_dy else None,
             "dpost_weight": self.dpost_weight if post_weight is not None and want_dy else None,
             "dpost_bias": self.dpost_bias if post_bias is not None and want_dy else None,
             "dpre_weight": self.dpre_weight if pre_weight is not None else None,
             "dpre_bias": self.dpre_bias if pre_bias is not None else None, "dgate": None}
        if self.gate is not None and want_dy:
            g["dgate"] = self._buf("dgate", (T,) if self.gate == "token" else (T, d), f32 if self.gate == "token" else self.tdtype)
        if self.ws is None:   # enough for every parameter
            full = B.make_block_norm(*self._fixed, *[self.h if k else None for k in (self.post, self.post, self.pre, self.pre, self.gate)])
            self.ws = torch.empty(max(4, B.occult_block_norm_backward_ws_bytes(self.cfg, full) // 4), dtype=f32, device=self.device)
            self._ws_bytes = self.ws.numel() * 4
        at = {name: None if t is None else t.data_ptr() for name, t in g.items()}   # this object's own buffers
        grads = B.occult_block_norm_grads_t(at["dpost_weight"], at["dpost_bias"], at["dpre_weight"], at["dpre_bias"], at["dgate"])
        B._check(self._lib.occult_block_norm_backward(
            ctypes.byref(self.cfg), ctypes.byref(desc), *rows, at["dx"], at["dy"], ctypes.byref(grads), int(bool(accumulate)),
            self.ws.data_ptr(), self._ws_bytes, B._stream_of(self.device.index)))
        return g
