"""The norms around a block with its gate, residual scale and residual sum: device buffers and calls, forward and backward.

    out = x_scale * x + y_scale * gate * N_post(y);   h = N_pre(out)

``y`` is the block's output (``OccultLayer.forward``'s), ``x`` the residual stream in front of it, ``h`` the input of
the next block.  Memory plumbing only, like layer.py: buffers are allocated once (the backward pass's on first use), a
call is one call into the C library on the current stream, and nothing here synchronises or computes.
"""
from __future__ import annotations

import torch

from . import binding as B

_NORMS = {None: B.OCCULT_NORM_NONE, "rms": B.OCCULT_NORM_RMS, "layer": B.OCCULT_NORM_LAYER}
_GATES = {None: B.OCCULT_GATE_NONE, "channel": B.OCCULT_GATE_CHANNEL, "token": B.OCCULT_GATE_TOKEN, "element": B.OCCULT_GATE_ELEMENT}


class BlockNorm:
    """post, pre: "rms", "layer" or None (no norm there); gate: "channel" ([d]), "token" ([T]), "element" ([T, d]) or None.
    Parameters are passed to the calls: weights and biases [d] and the gate in the layer's type, each may be left out
    (factor 1, summand 0)."""

    def __init__(self, T, d, dtype="bf16", post=None, pre="rms", gate=None, x_scale=1.0, y_scale=1.0, post_eps=1e-6, pre_eps=1e-6,
                 weight_offset=0.0, device="cuda:0"):
        B.load_library()          # fail early and loudly if the HIP library is missing
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
        self.out = torch.zeros((T, d), dtype=self.tdtype, device=self.device)
        self.h = torch.zeros((T, d), dtype=self.tdtype, device=self.device)

    def _expect(self, t, name, numel):
        if t is not None and t.device != self.device:
            raise ValueError(f"occult: {name} is on {t.device}, the buffers are on {self.device}")
        return B.expect(t, name, self.tdtype, numel)

    def _rows(self, t, name):
        return self._expect(t, name, self.T * self.d)

    def _on_device(self):
        """The library launches on the current device's stream."""
        if torch.cuda.current_device() != self.device.index:
            raise ValueError(f"occult: the current device is cuda:{torch.cuda.current_device()}, the buffers are on {self.device}")

    def _norm(self, gate, post_weight, post_bias, pre_weight, pre_bias):
        self._on_device()
        for t, name in ((post_weight, "post_weight"), (post_bias, "post_bias"), (pre_weight, "pre_weight"), (pre_bias, "pre_bias")):
            self._expect(t, name, self.d)
        self._expect(gate, "gate", self._gate_len)
        return B.make_block_norm(*self._fixed, post_weight, post_bias, pre_weight, pre_bias, gate)

    def forward(self, x, y=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None, out=None, h=None):
        """x, y [T, d] -> out [T, d], h [T, d] (None without a pre norm); without y the pre norm alone: out is x.
        Results go to this object's buffers unless others are given (out may be x, the residual stream in place)."""
        norm = self._norm(gate, post_weight, post_bias, pre_weight, pre_bias)
        out = None if y is None else self.out if out is None else out
        h = None if self.pre is None else self.h if h is None else h
        for t, name in ((x, "x"), (y, "y"), (out, "out"), (h, "h")):
            self._rows(t, name)
        B.occult_block_norm(self.cfg, norm, x, y, out, h)
        return (x if y is None else out), h

    def _buf(self, name, shape, dtype):
        if getattr(self, name, None) is None:
            setattr(self, name, torch.zeros(shape, dtype=dtype, device=self.device))
        return getattr(self, name)

    def backward(self, out, dout, dh=None, y=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None,
                 accumulate=False, want_dy=None):
        """out and y as the forward pass had them (y may be left out where there is neither post norm nor gate; want_dy then says
        whether dy is wanted), dout the gradient of out from where it is read beside h (None = none), dh that
        of h -> dict of dx, dy, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias: each None where there is
        nothing of that name; sums over tokens are f32 (accumulate: added to what the last call left)."""
        norm = self._norm(gate, post_weight, post_bias, pre_weight, pre_bias)
        for t, name in ((out, "out"), (dout, "dout"), (dh, "dh"), (y, "y")):
            self._rows(t, name)
        T, d, f32 = self.T, self.d, torch.float32
        want_dy = y is not None if want_dy is None else want_dy
        g = {"dx": self._buf("dx", (T, d), self.tdtype), "dy": self._buf("dy", (T, d), self.tdtype) if want_dy else None}
        for name, given in (("dpost_weight", post_weight), ("dpost_bias", post_bias), ("dpre_weight", pre_weight),
                            ("dpre_bias", pre_bias)):
            g[name] = None if given is None or (name.startswith("dpost") and not want_dy) else self._buf(name, (d,), f32)
        g["dgate"] = None
        if self.gate is not None and want_dy:
            shape, dtype = {"channel": ((d,), f32), "token": ((T,), f32), "element": ((T, d), self.tdtype)}[self.gate]
            g["dgate"] = self._buf("dgate", shape, dtype)
        ws = None
        n = B.occult_block_norm_backward_ws_bytes(self.cfg, norm)
        if n:
            if getattr(self, "ws", None) is None or self.ws.numel() * 4 < n:
                self.ws = torch.empty(n // 4, dtype=f32, device=self.device)
            ws = self.ws
        B.occult_block_norm_backward(self.cfg, norm, y, out, dout, dh, accumulate=accumulate, ws=ws, **g)
        return g
