"""Device buffers for one layer and the call sequence of its hot path (forward, and the backward
pass of the data movement).

Memory plumbing only: torch allocates the worst-case-sized buffers once (N_sfd <= T*min(k, D),
N_epd = T*k), every step is one call into the C library on the current stream, and nothing here
synchronises or computes.  Table views onto the plan block are for tests and reports.
"""
from __future__ import annotations

import operator
from typing import NamedTuple, Optional

import torch

from . import binding as B


class W4Weights(NamedTuple):
    """Expert weights in 4 bits, weight = scale * (code - zero), each field three tensors in the order gate, up, down:
    codes uint8 [E+S, rows, K / 2] (two along K per byte, the lower one in the low bits), scales bfloat16 and zeros uint8
    [E+S, rows, ceil(K / group)]; zeros is None, or three Nones, where every zero point is 8.  Scales of another type are the
    caller's to round to bfloat16 (from float16 three bits of each are lost)."""
    group: int
    codes: tuple
    scales: tuple
    zeros: Optional[tuple] = None

    @property
    def has_zeros(self):
        return self.zeros is not None and self.zeros[0] is not None


class OccultLayer:
    def __init__(self, T, d, f, E, S, k, D, dtype="bf16", n_d=0, prune_mode=1, renorm=1,
                 expert_pos=None, device="cuda:0", with_ffn=True, sim_table=None):
        B.load_library()          # fail early and loudly if the HIP library is missing
        self.device = torch.device(device)
        self.shape = dict(T=T, d=d, f=f, E=E, S=S, k=k, D=D)
        self.dtype_name = dtype
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        dev = self.device
        self.expert_pos = None
        if expert_pos is not None:
            self.expert_pos = torch.as_tensor(expert_pos, dtype=torch.int32).to(dev).contiguous()
        self.sim_table = None
        if sim_table is not None:
            self.sim_table = torch.as_tensor(sim_table, dtype=torch.int32).to(dev).contiguous()
        self.cfg = B.make_cfg(T, d, f, E, S, k, D, dtype, n_d, prune_mode, renorm, self.expert_pos, self.sim_table)
        plan_bytes, ws_bytes = B.occult_plan_sizes(self.cfg)
        self.plan_mem = torch.zeros(plan_bytes, dtype=torch.uint8, device=dev)
        self.ws = torch.zeros(ws_bytes, dtype=torch.uint8, device=dev)
        self.plan = B.occult_plan_bind(self.cfg, self.plan_mem)
        n_sfd_max = T * min(k, D)
        self.n_sfd_max = n_sfd_max
        self.ids = torch.zeros((T, k), dtype=torch.int32, device=dev)
        self.w = torch.zeros((T, k), dtype=torch.float32, device=dev)
        self.sfd_x = torch.zeros((n_sfd_max, d), dtype=self.tdtype, device=dev)
        self.sfd_y = torch.zeros((n_sfd_max, d), dtype=self.tdtype, device=dev)
        self.y = torch.zeros((T, d), dtype=self.tdtype, device=dev)
        self.epd_h = self.epd_y = self.h_shared = self.y_shared = self.ffn_ws = None
        # epd_gu and gu_shared hold the pre-activations of the present plan, rows and inputs: set by expert_ffn_train(),
        # cleared by every step that brings another plan, other rows or other outputs, and by the backward that overwrites them
        self.gu_saved = False
        # whether weight gradients are to be expected after the next input gradients: they came after the last ones
        self.weights_follow = True
        if with_ffn:
            ws_bytes = B.occult_expert_ffn_ws_bytes(self.cfg)
            if ws_bytes:
                self.ffn_ws = torch.empty(ws_bytes // 4, dtype=torch.float32, device=dev)
            self.epd_h = torch.zeros((T * k, f), dtype=self.tdtype, device=dev)
            self.epd_y = torch.zeros((T * k, d), dtype=self.tdtype, device=dev)
            if S > 0:
                self.h_shared = torch.zeros((T, S * f), dtype=self.tdtype, device=dev)
                self.y_shared = torch.zeros((T, d), dtype=self.tdtype, device=dev)

    # ---- element type and size of the caller's tensors (the library sees raw pointers) --------
    def _hidden(self, t, name, rows=None):
        s = self.shape
        return B.expect(t, name, self.tdtype, (s["T"] if rows is None else rows) * s["d"])

    def _weights(self, w_gate, w_up, w_down):
        s = self.shape
        n = (s["E"] + s["S"]) * s["d"] * s["f"]
        for t, name in ((w_gate, "w_gate"), (w_up, "w_up"), (w_down, "w_down")):
            B.expect(t, name, self.tdtype, n)

    def _routing(self, ids, w):
        s = self.shape
        B.expect(ids, "ids", torch.int32, s["T"] * s["k"])
        B.expect(w, "w", torch.float32, s["T"] * s["k"])

    # ---- steps (each = one library call on the current stream) -------------------------------
    def route(self, logits):
        B.expect(logits, "logits", torch.float32, self.shape["T"] * self.shape["E"])
        B.occult_route(self.cfg, logits, self.ids, self.w)

    def route_from_hidden(self, x, w_router, logits_out):
        """Router projection x w_router^T -> logits_out [T, E] f32, then routing, in one call."""
        s = self.shape
        self._hidden(x, "x")
        B.expect(w_router, "w_router", self.tdtype, s["E"] * s["d"])
        B.expect(logits_out, "logits_out", torch.float32, s["T"] * s["E"])
        B.occult_router(self.cfg, x, w_router, logits_out, self.ids, self.w)

    def make_plan(self, ids=None, w=None):
        self._routing(ids, w)
        self.gu_saved = False
        B.occult_plan(self.cfg, self.ids if ids is None else ids, self.w if w is None else w,
                      self.plan, self.ws)

    def dispatch(self, x):
        self._hidden(x, "x")
        self.gu_saved = False
        B.occult_dispatch(self.cfg, self.plan, x, self.sfd_x)

    def pack_weights(self, w_gate, w_up, w_down):
        """One-time repacking of the weights for decode-shaped batches (again after a weight update);
        expert_ffn() then reads the packed copy wherever the weight-streaming kernel runs."""
        n = B.occult_pack_weights_bytes(self.cfg)
        if n == 0:
            return None
        if getattr(self, "packed", None) is None:
            self.packed = torch.empty(n // 2, dtype=torch.bfloat16, device=self.device)
        B.occult_pack_weights(self.cfg, w_gate, w_up, w_down, self.packed)
        return self.packed

    def expert_ffn(self, x, w_gate, w_up, w_down, use_ws=True):
        self._hidden(x, "x")
        self._weights(w_gate, w_up, w_down)
        self.gu_saved = False
        if getattr(self, "packed", None) is not None:
            B.occult_expert_ffn_packed(self.cfg, self.plan, self.sfd_x, x, w_gate, w_up, w_down, self.packed, self.epd_h,
                                       self.epd_y, self.h_shared, self.y_shared, self.ffn_ws if use_ws else None)
            return
        if use_ws and self.ffn_ws is not None:
            B.occult_expert_ffn_ws(self.cfg, self.plan, self.sfd_x, x, w_gate, w_up, w_down, self.epd_h,
                                   self.epd_y, self.h_shared, self.y_shared, self.ffn_ws)
        else:
            B.occult_expert_ffn(self.cfg, self.plan, self.sfd_x, x, w_gate, w_up, w_down, self.epd_h,
                                self.epd_y, self.h_shared, self.y_shared)

    def expert_ffn_train(self, x, w_gate, w_up, w_down):
        """expert_ffn() that also keeps the pre-activations [g | u] for expert_ffn_backward(gu_saved=True)."""
        self._hidden(x, "x")
        self._weights(w_gate, w_up, w_down)
        epd_gu, gu_sh = self._pre_activations()
        self.gu_saved = False   # (until the call has succeeded)
        B.occult_expert_ffn_train(self.cfg, self.plan, self.sfd_x, x, w_gate, w_up, w_down, self.epd_h, self.epd_y,
                                  self.h_shared, self.y_shared, epd_gu, gu_sh, self.ffn_ws)
        self.gu_saved = True

    def _pre_activations(self):
        s = self.shape
        T, k, f, S = s["T"], s["k"], s["f"], s["S"]
        return (self._buf("epd_gu", (T * k, 2 * f), self.tdtype),
                self._buf("gu_shared", (T, S * 2 * f), self.tdtype) if S > 0 else None)

    # ---- 4-bit weights -------------------------------------------------------------------------
    def _w4_shapes(self, group):
        s = self.shape
        n = s["E"] + s["S"]
        return [(n, rows, K, (K + group - 1) // group) for rows, K in ((s["f"], s["d"]), (s["f"], s["d"]), (s["d"], s["f"]))]

    def _expect_w4(self, w4):
        B.occult_pack_w4_bytes(self.cfg, w4.group, w4.has_zeros)   # refuses the group and the layer's rows
        self._here(*w4.codes, *w4.scales, *(w4.zeros or ()))
        for i, ((n, rows, K, groups), name) in enumerate(zip(self._w4_shapes(w4.group), ("gate", "up", "down"))):
            B.expect(w4.codes[i], f"codes of {name}", torch.uint8, n * rows * K // 2)
            B.expect(w4.scales[i], f"scales of {name}", torch.bfloat16, n * rows * groups)
            if w4.has_zeros:
                B.expect(w4.zeros[i], f"zeros of {name}", torch.uint8, n * rows * groups)

    def quantize_weights(self, w_gate, w_up, w_down, group=128, zeros=False):
        """The layer's weights rounded to 4 bits with a scale (and, if asked for, a zero point) per `group` weights along K."""
        self._weights(w_gate, w_up, w_down)
        self._here(w_gate, w_up, w_down)
        B.occult_pack_w4_bytes(self.cfg, group, zeros)
        shapes = self._w4_shapes(group)
        empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=self.device)
        w4 = W4Weights(group, tuple(empty((n, rows, K // 2), torch.uint8) for n, rows, K, _ in shapes),
                       tuple(empty((n, rows, g), torch.bfloat16) for n, rows, _, g in shapes),
                       tuple(empty((n, rows, g), torch.uint8) for n, rows, _, g in shapes) if zeros else None)
        B.occult_quantize_weights(self.cfg, w_gate, w_up, w_down, *w4)
        return w4

    def dequantize_weights(self, w4):
        """The values that 4-bit weights stand for, in the layer's type: w_gate, w_up, w_down for forward() on large batches."""
        self._expect_w4(w4)
        w = tuple(torch.empty((n, rows, K), dtype=self.tdtype, device=self.device) for n, rows, K, _ in self._w4_shapes(w4.group))
        B.occult_dequantize_weights(self.cfg, *w4, *w)
        return w

    def pack_weights_w4(self, w4):
        """4-bit weights in the order that expert_ffn_w4() and forward_w4() read (again after every change of the weights, which
        are not read after this).  The layer keeps one buffer per group and kind of zero points: weights of a form go to that form's
        buffer, which the graphs captured with it go on reading; the eager calls read what was packed last."""
        self._expect_w4(w4)
        form = (w4.group, w4.has_zeros)
        forms = self.__dict__.setdefault("_packed_forms", {})
        packed = forms.get(form)
        if packed is None:
            packed = torch.empty(B.occult_pack_w4_bytes(self.cfg, *form), dtype=torch.uint8, device=self.device)
        B.occult_pack_w4(self.cfg, *w4, packed)
        forms[form] = packed   # kept: a captured graph holds its address
        self.packed_w4, self.w4_format = packed, form
        return packed

    def _packed_w4(self):
        if getattr(self, "packed_w4", None) is None:
            raise ValueError("occult: no 4-bit weights: call pack_weights_w4() first")
        return (self.packed_w4, *self.w4_format)

    def _here(self, *tensors):
        """The library launches on the current device's stream, and its kernels read this layer's buffers and the caller's tensors."""
        at = self.ws.get_device()
        if at != torch.cuda.current_device():
            raise ValueError(f"occult: the current device is cuda:{torch.cuda.current_device()}, the layer's buffers are on cuda:{at}")
        for t in tensors:
            if t is not None and t.is_cuda and t.get_device() != at:
                raise ValueError(f"occult: a tensor is on cuda:{t.get_device()}, the layer's buffers are on cuda:{at}")

    def expert_ffn_w4(self, x):
        """expert_ffn() from 4-bit weights -> epd_y, y_shared (None without shared experts)."""
        self._hidden(x, "x")
        self._here(x)
        self.gu_saved = False
        B.occult_expert_ffn_w4(self.cfg, self.plan, self.sfd_x, x, *self._packed_w4(), self.epd_h, self.epd_y, self.h_shared,
                               self.y_shared)
        return self.epd_y, self.y_shared

    def forward_w4(self, logits, x):
        """forward() from 4-bit weights."""
        if _w4_steps_of(type(self)) != _W4_STEPS or not self.__dict__.keys().isdisjoint(_W4_STEP_NAMES):
            self.route(logits)
            self.make_plan()
            self.dispatch(x)
            self.expert_ffn_w4(x)
            self.combine()
            return self.y
        s = self.shape
        B.expect(logits, "logits", torch.float32, s["T"] * s["E"])
        self._hidden(x, "x")
        self._here(x, logits)
        self.gu_saved = False
        B.occult_forward_w4(self.cfg, self.plan, logits, x, *self._packed_w4(), self.ids, self.w, self.ws, self.sfd_x, self.epd_h,
                            self.epd_y, self.h_shared, self.y_shared, self.sfd_y, self.y)
        return self.y

    def forward_block(self, x, h, w_router, norm, weights=None, **params):
        """The layer inside its block: router scores of h [T, d] (the normed residual stream), the experts (weights = w_gate, w_up,
        w_down, or None for the 4-bit ones), and norm.forward(x, y, **params), a norm.BlockNorm that adds y to the residual stream x
        and norms it for the next block -> out, the next block's h.  Router scores stay in self.logits."""
        s = self.shape
        if (norm.T, norm.d, norm.tdtype) != (s["T"], s["d"], self.tdtype):   # its calls see addresses: other rows of the same total
            raise ValueError(f"occult: norm is for {norm.T} rows of {norm.d} {norm.tdtype}, the layer for {s['T']} of {s['d']} {self.tdtype}")
        self.route_from_hidden(h, w_router, self._buf("logits", (s["T"], s["E"]), torch.float32))
        self.make_plan()
        self.dispatch(h)
        if weights is None:
            self.expert_ffn_w4(h)
        else:
            self.expert_ffn(h, *weights)
        self.combine()
        return norm.forward(x, self.y, **params)

    def combine(self, epd_y=None):
        self._hidden(epd_y, "epd_y", self.shape["T"] * self.shape["k"])
        B.occult_combine(self.cfg, self.plan, self.epd_y if epd_y is None else epd_y, self.sfd_y,
                         self.y_shared, self.y)

    def combine_atomic(self, epd_y=None, mode=0):
        """combine() with the paper's atomic merge as its first stage (mode 0: float32 atomics into a scratch
        tensor allocated on first use; mode 1: packed bf16 atomics into sfd_y)."""
        s = self.shape
        self._hidden(epd_y, "epd_y", s["T"] * s["k"])
        acc = self._buf("sfd_acc", (self.n_sfd_max, s["d"]), torch.float32) if mode == 0 else None
        B.occult_combine_atomic(self.cfg, self.plan, self.epd_y if epd_y is None else epd_y, acc, self.sfd_y,
                                self.y_shared, self.y, mode)

    def forward(self, logits, x, w_gate, w_up, w_down, train=False):
        """route(), make_plan(), dispatch(), expert_ffn() or expert_ffn_train(), combine(): in one call into the library, or
        one by one where a subclass or this object has its own version of one of them."""
        if self._has_own_steps():
            self.route(logits)
            self.make_plan()
            self.dispatch(x)
            (self.expert_ffn_train if train else self.expert_ffn)(x, w_gate, w_up, w_down)
            self.combine()
            return self.y
        s = self.shape
        B.expect(logits, "logits", torch.float32, s["T"] * s["E"])
        self._hidden(x, "x")
        self._weights(w_gate, w_up, w_down)
        packed = epd_gu = gu_sh = None
        if train:
            epd_gu, gu_sh = self._pre_activations()
        else:
            packed = getattr(self, "packed", None)
        self.gu_saved = False
        B.occult_forward(self.cfg, self.plan, logits, x, w_gate, w_up, w_down, packed, self.ids, self.w, self.ws, self.sfd_x,
                         self.epd_h, self.epd_y, self.h_shared, self.y_shared, self.ffn_ws, epd_gu, gu_sh, self.sfd_y, self.y)
        self.gu_saved = bool(train)
        return self.y

    def _has_own_steps(self):
        return _steps_of(type(self)) != _STEPS or not self.__dict__.keys().isdisjoint(_STEP_NAMES)

    # ---- backward of the data movement (buffers allocated on first use) -----------------------
    def _buf(self, name, shape, dtype):
        if getattr(self, name, None) is None:
            setattr(self, name, torch.zeros(shape, dtype=dtype, device=self.device))
        return getattr(self, name)

    def combine_backward(self, dy, ids=None, epd_y=None, want_sfd=True, want_epd=True, want_dw=True):
        """dy [T, d] -> sfd_dy, epd_dy, dw (each None if not asked for)."""
        s = self.shape
        sfd_dy = self._buf("sfd_dy", (self.n_sfd_max, s["d"]), self.tdtype) if want_sfd else None
        epd_dy = self._buf("epd_dy", (s["T"] * s["k"], s["d"]), self.tdtype) if want_epd else None
        dw = self._buf("dw", (s["T"], s["k"]), torch.float32) if want_dw else None
        self._hidden(dy, "dy")
        self._hidden(epd_y, "epd_y", s["T"] * s["k"])
        B.expect(ids, "ids", torch.int32, s["T"] * s["k"])
        B.occult_combine_backward(self.cfg, self.plan, self.ids if ids is None else ids, dy,
                                  self.epd_y if epd_y is None else epd_y, sfd_dy, epd_dy, dw)
        return sfd_dy, epd_dy, dw

    def dispatch_backward(self, epd_dx, dx_shared=None):
        """epd_dx [T*k, d] -> sfd_dx, dx."""
        s = self.shape
        sfd_dx = self._buf("sfd_dx", (self.n_sfd_max, s["d"]), self.tdtype)
        dx = self._buf("dx", (s["T"], s["d"]), self.tdtype)
        self._hidden(epd_dx, "epd_dx", s["T"] * s["k"])
        self._hidden(dx_shared, "dx_shared")
        B.occult_dispatch_backward(self.cfg, self.plan, epd_dx, sfd_dx, dx_shared, dx)
        return sfd_dx, dx

    def transpose_weights(self, w_gate, w_up, w_down):
        """Transposed weight copies for the backward products (again after every weight update)."""
        s = self.shape
        n = s["E"] + s["S"]
        w_down_t = self._buf("w_down_t", (n, s["f"], s["d"]), self.tdtype)
        w_gu_t = self._buf("w_gu_t", (n, s["d"], 2 * s["f"]), self.tdtype)
        self._weights(w_gate, w_up, w_down)
        B.occult_transpose_weights(self.cfg, w_gate, w_up, w_down, w_down_t, w_gu_t)
        return w_down_t, w_gu_t

    def expert_ffn_backward(self, x, w_gate, w_up, epd_dy, dy, gu_saved=None):
        """epd_dy [T*k, d] (and dy [T, d] for shared experts) -> epd_dx, dx_shared (None if S == 0);
        needs transpose_weights() first and the forward's sfd_x."""
        s = self.shape
        T, k, d, f, S = s["T"], s["k"], s["d"], s["f"], s["S"]
        epd_gu = self._buf("epd_gu", (T * k, 2 * f), self.tdtype)
        epd_dh = self._buf("epd_dh", (T * k, f), self.tdtype)
        epd_dx = self._buf("epd_dx", (T * k, d), self.tdtype)
        gu_sh = dh_sh = dx_sh = None
        if S > 0:
            gu_sh = self._buf("gu_shared", (T, S * 2 * f), self.tdtype)
            dh_sh = self._buf("dh_shared", (T, S * f), self.tdtype)
            dx_sh = self._buf("dx_shared", (T, d), self.tdtype)
        self._hidden(x, "x")
        self._hidden(dy, "dy")
        self._hidden(epd_dy, "epd_dy", T * k)
        self._weights(w_gate, w_up, None)
        if gu_saved is None:   # pre-activations kept by expert_ffn_train() for this very batch
            gu_saved = self.gu_saved
        B.occult_expert_ffn_backward(self.cfg, self.plan, self.sfd_x, x, w_gate, w_up, self.w_down_t, self.w_gu_t,
                                     epd_dy, dy, epd_gu, epd_dh, epd_dx, gu_sh, dh_sh, dx_sh, gu_saved,
                                     weights_follow=self.weights_follow)
        self.gu_saved = False      # overwritten with [dg | du]
        self.weights_follow = False
        return epd_dx, dx_sh

    def expert_ffn_backward_weights(self, x, dy, accumulate=False, use_ws=True):
        """f32 weight gradients dw_gate, dw_up [E+S, f, d], dw_down [E+S, d, f]; after expert_ffn_backward()."""
        s = self.shape
        n = s["E"] + s["S"]
        dw_gate = self._buf("dw_gate", (n, s["f"], s["d"]), torch.float32)
        dw_up = self._buf("dw_up", (n, s["f"], s["d"]), torch.float32)
        dw_down = self._buf("dw_down", (n, s["d"], s["f"]), torch.float32)
        self._hidden(x, "x")
        self._hidden(dy, "dy")
        ws = None
        if use_ws:   # scratch for the row slices of the shared experts' products (large T, few shared experts)
            n = B.occult_expert_ffn_backward_weights_ws_bytes(self.cfg)
            if n:
                ws = self._buf("wgrad_ws", (n // 4,), torch.float32)
        B.occult_expert_ffn_backward_weights_ws(self.cfg, self.plan, self.sfd_x, x, self.epd_h, self.h_shared, self.epd_dy,
                                                dy, self.epd_gu, getattr(self, "gu_shared", None), dw_gate, dw_up, dw_down,
                                                ws, accumulate)
        self.weights_follow = True
        return dw_gate, dw_up, dw_down

    def backward_input(self, x, w_gate, w_up, dy):
        """dy [T, d] -> dx [T, d], dw [T, k]: the three backward calls in order (after forward())."""
        _, epd_dy, dw = self.combine_backward(dy, want_sfd=True)
        epd_dx, dx_sh = self.expert_ffn_backward(x, w_gate, w_up, epd_dy, dy)
        _, dx = self.dispatch_backward(epd_dx, dx_sh)
        return dx, dw

    def route_backward(self, logits, dw, dlogits, ids=None):
        s = self.shape
        B.expect(logits, "logits", torch.float32, s["T"] * s["E"])
        B.expect(dlogits, "dlogits", torch.float32, s["T"] * s["E"])
        self._routing(ids, dw)
        B.occult_route_backward(self.cfg, logits, self.ids if ids is None else ids, dw, dlogits)

    def stats(self):
        return B.occult_plan_stats(self.cfg, self.plan)

    # ---- views onto the plan block ------------------------------------------------------------
    def _view(self, field, count, dtype):
        base = self.plan_mem.data_ptr()
        off = getattr(self.plan, field) - base
        nbytes = count * torch.empty((), dtype=dtype).element_size()
        return self.plan_mem[off:off + nbytes].view(dtype)

    def tables(self):
        s = self.shape
        T, E, D, k = s["T"], s["E"], s["D"], s["k"]
        m1 = min(k, E // D)
        i32 = torch.int32
        return {
            "tok_devmask": self._view("tok_devmask", T, torch.int64),
            "dev_count": self._view("dev_count", D, i32),
            "dev_offset": self._view("dev_offset", D + 1, i32),
            "tok_sfd_row": self._view("tok_sfd_row", T * D, i32).view(T, D),
            "sfd_token": self._view("sfd_token", self.n_sfd_max, i32),
            "exp_count": self._view("exp_count", E, i32),
            "exp_offset": self._view("exp_offset", E + 1, i32),
            "pos_expert": self._view("pos_expert", E, i32),
            "epd_sfd_row": self._view("epd_sfd_row", T * k, i32),
            "epd_gate": self._view("epd_gate", T * k, torch.float32),
            "sfd_epd_rows": self._view("sfd_epd_rows", self.n_sfd_max * m1, i32).view(self.n_sfd_max, m1),
            "counters": self._view("counters", 8, torch.int64),
        }


# the steps that forward() stands for (one attribute lookup for all of them: this runs on every pass)
_STEP_NAMES = ("route", "make_plan", "dispatch", "expert_ffn", "expert_ffn_train", "combine")
_steps_of = operator.attrgetter(*_STEP_NAMES)
_STEPS = _steps_of(OccultLayer)
_W4_STEP_NAMES = ("route", "make_plan", "dispatch", "expert_ffn_w4", "combine")
_w4_steps_of = operator.attrgetter(*_W4_STEP_NAMES)
_W4_STEPS = _w4_steps_of(OccultLayer)
