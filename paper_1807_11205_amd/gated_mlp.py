"""A stack of gated feed-forward residual blocks as a sequence of libjz calls: a training step in mixed precision, and its answers
for rows that come one at a time (sequencing and buffer bookkeeping only: every arithmetic step runs in the library's kernels).

    n_0 = norm(r_0) w_pre_0
    block i:   y = (silu(n_i W_gate^T) * (n_i W_up^T)) W_down^T
               r_{i+1} = r_i + scale gate_i norm(y) w_post_i,    n_{i+1} = norm(r_{i+1}) w_pre_{i+1}        one call
    logits = n_last W_fc^T

One step = forward; softmax cross-entropy gradient times the loss scale; backward into the fused FP16 gradient buffer; clipping of all gradients
by their global norm; the mixed-precision LARS update with the device-resident dynamic loss scale.  The residual stream and its gradient
are FP32, everything between a block's norms FP16.  The norms' and gates' parameters are exempt from weight decay.
"""
from typing import Optional

import numpy as np
import torch

from . import api

EPS = 1e-5


class GatedMLP:
    def __init__(self, rows: int, width: int, hidden: int, classes: int, blocks: int, scale: float = 0.5, max_norm: float = 1.0, seed: int = 1,
                 initial_loss_scale: float = 1024.0, hparams: Optional[dict] = None, policy: Optional[dict] = None, device: str = "cuda:0"):
        if width % 8 or hidden % 8 or classes % 8:
            raise ValueError("width, hidden and classes must be multiples of 8: tensors of the fused buffers start on 16 bytes")
        self.rows, self.width, self.hidden, self.classes, self.blocks, self.max_norm = rows, width, hidden, classes, blocks, float(max_norm)
        self.device = torch.device(device)
        D, F, h, f = width, hidden, torch.float16, torch.float32
        weights, others = api.JZ_PARAM_LARS | api.JZ_PARAM_WEIGHT_DECAY, api.JZ_PARAM_LARS
        self.shapes, flags = {}, []

        def add(name, shape, flag):
            self.shapes[name] = shape
            flags.append(flag)
        for i in range(blocks):
            add("w_pre_%d" % i, (D,), others)
            add("w_gate_%d" % i, (F, D), weights)
            add("w_up_%d" % i, (F, D), weights)
            add("w_down_%d" % i, (D, F), weights)
            add("w_post_%d" % i, (D,), others)
            add("gate_%d" % i, (1, D), others)
        add("w_pre_%d" % blocks, (D,), others)
        add("w_fc", (classes, D), weights)
        sizes = [int(np.prod(s)) for s in self.shapes.values()]
        offsets = np.concatenate([[0], np.cumsum(sizes)])
        self.place = {n: (int(a), int(b)) for n, a, b in zip(self.shapes, offsets[:-1], offsets[1:])}

        g = torch.Generator(device="cpu").manual_seed(seed)
        self.master = torch.cat([torch.randn(n, generator=g) * s[-1] ** -0.5 if len(s) == 2 and not name.startswith("gate_") else torch.ones(n)
                                 for n, (name, s) in zip(sizes, self.shapes.items())]).to(self.device)
        self.momentum = torch.zeros_like(self.master)
        self.w16 = self.master.to(h)
        self.grad = torch.zeros(self.master.numel(), dtype=h, device=self.device)
        self.ps = api.ParamSet(offsets, flags, self.master, self.momentum, self.grad, self.w16)
        self.lars_ws = torch.zeros(api.jz_lars_workspace_bytes(self.ps), dtype=torch.uint8, device=self.device)
        api.jz_lars_prepare(self.ps, self.lars_ws)
        self.hp = api.lars_hparams(**{**dict(lr=1.0, momentum=0.9, weight_decay=5e-5, trust_coef=0.001, loss_scale=1.0), **(hparams or {})})
        self.policy = api.loss_scale_policy(**(policy or {}))
        self.ls_state = torch.zeros(2, dtype=torch.int32, device=self.device)
        api.jz_loss_scale_init(self.ls_state, initial_loss_scale)
        self.found_inf, self.clip_found_inf = self._buf(1, torch.int32), self._buf(1, torch.int32)

        # clipping in place: every gradient of the fused buffer as a tensor of its own
        self.grad_list = api.GradList([self._param(self.grad, n) for n in self.shapes])
        self.clip_ws = torch.zeros(api.jz_grad_clip_workspace_bytes(self.grad_list), dtype=torch.uint8, device=self.device)
        api.jz_grad_clip_prepare(self.grad_list, self.clip_ws)
        self.norm = self._buf(1, f)

        # activations that the backward pass reads
        self.r = [self._buf((rows, D), f) for _ in range(blocks + 1)]
        self.n = [self._buf((rows, D)) for _ in range(blocks + 1)]
        self.y = [self._buf((rows, D)) for _ in range(blocks)]
        self.gate, self.up, self.h = ([self._buf((rows, F)) for _ in range(blocks)] for _ in range(3))
        self.rstd_post, self.rstd_pre = [self._buf(rows, f) for _ in range(blocks)], [self._buf(rows, f) for _ in range(blocks + 1)]
        self.logits, self.dlogits = self._buf((rows, classes)), self._buf((rows, classes))
        self.loss = self._buf(rows, f)
        self.labels = self._buf(rows, torch.int32)
        self.dr, self.dn, self.dy = self._buf((rows, D), f), self._buf((rows, D)), self._buf((rows, D))

        self.scale = float(scale)
        self.ffn = api.ffn_desc(rows, D, F, D, api.JZ_ACT_SILU, api.JZ_F16)
        self.around = self._around(rows)
        need = [api.jz_ffn_fwd_workspace_bytes(self.ffn), api.jz_ffn_bwd_workspace_bytes(self.ffn), api.jz_norm_residual_bwd_workspace_bytes(self.around)]
        need += [api.jz_gemm_fc_workspace_bytes(mode, rows, D, classes) for mode in (api.JZ_FWD, api.JZ_BWD_DATA, api.JZ_BWD_WEIGHT)]
        self.ws = torch.zeros(max(16, *need), dtype=torch.uint8, device=self.device)
        torch.cuda.current_stream(self.device).synchronize()    # whatever stream a step runs on, the buffers' fills are behind it

    # ---- buffers and parameter views --------------------------------------------------------------------------------
    def _buf(self, shape, dtype=torch.float16):
        return torch.zeros(shape, dtype=dtype, device=self.device)

    def _param(self, buf, name):
        a, b = self.place[name]
        return buf[a:b].view(self.shapes[name])

    def _around(self, rows):
        return api.norm_residual_desc(rows, self.width, 0, api.JZ_F16, api.JZ_F32, EPS, 1.0, self.scale)

    def _ffn_weights(self, i):
        return tuple(self._param(self.w16, "%s_%d" % (n, i)) for n in ("w_gate", "w_up", "w_down"))

    # ---- the step ------------------------------------------------------------------------------------------------------
    def set_batch(self, x: torch.Tensor, labels: torch.Tensor, stream=None):
        """r_0 (float32 [rows, width]) and the classes of the rows, copied on the stream of the step that takes them."""
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
            self.r[0].copy_(x)
            self.labels.copy_(labels)

    def forward(self, stream=None):
        m = lambda n: self._param(self.master, n)
        api.jz_norm_residual_fwd(self.around, self.r[0], None, None, None, m("w_pre_0"), None, self.n[0], None, self.rstd_pre[0], stream)
        for i in range(self.blocks):
            api.jz_ffn_fwd(self.ffn, self.n[i], *self._ffn_weights(i), self.h[i], self.y[i], self.gate[i], self.up[i], self.ws, stream)
            api.jz_norm_residual_fwd(self.around, self.r[i], self.y[i], m("w_post_%d" % i), m("gate_%d" % i), m("w_pre_%d" % (i + 1)), self.r[i + 1], self.n[i + 1],
                                     self.rstd_post[i], self.rstd_pre[i + 1], stream)
        api.jz_gemm_fc(api.JZ_FWD, self.rows, self.width, self.classes, self.n[-1], self._param(self.w16, "w_fc"), self.logits, self.ws, stream)
        api.jz_softmax_xent_bwd(self.rows, self.classes, self.logits, self.labels, self.dlogits, self.loss, state=self.ls_state, stream=stream)

    def backward(self, stream=None):
        m, d = lambda n: self._param(self.master, n), lambda n: self._param(self.grad, n)
        api.jz_gemm_fc(api.JZ_BWD_WEIGHT, self.rows, self.width, self.classes, self.dlogits, self.n[-1], d("w_fc"), self.ws, stream)
        api.jz_gemm_fc(api.JZ_BWD_DATA, self.rows, self.width, self.classes, self.dlogits, self._param(self.w16, "w_fc"), self.dn, self.ws, stream)
        arrives = None                          # of the residual stream's gradient nothing arrives behind the last norm
        for i in reversed(range(self.blocks)):
            api.jz_norm_residual_bwd(self.around, self.y[i], self.r[i + 1], m("w_post_%d" % i), m("gate_%d" % i), m("w_pre_%d" % (i + 1)), self.rstd_post[i],
                                     self.rstd_pre[i + 1], arrives, self.dn, self.dr, self.dy, d("w_post_%d" % i), d("gate_%d" % i), d("w_pre_%d" % (i + 1)), self.ws, stream)
            api.jz_ffn_bwd(self.ffn, self.n[i], *self._ffn_weights(i), self.gate[i], self.up[i], self.h[i], self.dy, self.dn, d("w_gate_%d" % i), d("w_up_%d" % i),
                           d("w_down_%d" % i), self.ws, stream)
            arrives = self.dr
        api.jz_norm_residual_bwd(self.around, None, self.r[0], None, None, m("w_pre_0"), None, self.rstd_pre[0], arrives, self.dn, self.dr, None, None, None,
                                 d("w_pre_0"), self.ws, stream)

    def update(self, stream=None):
        api.jz_grad_clip(self.grad_list, self.max_norm, self.norm, self.clip_found_inf, self.clip_ws, state=self.ls_state, stream=stream)
        api.jz_lars_mp_update_dyn(self.ps, self.hp, self.policy, self.ls_state, self.found_inf, self.lars_ws, stream)

    def step(self, stream=None):
        self.forward(stream)
        self.backward(stream)
        self.update(stream)

    def mean_loss(self) -> float:
        """Of the last forward pass, on whatever stream it ran (synchronizes)."""
        torch.cuda.synchronize(self.device)
        return float(self.loss.double().mean().item())

    # ---- answers -------------------------------------------------------------------------------------------------------
    def answer(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """Logits (float16) of the rows of x (float32 [any number of rows, width]), nothing kept for a backward pass.  x is as the current stream
        leaves it; the logits are ready once `stream` is (None: the current one)."""
        current = torch.cuda.current_stream(self.device)
        if stream is None or api._stream(stream) == api._stream(current):
            return self._answer(x)
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), self.device) if int(stream) else torch.cuda.default_stream(self.device)
        stream.wait_stream(current)
        with torch.cuda.stream(stream):         # copies, temporaries and launches all belong to it
            logits = self._answer(x)
        x.record_stream(stream)
        logits.record_stream(current)
        return logits

    def _answer(self, x):
        """On the current stream."""
        rows, D, F = x.shape[0], self.width, self.hidden
        m = lambda n: self._param(self.master, n)
        ffn, around = api.ffn_desc(rows, D, F, D, api.JZ_ACT_SILU, api.JZ_F16), self._around(rows)
        r, n, y, h, k1, k2 = x.to(torch.float32).clone(), self._buf((rows, D)), self._buf((rows, D)), self._buf((rows, F)), self._buf(rows, torch.float32), self._buf(rows, torch.float32)
        logits = self._buf((rows, self.classes))
        ws = self._buf(max(16, api.jz_ffn_fwd_workspace_bytes(ffn), api.jz_gemm_fc_workspace_bytes(api.JZ_FWD, rows, D, self.classes)), torch.uint8)
        api.jz_norm_residual_fwd(around, r, None, None, None, m("w_pre_0"), None, n, None, k2)
        for i in range(self.blocks):
            api.jz_ffn_fwd(ffn, n, *self._ffn_weights(i), h, y, ws=ws)
            api.jz_norm_residual_fwd(around, r, y, m("w_post_%d" % i), m("gate_%d" % i), m("w_pre_%d" % (i + 1)), r, n, k1, k2)
        api.jz_gemm_fc(api.JZ_FWD, rows, D, self.classes, n, self._param(self.w16, "w_fc"), logits, ws)
        return logits
