"""A stack of gated feed-forward residual blocks as a sequence of libjz calls: a training step in mixed precision, and its answers
for rows that come one at a time (sequencing and buffer bookkeeping only: every arithmetic step runs in the library's kernels).

    r_0: the rows given, or, with a vocabulary, embed_scale E[token]
    n_0 = norm(r_0) w_pre_0
    block i:   y = (silu(n_i W_gate^T) * (n_i W_up^T)) W_down^T
               r_{i+1} = r_i + scale gate_i norm(y) w_post_i,    n_{i+1} = norm(r_{i+1}) w_pre_{i+1}        one call
    logits = n_last W_fc^T         (tied: W_fc is E)

Rows are independent of each other: nothing mixes them, so that with a vocabulary a row's logits depend on its one token alone (a bigram model, where the classes are the tokens that follow).

One step = forward; softmax cross-entropy gradient times the loss scale; backward into the fused FP16 gradient buffer; clipping of all gradients
by their global norm; the mixed-precision LARS update with the device-resident dynamic loss scale.  The residual stream and its gradient
are FP32, everything between a block's norms FP16.  The norms' and gates' parameters are exempt from weight decay.

With optimizer="muon" the blocks' matrices get orthogonalised updates instead, all of a shape in one call, and LARS has the other parameters; all of them skip the
step where a gradient, or a matrix's momentum, overflows.  Answers can also run with the matrices in 8-bit integers (prepare_answers_i8).
"""
import contextlib
import threading
from typing import Optional

import numpy as np
import torch

from . import api

EPS = 1e-5


def _within_int32(t):
    """Tokens or classes of 64 bits without their wrapping around: what int32 does not hold stays outside of every vocabulary, at -1 or 2^31 - 1."""
    return t.clamp(-1, 2 ** 31 - 1) if t.dtype == torch.int64 else t


class GatedMLP:
    vocab, fc, i8 = 0, "w_fc", None     # without a vocabulary, a classifier of its own, no codes

    def __init__(self, rows: int, width: int, hidden: int, classes: int, blocks: int, scale: float = 0.5, max_norm: float = 1.0, seed: int = 1,
                 initial_loss_scale: float = 1024.0, hparams: Optional[dict] = None, policy: Optional[dict] = None, device: str = "cuda:0", vocab: int = 0,
                 embed_scale: float = 1.0, tied: bool = False, optimizer: str = "lars", muon: Optional[dict] = None):
        """vocab > 0: the rows are tokens (set_tokens; answer takes tokens too); tied: the classes are the vocabulary and the classifier's matrix is the embedding's table.
        muon: settings of the orthogonalised updates (lr, momentum, weight_decay, nesterov, steps)."""
        if width % 8 or hidden % 8 or classes % 8:
            raise ValueError("width, hidden and classes must be multiples of 8: tensors of the fused buffers start on 16 bytes")
        if vocab < 0 or tied and vocab != classes:
            raise ValueError("a tied classifier's classes are the vocabulary")
        if optimizer not in ("lars", "muon"):
            raise ValueError("optimizer: lars or muon")
        self.vocab, self.tied, self.muon = vocab, tied, optimizer == "muon"
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
        self.fc = "embed" if tied else "w_fc"
        add(self.fc, (classes, D), weights)
        if vocab and not tied:
            add("embed", (vocab, D), weights)
        if self.muon:       # LARS' parameters, then the matrices, those of a shape side by side
            kind = lambda n: 2 if n.startswith("w_down_") else 1 if n.startswith(("w_gate_", "w_up_")) else 0
            order = sorted(range(len(flags)), key=lambda k: kind(list(self.shapes)[k]))
            names, flags = [list(self.shapes)[k] for k in order], [flags[k] for k in order]
            self.shapes = {n: self.shapes[n] for n in names}
        sizes = [int(np.prod(s)) for s in self.shapes.values()]
        offsets = np.concatenate([[0], np.cumsum(sizes)])
        self.place = {n: (int(a), int(b)) for n, a, b in zip(self.shapes, offsets[:-1], offsets[1:])}

        g = torch.Generator(device="cpu").manual_seed(seed)
        self.master = torch.cat([torch.randn(n, generator=g) * s[-1] ** -0.5 if len(s) == 2 and not name.startswith("gate_") else torch.ones(n)
                                 for n, (name, s) in zip(sizes, self.shapes.items())]).to(self.device)
        self.momentum = torch.zeros_like(self.master)
        self.w16 = self.master.to(h)
        self.grad = torch.zeros(self.master.numel(), dtype=h, device=self.device)
        if self.muon:
            # of each shape an empty tensor stands in LARS' set, whose sink passes on that a matrix's gradient is not finite
            of_lars = sum(not name.startswith(("w_gate_", "w_up_", "w_down_")) for name in self.shapes)
            end = int(offsets[of_lars])
            self.ps = api.ParamSet(list(offsets[:of_lars + 1]) + [end, end], flags[:of_lars] + [others, others], self.master[:end], self.momentum[:end], self.grad[:end], self.w16[:end])
        else:
            self.ps = api.ParamSet(offsets, flags, self.master, self.momentum, self.grad, self.w16)
        self.lars_ws = torch.zeros(api.jz_lars_workspace_bytes(self.ps), dtype=torch.uint8, device=self.device)
        api.jz_lars_prepare(self.ps, self.lars_ws)
        self.hp = api.lars_hparams(**{**dict(lr=1.0, momentum=0.9, weight_decay=5e-5, trust_coef=0.001, loss_scale=1.0), **(hparams or {})})
        self.policy = api.loss_scale_policy(**(policy or {}))
        self.ls_state = torch.zeros(2, dtype=torch.int32, device=self.device)
        api.jz_loss_scale_init(self.ls_state, initial_loss_scale)
        self.found_inf, self.clip_found_inf = self._buf(1, torch.int32), self._buf(1, torch.int32)

        if self.muon:
            m = {**dict(lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5), **(muon or {})}
            steps = m.pop("steps")
            self.groups, ws = [], 16
            for k, (first, count, shape) in enumerate((("w_gate_0", 2 * blocks, (F, D)), ("w_down_0", blocks, (D, F)))):
                desc = api.ortho_desc(count, *shape, api.JZ_F16, steps=steps)
                a = self.place[first][0] if blocks else 0
                b = a + count * shape[0] * shape[1]
                sink = api.jz_lars_sumsq_sink(self.ps, self.lars_ws, of_lars + k)
                self.groups.append((desc, api.muon_hparams(update_scale=max(1.0, shape[0] / shape[1]) ** 0.5, **m), slice(a, b), sink.nonfinite))
                ws = max(ws, api.jz_muon_mp_update_workspace_bytes(desc))
            self.muon_ws, self.muon_found_inf = self._buf(ws, torch.uint8), self._buf(1, torch.int32)

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
        self.ids = self._buf(rows, torch.int32) if vocab else None
        self.dr, self.dn, self.dy = self._buf((rows, D), f), self._buf((rows, D)), self._buf((rows, D))

        self.scale = float(scale)
        self.ffn = api.ffn_desc(rows, D, F, D, api.JZ_ACT_SILU, api.JZ_F16)
        self.around = self._around(rows)
        self.embed_scale = float(embed_scale)
        self.embed = self._embed(rows) if vocab else None
        need = [api.jz_ffn_fwd_workspace_bytes(self.ffn), api.jz_ffn_bwd_workspace_bytes(self.ffn), api.jz_norm_residual_bwd_workspace_bytes(self.around)]
        need += [api.jz_gemm_fc_workspace_bytes(mode, rows, D, classes) for mode in (api.JZ_FWD, api.JZ_BWD_DATA, api.JZ_BWD_WEIGHT)]
        if vocab:
            need.append(api.jz_embed_bwd_workspace_bytes(self.embed))
        self.ws = torch.zeros(max(16, *need), dtype=torch.uint8, device=self.device)
        self.i8, self.i8_lock = None, threading.Lock()
        torch.cuda.current_stream(self.device).synchronize()    # whatever stream a step runs on, the buffers' fills are behind it

    # ---- buffers and parameter views --------------------------------------------------------------------------------
    def _buf(self, shape, dtype=torch.float16):
        return torch.zeros(shape, dtype=dtype, device=self.device)

    def _param(self, buf, name):
        a, b = self.place[name]
        return buf[a:b].view(self.shapes[name])

    def _around(self, rows):
        return api.norm_residual_desc(rows, self.width, 0, api.JZ_F16, api.JZ_F32, EPS, 1.0, self.scale)

    def _embed(self, rows):
        return api.embed_desc(rows, self.vocab, self.width, api.JZ_F16, api.JZ_F32, self.embed_scale)

    def _ffn_weights(self, i):
        return tuple(self._param(self.w16, "%s_%d" % (n, i)) for n in ("w_gate", "w_up", "w_down"))

    # ---- the step ------------------------------------------------------------------------------------------------------
    def set_batch(self, x: torch.Tensor, labels: torch.Tensor, stream=None):
        """r_0 (float32 [rows, width]) and the classes of the rows (int32 or int64), copied on the stream of the step that takes them."""
        if self.vocab:
            raise ValueError("the network's rows are tokens: set_tokens")
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
            self.r[0].copy_(x)
            self.labels.copy_(_within_int32(labels))

    def set_tokens(self, ids: torch.Tensor, labels: torch.Tensor, stream=None):
        """The rows' tokens (int32 or int64 [rows]; one outside the vocabulary is a row of zeros) and classes, as set_batch."""
        if not self.vocab:
            raise ValueError("the network has no vocabulary")
        if ids.is_floating_point():
            raise ValueError("the network's rows are tokens")
        if ids.shape != (self.rows,) or labels.shape != (self.rows,):
            raise ValueError("a step takes %d tokens and as many classes" % self.rows)
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
            self.ids.copy_(_within_int32(ids))
            self.labels.copy_(_within_int32(labels))

    def forward(self, stream=None):
        m = lambda n: self._param(self.master, n)
        if self.vocab:
            api.jz_embed_fwd(self.embed, self.ids, self._param(self.w16, "embed"), self.r[0], stream)
        api.jz_norm_residual_fwd(self.around, self.r[0], None, None, None, m("w_pre_0"), None, self.n[0], None, self.rstd_pre[0], stream)
        for i in range(self.blocks):
            api.jz_ffn_fwd(self.ffn, self.n[i], *self._ffn_weights(i), self.h[i], self.y[i], self.gate[i], self.up[i], self.ws, stream)
            api.jz_norm_residual_fwd(self.around, self.r[i], self.y[i], m("w_post_%d" % i), m("gate_%d" % i), m("w_pre_%d" % (i + 1)), self.r[i + 1], self.n[i + 1],
                                     self.rstd_post[i], self.rstd_pre[i + 1], stream)
        api.jz_gemm_fc(api.JZ_FWD, self.rows, self.width, self.classes, self.n[-1], self._param(self.w16, self.fc), self.logits, self.ws, stream)
        api.jz_softmax_xent_bwd(self.rows, self.classes, self.logits, self.labels, self.dlogits, self.loss, state=self.ls_state, stream=stream)

    def backward(self, stream=None):
        m, d = lambda n: self._param(self.master, n), lambda n: self._param(self.grad, n)
        api.jz_gemm_fc(api.JZ_BWD_WEIGHT, self.rows, self.width, self.classes, self.dlogits, self.n[-1], d(self.fc), self.ws, stream)
        api.jz_gemm_fc(api.JZ_BWD_DATA, self.rows, self.width, self.classes, self.dlogits, self._param(self.w16, self.fc), self.dn, self.ws, stream)
        arrives = None                          # of the residual stream's gradient nothing arrives behind the last norm
        for i in reversed(range(self.blocks)):
            api.jz_norm_residual_bwd(self.around, self.y[i], self.r[i + 1], m("w_post_%d" % i), m("gate_%d" % i), m("w_pre_%d" % (i + 1)), self.rstd_post[i],
                                     self.rstd_pre[i + 1], arrives, self.dn, self.dr, self.dy, d("w_post_%d" % i), d("gate_%d" % i), d("w_pre_%d" % (i + 1)), self.ws, stream)
            api.jz_ffn_bwd(self.ffn, self.n[i], *self._ffn_weights(i), self.gate[i], self.up[i], self.h[i], self.dy, self.dn, d("w_gate_%d" % i), d("w_up_%d" % i),
                           d("w_down_%d" % i), self.ws, stream)
            arrives = self.dr
        api.jz_norm_residual_bwd(self.around, None, self.r[0], None, None, m("w_pre_0"), None, self.rstd_pre[0], arrives, self.dn, self.dr, None, None, None,
                                 d("w_pre_0"), self.ws, stream)
        if self.vocab:                          # a tied table has the classifier's gradient already
            api.jz_embed_bwd(self.embed, self.ids, self.dr, d("embed"), self.ws, accumulate=self.tied, stream=stream)

    def update(self, stream=None):
        api.jz_grad_clip(self.grad_list, self.max_norm, self.norm, self.clip_found_inf, self.clip_ws, state=self.ls_state, stream=stream)
        if self.muon:
            api.jz_lars_begin_step(self.ps, self.lars_ws, self.ls_state, stream)
            api.jz_lars_grad_sumsq(self.ps, 0, len(self.ps.flags), self.lars_ws, stream)
            # one step over both shapes and LARS: the second shape's flag before the first is written, and each later update behind the flags of all before it
            desc, hp, at, _ = self.groups[1]
            skip = self.muon_found_inf
            api.jz_muon_mp_overflow(desc, hp, self.momentum[at], self.grad[at], skip, self.muon_ws, self.ls_state, self.clip_found_inf, stream)
            for desc, hp, at, flag in self.groups:
                api.jz_muon_mp_update(desc, hp, self.master[at], self.momentum[at], self.grad[at], self.w16[at], flag, self.muon_ws, self.ls_state, skip, stream)
                skip = flag
            api.jz_lars_mp_update_presummed_dyn(self.ps, self.hp, self.policy, self.ls_state, self.found_inf, self.lars_ws, stream)
            return
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
    def prepare_answers_i8(self, stream=None):
        """Codes and scales of all matrices as `stream` (None: the current one) finds them, for answer(i8=True): again after every update that is to be seen.  Answers
        that follow, on whatever stream, wait for the codes, and the codes for the answers before them.  In a capture both are left out, since a graph cannot wait for what is outside it:
        there the order is the caller's.  Threads may call both: the launches of one call lie together."""
        with self.i8_lock:
            self._write_codes(stream)

    def _write_codes(self, stream):
        codes = self.i8
        if codes is None:
            names = [n for n in self.shapes if n.startswith(("w_gate_", "w_up_", "w_down_"))] + [self.fc]
            codes = {n: (self._buf((self.shapes[n][0], api.i8_pitch(self.shapes[n][1])), torch.int8), self._buf(self.shapes[n][0], torch.float32)) for n in names}
            torch.cuda.current_stream(self.device).synchronize()
            self.i8_written, self.i8_read = None, {}        # events: the last codes, and each stream's last answer
        stream = self._stream_object(stream)
        with torch.cuda.stream(stream):
            captured = torch.cuda.is_current_stream_capturing()
            if not captured:
                for event in ([self.i8_written] if self.i8_written else []) + list(self.i8_read.values()):
                    stream.wait_event(event)
                self.i8_read = {}
            for n, (q, s) in codes.items():
                api.jz_quantize_i8(*self.shapes[n], self._param(self.w16, n), q, s)
            if not captured:
                self.i8_written = stream.record_event()
        self.i8 = codes

    def _stream_object(self, stream):
        if stream is None:
            return torch.cuda.current_stream(self.device)
        if hasattr(stream, "cuda_stream"):
            return stream
        return torch.cuda.ExternalStream(int(stream), self.device) if int(stream) else torch.cuda.default_stream(self.device)

    def answer(self, x: torch.Tensor, stream=None, i8: bool = False) -> torch.Tensor:
        """Logits (float16) of the rows of x (float32 [any number of rows, width], or tokens as set_tokens takes them), nothing kept for a backward pass; i8: with the codes of
        prepare_answers_i8.  x is as the current stream leaves it; the logits are ready once `stream` is (None: the current one)."""
        if i8 and self.i8 is None:
            raise ValueError("prepare_answers_i8 comes first")
        if self.vocab and x.is_floating_point():
            raise ValueError("the network's rows are tokens")
        current, one = torch.cuda.current_stream(self.device), self.i8_lock if i8 else contextlib.nullcontext()
        if stream is None or api._stream(stream) == api._stream(current):
            with one:
                return self._answer(x, i8)
        stream = self._stream_object(stream)
        stream.wait_stream(current)
        with one, torch.cuda.stream(stream):    # copies, temporaries and launches all belong to it
            logits = self._answer(x, i8)
        x.record_stream(stream)
        logits.record_stream(current)
        return logits

    def _answer(self, x, i8=False):
        """On the current stream."""
        rows, D, F = x.shape[0], self.width, self.hidden
        m = lambda n: self._param(self.master, n)
        ffn, around = api.ffn_desc(rows, D, F, D, api.JZ_ACT_SILU, api.JZ_F16), self._around(rows)
        n, y, k1, k2 = self._buf((rows, D)), self._buf((rows, D)), self._buf(rows, torch.float32), self._buf(rows, torch.float32)
        if self.vocab:
            r = self._buf((rows, D), torch.float32)
            api.jz_embed_fwd(self._embed(rows), _within_int32(x).to(torch.int32).contiguous(), self._param(self.w16, "embed"), r)
        else:
            r = x.to(torch.float32).clone()
        logits = self._buf((rows, self.classes))
        if i8:
            stream, captured = torch.cuda.current_stream(self.device), torch.cuda.is_current_stream_capturing()
            if not captured:
                stream.wait_event(self.i8_written)
            fc = api.linear_i8_desc(rows, D, self.classes, api.JZ_F16)
            ws = self._buf(max(16, api.jz_ffn_i8_workspace_bytes(ffn), api.jz_linear_i8_workspace_bytes(fc)), torch.uint8)
        else:
            h = self._buf((rows, F))
            ws = self._buf(max(16, api.jz_ffn_fwd_workspace_bytes(ffn), api.jz_gemm_fc_workspace_bytes(api.JZ_FWD, rows, D, self.classes)), torch.uint8)
        api.jz_norm_residual_fwd(around, r, None, None, None, m("w_pre_0"), None, n, None, k2)
        for i in range(self.blocks):
            if i8:
                api.jz_ffn_i8_fwd(ffn, n, *self.i8["w_gate_%d" % i], *self.i8["w_up_%d" % i], *self.i8["w_down_%d" % i], y, ws)
            else:
                api.jz_ffn_fwd(ffn, n, *self._ffn_weights(i), h, y, ws=ws)
            api.jz_norm_residual_fwd(around, r, y, m("w_post_%d" % i), m("gate_%d" % i), m("w_pre_%d" % (i + 1)), r, n, k1, k2)
        if i8:
            api.jz_linear_i8(fc, n, *self.i8[self.fc], logits, ws)
            if not captured:
                self.i8_read[stream.cuda_stream] = stream.record_event(self.i8_read.get(stream.cuda_stream))
        else:
            api.jz_gemm_fc(api.JZ_FWD, rows, D, self.classes, n, self._param(self.w16, self.fc), logits, ws)
        return logits
