"""Greedy decode of a sweep around the spliced attention (Algorithm 1 of the
paper: per decode step one forward pass, which appends the step's K/V to the
generated cache and attends, then the argmax token; a trajectory stops at
EOS or T_max).

The decoder is a stand-in with synthetic weights (``workloads.model``):
pre-norm blocks of grouped-query attention and a gated MLP.  Per layer and
step the attention -- the current token's K/V appended to each cell's
generated cache, then single-query attention over the cell's spliced prompt
and its generated rows -- is one ``splice_decode_step`` launch of this
library's kernel. Around it, with dense bf16 weights on the GPU, what lies
between the products, the head, the argmax and the products it has better
tiles for are this library's kernels too (``include/splice_decoder.h``); the
other products, and passes with other weights, are PyTorch operations.
``SweepDecoder.score_tree`` is a pass over a tree of candidate tokens per cell
(``tree``): what the model says about each of them, without a pass per token.
``SweepDecoder.page_logits`` is a pass over caches in 4 bits, in pages that the
cells share (``pages``).

Readings of what the paper leaves to the model (the same on the CPU
reference in ``oracle.decoder``):
  * RMSNorm x / sqrt(mean(x^2) + eps) * gain; residual stream in float32;
  * rotary embedding on q and k, pairs (i, i + D/2), angle
    pos * theta^(-2i/D), position T_p + s for decode step s;
  * MLP down(silu(gate(h)) * up(h)); logits from the final norm;
  * the next token is the lowest index of the maximal logit; a cell that
    emits EOS stops (its step becomes -1) and is skipped from then on.
"""
from __future__ import annotations

import ctypes
from typing import List, NamedTuple, Optional

import numpy as np
import torch
from torch.autograd import forward_ad
from torch.utils._device import DeviceContext

from . import pages as P
from . import splice as S
from . import tree as T

ARGMAX_PARTS = 64   # SPLICE_ARGMAX_PARTS
_declared = None


def _library():
    """The library with the prototypes of include/splice_decoder.h."""
    global _declared
    lib = S.load_library()
    if _declared is not lib:
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        for name, args in (("residual", [vp, vp, vp, i64, i32, vp]),
                           ("norm", [vp, vp, vp, vp, i32, i32, ctypes.c_float, i32, vp]),
                           ("add_norm", [vp, vp, vp, vp, vp, i32, i32, ctypes.c_float, i32, vp]),
                           ("rope_table", [vp, vp, vp, i32, i32, i32, ctypes.c_double, vp]),
                           ("rope", [vp, vp, vp, i32, i32, i32, i32, vp]),
                           ("round", [vp, vp, i32, i32, i32, vp]),
                           ("silu", [vp, vp, vp, i32, i32, i32, vp]), ("product_takes", [i32, i32, i32]), ("head_takes", [i32, i32, i32]),
                           ("product", [vp, vp, vp, i32, i32, i32, vp]),
                           ("head", [vp, vp, vp, i32, i32, i32, vp, ctypes.c_size_t, vp]), ("argmax", [vp, i32, i32, vp, vp, vp])):
            f = getattr(lib, "splice_decoder_" + name)
            f.restype, f.argtypes = i32, args
        lib.splice_decoder_head_bytes.restype, lib.splice_decoder_head_bytes.argtypes = i64, [i32, i32, i32]
        _declared = lib
    return lib


def _unwatched() -> bool:
    """Whether nothing follows the operations of a pass but autograd's backward graph (see _plain): no function
    transform (vmap, jvp, ...), no forward-mode level, no tracer and no mode that sees each operation."""
    return not (torch._C._are_functorch_transforms_active() or forward_ad._current_level >= 0 or
                torch._C._len_torch_dispatch_stack() > 0 or torch._C._get_tracing_state() is not None or
                torch.compiler.is_compiling() or
                any(type(m) is not DeviceContext for m in torch.overrides._get_current_function_mode_stack()))


def _plain(t, device, *shape) -> bool:
    """A bf16 matrix of this shape on the device that autograd does not follow (any strides)."""
    return (type(t) in (torch.Tensor, torch.nn.Parameter) and t.dtype == torch.bfloat16 and t.device == device and
            t.layout == torch.strided and tuple(t.shape) == shape and not (t.requires_grad and torch.is_grad_enabled()))


def _columns(t) -> int:
    """Columns of a weight that is a matrix, else 0 (an object that only knows how to be multiplied, say)."""
    return t.shape[1] if isinstance(t, torch.Tensor) and t.dim() == 2 else 0


def _dense(t) -> bool:
    return t.is_contiguous() and t.data_ptr() % 16 == 0


def _current(device) -> bool:
    """Whether kernels are launched on this GPU: a launch goes to the current device, an operation to its tensors'."""
    return device.index == torch.cuda.current_device()


def greedy(logits: torch.Tensor) -> torch.Tensor:
    """The lowest index of the largest logit of every row (int64)."""
    if not (type(logits) is torch.Tensor and _unwatched() and logits.is_cuda and _current(logits.device) and
            logits.dim() == 2 and logits.is_contiguous() and logits.dtype == torch.float32 and
            0 < logits.shape[0] <= 65535 and 0 < logits.shape[1] <= 1 << 24):
        return torch.argmax(logits, dim=-1)
    n, vocab = logits.shape
    tokens = torch.empty(n, dtype=torch.int64, device=logits.device)
    keys = torch.empty(n * ARGMAX_PARTS, dtype=torch.int64, device=logits.device)
    S._check(_library().splice_decoder_argmax(logits.data_ptr(), n, vocab, tokens.data_ptr(), keys.data_ptr(),
                                              S._stream_ptr(None, logits.device)), "splice_decoder_argmax")
    return tokens


def rms_norm(x: torch.Tensor, gain: torch.Tensor, eps: float) -> torch.Tensor:
    xf = x.float()
    return xf * torch.rsqrt(xf.pow(2).mean(-1, keepdim=True) + eps) * gain.float()


def rope(x: torch.Tensor, pos: torch.Tensor, theta: float) -> torch.Tensor:
    """x [C][H][D] float32, pos [C]: rotate pairs (i, i + D/2) by pos * theta^(-2i/D)."""
    D = x.shape[-1]
    half = D // 2
    inv = theta ** (-torch.arange(0, half, device=x.device, dtype=torch.float64) * 2.0 / D)
    ang = (pos.to(torch.float64)[:, None] * inv[None, :]).to(torch.float32)   # [C][D/2]
    cos, sin = torch.cos(ang)[:, None, :], torch.sin(ang)[:, None, :]
    return _rotated(x, cos, sin)


def _rotated(x: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor) -> torch.Tensor:
    """x [..][D]: pairs (i, i + D/2) turned by the angles of cos, sin [..][D/2]."""
    half = x.shape[-1] // 2
    x1, x2 = x[..., :half], x[..., half:]
    return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1)


class DecoderTree(NamedTuple):
    """A tree per cell on the decoder's device (SweepDecoder.make_tree)."""
    spec: T.SpliceTree
    depth: torch.Tensor       # int32 [C][T]
    visible: torch.Tensor     # int64 [C][T]
    workspace: torch.Tensor   # of one pass at a time
    freq: torch.Tensor        # float64 [D / 2], of the rotary positions
    parents: np.ndarray       # int64 [C][T]


class DecoderPages(NamedTuple):
    """A cache in 4-bit pages on the decoder's device, and what passes of n tokens a cell over it need (SweepDecoder.make_pages)."""
    cache: P.PageCache
    spec: P.SplicePages
    depth: torch.Tensor       # int32 [C][n]: 0, 1, ...
    workspace: torch.Tensor   # of one pass at a time
    freq: torch.Tensor        # float64 [D / 2], of the rotary positions


def accept(parents: np.ndarray, tokens: np.ndarray, first: np.ndarray, best: np.ndarray):
    """(keep int32 [C][T], number int64 [C]) of the nodes of each cell that a greedy decode would have taken: a root whose
    token is first[c] (what the last pass chose), then, from node to node, a child whose token is best[c][t] (what
    the pass chose behind node t).  Of several children with that token the lowest index."""
    parents, tokens = np.asarray(parents), np.asarray(tokens)
    keep, number = np.full(parents.shape, -1, np.int32), np.zeros(parents.shape[0], np.int64)
    for c in range(parents.shape[0]):
        at, want = -1, first[c]
        while True:
            hits = np.flatnonzero((parents[c] == at) & (tokens[c] == want))
            if len(hits) == 0:
                break
            at = int(hits[0])
            keep[c, number[c]] = at
            number[c] += 1
            want = best[c][at]
    return keep, number


class SweepDecoder:
    """C sweep cells (L_c, W_c) decoding over one prompt, all N layers.

    ``weights`` as drawn by ``workloads.model.make_weights`` (on the device);
    ``caches[l]``: dict clean_k, clean_v, donor_k, donor_v (prompt caches of
    layer l, shared by the cells) and gen_k, gen_v ([C][Hkv][S][D], rows
    written by the decode itself)."""

    def __init__(self, w, m, weights, caches: List[dict], cell_LW, device="cuda"):
        self.w, self.m, self.wt, self.caches = w, m, weights, caches
        self.lw = np.ascontiguousarray(np.asarray(cell_LW, dtype=np.int32).reshape(-1, 2))
        C = self.lw.shape[0]
        self.C, self.N = C, len(weights["layers"])
        self.shape = S.make_shape(C, self.N, w.n_q_heads, w.n_kv_heads, w.head_dim, w.prompt_len, w.span,
                                  w.n_steps, w.donor == "zero", "bf16")
        self.ws = S.new_workspace(self.shape, device=device)
        self.out = torch.empty((C, w.n_q_heads, w.head_dim), dtype=torch.float32, device=device)
        self.lse = torch.empty((C, w.n_q_heads), dtype=torch.float32, device=device)
        self.calls = [S.make_call(l, 0, w.window(l), w.head_dim ** -0.5) for l in range(self.N)]
        self.device = device

    def positions(self, steps: np.ndarray) -> torch.Tensor:
        """Device positions T_p + s of the cells' current tokens."""
        return torch.as_tensor(self.w.prompt_len + np.maximum(steps, 0), device=self.device)

    def forward(self, tokens: torch.Tensor, steps: np.ndarray, pos: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Logits [C][V] (float32) of one decode pass; steps[c] < 0: finished.
        pos: the device positions (self.positions(steps)), given when the pass
        is captured in a graph."""
        w, m, wt = self.w, self.m, self.wt
        C, Hq, Hkv, D = self.C, w.n_q_heads, w.n_kv_heads, w.head_dim
        cdt = wt["embed"].dtype
        x = wt["embed"][tokens]
        if pos is None and getattr(self.positions, "__func__", None) is not SweepDecoder.positions:
            pos = self.positions(steps)   # not the T_p + s that the kernels compute
        if self._fused(x, pos):
            return self._forward_fused(x, steps, pos)
        x = x.float()
        if pos is None:
            pos = self.positions(steps)
        for l in range(self.N):
            p = wt["layers"][l]
            h = rms_norm(x, p["norm_1"], m.rms_eps).to(cdt)
            q = rope((h @ p["w_q"]).float().view(C, Hq, D), pos, m.rope_theta)
            k = rope((h @ p["w_k"]).float().view(C, Hkv, D), pos, m.rope_theta)
            v = (h @ p["w_v"]).float().view(C, Hkv, D)
            c = self.caches[l]
            S.splice_decode_step(self.shape, self.calls[l], self.lw, steps,
                                 q.to(torch.bfloat16).contiguous(), k.to(torch.bfloat16).contiguous(),
                                 v.to(torch.bfloat16).contiguous(), c["clean_k"], c["clean_v"], c["donor_k"],
                                 c["donor_v"], c["gen_k"], c["gen_v"], self.out, self.lse, self.ws)
            x = x + (self.out.view(C, Hq * D).to(cdt) @ p["w_o"]).float()
            h = rms_norm(x, p["norm_2"], m.rms_eps).to(cdt)
            x = x + ((torch.nn.functional.silu((h @ p["w_gate"]).float()).to(cdt) * (h @ p["w_up"]))
                     @ p["w_down"]).float()
        return (rms_norm(x, wt["norm_f"], m.rms_eps).to(cdt) @ wt["lm_head"]).float()

    def _fused(self, x: torch.Tensor, pos: Optional[torch.Tensor], rows: Optional[int] = None) -> bool:
        """Whether the library's kernels take this pass (x: the embedded tokens, a row per cell or ``rows``)."""
        w, wt = self.w, self.wt
        C, Hq, Hkv, D, dev, d = rows or self.C, w.n_q_heads, w.n_kv_heads, w.head_dim, x.device, x.shape[-1]
        if torch.is_autocast_enabled("cuda") and torch.get_autocast_dtype("cuda") != torch.bfloat16:
            return False   # the products are another type's
        if not (_unwatched() and x.is_cuda and _current(dev) and C > 0 and d % 8 == 0 and _plain(x, dev, C, d) and
                _dense(x) and (pos is None or (pos.device == dev and tuple(pos.shape) == (C,)))):
            return False
        for p in wt["layers"]:
            F = _columns(p["w_gate"])
            if not (F % 8 == 0 and F > 0 and _plain(p["w_gate"], dev, d, F) and _plain(p["w_up"], dev, d, F) and
                    _plain(p["w_down"], dev, F, d) and _plain(p["w_q"], dev, d, Hq * D) and
                    _plain(p["w_k"], dev, d, Hkv * D) and _plain(p["w_v"], dev, d, Hkv * D) and
                    _plain(p["w_o"], dev, Hq * D, d) and _plain(p["norm_1"], dev, d) and _dense(p["norm_1"]) and
                    _plain(p["norm_2"], dev, d) and _dense(p["norm_2"])):
                return False
        head = wt["lm_head"]
        return _plain(wt["norm_f"], dev, d) and _dense(wt["norm_f"]) and _plain(head, dev, d, _columns(head))

    def _forward_fused(self, delta: torch.Tensor, steps, pos: Optional[torch.Tensor]) -> torch.Tensor:
        """forward() with the library's kernels between the products: the same roundings, so the same bits up to the head."""
        w, m, wt, lib = self.w, self.m, self.wt, _library()
        C, Hq, Hkv, D, d, dev = self.C, w.n_q_heads, w.n_kv_heads, w.head_dim, delta.shape[1], delta.device
        bf16, stream = torch.bfloat16, S._stream_ptr(None, delta.device)
        ok = S._check
        # one kernel a norm where it adds in the order of mean(), so that the
        # bits stay: fewer rows, shorter and longer ones are added in others
        # (measured: 8184 values differ, 7680 do not)
        one_norm = C >= 8 and 256 <= d <= 7680
        x = torch.empty((C, d), dtype=torch.float32, device=dev)   # the residual stream
        sq = None if one_norm else torch.empty_like(x)
        h = torch.empty(((C + 15) // 16 * 16, d), dtype=bf16, device=dev)[:C]
        o = torch.empty((C, Hq * D), dtype=bf16, device=dev)
        tab = torch.empty((C, D), dtype=torch.float32, device=dev)
        xp, hp, op, tp, outp = (t.data_ptr() for t in (x, h, o, tab, self.out))
        st, stp = S._steps(steps, C)
        if pos is not None:
            pos = pos.to(torch.float64).contiguous()
        ok(lib.splice_decoder_rope_table(tp, None if pos is None else pos.data_ptr(), stp, C, D, w.prompt_len,
                                         float(m.rope_theta), stream), "splice_decoder_rope_table")

        def norm(delta, gain, assign=0, packed=0):
            """x += delta (the first: x = delta); h = bf16(rms_norm(x)), packed for the head (2: both, packed in hq)."""
            if one_norm:
                ok(lib.splice_decoder_add_norm(xp, delta.data_ptr(), gain.data_ptr(), None if packed == 1 else hp,
                                               (None, hp, hqp)[packed], C, d, m.rms_eps, assign, stream),
                   "splice_decoder_add_norm")
                return
            ok(lib.splice_decoder_residual(xp, delta.data_ptr(), sq.data_ptr(), C * d, assign, stream),
               "splice_decoder_residual")
            mean = sq.mean(-1, keepdim=True)
            ok(lib.splice_decoder_norm(xp, mean.data_ptr(), gain.data_ptr(), hp, C, d, m.rms_eps, packed, stream),
               "splice_decoder_norm")

        def own(w):
            """Whether the library's own product takes this weight."""
            return one_norm and _dense(w) and lib.splice_decoder_product_takes(C, w.shape[0], w.shape[1]) == 1

        def product(x_packed, w):
            y = torch.empty((C, w.shape[1]), dtype=bf16, device=dev)
            ok(lib.splice_decoder_product(x_packed, w.data_ptr(), y.data_ptr(), C, w.shape[0], w.shape[1], stream),
               "splice_decoder_product")
            return y

        hq = torch.empty_like(h) if any(own(p["w_q"]) for p in wt["layers"]) else h
        hqp = hq.data_ptr()
        first = 1
        for l in range(self.N):
            p, c = wt["layers"][l], self.caches[l]
            own_q, own_o, own_down = own(p["w_q"]), own(p["w_o"]), own(p["w_down"])
            norm(delta, p["norm_1"], first, 2 if own_q else 0)
            first = 0
            q = product(hqp, p["w_q"]) if own_q else h @ p["w_q"]
            k, v = h @ p["w_k"], h @ p["w_v"]
            ok(lib.splice_decoder_rope(q.data_ptr(), k.data_ptr(), tp, C, Hq, Hkv, D, stream), "splice_decoder_rope")
            S.splice_decode_step(self.shape, self.calls[l], self.lw, st, q, k, v, c["clean_k"], c["clean_v"],
                                 c["donor_k"], c["donor_v"], c["gen_k"], c["gen_v"], self.out, self.lse, self.ws)
            ok(lib.splice_decoder_round(outp, op, C, Hq * D, own_o, stream), "splice_decoder_round")
            norm(product(op, p["w_o"]) if own_o else o @ p["w_o"], p["norm_2"])
            gate, up = h @ p["w_gate"], h @ p["w_up"]
            act = torch.empty_like(gate) if own_down else gate
            ok(lib.splice_decoder_silu(gate.data_ptr(), up.data_ptr(), act.data_ptr(), C, gate.shape[1], own_down, stream),
               "splice_decoder_silu")
            delta = product(act.data_ptr(), p["w_down"]) if own_down else act @ p["w_down"]
        head = wt["lm_head"]
        vocab = head.shape[1]
        own_head = _dense(head) and lib.splice_decoder_head_takes(C, d, vocab) == 1
        norm(delta, wt["norm_f"], first, own_head)
        if not own_head:
            return (h @ head).float()
        logits = torch.empty((C, vocab), dtype=torch.float32, device=dev)
        need = ok(lib.splice_decoder_head_bytes(C, d, vocab), "splice_decoder_head_bytes")
        part = torch.empty(need, dtype=torch.uint8, device=dev)
        ok(lib.splice_decoder_head(hp, head.data_ptr(), logits.data_ptr(), C, d, vocab, part.data_ptr(), need, stream),
           "splice_decoder_head")
        return logits

    # ------------------------------------------------------------- trees of candidate tokens

    def _kv_format(self) -> str:
        kinds = {(c["gen_k"].dtype, c["gen_v"].dtype) for c in self.caches}
        if kinds == {(torch.bfloat16, torch.bfloat16)}:
            return "bf16"
        if kinds == {(torch.uint8, torch.uint8)}:
            return "e4m3"
        raise ValueError(f"generated caches are bfloat16, or uint8 with exponents, in every layer: got {kinds}")

    def make_tree(self, parents) -> DecoderTree:
        """Trees of T nodes per cell (``tree.tree_layout``: parents [C][T], -1 a root, less padding) for score_tree and
        keep_nodes.  Generated caches may be bfloat16, or uint8 (e4m3) with ``gen_k_exp`` and ``gen_v_exp`` (which
        ``step`` does not take).  Passes over one tree object share its workspace: order them on one stream."""
        parents = np.asarray(parents)
        depth, visible = T.tree_layout(parents)
        if depth.shape[0] != self.C:
            raise ValueError(f"parents has {depth.shape[0]} rows, the decoder {self.C} cells")
        spec = T.make_tree(depth.shape[1], self._kv_format())
        need = max((T.splice_tree_attn_workspace_bytes(self.shape, call, spec) for call in self.calls), default=0)
        return DecoderTree(spec, torch.from_numpy(depth).to(self.device), torch.from_numpy(visible.view(np.int64)).to(self.device),
                           torch.empty(need, dtype=torch.uint8, device=self.device),
                           torch.from_numpy(T.rope_frequencies(self.w.head_dim, float(self.m.rope_theta))[0]).to(self.device),
                           parents.astype(np.int64))

    def _node_positions(self, tree: DecoderTree, steps: np.ndarray) -> Optional[torch.Tensor]:
        """Positions [C][T] of the nodes where they are not T_p + step + depth (None): what a decoder's own positions() says of
        each node's step, asked depth by depth, as passes of one token would."""
        if getattr(self.positions, "__func__", None) is SweepDecoder.positions:
            return None
        most = max(int(T.tree_layout(tree.parents)[0].max(initial=0)), 0)
        pos = [self.positions(np.where(steps >= 0, steps + d, steps)) for d in range(most + 1)]
        pos = torch.stack(pos, 1).gather(1, tree.depth.clamp(min=0).to(torch.int64))
        return pos.to(torch.float64 if pos.is_floating_point() else torch.int64)

    def _turns(self, tree, steps: np.ndarray, pos: Optional[torch.Tensor]):
        """(cos, sin) float32 [C][T][1][D / 2] of the nodes' (or tokens') positions: pos [C][T], or T_p + step + depth, whose
        T_p + step is the cells' (from the steps by value, so that a pass can be captured), the depth's angle added to it."""
        C, D, (_, dev) = self.C, self.w.head_dim, T._anchor(tree.depth, "depth")
        ang = (tree.depth if pos is None else pos).to(torch.float64)[:, :, None, None] * tree.freq
        cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
        if pos is not None or C == 0:
            return cos, sin
        tab = torch.empty((C, 1, 1, D // 2, 2), dtype=torch.float32, device=dev)
        S._check(_library().splice_decoder_rope_table(tab.data_ptr(), None, S._steps(steps, C)[1], C, D, self.w.prompt_len,
                                                      float(self.m.rope_theta), S._stream_ptr(None, dev)),
                 "splice_decoder_rope_table")
        c, s = tab[..., 0], tab[..., 1]
        return c * cos - s * sin, s * cos + c * sin

    @torch.no_grad()
    def tree_logits(self, tokens: torch.Tensor, tree: DecoderTree, steps: np.ndarray) -> torch.Tensor:
        """Logits [C * T][V] of one pass over the trees' nodes (bfloat16 where the head's product is, else float32): node t
        of cell c is the token tokens[c][t] (int64) at decode step steps[c] + its depth (at the position that positions()
        gives for that step), behind the steps[c] rows of the cell's generated caches and its ancestors.  Its K/V become row
        steps[c] + t, so steps[c] + T must not pass the caches' rows; cells with a negative step are skipped.  Rows of
        padding and of skipped cells hold no meaning (their tokens are any of the vocabulary).  No gradients."""
        w = self.w
        C, Hq, Hkv, D, n = self.C, w.n_q_heads, w.n_kv_heads, w.head_dim, tree.spec.n_nodes
        if tuple(tokens.shape) != (C, n):
            raise ValueError(f"tokens has shape {tuple(tokens.shape)}, expected ({C}, {n})")
        st, _ = S._steps(steps, C)
        pos = self._node_positions(tree, st)
        x = self.wt["embed"][tokens.reshape(-1)]
        dev, bf16 = x.device, torch.bfloat16
        out = torch.zeros((C, n, Hq, D), dtype=bf16, device=dev)
        lse = torch.empty((C, n, Hq), dtype=torch.float32, device=dev)
        exps = ("gen_k_exp", "gen_v_exp") if tree.spec.kv_format == T.SPLICE_KV_E4M3 else ()
        turned = self._turner(tree, st, pos)

        def attend(l, q, k, v):
            c = self.caches[l]
            e = [c[name] for name in exps] or [None, None]
            q, k, v = q.view(C, n, Hq, D), k.view(C, n, Hkv, D), v.to(bf16).view(C, n, Hkv, D)
            q, k, rotary, freq, at = turned(q, k)
            T.splice_tree_append(self.shape, tree.spec, rotary, freq, st, tree.depth, q, k, v, q, c["gen_k"], c["gen_v"], *e, pos=at)
            T.splice_tree_attn(self.shape, self.calls[l], tree.spec, self.lw, st, tree.depth, tree.visible, q, c["clean_k"],
                               c["clean_v"], c["donor_k"], c["donor_v"], c["gen_k"], c["gen_v"], *e, out, lse, tree.workspace)
            return out.view(C * n, Hq * D)

        return self._pass(x, attend)

    def _turner(self, tree, st: np.ndarray, pos: Optional[torch.Tensor]):
        """What a pass's entries take of q and k [C][n][..][D]: (q, k, rope, freq, pos)."""
        D, bf16 = self.w.head_dim, torch.bfloat16
        rope_of, unturned, whole = T.make_rope("half", D), T.make_rope("half", 0), pos is None or not pos.is_floating_point()
        turns = None   # (cos, sin) of the positions, where products of other types need them

        def turned(q, k):
            nonlocal turns
            # of more bits: rotated before they are rounded, as in forward; and the kernel's positions are whole numbers
            if q.dtype != bf16 or k.dtype != bf16 or not whole:
                turns = turns or self._turns(tree, st, pos)
                return *(_rotated(y.float(), *turns).to(bf16) for y in (q, k)), unturned, None, None
            return q, k, rope_of, tree.freq, pos
        return turned

    def _pass(self, x: torch.Tensor, attend) -> torch.Tensor:
        """Logits [rows][V] of embedded tokens x [rows][d]; attend(l, q, k, v): the layer's attention over them."""
        m, wt = self.m, self.wt
        cdt, dev, rows, bf16 = x.dtype, x.device, x.shape[0], torch.bfloat16
        fused = self._fused(x, None, rows) and x.shape[1] <= 8192   # SPLICE_ADD_NORM_MAX_D

        if not fused:
            x = x.float()
            for l in range(self.N):
                p = wt["layers"][l]
                h = rms_norm(x, p["norm_1"], m.rms_eps).to(cdt)
                x = x + (attend(l, h @ p["w_q"], h @ p["w_k"], h @ p["w_v"]).to(cdt) @ p["w_o"]).float()
                h = rms_norm(x, p["norm_2"], m.rms_eps).to(cdt)
                x = x + ((torch.nn.functional.silu((h @ p["w_gate"]).float()).to(cdt) * (h @ p["w_up"])) @ p["w_down"]).float()
            logits = rms_norm(x, wt["norm_f"], m.rms_eps).to(cdt) @ wt["lm_head"]
            return logits if logits.dtype in (bf16, torch.float32) else logits.float()   # (what splice_token_scores takes)

        lib, ok, stream, d = _library(), S._check, S._stream_ptr(None, dev), x.shape[1]
        res, h = torch.empty((rows, d), dtype=torch.float32, device=dev), torch.empty((rows, d), dtype=bf16, device=dev)

        def norm(delta, gain, assign=0):
            ok(lib.splice_decoder_add_norm(res.data_ptr(), delta.data_ptr(), gain.data_ptr(), h.data_ptr(), None, rows, d,
                                           m.rms_eps, assign, stream), "splice_decoder_add_norm")

        delta, first = x, 1
        for l in range(self.N):
            p = wt["layers"][l]
            norm(delta, p["norm_1"], first)
            first = 0
            norm(attend(l, h @ p["w_q"], h @ p["w_k"], h @ p["w_v"]) @ p["w_o"], p["norm_2"])
            gate, up = h @ p["w_gate"], h @ p["w_up"]
            ok(lib.splice_decoder_silu(gate.data_ptr(), up.data_ptr(), gate.data_ptr(), rows, gate.shape[1], 0, stream),
               "splice_decoder_silu")
            delta = gate @ p["w_down"]
        norm(delta, wt["norm_f"], first)
        return h @ wt["lm_head"]

    def score_tree(self, tokens: torch.Tensor, tree: DecoderTree, steps: np.ndarray, targets: torch.Tensor, top: int = 0,
                   scale: float = 1.0) -> T.TokenScores:
        """What the model says behind every node of the trees (tree_logits): log probability, entropy, rank of the token
        targets[c][t] (int64 [C][T]), and the ``top`` most probable tokens; fields [C][T] and [C][T][top].  scale: an
        inverse temperature."""
        if targets.shape != tokens.shape:
            raise ValueError(f"targets has shape {tuple(targets.shape)}, tokens {tuple(tokens.shape)}")
        logits = self.tree_logits(tokens, tree, steps)
        got = T.token_scores(logits, targets.reshape(-1).contiguous(), top, scale)
        shape = (self.C, tree.spec.n_nodes)
        return T.TokenScores(*(None if f is None else f.view(*shape, *f.shape[1:]) for f in got))

    def keep_nodes(self, tree: DecoderTree, steps: np.ndarray, keep: torch.Tensor) -> None:
        """Move the K/V of each cell's nodes keep[c] (int32 [C][T], ascending, ended by -1: ``accept``) to its rows
        steps[c], steps[c] + 1, ... in every layer: the decode goes on at steps[c] + their number."""
        if tuple(keep.shape) != (self.C, tree.spec.n_nodes):
            raise ValueError(f"keep has shape {tuple(keep.shape)}, expected ({self.C}, {tree.spec.n_nodes})")
        for c in self.caches:
            e = [c[name] for name in ("gen_k_exp", "gen_v_exp")] if tree.spec.kv_format == T.SPLICE_KV_E4M3 else []
            T.splice_tree_keep(self.shape, tree.spec, steps, keep, c["gen_k"], c["gen_v"], *e)

    # ------------------------------------------------------------- caches in 4-bit pages

    def make_pages(self, n_tokens: int = 1, n_pages: Optional[int] = None, cache: Optional[P.PageCache] = None) -> DecoderPages:
        """A cache in 4-bit pages for passes of ``n_tokens`` tokens a cell (``page_logits``), the prompts of ``caches`` in it,
        or passes of another number of tokens over the cache of an earlier one.  ``n_pages``: pages of each layer, by default
        as many as they and all cells can fill.  Passes over one object share its workspace: order them on one stream."""
        w, dev = self.w, self.device
        if cache is None:
            prompt, rows = -(-w.prompt_len // P.SPLICE_PAGE_ROWS) * (1 if w.donor == "zero" else 2), -(-w.n_steps // P.SPLICE_PAGE_ROWS)
            cache = P.PageCache(self.C, self.N, w.n_q_heads, w.n_kv_heads, w.head_dim, w.prompt_len, w.span, w.n_steps,
                                prompt + self.C * rows if n_pages is None else n_pages, w.donor == "zero", dev)
            for l, c in enumerate(self.caches):
                cache.load_prompt(l, c["clean_k"], c["clean_v"])
                if w.donor != "zero":
                    cache.load_prompt(l, c["donor_k"], c["donor_v"], donor=True)
        spec = cache.pages(n_tokens)
        need = max((P.splice_page_attn_workspace_bytes(cache.shape, call, spec) for call in self.calls), default=0)
        depth = torch.arange(n_tokens, dtype=torch.int32, device=dev).repeat(self.C, 1)
        return DecoderPages(cache, spec, depth, torch.empty(need, dtype=torch.uint8, device=dev),
                            torch.from_numpy(T.rope_frequencies(w.head_dim, float(self.m.rope_theta))[0]).to(dev))

    @torch.no_grad()
    def page_logits(self, tokens: torch.Tensor, pages: DecoderPages, steps: np.ndarray, new=None) -> torch.Tensor:
        """Logits [C * n][V] (bfloat16 where the head's product is, else float32) of one pass over n tokens a cell: token t of
        cell c is tokens[c][t] (int64) at decode step steps[c] + t, behind the cell's steps[c] rows and the tokens before it;
        its K/V become row steps[c] + t, for which the cell has its pages (``pages.cache.reserve``, ``fork``: tokens behind
        ``pages.cache.rows`` are refused, and a steps[c] in a page that other cells have too).  ``new``: how many tokens each cell
        has (host int32 [C]; all n without); cells with a negative step are skipped.  Logits of skipped cells and of tokens behind
        new[c] hold no meaning.  No gradients."""
        w, cache = self.w, pages.cache
        C, Hq, Hkv, D, n = self.C, w.n_q_heads, w.n_kv_heads, w.head_dim, pages.spec.n_tokens
        if tuple(tokens.shape) != (C, n):
            raise ValueError(f"tokens has shape {tuple(tokens.shape)}, expected ({C}, {n})")
        st, _ = S._steps(steps, C)
        cache._check_rows(st, np.int32(n) if new is None else S._host_i32(new, C, 1, "new", "entries")[0])
        pos = None
        if getattr(self.positions, "__func__", None) is not SweepDecoder.positions:   # a decoder's own, asked step by step
            # (none is asked for behind a cell's last token)
            last = n - 1 if new is None else np.maximum(np.asarray(new).reshape(-1), 1) - 1
            pos = torch.stack([self.positions(np.where(st >= 0, st + np.minimum(t, last), st).astype(np.int32)) for t in range(n)], 1)
            pos = pos.to(torch.float64 if pos.is_floating_point() else torch.int64)
        x = self.wt["embed"][tokens.reshape(-1)]
        bf16 = torch.bfloat16
        out = torch.zeros((C, n, Hq, D), dtype=bf16, device=x.device)
        lse = torch.empty((C, n, Hq), dtype=torch.float32, device=x.device)
        turned = self._turner(pages, st, pos)

        def attend(l, q, k, v):
            q, k, v = q.view(C, n, Hq, D), k.view(C, n, Hkv, D), v.to(bf16).view(C, n, Hkv, D)
            q, k, rotary, freq, at = turned(q, k)
            pool = cache.pools[l]
            P.splice_page_append(cache.shape, pages.spec, rotary, freq, st, new, cache.tables, q, k, v, q, pool, pos=at)
            P.splice_page_attn(cache.shape, self.calls[l], pages.spec, self.lw, st, new, cache.tables, cache.clean_table,
                               cache.donor_table, q, pool, out, lse, pages.workspace)
            return out.view(C * n, Hq * D)

        return self._pass(x, attend)

    def step(self, tokens: torch.Tensor, steps: np.ndarray, pos: Optional[torch.Tensor] = None):
        """One decode pass: (next tokens [C] int64, logits [C][V]); of equal
        largest logits the lowest index."""
        logits = self.forward(tokens, steps, pos)
        return greedy(logits), logits


def advance(steps: np.ndarray, next_tokens: np.ndarray, eos: int, n_steps: int) -> np.ndarray:
    """The cells' steps after a pass: +1, or -1 for a cell that emitted EOS or
    reached T_max (= the generated-cache capacity)."""
    s = steps.copy()
    act = s >= 0
    s[act] += 1
    s[act & (next_tokens == eos)] = -1
    s[s >= n_steps] = -1
    return s
