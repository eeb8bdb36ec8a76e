"""Python binding of include/splice_tree.h: several candidate tokens per sweep cell in one pass.

A tree of T drafted tokens hangs below each cell's last token; each node is one row of a forward
pass.  ``splice_tree_append`` turns the nodes' q and k by their positions and writes their K/V
behind the cell's generated rows, ``splice_tree_attn`` attends, ``splice_token_scores`` tells what
the logits say about given tokens, and ``splice_tree_keep`` moves the accepted nodes' rows
together.  ``decode.SweepDecoder.score_tree`` runs them as one pass.

As in ``splice``, functions have the C names, marshal arguments only and check every tensor's
device, dtype, layout and size before calling into C; a negative status raises ``SpliceError``.
The kernels run on the current device: tensors of another one are refused.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional, Sequence, Tuple

import numpy as np

from . import splice as S

SPLICE_MAX_NODES, SPLICE_MAX_TOP = 64, 64
SPLICE_KV_BF16, SPLICE_KV_E4M3 = 0, 1
SPLICE_ROPE_HALF, SPLICE_ROPE_INTERLEAVED = 0, 1

EXPORTS = ("splice_tree_append", "splice_tree_read", "splice_tree_attn", "splice_tree_attn_workspace_bytes",
           "splice_tree_keep", "splice_token_scores", "splice_token_scores_workspace_bytes")


class SpliceTree(ctypes.Structure):
    _fields_ = [("n_nodes", ctypes.c_int32), ("kv_format", ctypes.c_int32)]


class SpliceRope(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("mscale", ctypes.c_double)]


_declared = None


def _library():
    """The library with the prototypes of include/splice_tree.h."""
    global _declared
    lib = S.load_library()
    if _declared is not lib:
        vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        shp, cal = ctypes.POINTER(S.SpliceShape), ctypes.POINTER(S.SpliceCall)
        tre, rop = ctypes.POINTER(SpliceTree), ctypes.POINTER(SpliceRope)
        for name, res, args in (
                ("splice_tree_append", i32, [shp, tre, rop] + [vp] * 4 + [vp, i64] * 3 + [vp] * 6),
                ("splice_tree_read", i32, [shp, tre] + [vp] * 8),
                ("splice_tree_attn_workspace_bytes", i64, [shp, cal, tre]),
                ("splice_tree_attn", i32, [shp, cal, tre] + [vp] * 16 + [size, vp]),
                ("splice_tree_keep", i32, [shp, tre] + [vp] * 7),
                ("splice_token_scores_workspace_bytes", i64, [i64, i64, i32]),
                ("splice_token_scores", i32, [vp, i32, i64, i64, i64, ctypes.c_float, vp, i32] + [vp] * 7 + [size, vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args   # (a structure passes by reference where its pointer is declared)
        _declared = lib
    return lib


# ------------------------------------------------------------------ structs, trees, frequencies

def make_tree(n_nodes: int, kv_format: str = "bf16") -> SpliceTree:
    """T nodes per cell over generated caches of ``kv_format``, "bf16" or "e4m3"."""
    return SpliceTree(n_nodes, {"bf16": SPLICE_KV_BF16, "e4m3": SPLICE_KV_E4M3}[kv_format])


def make_rope(layout: str, rotary_dim: int, mscale: float = 1.0) -> SpliceRope:
    """Rotary pairs (i, i + R / 2) ("half") or (2 i, 2 i + 1) ("interleaved") of a head's first ``rotary_dim`` = R values."""
    return SpliceRope({"half": SPLICE_ROPE_HALF, "interleaved": SPLICE_ROPE_INTERLEAVED}[layout], rotary_dim, float(mscale))


def tree_layout(parents) -> Tuple[np.ndarray, np.ndarray]:
    """(depth int32 [C][T], visible uint64 [C][T]) of trees given by each node's parent.

    parents[c][t]: the index of node t's parent, below t; -1 for a root (a child of the cell's last
    token); less than -1 for padding.  A node sees itself and its ancestors."""
    p = np.asarray(parents)
    if p.ndim != 2 or not np.issubdtype(p.dtype, np.integer):
        raise ValueError("parents is an integer array [C][T]")
    C, T = p.shape
    if not 1 <= T <= SPLICE_MAX_NODES:
        raise ValueError(f"a tree has 1 to {SPLICE_MAX_NODES} nodes, not {T}")
    depth, visible = np.full((C, T), -1, np.int32), np.zeros((C, T), np.uint64)
    cells = np.arange(C)
    for t in range(T):
        up = p[:, t]
        if (up >= t).any():
            raise ValueError(f"the parent of node {t} must come before it")
        inner = up >= 0
        if (depth[cells[inner], up[inner]] < 0).any():
            raise ValueError(f"the parent of node {t} is padding")
        here = up >= -1
        depth[here, t] = 0
        depth[inner, t] = depth[cells[inner], up[inner]] + 1
        visible[inner, t] = visible[cells[inner], up[inner]]
        visible[here, t] |= np.uint64(1) << np.uint64(t)
    return depth, visible


def rope_frequencies(rotary_dim: int, theta: float, scaling: Optional[str] = None, factor: float = 1.0,
                     original_len: int = 0, low_freq_factor: float = 1.0, high_freq_factor: float = 4.0,
                     beta_fast: float = 32.0, beta_slow: float = 1.0) -> Tuple[np.ndarray, float]:
    """(frequencies float64 [R / 2] in radians a position, mscale) of rotary positions.

    f_i = theta^(-2 i / R); scaled for contexts ``factor`` times ``original_len`` long by
      "linear"   f / factor;
      "banded"   f / factor where the wavelength 2 pi / f is over original_len / low_freq_factor, f where it is under
                 original_len / high_freq_factor, and in between (1 - s) f / factor + s f with s linear in
                 original_len / wavelength;
      "yarn"     f / factor for pairs of under beta_slow turns in original_len, f for over beta_fast, and between, with
                 i(n) = R ln(original_len / (2 pi n)) / (2 ln theta) the index whose pair makes n turns, a ramp that is linear
                 in the index from floor i(beta_fast) to ceil i(beta_slow), both within 0..R - 1, as models are trained
                 with it (YaRN, arXiv 2309.00071, has it linear in the turns); mscale = 0.1 ln(factor) + 1, its equation 22."""
    if rotary_dim < 0 or rotary_dim % 2:
        raise ValueError("rotary_dim is an even number")
    if not factor >= 1.0 or not theta > 1.0:
        raise ValueError("factor is at least 1 and theta above 1")
    i = np.arange(0, rotary_dim, 2, dtype=np.float64)
    f = np.float64(theta) ** (-i / max(rotary_dim, 1))
    if scaling is None:
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling not in ("banded", "yarn"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if original_len < 1:
        raise ValueError(f"{scaling} needs original_len")
    if scaling == "banded":
        if not high_freq_factor > low_freq_factor > 0:
            raise ValueError("high_freq_factor is above low_freq_factor, which is above 0")
        turns = original_len * f / (2 * math.pi)
        s = np.clip((turns - low_freq_factor) / (high_freq_factor - low_freq_factor), 0.0, 1.0)
        return (1 - s) * f / factor + s * f, 1.0
    if not beta_fast > beta_slow > 0:
        raise ValueError("beta_fast is above beta_slow, which is above 0")
    pair = lambda turns: rotary_dim * math.log(original_len / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    low, high = max(math.floor(pair(beta_fast)), 0), min(math.ceil(pair(beta_slow)), max(rotary_dim - 1, 0))
    s = np.clip((i / 2 - low) / max(high - low, 1e-3), 0.0, 1.0)   # 0: as it was, 1: by factor
    return (1 - s) * f + s * f / factor, 0.1 * math.log(factor) + 1.0


# ------------------------------------------------------------------ checks

def _anchor(t, name: str):
    """(device index, device) of the tensor that the others of a call are compared with: the current device, on which
    kernels are launched."""
    if t is None or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    index = t.get_device()
    if index != S._torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {t.device}, which is not the current device")
    return index, t.device


def _ptr(t, name: str, numel: int, dtype, dev) -> Optional[int]:
    """S._ptr, the usual case first: a call makes up to a dozen of these checks."""
    if t is not None and t.dtype is dtype and t.get_device() == dev[0] and t.numel() == numel > 0 and t.is_contiguous():
        return t.data_ptr()
    return S._ptr(t, name, numel, dtype, dev)


def _stream(stream, dev) -> int:
    if stream is None and S._current_raw_stream is not None:
        return S._current_raw_stream(dev[0])
    return S._stream_ptr(stream, dev[1])


_INT32 = np.dtype(np.int32)


def _host(x, rows: int, cols: int, name: str, what: str):
    """Host int32 values [rows][cols] as what ctypes passes the address of: a copy, for an array of that many a quicker one
    than asking for its address."""
    if type(x) is np.ndarray and x.dtype == _INT32 and x.size == rows * cols:
        return x.tobytes()
    return S._host_i32(x, rows, cols, name, what)[0].tobytes()


def _steps(cell_step, n_cells: int):
    return _host(cell_step, n_cells, 1, "cell_step", "entries")


def _caches(shape, tree, dev, gen_k, gen_v, gen_k_exp, gen_v_exp):
    n = shape.n_cells * shape.n_kv_heads * shape.gen_capacity
    if tree.kv_format != SPLICE_KV_E4M3:
        if gen_k_exp is not None or gen_v_exp is not None:
            raise ValueError("bf16 caches take no exponents")
        dt = S._torch.bfloat16
        return (_ptr(gen_k, "gen_k", n * shape.head_dim, dt, dev), _ptr(gen_v, "gen_v", n * shape.head_dim, dt, dev),
                None, None)
    u8 = S._torch.uint8
    return (_ptr(gen_k, "gen_k", n * shape.head_dim, u8, dev), _ptr(gen_v, "gen_v", n * shape.head_dim, u8, dev),
            _ptr(gen_k_exp, "gen_k_exp", n, u8, dev), _ptr(gen_v_exp, "gen_v_exp", n, u8, dev))


def _rows(t, name: str, shape, T: int, heads: int, dev) -> Tuple[int, int]:
    """(address, values from one token to the next) of bf16 [C][T][heads][D], tokens evenly apart, each one's heads dense."""
    D = shape.head_dim
    dims = (shape.n_cells, T, heads, D)
    if t is None or t.get_device() != dev[0]:
        raise ValueError(f"{name} must be a tensor on {dev[1]}")
    if t.dtype is not S._torch.bfloat16:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {S._torch.bfloat16}")
    if t.shape != dims:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {dims}")
    if t.is_contiguous():
        return t.data_ptr(), heads * D
    sc, st, sh, sd = t.stride()
    C = dims[0]
    if C * T == 1:
        st = heads * D
    elif T == 1:
        st = sc
    if (D > 1 and sd != 1) or (heads > 1 and sh != D) or (C > 1 and T > 1 and sc != T * st) or st < heads * D:
        raise ValueError(f"{name}: a token's heads must be dense and the tokens evenly apart")
    return t.data_ptr(), st


# ------------------------------------------------------------------ C entry points

def splice_tree_append(shape, tree, rope, freq, cell_step, depth, q, k, v, q_out, gen_k, gen_v, gen_k_exp=None,
                       gen_v_exp=None, pos=None, stream=None) -> None:
    """Rotate the nodes' ``q`` [C][T][Hq][D] into ``q_out`` and write their rotated ``k`` and their ``v``
    ([C][T][Hkv][D]) as rows s_c .. s_c + T - 1 of the generated caches (uint8 with exponents for "e4m3")."""
    lib = _library()
    dev = _anchor(q_out, "q_out")
    T, C = tree.n_nodes, shape.n_cells
    t, n_q = S._torch, C * T * shape.n_q_heads * shape.head_dim
    qo = _ptr(q_out, "q_out", n_q, t.bfloat16, dev)
    qp, qs = _rows(q, "q", shape, T, shape.n_q_heads, dev)
    kp, ks = _rows(k, "k", shape, T, shape.n_kv_heads, dev)
    vp, vs = _rows(v, "v", shape, T, shape.n_kv_heads, dev)
    dp = _ptr(depth, "depth", C * T, t.int32, dev)
    pp = None if pos is None else _ptr(pos, "pos", C * T, t.int64, dev)
    fp = None if rope.rotary_dim == 0 and freq is None else _ptr(freq, "freq", rope.rotary_dim // 2, t.float64, dev)
    stp = _steps(cell_step, C)
    S._check(lib.splice_tree_append(shape, tree, rope, stp, dp, pp, fp, qp, qs, kp, ks, vp, vs, qo,
                                    *_caches(shape, tree, dev, gen_k, gen_v, gen_k_exp, gen_v_exp), _stream(stream, dev)),
             "splice_tree_append")


def splice_tree_read(shape, tree, cell_step, gen_k, gen_v, gen_k_exp, gen_v_exp, rows_k, rows_v, stream=None) -> None:
    """``rows_k``, ``rows_v`` (bf16 [C][Hkv][T][D]) = rows s_c .. s_c + T - 1 of the generated caches."""
    lib = _library()
    dev = _anchor(rows_k, "rows_k")
    n = shape.n_cells * shape.n_kv_heads * tree.n_nodes * shape.head_dim
    rk, rv = (_ptr(x, name, n, S._torch.bfloat16, dev) for x, name in ((rows_k, "rows_k"), (rows_v, "rows_v")))
    stp = _steps(cell_step, shape.n_cells)
    S._check(lib.splice_tree_read(shape, tree, stp,
                                  *_caches(shape, tree, dev, gen_k, gen_v, gen_k_exp, gen_v_exp), rk, rv,
                                  _stream(stream, dev)), "splice_tree_read")


def splice_tree_attn_workspace_bytes(shape, call, tree) -> int:
    return S._check(_library().splice_tree_attn_workspace_bytes(shape, call, tree),
                    "splice_tree_attn_workspace_bytes")


def _workspace(workspace, dev) -> Tuple[Optional[int], int]:
    """(address, bytes) of a workspace; None, or an empty tensor, where none is needed."""
    if workspace is None:
        return None, 0
    n = workspace.numel()
    if n == 0:
        return None, 0
    if workspace.dtype is S._torch.uint8 and workspace.get_device() == dev[0] and workspace.is_contiguous():
        return workspace.data_ptr(), n
    return S._dev_ptr(workspace, "workspace", None, None, dev[1])[0], workspace.numel() * workspace.element_size()


def splice_tree_attn(shape, call, tree, cell_LW, cell_step, depth, visible, q, clean_k, clean_v, donor_k, donor_v, gen_k,
                     gen_v, gen_k_exp, gen_v_exp, out, lse, workspace, stream=None) -> None:
    """Spliced attention of every cell's nodes: ``out`` bf16 [C][T][Hq][D], ``lse`` float32 [C][T][Hq].

    ``depth`` int32 and ``visible`` int64 or uint64 [C][T] on the device (``tree_layout``)."""
    lib = _library()
    dev = _anchor(q, "q")
    t, C, T, Hq, D = S._torch, shape.n_cells, tree.n_nodes, shape.n_q_heads, shape.head_dim
    n_prompt, bf16 = shape.n_kv_heads * shape.prompt_len * D, t.bfloat16
    qp = _ptr(q, "q", C * T * Hq * D, bf16, dev)
    ck, cv = _ptr(clean_k, "clean_k", n_prompt, bf16, dev), _ptr(clean_v, "clean_v", n_prompt, bf16, dev)
    if shape.donor_kind == S.SPLICE_DONOR_ZERO:
        if donor_k is not None or donor_v is not None:
            raise ValueError("the ZERO donor takes no donor buffers")
        dk = dv = None
    else:
        dk, dv = _ptr(donor_k, "donor_k", n_prompt, bf16, dev), _ptr(donor_v, "donor_v", n_prompt, bf16, dev)
    gen = _caches(shape, tree, dev, gen_k, gen_v, gen_k_exp, gen_v_exp)
    dp = _ptr(depth, "depth", C * T, t.int32, dev)
    words = t.int64 if visible is None or visible.dtype is t.int64 else getattr(t, "uint64", t.int64)
    vp = _ptr(visible, "visible", C * T, words, dev)
    op, lp = _ptr(out, "out", C * T * Hq * D, bf16, dev), _ptr(lse, "lse", C * T * Hq, t.float32, dev)
    wp, wbytes = _workspace(workspace, dev)
    lwp, stp = _host(cell_LW, C, 2, "cell_LW", "rows"), _steps(cell_step, C)
    S._check(lib.splice_tree_attn(shape, call, tree, lwp, stp, dp, vp, qp, ck, cv,
                                  dk, dv, *gen, op, lp, wp, wbytes, _stream(stream, dev)), "splice_tree_attn")


def splice_tree_keep(shape, tree, cell_step, keep, gen_k, gen_v, gen_k_exp=None, gen_v_exp=None, stream=None) -> None:
    """Row s_c + i of the generated caches = row s_c + keep[c][i] (``keep`` int32 [C][T], ascending, ended by -1)."""
    lib = _library()
    dev = _anchor(keep, "keep")
    kp = _ptr(keep, "keep", shape.n_cells * tree.n_nodes, S._torch.int32, dev)
    stp = _steps(cell_step, shape.n_cells)
    S._check(lib.splice_tree_keep(shape, tree, stp, kp,
                                  *_caches(shape, tree, dev, gen_k, gen_v, gen_k_exp, gen_v_exp),
                                  _stream(stream, dev)), "splice_tree_keep")


def splice_token_scores_workspace_bytes(rows: int, vocab: int, k: int) -> int:
    return S._check(_library().splice_token_scores_workspace_bytes(rows, vocab, k), "splice_token_scores_workspace_bytes")


def splice_token_scores(logits, tokens, logp, lse, entropy, rank, top, top_logp, workspace, scale: float = 1.0,
                        stream=None) -> None:
    """Scores of ``tokens`` (int64 [rows]) under ``logits`` [rows][vocab] (bf16 or float32, rows any distance apart):
    ``logp``, ``lse``, ``entropy`` float32, ``rank`` int64, and the first k alternatives ``top`` (int64 [rows][k]) with
    ``top_logp`` (both None for none)."""
    lib = _library()
    dev = _anchor(logits, "logits")
    t = S._torch
    if logits.dtype not in (t.bfloat16, t.float32):
        raise ValueError(f"logits has dtype {logits.dtype}, expected bfloat16 or float32")
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits is a matrix with dense rows")
    rows, vocab = logits.shape
    stride = logits.stride(0) if rows > 1 else vocab
    if (top is None) != (top_logp is None):
        raise ValueError("top and top_logp come together")
    k = 0
    if top is not None:
        if top.dim() != 2 or top.shape[0] != rows:
            raise ValueError(f"top has shape {tuple(top.shape)}, expected ({rows}, k)")
        k = top.shape[1]
    f32, i64 = t.float32, t.int64
    tok, rk = _ptr(tokens, "tokens", rows, i64, dev), _ptr(rank, "rank", rows, i64, dev)
    out = [_ptr(x, name, rows, f32, dev) for x, name in ((logp, "logp"), (lse, "lse"), (entropy, "entropy"))]
    tp = tl = None
    if k:
        tp, tl = _ptr(top, "top", rows * k, i64, dev), _ptr(top_logp, "top_logp", rows * k, f32, dev)
    wp, wbytes = _workspace(workspace, dev)
    S._check(lib.splice_token_scores(logits.data_ptr(), S.SPLICE_BF16 if logits.dtype is t.bfloat16 else S.SPLICE_F32, rows,
                                     vocab, stride, float(scale), tok, k, *out, rk, tp, tl, wp, wbytes,
                                     _stream(stream, dev)), "splice_token_scores")


class TokenScores(NamedTuple):
    """What logits say about given tokens; ``top`` and ``top_logp`` are None when none were asked for."""
    logp: object
    lse: object
    entropy: object
    rank: object
    top: object
    top_logp: object


def token_scores(logits, tokens, top: int = 0, scale: float = 1.0) -> TokenScores:
    """``splice_token_scores`` on the current stream, with its outputs and workspace allocated by torch (whose
    memory is that stream's: for another one, ``with torch.cuda.stream(...)``)."""
    S.load_library()
    t, dev = S._torch, logits.device
    if logits.dim() != 2:
        raise ValueError("logits is a matrix")
    rows, vocab = logits.shape
    logp, lse, entropy = (t.empty(rows, dtype=t.float32, device=dev) for _ in range(3))
    rank = t.empty(rows, dtype=t.int64, device=dev)
    ids = t.empty((rows, top), dtype=t.int64, device=dev) if top else None
    vals = t.empty((rows, top), dtype=t.float32, device=dev) if top else None
    ws = t.empty(splice_token_scores_workspace_bytes(rows, vocab, top), dtype=t.uint8, device=dev)
    splice_token_scores(logits, tokens, logp, lse, entropy, rank, ids, vals, ws, scale)
    return TokenScores(logp, lse, entropy, rank, ids, vals)
