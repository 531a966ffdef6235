"""Several requests over one pool of pages: bookkeeping, norms / rotation / append and their gradients, and
attention of one new token each (include/locret.h)."""

from __future__ import annotations

import ctypes as C
import math
from typing import NamedTuple

import torch

from .binding import _check, lib, locret_pages, locret_rope_args

_DTYPES = {torch.bfloat16: 0, torch.float16: 1}


def _on_current_device(t: torch.Tensor, what: str) -> int:
    """The current stream's handle; the tensors of a call live on the current device."""
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what} must be a tensor of the current CUDA device")
    return torch.cuda.current_stream().cuda_stream


def _words(t: torch.Tensor, dtype, dim: int, what: str, like: torch.Tensor):
    if t.dtype != dtype or t.dim() != dim or t.device != like.device or (dim and t.stride(-1) != 1 and t.shape[-1] > 1):
        raise ValueError(f"{what} must be a {dtype} tensor of {dim} dimension(s) on {like.device}, contiguous in the last one")
    return t.data_ptr()


def _status(status, like):
    return None if status is None else _words(status.view(-1), torch.int32, 1, "status", like)


class Pages:
    """One layer's pool: keys and values [n_pages, n_kv_heads, page_size, head_dim], bf16 or fp16, views of any layout
    (the same for both) whose last dimension is contiguous."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device:
            raise ValueError("keys and values must be alike: [n_pages, n_kv_heads, page_size, head_dim]")
        if k.dtype not in _DTYPES or not k.is_cuda or k.stride(3) != 1:
            raise ValueError("pages must be CUDA bfloat16 or float16 tensors, contiguous in the last dimension")
        self.k, self.v = k, v
        n, hk, size, d = k.shape
        self.c = locret_pages(k.data_ptr(), v.data_ptr(), n, size, hk, d, _DTYPES[k.dtype], *k.stride()[:3])


class PagesStep(NamedTuple):
    slots: torch.Tensor      # int64 [n_tok]: page * page_size + offset, -1 where a row has no place
    positions: torch.Tensor  # int32 [n_tok]
    starts: torch.Tensor     # int32 [n_req + 1]: first row of every request
    lens: torch.Tensor       # int32 [n_req]: lengths after the step
    n_free: torch.Tensor     # int32 [1]


def pages_step(table: torch.Tensor, lens: torch.Tensor, new_lens: torch.Tensor, free_pages: torch.Tensor, n_free: torch.Tensor,
               page_size: int, n_tok: int, lens_out: torch.Tensor | None = None, n_free_out: torch.Tensor | None = None,
               status: torch.Tensor | None = None) -> PagesStep:
    """One step's bookkeeping: table int32 [n_req, width], lens, new_lens int32 [n_req] (< 0: the request has ended), free_pages
    int32 [number of pages], n_free int32 [1].  table and free_pages are updated in place, lens and n_free too unless lens_out
    and n_free_out are given."""
    stream = _on_current_device(table, "table")
    n, width = table.shape
    if lens.numel() != n or new_lens.numel() != n or n_free.numel() != 1:
        raise ValueError("one length and one number of new tokens for every row of the table, and one n_free")
    lens_out = lens if lens_out is None else lens_out
    n_free_out = n_free if n_free_out is None else n_free_out
    if lens_out.numel() != n or n_free_out.numel() != 1 or n_tok < 0:
        raise ValueError("lens_out and n_free_out must have the sizes of lens and n_free, and n_tok be >= 0")
    slots = torch.empty(n_tok, dtype=torch.int64, device=table.device)
    words = torch.empty(n_tok + n + 1, dtype=torch.int32, device=table.device)
    positions, starts = words[:n_tok], words[n_tok:]
    i32 = torch.int32
    _check(lib.locret_pages_step(_words(table, i32, 2, "table", table), table.stride(0), width,
                                 _words(lens, i32, 1, "lens", table), _words(lens_out, i32, 1, "lens_out", table),
                                 _words(new_lens, i32, 1, "new_lens", table), n, page_size,
                                 _words(free_pages, i32, 1, "free_pages", table), free_pages.numel(),
                                 _words(n_free, i32, 1, "n_free", table), _words(n_free_out, i32, 1, "n_free_out", table),
                                 n_tok, slots.data_ptr(), positions.data_ptr(), starts.data_ptr(), _status(status, table),
                                 stream), "locret_pages_step")
    return PagesStep(slots, positions, starts, lens_out, n_free_out)


def rope_turns(rot: int, theta: float, scaling: dict | None = None, device="cuda"):
    """(turns, factor) of locret_norm_rope for a rotation of `rot` elements with base `theta`: pair i turns by
    theta^(-2i / rot) radians per position, kept in 64 bits as a fraction of a turn.  scaling, for contexts beyond the trained
    one (original_max_position):

    {"type": "linear", "factor"}           positions divided by factor
    {"type": "ntk", "factor"}              base raised to theta * factor^(rot / (rot - 2))
    {"type": "llama3", "factor", "low_freq_factor", "high_freq_factor", "original_max_position"}
                                           waves longer than original / low divided by factor, those shorter than
                                           original / high kept, between them a linear mix
    {"type": "yarn", "factor", "original_max_position", "beta_fast" (32), "beta_slow" (1), "attention_factor"}
                                           pairs that turn less than beta_slow times within the original context divided by
                                           factor, those that turn more than beta_fast times kept, a linear ramp over the
                                           pairs between; cosines and sines times 0.1 ln(factor) + 1
    {"type": "longrope", "factors", "factor", "original_max_position", "attention_factor"}
                                           pair i divided by factors[i]; cosines and sines times
                                           sqrt(1 + ln(factor) / ln(original))
    """
    if rot % 2 or rot < 2 or not theta > 0:
        raise ValueError("rot must be a positive even number and theta positive")
    half, factor = rot // 2, 1.0
    s = dict(scaling or {"type": "none"})
    kind = s.get("type", "none")
    if kind != "none" and kind != "longrope" and not s.get("factor", 0) > 0:
        raise ValueError("scaling needs a positive factor")
    if kind == "ntk":
        if rot == 2:
            raise ValueError("ntk scaling needs more than one pair")
        theta = theta * s["factor"] ** (rot / (rot - 2))
    f = [theta ** (-i / half) for i in range(half)]
    if kind == "linear":
        f = [x / s["factor"] for x in f]
    elif kind == "llama3":
        low, high, original = s["low_freq_factor"], s["high_freq_factor"], s["original_max_position"]
        if not high > low:
            raise ValueError("high_freq_factor must be above low_freq_factor")
        keep = [min(1.0, max(0.0, (original * x / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [x * (m + (1.0 - m) / s["factor"]) for x, m in zip(f, keep)]
    elif kind == "yarn":
        original = s["original_max_position"]

        def pair(turns):   # the pair (a real number) that makes this many turns within the original context
            return half * math.log(original / (turns * 2 * math.pi)) / math.log(theta)
        low = max(0.0, math.floor(pair(s.get("beta_fast", 32.0))))
        high = min(half - 1.0, math.ceil(pair(s.get("beta_slow", 1.0))))
        ramp = [min(1.0, max(0.0, (i - low) / max(high - low, 1e-3))) for i in range(half)]
        f = [x * ((1.0 - r) + r / s["factor"]) for x, r in zip(f, ramp)]
        factor = s.get("attention_factor", 0.1 * math.log(s["factor"]) + 1.0 if s["factor"] > 1 else 1.0)
    elif kind == "longrope":
        if len(s["factors"]) != half or not all(x > 0 for x in s["factors"]):
            raise ValueError("one positive factor per pair")
        f = [x / y for x, y in zip(f, s["factors"])]
        if "attention_factor" in s:
            factor = s["attention_factor"]
        elif s.get("factor", 1.0) > 1.0:
            factor = math.sqrt(1.0 + math.log(s["factor"]) / math.log(s["original_max_position"]))
    elif kind not in ("none", "ntk"):
        raise ValueError(f"unknown scaling {kind!r}")
    turns = [int(round(x / (2 * math.pi) * 2.0 ** 64)) % 2 ** 64 for x in f]
    return torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], dtype=torch.int64, device=device), float(factor)


def _heads(t: torch.Tensor, what: str, like: torch.Tensor, shape=None):
    """(token stride, head stride) of [n_tok, heads, d]"""
    if t.dim() != 3 or t.dtype != like.dtype or t.device != like.device or t.stride(2) != 1 or (shape is not None and t.shape != shape):
        raise ValueError(f"{what} must be [n_tok, heads, d] of {like.dtype} on {like.device}, contiguous in the last dimension"
                         + (f", of shape {tuple(shape)}" if shape is not None else ""))
    return t.stride(0), t.stride(1)


def _rope_args(q, k, v, q_out, k_out, positions, turns, factor, interleaved, g_q, g_k, eps, pages, slots, status):
    n, h, d = q_out.shape
    for g, what in ((g_q, "g_q"), (g_k, "g_k")):
        if g is not None and (g.shape != (d,) or g.dtype != q_out.dtype or g.device != q_out.device or not g.is_contiguous()):
            raise ValueError(f"{what} must be a contiguous vector of {d} elements of {q_out.dtype}")
    if positions.shape != (n,) or (slots is not None and slots.shape != (n,)):
        raise ValueError("one position (and one slot) per token")
    none = (0, 0)
    k_like = k_out if k_out is not None else k
    return locret_rope_args(
        q.data_ptr() if q is not None else None, k.data_ptr() if k is not None else None,
        v.data_ptr() if v is not None else None, q_out.data_ptr(), k_out.data_ptr() if k_out is not None else None,
        *(_heads(q, "q", q_out, q_out.shape) if q is not None else none),
        *(_heads(k, "k", q_out) if k is not None else none),
        *(_heads(v, "v", q_out, k_like.shape) if v is not None else none),
        *_heads(q_out, "q_out", q_out), *(_heads(k_out, "k_out", q_out) if k_out is not None else none),
        _words(positions, torch.int32, 1, "positions", q_out), _words(turns, torch.int64, 1, "turns", q_out),
        g_q.data_ptr() if g_q is not None else None, g_k.data_ptr() if g_k is not None else None,
        C.pointer(pages.c) if pages is not None else None,
        _words(slots, torch.int64, 1, "slots", q_out) if slots is not None else None, _status(status, q_out),
        n, h, k_like.shape[1], d, 2 * turns.numel(), int(bool(interleaved)), _DTYPES.get(q_out.dtype, -1), factor, eps)


def norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, turns: torch.Tensor, factor: float = 1.0,
              interleaved: bool = False, g_q: torch.Tensor | None = None, g_k: torch.Tensor | None = None, eps: float = 1e-6,
              q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None, v: torch.Tensor | None = None,
              pages: Pages | None = None, slots: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """Per-head RMS norm (with gains g_q, g_k, if given), rotation at `positions` (int32 [n_tok]) and, with pages, the rotated
    keys and the values into `slots`: q [n_tok, h, d], k and v [n_tok, h_kv, d], of any token and head strides -> (q_out, k_out).
    Outputs are allocated where none are given, k_out only without pages; q_out may be q and k_out k.  turns, factor: of
    rope_turns."""
    stream = _on_current_device(q, "q")
    if k.dim() != 3 or q.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        raise ValueError("q and k must be [n_tok, heads, d], with the same tokens and head size")
    if (pages is None) != (v is None) or (pages is None) != (slots is None):
        raise ValueError("pages, v and slots come together")
    if pages is not None and pages.k.device != q.device:
        raise ValueError("pages must lie on the device of q")
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k_out is None and pages is None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    if q_out.shape != q.shape or (k_out is not None and k_out.shape != k.shape):
        raise ValueError("outputs must have the shapes of q and k")
    args = _rope_args(q, k, v, q_out, k_out, positions, turns, factor, interleaved, g_q, g_k, eps, pages, slots, status)
    _check(lib.locret_norm_rope(C.byref(args), stream), "locret_norm_rope")
    return q_out, k_out


def norm_rope_grad(dq_out: torch.Tensor, dk_out: torch.Tensor, q: torch.Tensor | None, k: torch.Tensor | None,
                   positions: torch.Tensor, turns: torch.Tensor, factor: float = 1.0, interleaved: bool = False,
                   g_q: torch.Tensor | None = None, g_k: torch.Tensor | None = None, eps: float = 1e-6):
    """Gradients of norm_rope from those of its outputs: (dq, dk, dg_q, dg_k), the latter fp32 [d] where a gain is given and
    None elsewhere.  q and k are the inputs of the forward call, needed where there is a gain."""
    stream = _on_current_device(dq_out, "dq_out")
    if dq_out.dim() != 3 or dk_out.dim() != 3 or dk_out.shape[0] != dq_out.shape[0] or dk_out.shape[2] != dq_out.shape[2]:
        raise ValueError("dq_out and dk_out must be [n_tok, heads, d], with the same tokens and head size")
    if (g_q is not None and q is None) or (g_k is not None and k is None) or (k is not None and k.shape != dk_out.shape):
        raise ValueError("q and k must be the forward call's inputs where there is a norm")
    d, dev = dq_out.shape[2], dq_out.device
    args = _rope_args(q, k, None, dq_out, dk_out, positions, turns, factor, interleaved, g_q, g_k, eps, None, None, None)
    dq = torch.empty(dq_out.shape, dtype=dq_out.dtype, device=dev)
    dk = torch.empty(dk_out.shape, dtype=dk_out.dtype, device=dev)
    dg_q = torch.empty(d, dtype=torch.float32, device=dev) if g_q is not None else None
    dg_k = torch.empty(d, dtype=torch.float32, device=dev) if g_k is not None else None
    need, ws = C.c_int64(), None
    if dg_q is not None or dg_k is not None:
        _check(lib.locret_norm_rope_grad_workspace(d, C.byref(need)), "locret_norm_rope_grad")
        ws = torch.empty(need.value, dtype=torch.uint8, device=dev)
    _check(lib.locret_norm_rope_grad(C.byref(args), dq.data_ptr(), dk.data_ptr(),
                                     dg_q.data_ptr() if dg_q is not None else None,
                                     dg_k.data_ptr() if dg_k is not None else None,
                                     ws.data_ptr() if ws is not None else None, need.value, stream), "locret_norm_rope_grad")
    return dq, dk, dg_q, dg_k


def paged_attention(q: torch.Tensor, pages: Pages, table: torch.Tensor, lens: torch.Tensor, scale: float | None = None,
                    window: int = 0, sinks: int = 0, out: torch.Tensor | None = None, with_lse: bool = False,
                    status: torch.Tensor | None = None):
    """Attention of each request's newest token, q [n_req, h, d], over the keys and values in its pages: table int32
    [n_req, width], lens int32 [n_req] (the new token counted).  window > 0: only the last `window` and the first `sinks`
    tokens are visible.  scale: 1 / sqrt(d) by default.  Returns out, [n_req, h, d], or (out, lse fp32 [n_req, h])."""
    stream = _on_current_device(q, "q")
    if q.dim() != 3 or pages.k.device != q.device or q.dtype != pages.k.dtype or q.shape[2] != pages.c.head_dim:
        raise ValueError("q must be [n_req, h, d] of the pages' type, head size and device")
    n, h, d = q.shape
    if table.shape[:1] != (n,) or lens.shape != (n,):
        raise ValueError("one row of the table and one length for every request")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty((n, h), dtype=torch.float32, device=q.device) if with_lse else None
    need = C.c_int64()
    _check(lib.locret_paged_attention_workspace(h, pages.c.n_kv_heads, d, C.byref(need)), "locret_paged_attention")
    ws = torch.empty(need.value, dtype=torch.uint8, device=q.device)
    _check(lib.locret_paged_attention(q.data_ptr(), *_heads(q, "q", q), C.byref(pages.c),
                                      _words(table, torch.int32, 2, "table", q), table.stride(0), table.shape[1],
                                      _words(lens, torch.int32, 1, "lens", q), n, h, d ** -0.5 if scale is None else scale,
                                      window, sinks, out.data_ptr(), *_heads(out, "out", q, q.shape),
                                      lse.data_ptr() if with_lse else None, _status(status, q), ws.data_ptr(), need.value,
                                      stream), "locret_paged_attention")
    return (out, lse) if with_lse else out
