"""Several requests over one pool of pages: bookkeeping, norms / rotation / append and their gradients, and
attention of one new token each (include/locret.h).  The calls themselves are in csrc/paged_module.cpp."""

from __future__ import annotations

import math

import torch

try:
    from . import _paged
except ImportError as e:
    raise ImportError(f"the calls on pages need the compiled module _paged.so, which is missing or was built for another torch or "
                      f"Python ({e}): run `python paper_2410_01805_b200/build.py`") from e
from ._paged import Pages, PagesStep, norm_rope, norm_rope_grad, paged_attention, pages_step  # noqa: F401
from .binding import LocretError

_paged.LocretError = LocretError   # what the calls raise for an error code of the library


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
        high = min(rot - 1.0, math.ceil(pair(s.get("beta_slow", 1.0))))   # (behind the last pair, if all turn that often)
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

