"""The calls around a decode step (rotation, bounds and choice of blocks), from their definitions, in 64 bits or whole
numbers on the CPU. Shares no code with the package."""
from __future__ import annotations

import math

import numpy as np
import torch


def positions(offsets, context):
    """(row, position) of every row that belongs to a sequence."""
    out = []
    for r in range(len(offsets) - 1):
        out += [(t, max(0, context[r]) + t - offsets[r]) for t in range(offsets[r], offsets[r + 1])]
    return out


def rotate(x, position, freq, interleaved, magnitude, norm, eps):
    """x [H, D] float64 of one token. Returns its rows, and for every element the sum of magnitudes that goes into it."""
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * norm.double()
    rot = 0 if freq is None else 2 * len(freq)
    out, size = x.clone(), x.abs()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        # the angle as defined: a product in 64 bits
        angle = float(position) * float(freq[i])
        c, s = magnitude * math.cos(angle), magnitude * math.sin(angle)
        out[:, a], out[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
        size[:, a] = size[:, b] = (x[:, a].abs() + x[:, b].abs()) * abs(magnitude)
    return out, size


def rotate_bound(out, size, dtype, dim, position):
    """|computed - exact|: the rounding to the type (half a step: 2^-8 or 2^-11 of the number, or half a float16
    subnormal) of a number that is itself off by: the norm, a sum of dim squares (dim 2^-24 of it, halved by the root)
    and five more operations; the cosine and sine, off by 2^-22 for their argument's rounding (2 pi 2^-26 of a turn) and
    their own two units, and by what 64 bits leave of position times frequency (three roundings, 2 pi 2^-53 of up to
    `position` / 2 pi turns each); three operations of the rotation. All of `size`, the magnitudes that go in."""
    u, tiny = {torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}[dtype]
    inside = ((dim / 2 + 8) * 2.0 ** -24 + 2.0 ** -21 + 4 * position * 2.0 ** -53) * size
    return u * (out.abs() + inside) + inside + tiny


def bounds(pages, scales, page, tokens):
    """hi and lo [H, D] of a block's first `tokens` keys."""
    H = pages.shape[2]
    hi, lo = np.zeros((H, pages.shape[4]), np.int64), np.zeros((H, pages.shape[4]), np.int64)
    raw = pages.view(torch.uint8)[page, 0, :, :tokens].numpy()
    for h in range(H):
        if pages.dtype == torch.int8:
            x = raw[h].view(np.int8).astype(np.int64)
            up = down = np.clip(x, -127, 127)
        else:
            v = torch.from_numpy(raw[h].copy()).view(pages.dtype).double().numpy()
            nan = np.where(raw[h] & 0x80, -127, 127)
            up = np.where(np.isnan(v), nan, np.ceil(np.nan_to_num(v) / 4)).astype(np.int64)
            down = np.where(np.isnan(v), nan, np.floor(np.nan_to_num(v) / 4)).astype(np.int64)
        hi[h], lo[h] = up.max(0), down.min(0)
        if float(scales[page, 0, h]) < 0:
            hi[h], lo[h] = -lo[h], -hi[h]
    return hi, lo


def query_codes(q):
    """q [G, D] -> whole numbers and the exponents of their units."""
    x = q.double().numpy()
    fine = np.where(np.isfinite(x), np.abs(x), 0.0).max(1)
    e = np.array([math.frexp(v)[1] for v in fine]) - 7
    with np.errstate(invalid="ignore", over="ignore"):
        y = x * 2.0 ** -e[:, None].astype(np.float64)
    w = np.where(np.isnan(y), 0, np.clip(np.rint(np.where(np.isnan(y), 0, y)), -127, 127)).astype(np.int64)
    return w, e


def scores(q, hi, lo, scale, fmt):
    """q [G, D] of a kv head, hi, lo [nb, D], scale [nb] float32: float32 [nb]."""
    w, e = query_codes(q)
    dot = np.maximum(w[None] * hi[:, None], w[None] * lo[:, None]).sum(-1)            # [nb, G]
    with np.errstate(over="ignore", invalid="ignore"):
        best = np.ldexp(dot.astype(np.float64), e[None]).max(1).astype(np.float32)
        step = np.abs(scale.astype(np.float32)) * np.float32(1 if fmt == torch.int8 else 4)
        return best * step


def choose(score, nb, keep, sink, recent):
    """The blocks that stay, in order."""
    if nb <= keep:
        return list(range(nb))
    must = [b for b in range(nb) if b < sink or b >= nb - recent]
    rest = [b for b in range(sink, nb - recent)]
    rest.sort(key=lambda b: (not np.isnan(score[b]), 0.0 if np.isnan(score[b]) else -float(score[b]), b))
    return sorted(must + rest[:keep - len(must)])
