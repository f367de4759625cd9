"""The calls on the cache's contents, from their definitions, in 64 bits on the CPU.

Used by the GPU tests as the other side of every comparison; shares no code with the package. A cache is
pages [P, 2, H, B, D] (codes) with scales [P, 2, H]; tables are int lists per sequence.
"""
from __future__ import annotations

import math

import numpy as np
import torch

ROUNDOFF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}    # largest relative error of one rounding
# and absolute: half a float16 subnormal; bfloat16 has float32's range, below which a weight is nothing
SMALLEST = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def cached(pages, scales, row, tokens):
    """K and V [tokens, H, D] float64 of a sequence whose pages are `row`."""
    B = pages.shape[3]
    ids = torch.tensor([int(row[b]) for b in range(-(-tokens // B))], dtype=torch.int64)
    codes = pages.view(torch.uint8)[ids].view(pages.dtype).double()
    x = codes * scales[ids].double()[..., None, None]                # [blocks, 2, H, B, D]
    x = x.permute(1, 0, 3, 2, 4).reshape(2, -1, pages.shape[2], pages.shape[4])
    return x[0, :tokens], x[1, :tokens]


def attend(q, keys, values, scale, first_seen):
    """Rows q [T, Hq, D] over keys, values [S, H, D]; row i sees the first first_seen + i of them. Returns out, lse, the
    weights [Hq, T, S], and per (row, head): `spread` [T, Hq, D] = sum of weight * |value|, and `reach` [T, Hq] = the
    largest sum of |q k| * scale, the two quantities that rounding errors are proportional to."""
    T, Hq, D = q.shape
    S, H, _ = keys.shape
    q, keys, values = q.double(), keys.double(), values.double()
    group = Hq // H
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    weights, spread = torch.zeros(Hq, T, S, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    reach = torch.zeros(T, Hq, dtype=torch.float64)
    if S == 0:
        return out, lse, weights, spread, reach
    seen = torch.arange(S)[None] < (first_seen + torch.arange(T))[:, None]
    for h in range(Hq):
        k, v = keys[:, h // group], values[:, h // group]
        x = (q[:, h] @ k.T * scale).masked_fill(~seen, -math.inf)
        lse[:, h] = torch.logsumexp(x, 1)
        top = lse[:, h].clamp(min=-1e300)
        w = torch.exp(x - top[:, None])
        weights[h] = w
        out[:, h] = w @ v
        spread[:, h] = w @ v.abs()
        reach[:, h] = ((q[:, h].abs() @ k.abs().T) * abs(scale)).masked_fill(~seen, 0).amax(1)
    return out, lse, weights, spread, reach


def logit_error(reach, dim):
    """A logit is a sum of dim products held in 32 bits, times the scales: each of dim + 16 operations is off by at most
    2^-24 of the sum of magnitudes."""
    return (dim + 16) * 2.0 ** -24 * reach


def out_bound(out, spread, reach, dtype, tokens=0, most=0.0):
    """|computed - exact| of an output element: the output's own rounding, the rounding of each weight to the type, the
    weights' error through their logits (twice: above and below the fraction), and 2^-18 for sums, exponentials and
    scales in 32 bits. A weight below the type's normal range is off by up to SMALLEST of the largest: `tokens` of them,
    times the largest value that any scale lets a code stand for (`most`)."""
    u = ROUNDOFF[dtype]
    delta = logit_error(reach, out.shape[-1])[..., None]
    return u * out.abs() + (1 + u) * (u + 2.1 * delta + 2.0 ** -18) * spread + SMALLEST[dtype] * (1 + tokens * most)


def most_of(scales, fmt):
    """The largest value that a code of this pool can stand for (unused pages' scales are NaN), or 8 of fresh rows."""
    live = scales[~scales.isnan()]
    return max(8.0, float(live.max()) * (448 if fmt == torch.float8_e4m3fn else 127) if live.numel() else 0.0)


def lse_bound(lse, reach, dim):
    return logit_error(reach, dim) + 2.0 ** -20 * (1 + lse.abs())


def mass_bound(weight, reach, mass):
    """weight: what the call adds; reach: the largest of the group's heads."""
    return weight * (2.1 * logit_error(reach, 128) + 2.0 ** -16) + 2.0 ** -22 * mass.abs() + 1e-30


# ------------------------------------------------------------------ append
def e4m3_values():
    return torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()


def round_e4m3(y):
    """float64 -> the nearest e4m3 value, ties to the even code, magnitudes beyond 448 to 448, NaN kept."""
    grid = e4m3_values()[:127]                                       # 0 .. 448, ascending codes
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(grid, np.nan_to_num(a)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isnan(y), np.nan, np.copysign(grid[pick], y))


def block_scale(most, fmt):
    if fmt == torch.int8:
        s = np.float32(most) * (np.float32(1) / np.float32(127))     # 32 bits, as defined
        return float(np.clip(s, np.float32(2.0 ** -60), np.float32(2.0 ** 60)))
    e = -60 if most == 0 else math.ceil(math.log2(most / 448.0))
    while most > 448.0 * 2.0 ** e:
        e += 1
    while e > -60 and most <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** min(60, max(-60, e))


def quantised(x, scale, fmt):
    """Values (not bits) that x's codes stand for, before the scale; the quotient is one of 32 bits, as defined."""
    with np.errstate(invalid="ignore", over="ignore"):
        y = (x.astype(np.float32) / np.float32(scale)).astype(np.float64)
    if fmt == torch.int8:
        return np.where(np.isnan(y), 0.0, np.clip(np.rint(y), -127, 127))
    return round_e4m3(y)


def append(codes, scales, k, v, offsets, context, table, fmt):
    """codes [P, 2, H, B, D] float64 (values before the scale) and scales [P, 2, H] float64, changed in place."""
    B, H = codes.shape[3], codes.shape[2]
    for r in range(len(offsets) - 1):
        first, last = context[r], context[r] + offsets[r + 1] - offsets[r]
        for b in range(first // B, -(-last // B)):
            lo, hi = max(first, b * B), min(last, (b + 1) * B)
            if lo >= hi:
                continue
            p, at = int(table[r][b]), lo - b * B
            for part, x in enumerate((k, v)):
                for h in range(H):
                    new = x[offsets[r] + lo - first:offsets[r] + hi - first, h]
                    fine = np.abs(new[np.isfinite(new)])
                    s = block_scale(float(fine.max()) if fine.size else 0.0, fmt)
                    if at > 0:
                        held = scales[p, part, h]
                        if s > held:
                            old = codes[p, part, h, :at].astype(np.float32) * np.float32(held)
                            codes[p, part, h, :at] = quantised(old, s, fmt)
                        else:
                            s = held
                    scales[p, part, h] = s
                    codes[p, part, h, at:at + hi - lo] = quantised(new, s, fmt)


# ---------------------------------------------------------------- eviction
def evict(context, table, mass, keep, block, sink, recent):
    n, H, W = mass.shape
    table_out, freed = np.full((n, W), -1, np.int32), np.full((n, W), -1, np.int32)
    mass_out, ctx, count = np.zeros_like(mass), np.array(context, np.int32), np.zeros(n, np.int32)
    for r in range(n):
        nb = -(-int(ctx[r]) // block)
        score = mass[r, 0].copy()
        for h in range(1, H):
            score = (score + mass[r, h]).astype(np.float32)
        able = [b for b in range(sink, nb - recent)]
        able.sort(key=lambda b: (bool(np.isnan(score[b])), 0.0 if np.isnan(score[b]) else float(score[b]), b))
        gone = sorted(able[:max(0, nb - max(0, int(keep[r])))])
        stay = np.setdiff1d(np.arange(W), gone)
        table_out[r, :len(stay)] = table[r, stay]
        mass_out[r, :, :len(stay)] = mass[r][:, stay]
        freed[r, :len(gone)] = table[r, gone]
        count[r] = len(gone)
        ctx[r] -= block * len(gone)
    return ctx, table_out, mass_out, freed, count
