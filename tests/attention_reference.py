"""Plain implementations in 64 bits of the heads' norms and rotation, of the 4-bit cache and of attention over pages, on the CPU with numpy, and what
their tests share.  They share no code with the library."""
import math

import numpy as np
import torch

import paper_1603_02297_amd as ttc
from moves_reference import F32, ROUND, TYPES as MOVE_TYPES

TYPES = dict(MOVE_TYPES, q4=(ttc.TTC_Q4, torch.uint8))
EPS = 1e-5


def angles(rotated, base=10000.0):
    return [base ** (-2 * i / rotated) for i in range(rotated // 2)]


def pairs(rotated, paired):
    """The two elements of every rotation."""
    i = np.arange(rotated // 2)
    return (2 * i, 2 * i + 1) if paired else (i, i + rotated // 2)


def turn(x, positions, angle, rotated, paired, back=False):
    """x [tokens, heads, dim] turned by position: exact angles, reduced as Python integers times doubles would not be."""
    y = x.copy()
    a, b = pairs(rotated, paired)
    # a double angle is a whole number of 2^-k radians: its product with the position is exact in long double for the positions used here
    t = np.asarray(positions, np.longdouble)[:, None, None] * np.asarray(angle, np.longdouble)[None, None, :]
    c, s = np.cos(t).astype(np.float64), np.sin(t).astype(np.float64)
    if back:
        s = -s
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def heads(x, weight, positions, angle, rotated, paired, norm):
    """x [tokens, heads, dim] -> y, and for every element the magnitude that its 32-bit roundings are relative to."""
    u = x
    if norm:
        u = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * (1.0 if weight is None else weight)
    size = np.abs(u)
    if rotated:
        a, b = pairs(rotated, paired)
        size = size.copy()
        both = size[..., a] + size[..., b]
        size[..., a] = size[..., b] = both
        u = turn(u, positions, angle, rotated, paired)
    return u, size


def heads_grad(dy, x, weight, positions, angle, rotated, paired, norm):
    """dx and dw (over tokens and heads), each with such a magnitude."""
    du = turn(dy, positions, angle, rotated, paired, back=True) if rotated else dy
    size = np.abs(dy)
    if rotated:
        a, b = pairs(rotated, paired)
        size = size.copy()
        both = size[..., a] + size[..., b]
        size[..., a] = size[..., b] = both
    if not norm:
        return du, size, None, None
    w = 1.0 if weight is None else weight
    s = np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    g, gs, hat = du * w, size * np.abs(w), x / s
    dx = (g - hat * (g * hat).mean(-1, keepdims=True)) / s
    dx_size = (gs + np.abs(hat) * (gs * np.abs(hat)).mean(-1, keepdims=True)) / s
    return dx, dx_size, (du * hat).sum((0, 1)), (size * np.abs(hat)).sum((0, 1))


def bf16_towards(x, towards):
    x = np.asarray(x, np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))) - 7)
    return towards(x / step) * step


def to_records(x):
    """[..., dim] -> (step, minimum, codes), by the definition of the format."""
    low = bf16_towards(x.min(-1, keepdims=True), np.floor)
    step = bf16_towards((x.max(-1, keepdims=True) - low) / 15, np.ceil)
    with np.errstate(divide="ignore", invalid="ignore"):
        code = np.where(step > 0, np.clip(np.round((x - low) / step), 0, 15), 0)
    return step, low, code


def from_records(rec):
    """Records [..., 4 + dim/2] of bytes -> (step, minimum, codes)."""
    rec = np.asarray(rec, np.uint8)
    words = rec[..., :4].copy().view(np.uint16).astype(np.uint32) << 16
    head = words.view(np.float32).astype(np.float64)
    code = np.empty((*rec.shape[:-1], 2 * (rec.shape[-1] - 4)))
    code[..., 0::2], code[..., 1::2] = rec[..., 4:] & 15, rec[..., 4:] >> 4
    return head[..., :1], head[..., 1:2], code


def assert_within(got, want, limit, what=""):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    ok = np.isfinite(want)
    assert np.array_equal(got[~ok & ~np.isnan(want)], want[~ok & ~np.isnan(want)]), what
    off = np.abs(got[ok] - want[ok]) - np.broadcast_to(limit, want.shape)[ok]
    assert not off.size or off.max() <= 0, f"{what}: {off.max()} over the limit, {np.abs(got[ok] - want[ok]).max()} off"


def rounded(want, kind, err32):
    """How far a value within err32 of `want` is off after one rounding to `kind`."""
    rel, tiny = ROUND[kind]
    return err32 + rel * (np.abs(want) + err32) + tiny
