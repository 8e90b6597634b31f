"""The operators over a cache held in 4 bits written plainly: numpy, the interface's fp32 steps one by one where it says so, 64 bits
otherwise."""
from __future__ import annotations

import math

import numpy as np
import torch

from tests import serving_ref as R

GROUP = 16
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
f32 = np.float32


def e4m3(x):
    """float32 >= 0 -> bytes of the nearest e4m3 (ties to even, at most 448)."""
    return torch.from_numpy(np.minimum(x, f32(448)).astype(f32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def e4m3_value(b):
    return torch.from_numpy(np.ascontiguousarray(b)).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)


def e2m1(y):
    """float32 -> codes of the nearest e2m1 (ties to the even code, at most 6)."""
    gap = np.abs(np.abs(y.astype(np.float64))[..., None] - MAGNITUDES)
    best = gap.min(-1, keepdims=True)
    tied = gap == best
    code = np.where(tied.sum(-1) > 1, (tied & (np.arange(8) % 2 == 0)).argmax(-1), tied.argmax(-1))
    return (code | (np.signbit(y).astype(int) << 3)).astype(np.uint8)


def e2m1_value(code):
    return MAGNITUDES[code & 7] * np.where(code >= 8, -1.0, 1.0)


def hold(x, unit):
    """float32 [..., d] -> (codes [..., d], scale bytes [..., d/16])."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    s8 = e4m3(np.abs(g).max(-1) * f32(1.0 / (6.0 * unit)))
    s = e4m3_value(s8).astype(f32)
    r = np.divide(f32(1.0 / unit), s, out=np.zeros_like(s), where=s > 0)
    return e2m1(g * r[..., None]).reshape(x.shape), s8


def token(k, v, k_unit, v_unit):
    """k, v float32 [..., d] of tokens and heads -> the values that they are held as, float64 (NaN / 0 where not finite)."""
    out = []
    bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))
    for x, unit in ((k, k_unit), (v, v_unit)):
        codes, s8 = hold(np.where(bad[..., None], f32(0), x), unit)
        out.append((e2m1_value(codes).reshape(*s8.shape, GROUP) * e4m3_value(s8)[..., None]).reshape(x.shape) * unit)
    out[0][bad] = np.nan
    out[1][bad] = 0.0
    return out


def turn(x, pos, theta, sections, rot, interleaved):
    """x float32 [T][heads][d] turned as the append does: angles in 64 bits, their cosines in fp32, every step in fp32."""
    half = rot // 2
    ax = R.axis_of(half, sections, interleaved)
    ang = np.stack([pos[ax[j]].astype(np.float64) * theta ** (-2.0 * j / rot) for j in range(half)], -1)
    c, s = np.cos(ang).astype(f32)[:, None], np.sin(ang).astype(f32)[:, None]
    x1, x2 = x[..., :half], x[..., half:rot]
    return np.concatenate([x1 * c - x2 * s, x2 * c + x1 * s, x[..., rot:]], -1)


def unpack(blocks, d):
    """uint8 [n_pages][H][P/16][18 d] -> (K, V) float64 [n_pages][H][P][d] in units of 1, by the documented places of the bytes."""
    n, H, m, _ = blocks.shape
    tok, f = np.meshgrid(np.arange(16), np.arange(d), indexing="ij")
    lane = d // 8
    at = {0: tok * (d // 2) + f // 2, 1: 8 * d + (((tok // 8 * 8 + f // lane) * 4 + tok // 2 % 4) * 2 + tok % 2) * (d // 16) + f % lane // 2}
    sc = {0: 16 * d + tok * (d // 16) + f // 16, 1: 17 * d + f // 16 * 16 + tok}
    out = []
    for w in (0, 1):
        code = blocks[..., at[w]] >> (f % 2 * 4) & 15
        out.append((e2m1_value(code) * e4m3_value(blocks[..., sc[w]])).reshape(n, H, m * 16, d))
    return out


def bounds(k):
    """keys [tokens][d] in units of k_unit -> (int8 [2][d], scale float32)."""
    if np.isnan(k).any():
        return np.zeros((2, k.shape[1]), np.int8), f32(np.nan)
    both = np.stack([k.max(0), k.min(0)]).astype(f32)
    scale = np.maximum(np.abs(both).max() * f32(1.0 / 127.0), f32(2.0 ** -60))
    return np.clip(np.rint(both * (f32(1) / scale)), -127, 127).astype(np.int8), scale


def select(q, bnd, scales, pos, page, n_select, n_first, n_recent):
    """q float32 [Hq][d] of one token, bounds [pages][H][2][d] and scales [pages][H] of its sequence's pages -> [H][n_select]."""
    H, Hq = bnd.shape[1], len(q)
    own = pos // page
    out = np.full((H, n_select), -1)
    for h in range(H):
        best = np.full(own + 1, -np.inf, f32)
        for j in range(h * Hq // H, (h + 1) * Hq // H):
            row = q[j]
            if not np.isfinite(row).all():
                row = np.zeros_like(row)
            s_q = np.clip(np.abs(row).max() * f32(1.0 / 127.0), f32(2.0 ** -60), f32(2.0 ** 100))
            code = np.clip(np.rint(row * (f32(1) / s_q)), -127, 127).astype(np.int64)
            top, low = bnd[:own + 1, h, 0].astype(np.int64), bnd[:own + 1, h, 1].astype(np.int64)
            whole = top @ np.maximum(code, 0) + low @ np.minimum(code, 0)
            with np.errstate(invalid="ignore"):
                score = (s_q * scales[:own + 1, h]).astype(f32) * whole.astype(f32)
            best = np.maximum(best, np.where(np.isnan(score), np.finfo(f32).max, score))
        j = np.arange(own + 1)
        key = np.where((j < n_first) | (j > own - n_recent), np.inf, best.astype(np.float64))
        take = np.sort(np.argsort(-key, kind="stable")[:n_select])
        out[h, :len(take)] = take
    return out


def attend_pages(q, k, v, pos, pages, page, scale, softcap=0.0, slopes=None):
    """One token: q [Hq][d], k, v [L][H][d] float64, pages [H][n] -> (out [Hq][d], size [Hq][2]) as serving_ref.attend's."""
    Hq, d = q.shape
    H = k.shape[1]
    out, size = np.zeros((Hq, d)), np.zeros((Hq, 2))
    for h in range(Hq):
        t = np.concatenate([np.arange(p * page, (p + 1) * page) for p in pages[h * H // Hq] if p >= 0] + [np.zeros(0, int)]).astype(int)
        t = t[t <= pos]
        if not len(t):
            continue
        kk, vv = k[t, h * H // Hq], v[t, h * H // Hq]
        x = kk @ q[h] * scale
        if softcap:
            x = softcap * np.tanh(x / softcap)
        if slopes is not None:
            x = x - float(slopes[h]) * np.abs(pos - t)
        w = np.exp(x - x.max())
        out[h] = (w / w.sum()) @ vv
        size[h] = (np.abs(kk) @ np.abs(q[h])).max() * scale, np.abs(vv).max()
    return out, size


def tolerance(ref, size, L, out_eps, bf16, chunk=False, softcap=0.0, slopes=None):
    """serving_ref.tolerance without what that cache's scales cost: values are exact in their operands.  bf16: a probability is rounded to
    fp16 (2^-11 of it), and one far below the row's largest to a multiple of 2^-24: by rows that is 2^-30 of the largest, in chunks
    2^-25, for each of L keys.  Beside that 2^-22 each for the exponential and the fp32 sums of L / 16 blocks."""
    base = R.tolerance(ref, size, L, out_eps, bf16, False, softcap, slopes)
    small = L * (2.0 ** -25 if chunk else 2.0 ** -30) if bf16 else 0.0
    return base + (small * size[..., 1])[..., None]


def scale_of(d):
    return 1.0 / math.sqrt(d)
