"""The serving step's operators written plainly (Python integers, numpy in 64 bits), one sequence at a time."""
from __future__ import annotations

import math

import numpy as np
import torch

BLOCK = 16
QMAX = {"int8": 127.0, "e4m3": 448.0}


def plan(table, slots, lens, new, free_pages, free_count, n_tokens, page, max_batch, n_pages):
    """-> dict(table, cu, positions, seqs, rows, lens, count, status)."""
    table = [list(r) for r in table]
    cap = len(table[0]) * page
    status, taken, asked_pages, asked_tokens = 0, 0, 0, 0
    count = min(max(free_count, 0), n_pages)
    cu, positions, seqs, rows, after = [0], [], [], [], []

    def tell(code):
        nonlocal status
        status = status or code
    for b, (slot, n, k) in enumerate(zip(slots, lens, new)):
        if not 0 <= slot < max_batch:
            tell(-8)
            k = 0
        elif n < 0 or k < 0 or n + k > cap:
            tell(-11)
            k = 0
        else:
            old = -(-n // page)
            need = -(-(n + k) // page) - old
            asked_pages += need
            asked_tokens += k
            if (need and asked_pages > count) or asked_tokens > n_tokens:
                tell(-4)
                k = need = 0
            for j in range(need):
                table[slot][old + j] = free_pages[count - 1 - taken]
                taken += 1
        for i in range(k):
            p = table[slot][(n + i) // page]
            positions.append(n + i)
            seqs.append(b)
            ok = 0 <= p < n_pages
            if not ok:
                tell(-8)
            rows.append(p * page + (n + i) % page if ok else -1)
        cu.append(len(positions))
        after.append(n + k)
    pad = [-1] * (n_tokens - len(positions))
    return dict(table=table, cu=cu, positions=positions + pad, seqs=seqs + pad, rows=rows + pad, lens=after,
                count=count - taken, status=status)


def axis_of(half, sections, interleaved):
    out = []
    for j in range(half):
        if interleaved:
            a = j % len(sections)
            out.append(a if j // len(sections) < sections[a] else 0)
        else:
            a, until = 0, sections[0]
            while j >= until:
                a += 1
                until += sections[a]
            out.append(a)
    return out


def rotate(x, pos, theta, sections, rot, interleaved, inverse):
    """x [T][heads][d] float64, pos [axes][T]."""
    half = rot // 2
    y = x.copy()
    ax = axis_of(half, sections, interleaved)
    for j in range(half):
        a = pos[ax[j]].astype(np.float64) * theta ** (-2.0 * j / rot) * (-1.0 if inverse else 1.0)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        y[:, :, j] = x[:, :, j] * c - x[:, :, j + half] * s
        y[:, :, j + half] = x[:, :, j + half] * c + x[:, :, j] * s
    return y


def quantise_block(x, fmt):
    """x [16][d] float32 -> (scale float32, codes as float32 values); the interface's fp32 steps one by one."""
    a = np.abs(x).max()
    if not np.isfinite(a):
        return np.float32(np.nan), np.zeros_like(x)
    scale = np.maximum(np.float32(a) * (np.float32(1) / np.float32(QMAX[fmt])), np.float32(2.0 ** -100))
    y = x * (np.float32(1) / scale)
    if fmt == "int8":
        return scale, np.clip(np.rint(y), -127, 127).astype(np.float32)
    return scale, torch.from_numpy(np.clip(y, -448, 448)).to(torch.float8_e4m3fn).float().numpy()


class Cache:
    """All tokens of every sequence; what the 8-bit cache stands for is derived from them."""

    def __init__(self, fmt, batch):
        self.fmt, self.k, self.v = fmt, [None] * batch, [None] * batch

    def append(self, b, k, v):
        self.k[b] = k if self.k[b] is None else np.concatenate([self.k[b], k])
        self.v[b] = v if self.v[b] is None else np.concatenate([self.v[b], v])

    def values(self, x):
        """[n][H][d] float32 -> float64 values, whole blocks through their codes, the open block as it is."""
        y = x.astype(np.float64)
        n = len(x)
        for t in range(0, n, BLOCK):
            for h in range(x.shape[1]):
                blk = x[t:t + BLOCK, h]
                if len(blk) == BLOCK:
                    scale, codes = quantise_block(blk, self.fmt)
                    y[t:t + BLOCK, h] = codes.astype(np.float64) * float(scale)
                elif not np.isfinite(blk).all():
                    y[t:t + BLOCK, h] = np.nan
        return y


def attend(q, k, v, scale, softcap=0.0, slopes=None, prefix=0, only=None):
    """q [n][Hq][d] = the last n tokens, k, v [L][H][d] float64 -> (out [n][Hq][d], size [n][Hq][2]: the largest sum |q_i k_i| scale
    of a seen key, and the largest |v| of one); only: the queries that are worked out (the others' rows stay 0)."""
    n, Hq, d = q.shape
    L, H, _ = k.shape
    out = np.zeros((n, Hq, d))
    size = np.zeros((n, Hq, 2))
    t = np.arange(L)
    for i in range(n) if only is None else only:
        p = L - n + i
        seen = (t <= p) | (t < prefix)
        for h in range(Hq):
            kk, vv = k[seen, h * H // Hq], v[seen, h * H // Hq]
            x = kk @ q[i, h] * scale
            if softcap:
                x = softcap * np.tanh(x / softcap)
            if slopes is not None:
                x = x - float(slopes[h]) * np.abs(p - t[seen])
            w = np.exp(x - x.max())
            out[i, h] = (w / w.sum()) @ vv
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale, np.abs(vv).max()
    return out, size


def tolerance(ref, size, L, out_eps, half_p, half_v=False, softcap=0.0, slopes=None):
    """How far a row may be off, from the roundings on its way (first order, absolute, per element).

    x: products accumulate in fp32, 16 at a time: at most d / 16 = 8 sums of partly truncated terms, and the operands carry 22 bits
       (2^-22 each): (8 + 4) 2^-23 < 2^-19 of sum |q k| scale.  tanh: 2^-20 of the cap.  bias: one fp32 product, one sum, in base-2
       units: 2^-22 of the largest |bias|.  A probability is off by the score's error, the output by twice that times max |v|.
    p: 2^x 2^-21, times the V scale and back 2^-21, as an fp16 pair 2^-21; summed over L / 16 blocks in fp32: L / 16 2^-23.
    half_p (bf16 queries): probabilities as single fp16, half a step of which is 2^-11 of each.
    half_v (chunks): a value is its code times its block's scale over the largest, both rounded to fp16: 2^-11 each.
    out: half a step of its type, out_eps / 2 = 2^-8 |ref| in bf16 and 2^-24 |ref| in fp32."""
    dx = 2.0 ** -19 * size[..., 0]
    if softcap:
        dx = dx + 2.0 ** -20 * softcap
    if slopes is not None:
        dx = dx + 2.0 ** -22 * np.abs(np.asarray(slopes, dtype=np.float64))[None, :] * L * math.log2(math.e)
    dp = 3 * 2.0 ** -21 + L / 16 * 2.0 ** -23 + (2.0 ** -11 if half_p else 0.0) + (2.0 ** -10 if half_v else 0.0)
    return (out_eps / 2) * np.abs(ref) + ((2 * dx + dp) * size[..., 1])[..., None] * (1 + out_eps)
