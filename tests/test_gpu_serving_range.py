"""Chunks over the 8-bit cache where the softmax's range matters: a key that holds most of a row's mass, scores near the cap.  All values
are positive, so that what a sum of probabilities loses cannot hide behind terms that cancel: bounds are relative to the output."""
import math

import numpy as np
import pytest
import torch

from tests import serving_ref as R
from tests.test_gpu_serving import EPS, Program, attend, check_attention, config, f64, sampled

pytestmark = pytest.mark.gpu
BASE = 0                # the feature that carries the scores' common part


def program(rng, L, n, n_q, n_kv, d, fmt, page=64, sigma=0.5, base_k=None):
    """A sequence of L tokens, the last n of them queries: scores of spread sigma from the features but BASE, where key t holds
    base_k[t] and every query 16."""
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=1, pages=-(-L // page), n_pages=-(-L // page))
    p = Program(cfg, fmt, seed=L + n)
    k = rng.standard_normal((L, n_kv, d)).astype(np.float32)
    v = (1.0 + 0.25 * rng.uniform(-1, 1, (L, n_kv, d))).astype(np.float32)
    k[..., BASE] = base_k[:, None]
    q = rng.standard_normal((n, n_q, d)).astype(np.float32) * sigma
    q[..., BASE] = 16.0
    v[0] = 2.0 ** -9
    as_dev = lambda x: torch.tensor(x, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    p.step([L], as_dev(k), as_dev(v))
    return p, as_dev(q)


def check(p, q, out, only, softcap=0.0):
    """All values are positive, so every relative error of a term is at most that of the output.  2^-8: the output's rounding; 3 2^-11: the
    probability, its value and the value's scale as fp16; 2^-11: probabilities below fp16's normal numbers (2^-14) are off by up to 2^-25
    each, the largest is above 2^(r - 1) with 2^r >= L / 2^13, so L of them by less than 2^-11 of it; scores: 2^-19 of sum |q k| scale and 2^-20 of the cap, in numerator and denominator;
    the sums: 2^-23 for each 16 keys."""
    n, L, d = q.shape[0], p.lens[0], p.cfg.head_dim
    ref, size = R.attend(f64(q), p.ref.values(p.ref.k[0]), p.ref.values(p.ref.v[0]), d ** -0.5, softcap, only=only)
    rel = 2.0 ** -8 + 4 * 2.0 ** -11 + L / 16 * 2.0 ** -23 + 2 * (2.0 ** -19 * size[only, :, :1] + 2.0 ** -20 * softcap)
    err = np.abs(f64(out)[only] - ref[only]) / ref[only]
    assert n and np.isfinite(err).all() and (err <= rel * (1 + 2.0 ** -6)).all(), (float((err / rel).max()), float(err.max()))


@pytest.mark.parametrize("mass", [0.5, 0.9, 0.99])
@pytest.mark.parametrize("L,n,n_q,n_kv,d,fmt", [
    (2048, 200, 8, 4, 64, "int8"), (8192, 96, 4, 1, 128, "e4m3"), (32768, 70, 2, 2, 128, "int8"), (4096, 1900, 32, 32, 64, "int8")])
@pytest.mark.parametrize("softcap", [0.0, 100.0])
def test_chunk_whose_first_key_holds_most_of_the_mass(mass, L, n, n_q, n_kv, d, fmt, softcap):
    """Items cut along the keys, and (last sizes: more items than SMs) whole ones."""
    rng = np.random.default_rng(L + n)
    s = math.log(mass / (1 - mass)) + math.log(L) + 0.5 * 0.5 ** 2
    if softcap:
        s = softcap * math.atanh(s / softcap)
    base = np.zeros(L, dtype=np.float32)
    base[0] = s * math.sqrt(d) / 16.0
    p, q = program(rng, L, n, n_q, n_kv, d, fmt, base_k=base)
    out = attend(p, [n], q, **(dict(softcap=softcap) if softcap else {}))
    assert p.status.item() == 0
    check(p, q, out, sampled(rng, n)[:12], softcap)


@pytest.mark.parametrize("softcap,ratio", [(30.0, 0.7), (50.0, 0.9), (50.0, 1.2), (100.0, 1.0), (50.0, -1.1), (5.0, 4.0)])
@pytest.mark.parametrize("L,n,n_q,n_kv,d,fmt", [(8192, 96, 4, 1, 128, "int8"), (2048, 1200, 32, 32, 64, "e4m3"), (2048, 300, 8, 2, 128, "int8")])
def test_chunk_whose_scores_are_near_the_cap(softcap, ratio, L, n, n_q, n_kv, d, fmt):
    """Every score is about ratio times the cap, so the capped one is far below both."""
    rng = np.random.default_rng(n)
    base = np.full(L, softcap * ratio * math.sqrt(d) / 16.0, dtype=np.float32)
    p, q = program(rng, L, n, n_q, n_kv, d, fmt, base_k=base, sigma=2.0)
    out = attend(p, [n], q, softcap=softcap)
    assert p.status.item() == 0
    check(p, q, out, sampled(rng, n)[:12], softcap)


# ---- decode steps and drafts: values of very different sizes -------------------------------------------------------------
def values(p, L, H, blocks):
    """K and V rows of L tokens; V rows from token t on, for (t, size) in blocks, are standard normal times size."""
    k, v = p.rows(L, H), p.rows(L, H).float()
    size = torch.zeros(L, device="cuda")
    for t, s in blocks:
        size[t:] = s
    return k, (v * size[:, None, None]).to(k.dtype)


@pytest.mark.parametrize("size", [1e-6, 1e-12, 1e-20])
@pytest.mark.parametrize("d,L", [(128, 53), (64, 700)])
def test_open_block_of_zero_values_beside_small_ones(d, L, size):
    cfg = config(n_q=2, n_kv=2, d=d, batch=1, pages=48, n_pages=48, dtype="fp32")
    p = Program(cfg, "int8", seed=L, dtype="fp32")
    p.step([L], *values(p, L, 2, [(0, size), (L // 16 * 16, 0.0)]))
    q = p.rows(1, 2, 2.0)
    check_attention(p, [1], q, attend(p, [1], q))


@pytest.mark.parametrize("d,before,new", [(128, 16, 9), (64, 300, 11), (64, 0, 14)])
def test_a_large_value_of_the_open_block_that_the_first_drafts_do_not_see(d, before, new):
    cfg = config(n_q=2, n_kv=2, d=d, batch=1, pages=48, n_pages=48, dtype="fp32")
    p = Program(cfg, "e4m3", seed=new, dtype="fp32")
    L = before + new
    p.step([L], *values(p, L, 2, [(0, 1.0), (L - 2, 1e12), (L - 1, 1e30)]))
    q = p.rows(new, 2, 2.0)
    check_attention(p, [new], q, attend(p, [new], q))


@pytest.mark.parametrize("dtype,d,n_q,before,new", [("fp32", 128, 2, 8, 40), ("bf16", 128, 2, 8, 40), ("bf16", 64, 8, 294, 10),
                                                    ("fp32", 64, 4, 24, 24)])
def test_a_large_value_of_a_block_that_the_first_drafts_do_not_see(dtype, d, n_q, before, new):
    """The last block of codes holds large values; the queries before it are attended beside it, eight rows at a time."""
    cfg = config(n_q=n_q, n_kv=2, d=d, batch=1, pages=48, n_pages=48, dtype=dtype)
    p = Program(cfg, "int8", seed=new, dtype=dtype)
    L = before + new
    p.step([L], *values(p, L, 2, [(0, 1.0), (L // 16 * 16 - 16, 1e12), (L // 16 * 16, 1e-12)]))
    q = p.rows(new, n_q, 2.0)
    check_attention(p, [new], q, attend(p, [new], q))


@pytest.mark.parametrize("kv", [0, 1])
def test_a_large_key_or_value_of_the_open_block_and_a_prefix(kv):
    cfg = config(n_q=2, n_kv=2, d=64, batch=1, pages=48, n_pages=48, dtype="fp32")
    p = Program(cfg, "int8", seed=kv, dtype="fp32")
    x = [p.rows(78, 2), p.rows(78, 2)]
    x[kv][77] *= 1e25
    p.step([78], *x)
    q = p.rows(12, 2, 2.0)
    out = attend(p, [12], q, prefix=[70])
    check_attention(p, [12], q, out, prefix=[70])


@pytest.mark.parametrize("scale", ["as appended", 0.0])
@pytest.mark.parametrize("dtype,size", [("bf16", 3e7), ("bf16", 1e30), ("bf16", 1.0), ("fp32", 1e30)])
def test_blocks_of_zero_values_beside_large_ones(dtype, size, scale):
    """A block of zeros has the scale 2^-100, or 0 if the caller filled the cache so; then ordinary blocks, and the large open block."""
    cfg = config(n_q=4, n_kv=2, d=128, batch=2, pages=48, n_pages=96, dtype=dtype)
    p = Program(cfg, "int8", seed=5, dtype=dtype)
    kv = [values(p, 101, 2, [(96, size)]), values(p, 149, 2, [(32, 1e-3), (64, 0.0), (80, 1.0), (144, size)])]
    p.step([101, 149], torch.cat([kv[0][0], kv[1][0]]), torch.cat([kv[0][1], kv[1][1]]))
    if scale == 0.0:
        p.cache.v_scales[p.cache.v_scales < 1e-29] = 0.0
    q = p.rows(2, 4, 2.0)
    check_attention(p, [1, 1], q, attend(p, [1, 1], q))


@pytest.mark.parametrize("size", [1e-12, 1e7, 1e12, 1e30])
@pytest.mark.parametrize("d,n_q,n_kv,L,new,softcap", [(128, 8, 2, 900, 300, 0.0), (64, 32, 32, 1500, 700, 0.0), (128, 4, 1, 6007, 100, 20.0)])
def test_a_large_value_that_the_first_rows_of_a_chunk_do_not_see(d, n_q, n_kv, L, new, softcap, size):
    """Values change by `size` inside the chunk, at the end of a block and inside the open one: rows before that see ordinary ones."""
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=64, batch=1, pages=-(-L // 64), n_pages=-(-L // 64))
    p = Program(cfg, "int8", seed=L)
    p.step([L], *values(p, L, n_kv, [(0, 1.0), ((L - new // 2) // 16 * 16, size), ((L - new // 4) // 16 * 16, 1.0), (L - 2, size)]))
    q = p.rows(new, n_q, 2.0)
    out = attend(p, [new], q, softcap=softcap)
    only = sorted(set(sampled(p.rng, new)) | {new - new // 2 - 17, new - new // 4 - 17, new - 3})
    ref, seen = R.attend(f64(q), p.ref.values(p.ref.k[0]), p.ref.values(p.ref.v[0]), d ** -0.5, softcap, only=only)
    # (2^-11: probabilities below fp16's normal numbers, see above)
    tol = R.tolerance(ref, seen, L, EPS["bf16"], True, True, softcap) + 2.0 ** -11 * seen[..., 1:]
    err = np.abs(f64(out) - ref)[only]
    assert (err <= tol[only]).all(), float((err / tol[only]).max())
