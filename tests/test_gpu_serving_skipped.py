"""Appends in which some tokens of a sequence have no row (rejected drafts, cached prefixes, padding) or a bad one: the others are
held as if they had come alone."""
import numpy as np
import pytest
import torch

from tests.test_gpu_serving import DT, Program, config, dev

pytestmark = pytest.mark.gpu


def step_with_holes(p, keep, bad=()):
    """Append to every sequence b the tokens i with keep[b][i], the others of the step being skipped: slot -1, or `bad` values in turn."""
    kept = [int(np.sum(m)) for m in keep]
    plan = p.plan(kept)
    T, H, d = sum(len(m) for m in keep), p.cfg.n_kv_heads, p.cfg.head_dim
    mask = np.concatenate([np.asarray(m, dtype=bool) for m in keep])
    x = [torch.tensor(p.rng.standard_normal((T, H, d)) * s, dtype=DT[p.dtype][1], device="cuda") for s in (1.0, 2.0)]
    rows = np.full(T, -1, dtype=np.int64)
    for i, t in enumerate(np.flatnonzero(~mask)):
        rows[t] = bad[i % len(bad)] if bad else -1
    rows[mask] = plan.slot_map.cpu().numpy()[: sum(kept)]
    cu = np.concatenate([[0], np.cumsum([len(m) for m in keep])])
    seqs = np.repeat(np.arange(len(keep)), [len(m) for m in keep])
    p.cache.append(x[0], x[1], dev(rows, torch.int64), dev(seqs), dev(cu), seq_slots=dev(p.slots[: len(keep)]), status=p.status)
    host = [t.float().cpu().numpy() for t in x]
    for b, m in enumerate(keep):
        at = cu[b] + np.flatnonzero(m)
        if len(at):
            p.ref.append(b, host[0][at], host[1][at])
        p.lens[b] += len(at)
    assert p.status.item() == (-8 if bad and not mask.all() else 0)
    p.status.zero_()
    p.check_cache()


def program(dtype, d, n_kv, seed, fmt="int8", batch=4):
    cfg = config(n_q=n_kv, n_kv=n_kv, d=d, page=16, batch=batch, pages=256, n_pages=256 * batch, dtype=dtype)
    return Program(cfg, fmt, seed=seed, dtype=dtype)


def runs(*lengths):
    """Kept, skipped, kept, ... runs of these lengths."""
    return np.repeat(np.arange(len(lengths)) % 2 == 0, lengths)


@pytest.mark.parametrize("bad", [(), (1 << 40, 16384 + 7, -5)])
@pytest.mark.parametrize("dtype,d,n_kv", [("bf16", 128, 2), ("fp32", 64, 3), ("bf16", 64, 8)])
def test_skipped_last_tokens_leave_the_others(dtype, d, n_kv, bad):
    p = program(dtype, d, n_kv, 1)
    step_with_holes(p, [runs(2, 1), runs(5, 3), runs(16, 4), runs(0, 2)], bad)
    step_with_holes(p, [runs(14, 2), runs(12, 2), runs(31, 1), runs(3, 70)], bad)       # blocks that begin in the tail
    step_with_holes(p, [runs(1, 300), runs(40, 33), runs(2, 30), runs(50, 31)], bad)
    step_with_holes(p, [runs(15, 32), runs(1, 1), runs(16, 16), runs(11, 5)], bad)


@pytest.mark.parametrize("bad", [(), (1 << 40, -5)])
@pytest.mark.parametrize("dtype,d,n_kv", [("bf16", 128, 2), ("fp32", 128, 1)])
def test_skipped_first_and_middle_tokens(dtype, d, n_kv, bad):
    p = program(dtype, d, n_kv, 2, "e4m3")
    step_with_holes(p, [runs(0, 3, 5), runs(4, 1, 7), runs(0, 100, 3), runs(1, 1, 1, 1, 1)], bad)
    step_with_holes(p, [runs(0, 40, 20), runs(3, 65, 30, 2, 9), runs(7, 16, 7), runs(0, 1, 40, 1)], bad)
    step_with_holes(p, [runs(6, 31, 6, 32, 6, 33, 6), runs(0, 17, 1), runs(1, 15, 1, 14, 13, 200, 2), runs(0, 64, 64, 64, 64)], bad)


@pytest.mark.parametrize("share", [0.05, 0.5, 0.95])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("fp32", "e4m3")])
def test_tokens_skipped_at_random(dtype, fmt, share):
    p = program(dtype, 64, 2, 3, fmt, batch=7)
    for _ in range(6):
        step_with_holes(p, [p.rng.random(int(n)) >= share for n in p.rng.integers(0, 200, 7)])


def test_a_token_of_another_sequence_is_skipped_like_a_bad_row():
    """The last token names a sequence that does not hold it: the one before it ends the step."""
    p = program("bf16", 128, 2, 4, batch=2)
    p.step([13, 4])
    plan = p.plan([5, 2])
    k, v = p.rows(7, 2), p.rows(7, 2, 2.0)
    seqs = plan.token_seqs.clone()
    seqs[4] = 1                                          # token 4 is sequence 0's last
    p.cache.append(k, v, plan.slot_map, seqs, plan.cu_tokens, seq_slots=dev(p.slots[:2]), status=p.status)
    assert p.status.item() == -8
    p.status.zero_()
    for b, at in ((0, slice(0, 4)), (1, slice(5, 7))):
        p.ref.append(b, k[at].float().cpu().numpy(), v[at].float().cpu().numpy())
        p.lens[b] += at.stop - at.start
    p.check_cache()
