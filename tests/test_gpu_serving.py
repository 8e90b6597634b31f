"""The serving step over an 8-bit cache on the GPU: every operator against its plain form in 64 bits, their edge cases, and a
run of steps as a program makes them."""
import numpy as np
import pytest
import torch

from paper_2603_22910_b200 import binding
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": (binding.ECHOKV_BF16, torch.bfloat16), "fp32": (binding.ECHOKV_FP32, torch.float32)}
EPS = {"bf16": 2.0 ** -7, "fp32": 2.0 ** -23}
BLOCK = 16
CHUNK_ROWS = 64         # query rows per KV head from which bf16 sequences take the chunk kernel


def config(n_q=8, n_kv=2, d=128, page=16, batch=4, pages=16, n_pages=64, dtype="bf16", **kw):
    return binding.make_config(n_layers=1, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=d, group_size=1, n_retained_heads=0,
                               page_tokens=page, max_batch=batch, max_pages_per_seq=pages, n_pages=n_pages, dtype=DT[dtype][0], **kw)


def dev(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def f64(t):
    return t.detach().cpu().double().numpy()


# ---- plan and release -------------------------------------------------------------------------------------------
def run_plan(rng, B, page, pages, n_pages, lens, new, n_tokens, slots, free, count, bad_page=None, in_place=False, cfg=None):
    cfg = cfg or config(page=page, batch=max(B, max(slots) + 1 if slots else B), pages=pages, n_pages=n_pages)
    rows = cfg.max_batch
    table = rng.integers(0, n_pages, (rows, pages)).astype(np.int32)
    if bad_page is not None:
        table[bad_page[0], bad_page[1]] = n_pages + 3
    ref = R.plan(table.tolist(), slots or list(range(B)), lens, new, free, count, n_tokens, page, rows, n_pages)
    t, st = dev(table), dev([0])
    seq_lens, fc = dev(lens), dev([count])
    full = list(free) + [0] * (n_pages - len(free))
    out = None
    if in_place:
        out = binding.StepPlan(B, n_tokens, "cuda", seq_lens=seq_lens, free_count=fc)
    p = binding.plan_tokens(cfg, t, seq_lens, dev(new), dev(full), fc, n_tokens, seq_slots=dev(slots) if slots else None, out=out,
                            status=st)
    got = dict(table=t.tolist(), cu=p.cu_tokens.tolist(), positions=p.positions.tolist(), seqs=p.token_seqs.tolist(),
               rows=p.slot_map.tolist(), lens=p.seq_lens.tolist(), count=p.free_count.item(), status=st.item())
    for name in ref:
        if name == "status" and ref["status"] and got["status"]:
            continue                      # several sequences may have an error: any of them is the first one found
        assert got[name] == ref[name], name
    return p, ref


@pytest.mark.parametrize("B,page,hi_len,hi_new,in_place", [
    (1, 16, 0, 1, False), (1, 128, 300, 1, True), (7, 16, 70, 0, False), (256, 16, 500, 1, True), (33, 32, 400, 40, False),
    (5, 64, 3000, 2500, True), (700, 16, 90, 30, False), (3, 16, 10, 9000, False)])
def test_plan_matches_plain_form(B, page, hi_len, hi_new, in_place):
    rng = np.random.default_rng(B + page)
    lens, new = rng.integers(0, hi_len + 1, B).tolist(), rng.integers(0, hi_new + 1, B).tolist()
    pages = (hi_len + hi_new) // page + 1
    need = sum(-(-(a + b) // page) - -(-a // page) for a, b in zip(lens, new))
    n_pages = need + 13
    free = rng.permutation(n_pages)[: need + 5].tolist()
    slots = rng.permutation(B + 2)[:B].tolist()
    run_plan(rng, B, page, pages, n_pages, lens, new, sum(new) + 3, slots, free, len(free), in_place=in_place)


def test_plan_when_pages_or_tokens_run_out():
    rng = np.random.default_rng(0)
    run_plan(rng, 4, 16, 8, 40, [0, 15, 16, 3], [40, 2, 1, 2], 64, None, [3, 9, 1, 30], 4)      # third has no page, fourth needs none
    run_plan(rng, 3, 16, 8, 40, [0, 0, 0], [20, 20, 1], 30, None, list(range(20)), 20)           # second does not fit in 30 tokens
    run_plan(rng, 2, 16, 8, 40, [5, 5], [3, 3], 0, None, [1], 1)                                  # room for no token at all
    run_plan(rng, 2, 16, 8, 40, [16, 16], [1, 1], 4, None, [], 0)                                 # an empty list
    run_plan(rng, 2, 16, 8, 40, [16, 16], [1, 1], 4, None, [7] * 40, 1000)                        # a count beyond the pool: clamped
    run_plan(rng, 2, 16, 8, 40, [16, 16], [1, 1], 4, None, [7], -5)


def test_plan_bad_slots_lengths_and_pages():
    rng = np.random.default_rng(1)
    cfg = config(page=16, batch=6, pages=4, n_pages=40)
    run_plan(rng, 5, 16, 4, 40, [0, 3, 60, -1, 3], [4, 4, 5, 2, -2], 20, [0, 6, 2, 3, -1], list(range(9)), 9, cfg=cfg)
    run_plan(rng, 2, 16, 4, 40, [20, 1], [20, 1], 30, [1, 0], list(range(9)), 9, bad_page=(1, 1), cfg=cfg)
    run_plan(rng, 2, 16, 4, 40, [20, 1], [20, 1], 30, [1, 0], [5, 77, 2], 3, cfg=cfg)             # a bad id on the free list
    p, _ = run_plan(rng, 2, 16, 4, 40, [64, 0], [0, 64], 64, None, list(range(9)), 9)             # a full sequence
    assert p.seq_lens.tolist() == [64, 64]


def test_plan_largest_batch():
    rng = np.random.default_rng(2)
    B = 8192
    lens, new = rng.integers(0, 200, B).tolist(), rng.integers(0, 3, B).tolist()
    need = sum(-(-(a + b) // 16) - -(-a // 16) for a, b in zip(lens, new))
    run_plan(rng, B, 16, 13, need + 40, lens, new, sum(new) - 5, None, rng.permutation(need + 40)[: need - 3].tolist(), need - 3)


def test_release_gives_pages_back_in_order():
    cfg = config(page=16, batch=5, pages=4, n_pages=40)
    table = np.arange(20).reshape(5, 4) + 10
    table[2, 1] = 99
    free, count, st = dev([1, 2] + [0] * 38), dev([2]), dev([0])
    binding.release_pages(cfg, dev(table), dev([17, 0, 33, 65]), free, count, seq_slots=dev([4, 0, 2, 1]), status=st)
    assert free.tolist()[: count.item()] == [1, 2, 26, 27, 18, 20] and st.item() in (-8, -11)
    # a list that is full already takes nothing
    free, count, st = dev(list(range(40))), dev([39]), dev([0])
    binding.release_pages(cfg, dev(table), dev([64]), free, count, seq_slots=dev([0]), status=st)
    assert count.item() == 40 and free.tolist()[39] == 10 and st.item() == -4


def test_release_then_plan_takes_the_same_pages():
    rng = np.random.default_rng(3)
    cfg = config(page=32, batch=300, pages=40, n_pages=9000)
    table = torch.zeros(300, 40, dtype=torch.int32, device="cuda")
    free, count = dev(rng.permutation(9000)), dev([9000])
    before = free.tolist()
    new = rng.integers(0, 1200, 300)
    lens = torch.zeros(300, dtype=torch.int32, device="cuda")
    p = binding.plan_tokens(cfg, table, lens, dev(new), free, count, int(new.sum()),
                            out=binding.StepPlan(300, int(new.sum()), "cuda", seq_lens=lens, free_count=count))
    used = int((-(-new // 32)).sum())
    assert count.item() == 9000 - used and lens.tolist() == new.tolist()
    assert len(set(p.slot_map.tolist())) == int(new.sum())
    binding.release_pages(cfg, table, lens, free, count)
    assert count.item() == 9000 and sorted(free.tolist()) == sorted(before)


# ---- rotate -----------------------------------------------------------------------------------------------------
SECTIONS = {1: lambda h: [h], 2: lambda h: [h // 2, h - h // 2], 3: lambda h: [h // 4, 3 * h // 8, h - h // 4 - 3 * h // 8],
            4: lambda h: [0, h // 2, h // 4, h // 4]}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d,rot,axes,interleaved,inverse,place", [
    (1, 128, 128, 1, False, False, "new"), (5, 64, 64, 3, False, True, "new"), (700, 128, 64, 3, True, False, "in place"),
    (37, 128, 16, 2, True, True, "new"), (2, 64, 32, 4, False, False, "in place"), (601, 64, 48, 4, True, False, "slices")])
def test_rotate_matches_plain_form(dtype, T, d, rot, axes, interleaved, inverse, place):
    rng = np.random.default_rng(T + d + rot)
    cfg = config(n_q=6 if d == 64 else 4, n_kv=3 if d == 64 else 2, d=d, dtype=dtype)
    nq, nk, dt = cfg.n_q_heads, cfg.n_kv_heads, DT[dtype][1]
    qkv = torch.tensor(rng.standard_normal((T, (nq + 2 * nk) * d)), dtype=dt, device="cuda")
    q, k = qkv[:, : nq * d].view(T, nq, d), qkv[:, nq * d:(nq + nk) * d].view(T, nk, d)
    pos = rng.integers(-5, 1 << 20, (axes, T))
    pos[0, 0] = 0
    sec, theta = SECTIONS[axes](rot // 2), 10000.0
    q0, k0, v0 = f64(q), f64(k), qkv[:, (nq + nk) * d:].clone()
    kw = {}
    if place == "in place":
        kw = dict(q_out=q, k_out=k)
    elif place == "slices":
        other = torch.empty(T, 2 * (nq + nk) * d, dtype=dt, device="cuda")
        kw = dict(q_out=other[:, : nq * d].view(T, nq, d), k_out=other[:, nq * d:(nq + nk) * d].view(T, nk, d))
    qo, ko = binding.rotate(cfg, q, k, dev(pos), theta, sections=sec, rot_dim=rot, interleaved=interleaved, inverse=inverse, **kw)
    for got, x in ((qo, q0), (ko, k0)):
        ref = R.rotate(x, pos, theta, sec, rot, interleaved, inverse)
        # half a step of the result's type, and: cos and sin to 2^-22 (the remainder of a turn rounded to fp32, 2^-24 pi, and
        # their own two units), two products and a sum, 3 2^-24, each of |x1| + |x2|
        pair = np.abs(x).copy()
        half = rot // 2
        pair[..., :half] = pair[..., half:rot] = np.abs(x[..., :half]) + np.abs(x[..., half:rot])
        pair[..., rot:] = 0
        assert (np.abs(f64(got) - ref) <= EPS[dtype] / 2 * np.abs(ref) + 2.0 ** -21 * pair).all()
    assert torch.equal(qkv[:, (nq + nk) * d:], v0)


def test_rotate_is_its_own_gradient_and_turns_back():
    rng = np.random.default_rng(8)
    cfg = config(n_q=4, n_kv=2, d=64, dtype="fp32")
    T, sec = 9, [8, 12, 12]
    x, w = (torch.tensor(rng.standard_normal((T, 4, 64)), dtype=torch.float32, device="cuda") for _ in range(2))
    pos = dev(rng.integers(0, 3000, (3, T)))
    turn = lambda t, inv=False: binding.rotate(cfg, t, None, pos, 1e4, sections=sec, inverse=inv)[0]  # noqa: E731
    assert (turn(turn(x), True) - x).abs().max() < 1e-5
    # gradient of sum(w * rotate(x)) against differences: the map is linear, so a difference over h = 1/2 is exact
    grad = turn(w, True)
    for _ in range(20):
        i = tuple(rng.integers(0, n) for n in (T, 4, 64))
        up, dn = x.clone(), x.clone()
        up[i] += 0.5
        dn[i] -= 0.5
        diff = (w.double() * (turn(up).double() - turn(dn).double())).sum().item()
        assert abs(diff - grad[i].item()) < 1e-4
    q_only, none = binding.rotate(cfg, x, None, pos, 1e4, sections=sec)
    assert none is None and torch.equal(q_only, turn(x))
    k_none, k_only = binding.rotate(cfg, None, x[:, :2], pos, 1e4, sections=sec)
    assert k_none is None and torch.equal(k_only, turn(x)[:, :2])
    e, _ = binding.rotate(cfg, x[:0], None, pos[:, :0], 1e4, sections=sec)
    assert e.shape == (0, 4, 64)


# ---- append -----------------------------------------------------------------------------------------------------
class Program:
    """A cache, its block table and free list, and the plain copy of every token."""

    def __init__(self, cfg, fmt, seed=0, dtype="bf16"):
        self.cfg, self.fmt, self.dtype = cfg, fmt, dtype
        self.rng = np.random.default_rng(seed)
        B = cfg.max_batch
        self.cache = binding.QuantCache(cfg, fmt)
        self.table = torch.zeros(B, cfg.max_pages_per_seq, dtype=torch.int32, device="cuda")
        self.free, self.count = dev(self.rng.permutation(cfg.n_pages)), dev([cfg.n_pages])
        self.slots = self.rng.permutation(B)
        self.lens = [0] * B
        self.ref = R.Cache(fmt, B)
        self.status = dev([0])

    def rows(self, T, heads, scale=1.0):
        x = self.rng.standard_normal((T, heads, self.cfg.head_dim)) * scale
        return torch.tensor(x, dtype=DT[self.dtype][1], device="cuda")

    def plan(self, new):
        B = len(new)
        p = binding.plan_tokens(self.cfg, self.table, dev(self.lens[:B]), dev(new), self.free, self.count, sum(new),
                                seq_slots=dev(self.slots[:B]), status=self.status)
        self.count = p.free_count
        return p

    def step(self, new, k=None, v=None):
        """Append `new[b]` tokens to every sequence."""
        T, H = sum(new), self.cfg.n_kv_heads
        p = self.plan(new)
        k = self.rows(T, H) if k is None else k
        v = self.rows(T, H, 2.0) if v is None else v
        self.cache.append(k, v, p.slot_map, p.token_seqs, p.cu_tokens, seq_slots=dev(self.slots[: len(new)]), status=self.status)
        at = 0
        for b, n in enumerate(new):
            if n:
                self.ref.append(b, k[at:at + n].float().cpu().numpy(), v[at:at + n].float().cpu().numpy())
            at += n
            self.lens[b] += n
        return p

    def held(self, b):
        """What the cache stands for, read back through the block table: (k, v) [len][H][d] float64."""
        cfg, n = self.cfg, self.lens[b]
        P, full = cfg.page_tokens, n // BLOCK * BLOCK
        pages = self.table[int(self.slots[b])].long()[: -(-n // P)]
        out = []
        for codes, scales, tail in ((self.cache.k_codes, self.cache.k_scales, self.cache.k_tail),
                                    (self.cache.v_codes, self.cache.v_scales, self.cache.v_tail)):
            c = codes.view(torch.uint8)[pages].view(codes.dtype).float().double()
            x = c * scales[pages].double().repeat_interleave(BLOCK, -1)[..., None]
            x = x.permute(0, 2, 1, 3).reshape(-1, cfg.n_kv_heads, cfg.head_dim)[:full]
            w = tail[int(self.slots[b])].double().permute(1, 0, 2)[: n - full]
            out.append(torch.cat([x, w]).cpu().numpy())
        return out

    def check_cache(self):
        for b in range(self.cfg.max_batch):
            if self.lens[b]:
                k, v = self.held(b)
                for got, ref in ((k, self.ref.values(self.ref.k[b])), (v, self.ref.values(self.ref.v[b]))):
                    full = self.lens[b] // BLOCK * BLOCK
                    assert np.array_equal(got[:full], ref[:full], equal_nan=True)      # codes and scales to the bit
                    tail = (self.ref.k if got is k else self.ref.v)[b][full:]
                    assert np.array_equal(got[full:], tail.astype(np.float64), equal_nan=True)
        assert self.status.item() == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,page,n_kv", [("bf16", 128, 16, 8), ("bf16", 64, 64, 3), ("fp32", 128, 32, 2), ("fp32", 64, 128, 1)])
def test_append_matches_plain_form(fmt, dtype, d, page, n_kv):
    cfg = config(n_q=n_kv, n_kv=n_kv, d=d, page=page, batch=5, pages=1024 // page, n_pages=8192 // page, dtype=dtype)
    p = Program(cfg, fmt, seed=d + page, dtype=dtype)
    for new in ([1, 16, 15, 17, 0], [1, 1, 1, 1, 1], [40, 3, 200, 16, 14], [15, 33, 1, 31, 1], [7, 29, 64, 47, 1]):
        p.step(new)
        p.check_cache()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_does_not_depend_on_the_chunks(fmt):
    cfg = config(n_q=2, n_kv=2, d=64, batch=2, pages=16, n_pages=64)
    k, v = (torch.randn(2, 150, 2, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(i)).bfloat16() for i in (1, 2))
    held = []
    for cuts in ([150], [1] * 150, [5, 30, 48, 1, 2, 64], [31, 33, 86]):
        p = Program(cfg, fmt, seed=9)
        at = 0
        for n in cuts:
            kk, vv = k[:, at:at + n].reshape(-1, 2, 64), v[:, at:at + n].reshape(-1, 2, 64)
            p.step([n, n], kk, vv)
            at += n
        p.check_cache()
        held.append([x for b in (0, 1) for x in p.held(b)])
    for other in held[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(held[0], other))


def test_append_extremes():
    """Zeros, values at the ends of the range, infinities and NaN; another block and another head are left alone."""
    cfg = config(n_q=2, n_kv=2, d=128, batch=1, pages=16, n_pages=64, dtype="fp32")
    for fmt in ("int8", "e4m3"):
        p = Program(cfg, fmt, dtype="fp32")
        k = torch.randn(112, 2, 128, device="cuda")
        k[0:16, 0] = 0
        k[16:32, 0] *= 1e-36
        k[32:48, 0] *= 3e37
        k[48, 0, 5] = float("inf")
        k[64, 0, 7] = float("nan")
        k[95, 0, 127] = -float("inf")
        k[96:112, 0] *= 1e-44
        p.step([112], k, k.flip(1).contiguous())
        p.check_cache()
        s = p.cache.k_scales[p.table[int(p.slots[0])].long()[:7], :, 0].cpu().numpy()
        assert np.isnan(s[:, 0]).tolist() == [False, False, False, True, True, True, False] and not np.isnan(s[:, 1]).any()
        assert s[0, 0] == np.float32(2.0 ** -100)


def test_append_strided_rows_and_skipped_tokens():
    cfg = config(n_q=4, n_kv=2, d=128, batch=2, pages=8, n_pages=16)
    p, q = Program(cfg, "int8", seed=4), Program(cfg, "int8", seed=4)
    qkv = torch.randn(50, 8 * 128, device="cuda").bfloat16()
    k, v = qkv[:, 512:768].view(50, 2, 128), qkv[:, 768:].view(50, 2, 128)
    p.step([20, 30], k, v)
    q.step([20, 30], k.contiguous(), v.contiguous())
    p.check_cache()
    for a, b in zip(p.held(0) + p.held(1), q.held(0) + q.held(1)):
        assert np.array_equal(a, b)
    # rows that are skipped (-1), outside the pool, or of no sequence: nothing is written, the status tells of the bad ones
    before = [t.clone() for t in (p.cache.k_codes, p.cache.v_codes, p.cache.k_scales, p.cache.v_scales, p.cache.k_tail, p.cache.v_tail)]
    st = dev([0])
    p.cache.append(k[:3], v[:3], dev([-1, -1, -1], torch.int64), dev([0, 0, 1]), dev([0, 2, 3]), status=st)
    assert st.item() == 0
    for rows, seqs, cu in (([256, 5, 6], [0, 0, 0], [0, 3, 3]), ([-7, 300, 1 << 40], [0, 0, 1], [0, 2, 3]), ([1, 2, 3], [2, -1, 9], [0, 2, 3]),
                           ([1, 2, 3], [0, 0, 1], [2, 9, -1])):
        st.zero_()
        p.cache.append(k[:1], v[:1], dev(rows[:1], torch.int64), dev(seqs[:1]), dev(cu), status=st)
        assert st.item() == -8
    after = (p.cache.k_codes, p.cache.v_codes, p.cache.k_scales, p.cache.v_scales, p.cache.k_tail, p.cache.v_tail)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, after))


# ---- attention --------------------------------------------------------------------------------------------------
def check_attention(p, new, q, out, softcap=0.0, slopes=None, prefix=None):
    cfg = p.cfg
    at = 0
    for b, n in enumerate(new):
        if n:
            k, v = p.ref.values(p.ref.k[b]), p.ref.values(p.ref.v[b])
            ref, size = R.attend(f64(q[at:at + n]), k, v, cfg.head_dim ** -0.5, softcap, slopes, prefix[b] if prefix else 0)
            tol = R.tolerance(ref, size, p.lens[b], EPS[p.dtype], p.dtype == "bf16",
                              p.dtype == "bf16" and n * cfg.n_q_heads // cfg.n_kv_heads >= CHUNK_ROWS, softcap, slopes)
            err = np.abs(f64(out[at:at + n]) - ref)
            assert (err <= tol).all(), (b, n, p.lens[b], float((err / tol).max()))
        at += n


def attend(p, new, q, **kw):
    cu = dev(np.concatenate([[0], np.cumsum(new)]))
    B = len(new)
    if "slopes" in kw:
        kw["alibi_slopes"] = dev(kw.pop("slopes"), torch.float32)
    if "prefix" in kw:
        kw["prefix_lens"] = dev(kw.pop("prefix"))
    return p.cache.attention(q, p.table, dev(p.lens[:B]), cu_tokens=cu, max_new=max(1, max(new)), seq_slots=dev(p.slots[:B]), status=p.status, **kw)


SHAPES = [("bf16", 128, 16, 8, 2), ("bf16", 64, 32, 4, 4), ("bf16", 128, 64, 8, 1), ("fp32", 128, 16, 4, 2), ("fp32", 64, 128, 8, 1),
          ("bf16", 64, 16, 2, 1)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,page,n_q,n_kv", SHAPES)
def test_decode_matches_plain_form(fmt, dtype, d, page, n_q, n_kv):
    lens = [1, 15, 16, 17, 300, 333, 128, 2]
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=8, pages=512 // page, n_pages=4096 // page, dtype=dtype)
    p = Program(cfg, fmt, seed=d + n_q, dtype=dtype)
    p.step(lens)
    q = p.rows(8, n_q, 2.0)
    out = p.cache.attention(q, p.table, dev(p.lens), seq_slots=dev(p.slots), status=p.status)
    check_attention(p, [1] * 8, q, out)
    assert torch.equal(out, attend(p, [1] * 8, q))
    assert p.status.item() == 0


@pytest.mark.parametrize("opts", [dict(softcap=5.0), dict(softcap=50.0), dict(slopes=True), dict(prefix=True),
                                  dict(softcap=20.0, slopes=True, prefix=True)])
@pytest.mark.parametrize("fmt,dtype,d,n_q,n_kv", [("int8", "bf16", 128, 8, 2), ("e4m3", "fp32", 64, 4, 4), ("int8", "fp32", 128, 8, 1)])
def test_score_options_and_drafts(opts, fmt, dtype, d, n_q, n_kv):
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=16, batch=6, pages=32, n_pages=160, dtype=dtype)
    p = Program(cfg, fmt, seed=7, dtype=dtype)
    p.step([0, 16, 200, 37, 3, 250])
    new = [2, 1, 8, 5, 0, 7]
    p.step(new)
    kw = dict(opts)
    slopes = [2.0 ** (-8.0 * (h + 1) / n_q) for h in range(n_q)]
    if "slopes" in kw:
        kw["slopes"] = slopes
    if "prefix" in kw:
        kw["prefix"] = [2, 0, 100, 42, 7, 254]
    q = p.rows(sum(new), n_q, 3.0)
    out = attend(p, new, q, **dict(kw))
    check_attention(p, new, q, out, softcap=kw.get("softcap", 0.0), slopes=kw.get("slopes"), prefix=kw.get("prefix"))
    assert p.status.item() == 0


@pytest.mark.parametrize("fmt,dtype,d,page,n_q,n_kv,before,new", [
    ("int8", "bf16", 128, 16, 8, 2, [0, 100, 3], [40, 70, 1]), ("e4m3", "bf16", 64, 64, 4, 4, [0, 500], [300, 129]),
    ("e4m3", "bf16", 128, 32, 8, 1, [17, 0, 0], [130, 1, 64]), ("int8", "fp32", 64, 16, 2, 2, [5, 0], [33, 50]),
    ("int8", "bf16", 128, 128, 2, 2, [1, 255], [257, 128]), ("int8", "bf16", 64, 16, 8, 4, [0], [1])])
@pytest.mark.parametrize("opts", [{}, dict(softcap=10.0, slopes=True, prefix=True)])
def test_chunks_match_plain_form(fmt, dtype, d, page, n_q, n_kv, before, new, opts):
    B = len(new)
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=1024 // page, n_pages=4096 // page, dtype=dtype)
    p = Program(cfg, fmt, seed=3, dtype=dtype)
    p.step(before)
    p.step(new)
    kw = dict(opts)
    if kw:
        kw["slopes"] = [2.0 ** (-8.0 * (h + 1) / n_q) for h in range(n_q)]
        kw["prefix"] = [(n + o) * 2 // 3 for n, o in zip(new, before)]
    q = p.rows(sum(new), n_q, 2.0)
    out = attend(p, new, q, **dict(kw))
    check_attention(p, new, q, out, softcap=kw.get("softcap", 0.0), slopes=kw.get("slopes"), prefix=kw.get("prefix"))
    assert p.status.item() == 0


def sampled(rng, n):
    return sorted({0, 1, n // 2, n - 2, n - 1} | set(rng.integers(0, n, 12).tolist()) | set(range(60, min(n, 70))))


@pytest.mark.parametrize("opts", [{}, dict(softcap=50.0), dict(softcap=6.0), dict(softcap=0.5), dict(slopes=True), dict(prefix=True),
                                  dict(softcap=10.0, slopes=True, prefix=True)])
@pytest.mark.parametrize("fmt,d,page,n_q,n_kv,before,new", [
    ("int8", 128, 16, 16, 8, [0, 77], [400, 513]), ("e4m3", 64, 64, 8, 8, [300], [700]), ("e4m3", 128, 128, 32, 4, [1003, 0, 0], [150, 299, 1]),
    ("int8", 64, 32, 4, 4, [0, 9, 130], [640, 640, 641])])
def test_large_chunks_match_plain_form(opts, fmt, d, page, n_q, n_kv, before, new):
    """Sizes that go to the tcgen05 kernel: odd lengths, several items, open blocks in the last tile, every score transform."""
    B = len(new)
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=1280 // page, n_pages=B * 1280 // page)
    p = Program(cfg, fmt, seed=n_q + d)
    p.step(before)
    p.step(new)
    kw = dict(opts)
    if "slopes" in kw:
        kw["slopes"] = [2.0 ** (-8.0 * (h + 1) / n_q) for h in range(n_q)]
    if "prefix" in kw:
        kw["prefix"] = [(n + o) * 2 // 3 for n, o in zip(new, before)]
    q = p.rows(sum(new), n_q, 2.5)
    out = attend(p, new, q, **dict(kw))
    assert p.status.item() == 0 and torch.isfinite(out).all()
    at = 0
    for b, n in enumerate(new):
        only = sampled(p.rng, n) if n > 1 else [0]
        ref, size = R.attend(f64(q[at:at + n]), p.ref.values(p.ref.k[b]), p.ref.values(p.ref.v[b]), d ** -0.5, kw.get("softcap", 0.0),
                             kw.get("slopes"), kw["prefix"][b] if "prefix" in kw else 0, only=only)
        tol = R.tolerance(ref, size, p.lens[b], EPS["bf16"], True, True, kw.get("softcap", 0.0), kw.get("slopes"))
        err = np.abs(f64(out[at:at + n]) - ref)[only]
        assert (err <= tol[only]).all(), (b, n, float((err / tol[only]).max()))
        at += n


def test_chunk_whose_scores_grow_and_whose_prefix_is_all():
    """A reference that has to move in the middle of tiles (keys that grow along the sequence), rows that see the whole sequence, and
    the same chunk again: the result does not depend on what ran before."""
    cfg = config(n_q=8, n_kv=8, d=128, page=64, batch=1, pages=12, n_pages=12)
    p = Program(cfg, "int8", seed=31)
    k, v = p.rows(700, 8), p.rows(700, 8)
    k = (k.float() * torch.linspace(0.1, 12, 700, device="cuda")[:, None, None]).bfloat16()
    p.step([700], k, v)
    q = p.rows(650, 8, 2.0)
    for prefix in (0, 700):
        outs = [attend(p, [650], q, prefix=[prefix]) for _ in range(2)]
        assert torch.equal(outs[0], outs[1])
        only = sampled(p.rng, 650)
        ref, size = R.attend(f64(q), p.ref.values(p.ref.k[0]), p.ref.values(p.ref.v[0]), 128 ** -0.5, prefix=prefix, only=only)
        tol = R.tolerance(ref, size, 700, EPS["bf16"], True, True)
        err = np.abs(f64(outs[0]) - ref)[only]
        assert (err <= tol[only]).all(), float((err / tol[only]).max())


@pytest.mark.parametrize("kv", [0, 1])
def test_infinities_and_nan_in_masked_places_of_chunks(kv):
    cfg = config(n_q=8, n_kv=8, d=64, page=16, batch=1, pages=48, n_pages=60)
    nan, inf = float("nan"), float("inf")
    p = Program(cfg, "e4m3", seed=6)
    for t in (p.cache.k_tail, p.cache.v_tail, p.cache.k_scales, p.cache.v_scales):
        t.fill_(nan)
    x = [p.rows(650, 8), p.rows(650, 8)]
    x[kv][330, 0, 3], x[kv][648, 1, 9] = nan, inf        # blocks 320.. (codes) of head 0 and 640.. (open) of head 1
    p.step([650], *x)
    q = p.rows(650, 8)
    bad = np.isnan(f64(attend(p, [650], q))).any(-1)
    first = np.arange(650)
    assert (bad[:, 0] == (first >= 320)).all() and (bad[:, 1] == (first >= 640)).all() and not bad[:, 2:].any()


@pytest.mark.parametrize("n_q,n_kv,d,new", [(8, 2, 64, [16] * 250), (4, 4, 128, [64, 1, 100, 3, 80, 128] * 40), (8, 8, 64, [70, 260, 130] * 35)])
def test_many_chunks_of_few_rows(n_q, n_kv, d, new):
    """More items than SMs, several per CTA, most with one tile of query rows (the other one idle) beside sequences that the row
    kernel takes."""
    B = len(new)
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=32, batch=B, pages=12, n_pages=12 * B)
    p = Program(cfg, "e4m3", seed=21)
    before = [int(x) for x in p.rng.integers(0, 40, B)]
    p.step(before)
    p.step(new)
    q = p.rows(sum(new), n_q, 2.0)
    out = attend(p, new, q)
    assert p.status.item() == 0
    # (the oracle is slow: a sample of the sequences, all of them are finite)
    assert torch.isfinite(out).all()
    at = np.concatenate([[0], np.cumsum(new)])
    for b in sorted({0, 1, 2, B // 3, B // 2, B - 3, B - 2, B - 1}):
        k, v = p.ref.values(p.ref.k[b]), p.ref.values(p.ref.v[b])
        ref, size = R.attend(f64(q[at[b]:at[b + 1]]), k, v, d ** -0.5)
        tol = R.tolerance(ref, size, p.lens[b], EPS["bf16"], True, new[b] * n_q // n_kv >= CHUNK_ROWS)
        err = np.abs(f64(out[at[b]:at[b + 1]]) - ref)
        assert (err <= tol).all(), (b, new[b], float((err / tol).max()))


@pytest.mark.parametrize("opts", [{}, dict(softcap=8.0), dict(softcap=20.0, slopes=True, prefix=True)])
@pytest.mark.parametrize("fmt,d,page,n_q,n_kv,before,new", [
    ("int8", 128, 64, 32, 8, [6000], [64]), ("e4m3", 64, 16, 8, 1, [9001, 0, 40], [129, 0, 1]), ("int8", 128, 128, 4, 4, [3, 5007], [1, 301])])
def test_chunk_of_few_items_is_split_along_the_keys(opts, fmt, d, page, n_q, n_kv, before, new):
    """Fewer items than SMs over long caches: each is cut into parts of a few key tiles, the last ones masked, and joined."""
    B = len(new)
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=9216 // page, n_pages=B * 9216 // page)
    p = Program(cfg, fmt, seed=n_q + 3 * d)
    p.step(before)
    p.step(new)
    kw = dict(opts)
    if "slopes" in kw:
        kw["slopes"] = [2.0 ** (-8.0 * (h + 1) / n_q) for h in range(n_q)]
    if "prefix" in kw:
        kw["prefix"] = [max(0, n + o - 20) for n, o in zip(new, before)]
    q = p.rows(sum(new), n_q, 2.5)
    out = attend(p, new, q, **dict(kw))
    assert torch.equal(out, attend(p, new, q, **dict(kw)))
    check_attention(p, new, q, out, softcap=kw.get("softcap", 0.0), slopes=kw.get("slopes"), prefix=kw.get("prefix"))
    assert p.status.item() == 0


def test_nan_in_one_part_of_a_split_chunk():
    cfg = config(n_q=8, n_kv=2, d=128, page=64, batch=1, pages=128, n_pages=128)
    p = Program(cfg, "int8", seed=16)
    k, v = p.rows(8000, 2), p.rows(8000, 2)
    v[4321, 0, 77] = float("nan")                        # seen by every row of head 0's group
    k[7990, 1, 5] = float("inf")                         # a block that only the last rows of head 1's group see
    p.step([8000], k, v)
    q = p.rows(500, 8, 2.0)
    out = f64(attend(p, [500], q))
    pos = np.arange(7500, 8000)
    bad = np.isnan(out).any(-1)
    assert bad[:, :4].all() and (bad[:, 4:] == (pos >= 7984)[:, None]).all()


@pytest.mark.parametrize("opts", [{}, dict(softcap=8.0, prefix=True)])
def test_many_chunks_of_few_rows_over_longer_caches(opts):
    """Several items per CTA, whole and cut ones, most with one tile of query rows; bad sequences and sequences of the row kernel
    between them; captured and replayed over what another call left in the workspace."""
    new = [16, 70, 1, 0, 16, 16, 90, 16] * 9
    B, n_q, n_kv, d = len(new), 16, 4, 64
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=64, batch=B, pages=16, n_pages=16 * B)
    p = Program(cfg, "e4m3", seed=22)
    before = [int(x) for x in p.rng.integers(600, 900, B)]
    p.step(before)
    p.step(new)
    kw = dict(opts)
    if "prefix" in kw:
        kw["prefix"] = [int(x) for x in p.rng.integers(0, 1000, B)]
    q = p.rows(sum(new), n_q, 2.0)
    out = attend(p, new, q, **dict(kw))
    assert p.status.item() == 0
    at = np.concatenate([[0], np.cumsum(new)])
    for b in sorted({0, 1, 2, 6, B // 3, B // 2, B - 2, B - 1}):
        k, v = p.ref.values(p.ref.k[b]), p.ref.values(p.ref.v[b])
        ref, size = R.attend(f64(q[at[b]:at[b + 1]]), k, v, d ** -0.5, kw.get("softcap", 0.0), None, kw["prefix"][b] if "prefix" in kw else 0)
        tol = R.tolerance(ref, size, p.lens[b], EPS["bf16"], True, new[b] * n_q // n_kv >= CHUNK_ROWS, kw.get("softcap", 0.0))
        err = np.abs(f64(out[at[b]:at[b + 1]]) - ref)
        assert (err <= tol).all(), (b, new[b], float((err / tol).max()))
    # two sequences whose slots do not exist: zeros there, the others as they were
    lens, slots, cu = dev(p.lens[:B]), dev(p.slots[:B]), dev(at)
    slots[5], slots[9] = -1, B
    extra = dict(softcap=kw.get("softcap", 0.0), prefix_lens=dev(kw["prefix"]) if "prefix" in kw else None)
    bad = torch.empty_like(out)
    call = lambda: p.cache.attention(q, p.table, lens, cu_tokens=cu, max_new=90, seq_slots=slots, status=p.status, out=bad, **extra)
    call()
    assert p.status.item() != 0
    keep = torch.ones(len(q), dtype=torch.bool, device="cuda")
    for b in (5, 9):
        keep[at[b]:at[b + 1]] = False
        assert (bad[at[b]:at[b + 1]] == 0).all()
    want = bad.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    p.cache.workspace.fill_(0xff)
    for _ in range(2):
        bad.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(bad, want)
    assert torch.isfinite(out).all() and torch.isfinite(bad).all()


def test_chunk_calls_with_bad_lengths_spare_rows_and_two_streams():
    """Sequences over max_new or shorter than their new tokens are zeros, rows behind the last sequence stay, the others as they should
    be; two calls on two streams, each with a workspace of its own, do not disturb each other."""
    cfg = config(n_q=16, n_kv=8, d=128, page=64, batch=6, pages=40, n_pages=240)
    p = Program(cfg, "int8", seed=41)
    p.step([2000, 1800, 900, 1500, 30, 2200])
    new = [150, 90, 260, 129, 64, 1]
    p.step(new)
    q = p.rows(sum(new) + 9, 16, 2.0)
    good = attend(p, new, q[:sum(new)])
    check_attention(p, new, q, good)
    at = np.concatenate([[0], np.cumsum(new)])
    lens = dev(p.lens[:6])
    lens[4] = 63
    call = dict(cu_tokens=dev(at), max_new=200, seq_slots=dev(p.slots[:6]))
    out = torch.full_like(q, 7.0)
    p.cache.attention(q, p.table, lens, out=out, status=p.status, **call)
    assert p.status.item() != 0
    for b in (2, 4):
        assert (out[at[b]:at[b + 1]] == 0).all()
        out[at[b]:at[b + 1]] = good[at[b]:at[b + 1]]
    check_attention(p, new, q, out[:sum(new)])
    assert (out[at[-1]:] == 7).all()
    p.status.zero_()
    other = binding.QuantCache(cfg, "int8", k_codes=p.cache.k_codes, v_codes=p.cache.v_codes, k_scales=p.cache.k_scales,
                               v_scales=p.cache.v_scales, k_tail=p.cache.k_tail, v_tail=p.cache.v_tail)
    q = q[:sum(new)]
    call = dict(cu_tokens=dev(at), max_new=260, seq_slots=dev(p.slots[:6]))
    lens = dev(p.lens[:6])
    want = p.cache.attention(q, p.table, lens, status=p.status, **call)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for _ in range(8):
        for st, c in zip(streams, (p.cache, other)):
            with torch.cuda.stream(st):
                outs.append(c.attention(q, p.table, lens, status=p.status, **call))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs) and p.status.item() == 0


def test_more_sequences_than_threads_with_chunks_among_them():
    """640 sequences, every tenth a chunk over a longer cache, the others one token; query rows inside a wider tensor."""
    B, n_q, n_kv, d = 640, 16, 8, 64
    new = [16 + b % 7 if b % 10 == 3 else b % 3 % 2 for b in range(B)]
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=64, batch=B, pages=20, n_pages=64 * 20 + 640)
    p = Program(cfg, "int8", seed=29)
    before = [int(p.rng.integers(900, 1200)) if b % 10 == 3 else b % 40 for b in range(B)]
    p.step(before)
    new = [40 + n if n >= 16 else n for n in new]
    p.step(new)
    q = p.rows(sum(new), n_q + 2 * n_kv, 2.0)[:, :n_q]
    out = attend(p, new, q)
    assert p.status.item() == 0 and torch.isfinite(out).all()
    at = np.concatenate([[0], np.cumsum(new)])
    for b in (3, 4, 13, 313, 316, 633, 637):
        if new[b] == 0:
            continue
        k, v = p.ref.values(p.ref.k[b]), p.ref.values(p.ref.v[b])
        ref, size = R.attend(f64(q[at[b]:at[b + 1]]), k, v, d ** -0.5)
        tol = R.tolerance(ref, size, p.lens[b], EPS["bf16"], True, new[b] * n_q // n_kv >= CHUNK_ROWS)
        err = np.abs(f64(out[at[b]:at[b + 1]]) - ref)
        assert (err <= tol).all(), (b, new[b], float((err / tol).max()))


def test_one_long_sequence_is_split_over_the_machine():
    cfg = config(n_q=4, n_kv=1, d=128, page=16, batch=1, pages=2000, n_pages=2100)
    p = Program(cfg, "int8", seed=5)
    p.step([31000])
    q = p.rows(1, 4, 3.0)
    out = attend(p, [1], q)
    check_attention(p, [1], q, out)


def test_scales_that_grow_and_shrink_along_a_sequence():
    """Running references must follow V blocks of very different size, and a dominating token in a small block."""
    cfg = config(n_q=2, n_kv=2, d=64, batch=1, pages=32, n_pages=40, dtype="fp32")
    p = Program(cfg, "int8", dtype="fp32")
    k, v = p.rows(400, 2), p.rows(400, 2)
    size = torch.tensor([1e-6, 1.0, 1e4, 0.0, 1e-3, 1e8, 1e-8, 1.0], device="cuda").repeat(4)[:25].repeat_interleave(16)
    v *= size[:, None, None]
    k[7] *= 6
    p.step([400], k, v)
    q = p.rows(1, 2, 3.0)
    out = attend(p, [1], q)
    check_attention(p, [1], q, out)


def test_infinities_and_nan_in_masked_places():
    cfg = config(n_q=4, n_kv=2, d=64, batch=2, pages=8, n_pages=30)
    nan, inf = float("nan"), float("inf")
    for kv in (0, 1):
        p = Program(cfg, "int8", seed=6)
        # whatever lies behind the last token -- in the tail, on unused rows and pages -- must not matter
        for t in (p.cache.k_tail, p.cache.v_tail, p.cache.k_scales, p.cache.v_scales):
            t.fill_(nan)
        p.step([20, 40])
        x = [p.rows(30, 2), p.rows(30, 2)]
        x[kv][14, 0, 3], x[kv][25, 0, 9] = nan, inf       # sequence 0, positions 34 (a block held as codes) and 45 (its open block: 32..)
        p.step([30, 0], *x)
        q = p.rows(30, 4)
        out = f64(attend(p, [30, 0], q))
        bad = np.isnan(out).any(-1)
        # queries up to position 31 see no bad block; from 32 on the heads of KV head 0 see block 2 with its NaN
        assert not bad[:12].any() and bad[12:, :2].all() and not bad[:, 2:].any()
        check = np.isfinite(out[:12]).all() and np.isfinite(out[:, 2:]).all()
        assert check


def test_rows_of_bad_sequences_are_zero_and_other_rows_stay():
    cfg = config(n_q=4, n_kv=2, d=64, batch=3, pages=4, n_pages=30)
    p = Program(cfg, "int8", seed=2)
    p.step([20, 33, 5])
    q = p.rows(9, 4)
    good = p.cache.attention(q[:6], p.table, dev(p.lens), cu_tokens=dev([0, 2, 4, 6]), max_new=2, seq_slots=dev(p.slots))

    def run(slots=None, lens=None, cu=(0, 2, 4, 6), max_new=2):
        st, out = dev([0]), torch.full((9, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        p.cache.attention(q, p.table, dev(lens or p.lens), cu_tokens=dev(cu), max_new=max_new, seq_slots=dev(slots if slots is not None else p.slots),
                          out=out, status=st)
        return st.item(), out
    st, out = run()
    assert st == 0 and torch.equal(out[:6], good) and (out[6:] == 7).all()          # rows behind the last sequence
    for kw, code in ((dict(slots=[int(p.slots[0]), 3, int(p.slots[2])]), -8), (dict(slots=[int(p.slots[0]), -1, int(p.slots[2])]), -8),
                     (dict(lens=[20, 1, 5]), -11), (dict(lens=[20, 65, 5]), -11), (dict(lens=[20, -4, 5]), -11)):
        st, out = run(**kw)
        assert st == code and torch.equal(out[:2], good[:2]) and (out[2:4] == 0).all() and torch.equal(out[4:6], good[4:6])
    st, out = run(cu=(0, 2, 5, 6), max_new=2)                                      # more new tokens than max_new says
    assert st == -11 and torch.equal(out[:2], good[:2]) and (out[2:5] == 0).all()
    for cu in ((0, 2, 1, 3), (0, 2, 11, 12), (0, 2, -3, 2)):                       # offsets that decrease or pass the tokens
        st, out = run(cu=cu, max_new=9)
        assert st == -11 and torch.equal(out[:2], good[:2])
    st, out = run(cu=(0, 0, 0, 0))
    assert st == 0 and (out == 7).all()


def test_bad_page_is_reported_and_other_sequences_hold():
    cfg = config(n_q=4, n_kv=2, d=64, batch=2, pages=4, n_pages=30)
    p = Program(cfg, "e4m3", seed=2)
    p.step([50, 50])
    q = p.rows(2, 4)
    good = attend(p, [1, 1], q)
    for page in (30, -1, 1 << 30):
        t = p.table.clone()
        t[int(p.slots[0]), 1] = page
        st = dev([0])
        out = p.cache.attention(q, t, dev(p.lens), seq_slots=dev(p.slots), status=st)
        assert st.item() == -8 and torch.equal(out[1], good[1])


# ---- together ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("e4m3", "fp32")])
def test_a_run_of_steps(fmt, dtype):
    """Prompts, decode steps, a mixed step, a finished request whose pages another one takes: plan, rotate, append, attend."""
    cfg = config(n_q=8, n_kv=2, d=64, page=16, batch=4, pages=16, n_pages=24, dtype=dtype)
    p = Program(cfg, fmt, seed=11, dtype=dtype)
    dt = DT[dtype][1]

    def step(new):
        T, B = sum(new), len(new)
        plan = p.plan(new)
        qkv = torch.tensor(p.rng.standard_normal((T, 12 * 64)), dtype=dt, device="cuda")
        q, k, v = qkv[:, :512].view(T, 8, 64), qkv[:, 512:640].view(T, 2, 64), qkv[:, 640:].view(T, 2, 64)
        q, k = binding.rotate(cfg, q, k, plan.positions, 10000.0)
        p.cache.append(k, v, plan.slot_map, plan.token_seqs, plan.cu_tokens, seq_slots=dev(p.slots[:B]), status=p.status)
        out = p.cache.attention(q, p.table, plan.seq_lens, cu_tokens=plan.cu_tokens, max_new=max(new), seq_slots=dev(p.slots[:B]), softcap=30.0,
                                status=p.status)
        at = 0
        for b, n in enumerate(new):
            if n:
                p.ref.append(b, k[at:at + n].float().cpu().numpy(), v[at:at + n].float().cpu().numpy())
            p.lens[b] += n
            at += n
        assert plan.seq_lens.tolist() == p.lens
        p.check_cache()
        check_attention(p, new, q, out, softcap=30.0)
    step([33, 5, 70, 0])
    for _ in range(3):
        step([1, 1, 1, 0])
    step([1, 40, 1, 90])
    assert p.count.item() == 24 - 3 - 3 - 5 - 6
    # request 2 ends, another takes its slot
    binding.release_pages(cfg, p.table, dev([p.lens[2]]), p.free, p.count, seq_slots=dev(p.slots[2:3]))
    assert p.count.item() == 12
    p.lens[2], p.ref.k[2], p.ref.v[2] = 0, None, None
    step([2, 1, 100, 1])
    step([1, 1, 1, 1])


def test_a_captured_decode_step_replays_and_two_graphs_share_a_workspace():
    cfg = config(n_q=8, n_kv=2, d=128, page=16, batch=3, pages=16, n_pages=40)
    p = Program(cfg, "int8", seed=12)
    p.step([20, 31, 100])
    slots = dev(p.slots)
    new, lens = dev([1, 1, 1]), dev(p.lens)
    qkv = torch.zeros(3, 12 * 128, dtype=torch.bfloat16, device="cuda")
    plan = binding.StepPlan(3, 3, "cuda", seq_lens=lens, free_count=p.count)
    layers = [p.cache, binding.QuantCache(cfg, "int8", workspace=p.cache.workspace)]
    layers[1].k_codes.copy_(layers[0].k_codes); layers[1].v_codes.copy_(layers[0].v_codes)                 # noqa: E702
    layers[1].k_scales.copy_(layers[0].k_scales); layers[1].v_scales.copy_(layers[0].v_scales)             # noqa: E702
    layers[1].k_tail.copy_(layers[0].k_tail); layers[1].v_tail.copy_(layers[0].v_tail)                     # noqa: E702
    outs = [torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in layers]

    def begin():
        binding.plan_tokens(cfg, p.table, lens, new, p.free, p.count, 3, seq_slots=slots, out=plan, status=p.status)

    def layer(i):
        q, k, v = qkv[:, :1024].view(3, 8, 128), qkv[:, 1024:1280].view(3, 2, 128), qkv[:, 1280:].view(3, 2, 128)
        q, k = binding.rotate(cfg, q, k, plan.positions, 10000.0)
        layers[i].append(k, v, plan.slot_map, plan.token_seqs, plan.cu_tokens, seq_slots=slots, status=p.status)
        layers[i].attention(q, p.table, lens, seq_slots=slots, out=outs[i], status=p.status)
        return k, v
    keep = []
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0], stream=stream):
        begin()
        keep.append(layer(0))
    with torch.cuda.graph(graphs[1], stream=stream):
        keep.append(layer(1))
    for i in range(20):
        qkv.copy_(torch.randn(3, 12 * 128, device="cuda", generator=torch.Generator("cuda").manual_seed(i)))
        graphs[0].replay()
        graphs[1].replay()
        k, v = keep[0]
        for b in range(3):
            p.ref.append(b, k[b:b + 1].float().cpu().numpy(), v[b:b + 1].float().cpu().numpy())
            p.lens[b] += 1
        assert lens.tolist() == p.lens and torch.equal(outs[0], outs[1])
        if i in (0, 11, 12, 19):
            p.check_cache()
            q = binding.rotate(cfg, qkv[:, :1024].view(3, 8, 128), None, plan.positions, 10000.0)[0]
            check_attention(p, [1] * 3, q, outs[0])


def test_on_another_stream():
    cfg = config(n_q=8, n_kv=2, d=128, page=16, batch=2, pages=16, n_pages=40)
    p = Program(cfg, "e4m3", seed=13)
    p.step([40, 90])
    q = p.rows(2, 8)
    ref = attend(p, [1, 1], q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(ref)
    lens, slots = dev(p.lens), dev(p.slots)
    torch.cuda.synchronize()
    got = p.cache.attention(q, p.table, lens, seq_slots=slots, out=out, stream=s)
    s.synchronize()
    assert torch.equal(got, ref)
    with torch.cuda.stream(s):
        got = p.cache.attention(q, p.table, lens, seq_slots=slots)
    s.synchronize()
    assert torch.equal(got, ref)
