"""The 4-bit cache on the GPU: every operator against its plain form, their edge cases, and a run of steps as a program makes them."""
import numpy as np
import pytest
import torch

from paper_2603_22910_b200 import binding
from tests import fp4_ref as F
from tests import serving_ref as R
from tests.test_gpu_serving import CHUNK_ROWS, DT, EPS, config, dev, f64, sampled
from tests.test_gpu_streams import owner

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
SECTIONS = {1: lambda h: [h], 2: lambda h: [h // 2, h - h // 2], 3: lambda h: [h // 4, 3 * h // 8, h - h // 4 - 3 * h // 8],
            4: lambda h: [0, h // 2, h // 4, h // 4]}


class Program:
    """A cache, the block table of its sequences (pages in any order, block table rows too), and what every sequence should hold."""

    def __init__(self, cfg, seed=0, k_unit=0.25, v_unit=0.0625, garbage=True):
        self.cfg, self.dtype = cfg, "bf16" if cfg.dtype == binding.ECHOKV_BF16 else "fp32"
        self.rng = np.random.default_rng(seed)
        self.cache = binding.Fp4Cache(cfg, k_unit=k_unit, v_unit=v_unit)
        if garbage:                               # (whatever lies behind the last token must not matter: NaN scales everywhere)
            self.cache.blocks.fill_(0xff)
            self.cache.bounds.fill_(77)
            self.cache.bound_scales.fill_(NAN)
        B, N = cfg.max_batch, cfg.n_pages
        self.slots = self.rng.permutation(B).astype(np.int32)
        self.table = dev(np.full((B, cfg.max_pages_per_seq), N + 5))
        self.free, self.count, self.status = dev(self.rng.permutation(N)), dev([N]), dev([0])
        self.lens = [0] * B
        self.k, self.v = [np.zeros((0, cfg.n_kv_heads, cfg.head_dim))] * B, [np.zeros((0, cfg.n_kv_heads, cfg.head_dim))] * B

    def rows(self, T, heads, size=1.0):
        return torch.tensor(self.rng.standard_normal((T, heads, self.cfg.head_dim)) * size, dtype=DT[self.dtype][1], device="cuda")

    def plan(self, new):
        self.new = new
        return binding.plan_tokens(self.cfg, self.table, dev(self.lens[:len(new)]), dev(new), self.free, self.count, sum(new),
                                   seq_slots=dev(self.slots[:len(new)]), status=self.status, out=binding.StepPlan(
                                       len(new), sum(new), "cuda", free_count=self.count))

    def step(self, new, k=None, v=None, **kw):
        """`new` tokens of the first sequences (random ones), appended without a rotation."""
        T = sum(new)
        p = self.plan(new)
        k = self.rows(T, self.cfg.n_kv_heads) if k is None else k
        v = self.rows(T, self.cfg.n_kv_heads) if v is None else v
        if T:
            self.cache.append(k, v, p.slot_map, status=self.status, **kw)
        self.note(new, k.float().cpu().numpy(), v.float().cpu().numpy())
        return p

    def note(self, new, k, v):
        at = 0
        for b, n in enumerate(new):
            kk, vv = F.token(k[at:at + n], v[at:at + n], self.cache.k_unit, self.cache.v_unit)
            self.k[b], self.v[b] = np.concatenate([self.k[b], kk]), np.concatenate([self.v[b], vv])
            self.lens[b] += n
            at += n

    def pages_of(self, b):
        P = self.cfg.page_tokens
        return self.table[int(self.slots[b]), :-(-self.lens[b] // P)].cpu().numpy()

    def check_cache(self, bounds=True):
        P, d = self.cfg.page_tokens, self.cfg.head_dim
        blocks = self.cache.blocks.cpu().numpy()
        for b, n in enumerate(self.lens):
            if not n:
                continue
            pages = self.pages_of(b)
            k, v = [x.transpose(0, 2, 1, 3).reshape(len(pages) * P, -1, d)[:n] for x in F.unpack(blocks[pages], d)]
            assert np.array_equal(k * self.cache.k_unit, self.k[b], equal_nan=True) and np.array_equal(v * self.cache.v_unit, self.v[b])
            if not bounds:
                continue
            got, scales = self.cache.bounds[pages.tolist()].cpu().numpy(), self.cache.bound_scales[pages.tolist()].cpu().numpy()
            for j in range(len(pages)):
                for h in range(self.cfg.n_kv_heads):
                    want, s = F.bounds(k[j * P:min(n, (j + 1) * P), h])
                    assert np.array_equal(got[j, h], want) and np.array_equal(scales[j, h], s, equal_nan=True), (b, j, h)

    def attend(self, new, q, **kw):
        B = len(new)
        if "slopes" in kw:
            kw["alibi_slopes"] = dev(kw.pop("slopes"), torch.float32)
        if "prefix" in kw:
            kw["prefix_lens"] = dev(kw.pop("prefix"))
        return self.cache.attention(q, self.table, dev(self.lens[:B]), cu_tokens=dev(np.concatenate([[0], np.cumsum(new)])), max_new=max(1, max(new)),
                                    seq_slots=dev(self.slots[:B]), status=self.status, **kw)

    def check_attention(self, new, q, out, softcap=0.0, slopes=None, prefix=None, only=None):
        g, at = self.cfg.n_q_heads // self.cfg.n_kv_heads, 0
        for b, n in enumerate(new):
            if n:
                rows = sampled(self.rng, n) if only and n > 60 else list(range(n))
                ref, size = R.attend(f64(q[at:at + n]), self.k[b], self.v[b], self.cfg.head_dim ** -0.5, softcap, slopes, prefix[b] if prefix else 0,
                                     only=rows)
                tol = F.tolerance(ref, size, self.lens[b], EPS[self.dtype], self.dtype == "bf16", self.dtype == "bf16" and n * g >= CHUNK_ROWS,
                                  softcap, slopes)
                err = np.abs(f64(out[at:at + n]) - ref)[rows]
                assert (err <= tol[rows]).all(), (b, n, self.lens[b], float((err / tol[rows]).max()))
            at += n

    def tokens(self, new):
        """(sequence, position) of the last `new` tokens of the sequences."""
        seqs = np.repeat(np.arange(len(new)), new)
        pos = np.concatenate([np.arange(self.lens[b] - n, self.lens[b]) for b, n in enumerate(new)] + [np.zeros(0, int)])
        return seqs, pos


# ---- append and read ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,page,n_q,n_kv,rot,axes,interleaved,new,place", [
    (128, 16, 8, 2, 128, 1, False, [1, 1, 1, 1], "new"), (64, 32, 4, 4, 48, 3, True, [5, 0, 70, 33], "slices"), (128, 64, 8, 1, 64, 2, False, [200, 3, 64, 1], "in place"),
    (64, 128, 6, 3, 16, 4, True, [17, 150, 1, 16], "slices"), (128, 16, 4, 4, 96, 1, False, [640, 1, 0, 30], "new")])
def test_append_turns_and_holds(dtype, d, page, n_q, n_kv, rot, axes, interleaved, new, place):
    cfg = config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=4, pages=1024 // page, n_pages=4096 // page, dtype=dtype)
    p = Program(cfg, seed=d + rot)
    p.step([3, 40, 0, 15])
    T, dt = sum(new), DT[dtype][1]
    plan = p.plan(new)
    qkv = torch.tensor(p.rng.standard_normal((T, (n_q + 2 * n_kv) * d)), dtype=dt, device="cuda")
    q, k, v = [x.reshape(T, -1, d) for x in qkv.split([n_q * d, n_kv * d, n_kv * d], dim=1)] if place != "slices" else [
        x.view(T, -1, d) for x in qkv.split([n_q * d, n_kv * d, n_kv * d], dim=1)]
    pos = p.rng.integers(-3, 70000, (axes, T))
    sec = SECTIONS[axes](rot // 2)
    q_in, k_in, v_in = (x.float().cpu().numpy() for x in (q, k, v))
    r = binding.Rotation(cfg, 10000.0, n_axes=axes, sections=sec, rot_dim=rot, interleaved=interleaved)
    out = p.cache.append(k, v, plan.slot_map, q=q, rotation=r, positions=dev(pos if axes > 1 else pos[0]), q_out=q if place == "in place" else None,
                         status=p.status)
    assert (out.data_ptr() == q.data_ptr()) == (place == "in place")
    want = F.turn(q_in, pos, 10000.0, sec, rot, interleaved)
    # an element is two products and a sum in fp32 (cosines within 2^-24), half a step of the type on top: (4 2^-24 + eps / 2) (|x1| + |x2|)
    exact = R.rotate(q_in.astype(np.float64), pos, 10000.0, sec, rot, interleaved, False)
    assert (np.abs(f64(out) - exact) <= (2.0 ** -22 + EPS[dtype] / 2) * 2 * np.abs(q_in).max()).all()
    assert torch.equal(out, torch.tensor(want, device="cuda").to(dt))
    p.note(new, F.turn(k_in, pos, 10000.0, sec, rot, interleaved), v_in)
    p.check_cache()
    at = np.cumsum([0] + new)
    kk, vv = p.cache.read(plan.slot_map, status=p.status)
    for b, n in enumerate(new):
        for got, ref in ((kk, p.k), (vv, p.v)):
            assert np.array_equal(f64(got[at[b]:at[b + 1]]), ref[b][p.lens[b] - n:])
    assert p.status.item() == 0


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 16), ("fp32", 64, 64), ("bf16", 64, 128)])
def test_what_is_held_does_not_depend_on_how_it_came(dtype, d, page):
    cfg = config(n_q=4, n_kv=2, d=d, page=page, batch=2, pages=512 // page, n_pages=1024 // page, dtype=dtype)
    a = Program(cfg, seed=1)
    k, v = a.rows(300, 2), a.rows(300, 2)
    plan = a.step([300], k, v)
    a.check_cache()
    b = Program(cfg, seed=1)
    b.table.copy_(a.table)
    for i, n in ((0, 1), (1, 14), (15, 17), (32, 100), (132, 3), (131, 9), (140, 160)):        # (token 131 comes twice, 132 .. 134 too)
        b.cache.append(k[i:i + n], v[i:i + n], plan.slot_map[i:i + n])
    used = sorted(set((plan.slot_map // page).tolist()))
    assert torch.equal(a.cache.blocks[used], b.cache.blocks[used])
    assert torch.equal(a.cache.bounds[used], b.cache.bounds[used]) and torch.equal(a.cache.bound_scales[used], b.cache.bound_scales[used])
    rest = [x for x in range(cfg.n_pages) if x not in used]
    assert (b.cache.blocks[rest] == 0xff).all() and (b.cache.bounds[rest] == 77).all()          # nothing else was written


def test_append_skips_tokens_without_a_row_and_reports_bad_ones():
    cfg = config(n_q=4, n_kv=2, d=64, page=32, batch=2, pages=8, n_pages=16)
    p = Program(cfg, seed=2)
    k, v = p.rows(40, 2), p.rows(40, 2)
    plan = p.plan([40])
    rows = plan.slot_map.clone()
    rows[[3, 4, 20, 31, 39]] = -1
    p.cache.append(k, v, rows, status=p.status)
    assert p.status.item() == 0
    kk, vv = p.cache.read(plan.slot_map)
    wk, wv = F.token(k.float().cpu().numpy(), v.float().cpu().numpy(), 0.25, 0.0625)
    live = (rows >= 0).cpu().numpy()
    assert np.array_equal(f64(kk)[live], wk[live]) and np.array_equal(f64(vv)[live], wv[live])
    assert torch.isnan(kk[~torch.tensor(live, device="cuda")]).all()                              # (as they were)
    kk, vv = p.cache.read(rows)
    assert (kk[3] == 0).all() and (vv[39] == 0).all()                                             # no row: zeros
    # bounds go up to the last token with a row: 30 of the first page, 38 - 32 of the second
    first, second = (int(x) for x in p.table[int(p.slots[0]), :2])
    assert torch.isnan(p.cache.bound_scales[first]).all()                                         # (its skipped tokens are NaN here)
    p.cache.append(k[[3, 4, 20]], v[[3, 4, 20]], plan.slot_map[[3, 4, 20]])
    p.cache.append(k[21:31], v[21:31], plan.slot_map[21:31])
    for h in range(2):
        for page, tok in ((first, slice(0, 31)), (second, slice(32, 39))):
            want, s = F.bounds(wk[tok, h] / 0.25)
            assert np.array_equal(p.cache.bounds[page, h].cpu().numpy(), want) and p.cache.bound_scales[page, h].item() == s
    for bad in (16 * 32, -2, 1 << 40, -(1 << 40)):
        st = dev([0])
        before = p.cache.blocks.clone()
        p.cache.append(k[:2], v[:2], dev([bad, bad], torch.int64), status=st)
        assert st.item() == binding.ECHOKV_EBADPAGE and torch.equal(p.cache.blocks, before)
        st = dev([0])
        kk, vv = p.cache.read(dev([bad], torch.int64), status=st)
        assert st.item() == binding.ECHOKV_EBADPAGE and (kk == 0).all() and (vv == 0).all()


@pytest.mark.parametrize("gap,behind", [(5, 0), (16, 3), (40, 600), (300, 0), (700, 1), (1000, 5000)])
@pytest.mark.parametrize("page", [16, 64])
def test_bounds_see_every_row_however_many_tokens_without_one_lie_between(page, gap, behind):
    cfg = config(n_q=4, n_kv=2, d=64, page=page, batch=2, pages=8, n_pages=16)
    p = Program(cfg, seed=gap + behind)
    n = 2 * page + 5
    plan = p.plan([n])
    k, v = p.rows(n, 2, 0.1), p.rows(n, 2)
    k[n - 1] *= 100                               # (each page's last row is the one that its bounds come from)
    k[page - 1] *= 50
    rows = plan.slot_map.cpu().numpy()
    at = [0, 1, 2, page - 1, page, 2 * page - 1, 2 * page, 2 * page + 2]       # gaps in front of these, and tokens without a row at the end
    seen = np.full(n + gap * len(at) + behind, -1, np.int64)
    places = np.arange(n) + gap * np.searchsorted(at, np.arange(n), side="right")
    seen[places] = rows
    kk, vv = (torch.full((len(seen), 2, 64), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kk[places.tolist()], vv[places.tolist()] = k, v
    p.cache.append(kk, vv, dev(seen, torch.int64), status=p.status)
    p.note([n], k.float().cpu().numpy(), v.float().cpu().numpy())
    p.check_cache()
    assert p.status.item() == 0


def test_queries_of_skipped_tokens_are_turned_and_a_cache_without_bounds_works():
    cfg = config(n_q=4, n_kv=2, d=64, page=16, batch=1, pages=4, n_pages=4)
    cache = binding.Fp4Cache(cfg, selection=False)
    q, k = torch.randn(3, 4, 64, device="cuda").bfloat16(), torch.randn(3, 2, 64, device="cuda").bfloat16()
    r, pos = binding.Rotation(cfg, 1e4), dev([5, 6, 7])
    got = cache.append(k, k, dev([0, -1, 17], torch.int64), q=q, rotation=r, positions=pos)
    want = F.turn(q.float().cpu().numpy(), np.array([[5, 6, 7]]), 1e4, [32], 64, False)
    assert torch.equal(got, torch.tensor(want, device="cuda").bfloat16())
    assert cache.append(k, k, dev([0, -1, 17], torch.int64)) is None and cache.append(k[:0], k[:0], dev([], torch.int64)) is None
    assert cache.read(dev([], torch.int64))[0].shape == (0, 2, 64)


def test_tokens_that_are_not_finite():
    cfg = config(n_q=4, n_kv=2, d=128, page=16, batch=1, pages=16, n_pages=20)
    for kv, what in ((0, NAN), (1, INF), (0, -INF), (1, NAN)):
        p = Program(cfg, seed=3)
        x = [p.rows(100, 2), p.rows(100, 2)]
        x[kv][40, 0, 127], x[kv][77, 1, 0] = what, what
        p.step([100], *x)
        p.check_cache()
        q = p.rows(60, 4)
        bad = np.isnan(f64(p.attend([60], q)))                                # queries 40 .. 99, by the rows' kernel
        assert bad[:, :2].all() and not bad[:37, 2:].any() and bad[37:, 2:].all()


def test_values_of_every_size_are_held():
    """Groups from zero over the smallest scale to beyond the largest: scales saturate and vanish as the format says."""
    cfg = config(n_q=2, n_kv=1, d=64, page=16, batch=1, pages=8, n_pages=8, dtype="fp32")
    for unit in (1.0, 2.0 ** -20, 3.7, 2.0 ** 60, 2.0 ** -60):
        p = Program(cfg, seed=4, k_unit=unit, v_unit=unit)
        size = torch.tensor(2.0 ** np.arange(-16.0, 16, 0.5), dtype=torch.float32, device="cuda") * unit
        x = p.rows(64, 1) * size[:, None, None]
        x[7] = 0
        x[9, 0, :16] = 1e-42                                                  # (subnormal: held as zero, as anything below half the smallest step)
        p.step([64], x, -x)
        p.check_cache()


# ---- attention over the whole cache ----------------------------------------------------------------------------------
SHAPES = [("bf16", 128, 16, 8, 2), ("bf16", 64, 32, 4, 4), ("bf16", 128, 64, 8, 1), ("fp32", 128, 16, 4, 2), ("fp32", 64, 128, 8, 1), ("bf16", 64, 16, 2, 1),
          ("fp32", 128, 32, 2, 2)]


@pytest.mark.parametrize("dtype,d,page,n_q,n_kv", SHAPES)
def test_decode_matches_plain_form(dtype, d, page, n_q, n_kv):
    lens = [1, 15, 16, 17, 300, 333, 128, 2]
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=8, pages=512 // page, n_pages=4096 // page, dtype=dtype), seed=d + n_q)
    p.step(lens)
    q = p.rows(8, n_q, 2.0)
    out = p.cache.attention(q, p.table, dev(p.lens), seq_slots=dev(p.slots), status=p.status)
    p.check_attention([1] * 8, q, out)
    assert torch.equal(out, p.attend([1] * 8, q)) and p.status.item() == 0
    inside = q.clone()                                                         # (out may be q itself)
    assert torch.equal(p.attend([1] * 8, inside, out=inside), out)


OPTIONS = [{}, dict(softcap=5.0), dict(softcap=50.0), dict(slopes=True), dict(prefix=True), dict(softcap=20.0, slopes=True, prefix=True)]


def options(opts, n_q, prefix):
    kw = dict(opts)
    if "slopes" in kw:
        kw["slopes"] = [2.0 ** (-8.0 * (h + 1) / n_q) for h in range(n_q)]
    if "prefix" in kw:
        kw["prefix"] = prefix
    return kw


@pytest.mark.parametrize("opts", OPTIONS)
@pytest.mark.parametrize("dtype,d,n_q,n_kv", [("bf16", 128, 8, 2), ("fp32", 64, 4, 4), ("fp32", 128, 8, 1), ("bf16", 64, 16, 8)])
def test_score_options_and_drafts(opts, dtype, d, n_q, n_kv):
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=16, batch=6, pages=32, n_pages=160, dtype=dtype), seed=7)
    p.step([0, 16, 200, 37, 3, 250])
    new = [2, 1, 8, 5, 0, 7]
    p.step(new)
    kw = options(opts, n_q, [2, 0, 100, 42, 7, 254])
    q = p.rows(sum(new), n_q, 3.0)
    p.check_attention(new, q, p.attend(new, q, **dict(kw)), **kw)
    assert p.status.item() == 0


@pytest.mark.parametrize("opts", [{}, dict(softcap=50.0), dict(softcap=0.5), dict(slopes=True), dict(softcap=10.0, slopes=True, prefix=True)])
@pytest.mark.parametrize("d,page,n_q,n_kv,before,new", [
    (128, 16, 16, 8, [0, 77], [400, 513]), (64, 64, 8, 8, [300], [700]), (128, 128, 32, 4, [1003, 0, 0], [150, 299, 1]),
    (64, 32, 4, 4, [0, 9, 130], [640, 640, 641]), (128, 64, 32, 8, [6000], [64]), (64, 16, 8, 1, [9001, 0, 40], [129, 0, 1])])
def test_chunks_match_plain_form(opts, d, page, n_q, n_kv, before, new):
    """Sizes that go to the tcgen05 kernel: odd lengths, several items, ends inside a tile, items cut along the keys."""
    B, cap = len(new), 9216 if max(before) > 5000 else 1280
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=cap // page, n_pages=B * cap // page), seed=n_q + d)
    p.step(before)
    p.step(new)
    kw = options(opts, n_q, [(n + o) * 2 // 3 for n, o in zip(new, before)])
    q = p.rows(sum(new), n_q, 2.5)
    out = p.attend(new, q, **dict(kw))
    assert torch.equal(out, p.attend(new, q, **dict(kw))) and p.status.item() == 0
    p.check_attention(new, q, out, only=True, **kw)


def test_chunks_in_fp32_go_by_rows():
    p = Program(config(n_q=4, n_kv=2, d=64, page=16, batch=2, pages=32, n_pages=64, dtype="fp32"), seed=8)
    p.step([5, 0])
    p.step([133, 50])
    q = p.rows(183, 4, 2.0)
    p.check_attention([133, 50], q, p.attend([133, 50], q), only=True)


def test_not_finite_keys_in_masked_places_of_chunks():
    p = Program(config(n_q=8, n_kv=8, d=64, page=16, batch=1, pages=48, n_pages=60), seed=6)
    k, v = p.rows(650, 8), p.rows(650, 8)
    v[330, 0, 3], k[648, 1, 9], k[0, 2, 0] = NAN, INF, NAN
    p.step([650], k, v)
    q = p.rows(650, 8)
    bad = np.isnan(f64(p.attend([650], q))).any(-1)
    at = np.arange(650)
    assert (bad[:, 0] == (at >= 330)).all() and (bad[:, 1] == (at >= 648)).all() and bad[:, 2].all() and not bad[:, 3:].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scores_that_grow_along_the_sequence(dtype):
    """The reference has to move again and again; and one key that holds nearly everything, first or last."""
    p = Program(config(n_q=8, n_kv=8, d=128, page=64, batch=3, pages=12, n_pages=36, dtype=dtype), seed=31)
    k, v = p.rows(2100, 8), p.rows(2100, 8)
    grow = torch.linspace(0.1, 12, 700, device="cuda")
    k = (k.float() * torch.cat([grow, grow.flip(0), torch.ones(700, device="cuda")])[:, None, None]).to(k.dtype)
    k[1400] *= 8
    p.step([700] * 3, k, v)
    for n in (1, 5, 130):
        q = p.rows(3 * n, 8, 2.0)
        p.check_attention([n] * 3, q, p.attend([n] * 3, q), only=True)


def test_one_long_sequence_is_split_over_the_machine():
    p = Program(config(n_q=4, n_kv=1, d=128, page=16, batch=1, pages=2000, n_pages=2100), seed=5)
    p.step([31000])
    q = p.rows(1, 4, 3.0)
    p.check_attention([1], q, p.attend([1], q))


@pytest.mark.parametrize("B", [33, 400, 900])
def test_many_sequences(B):
    """More owners than a warp has lanes, than the kernels have threads: ragged, some without a token."""
    p = Program(config(n_q=8, n_kv=2, d=64, page=16, batch=B, pages=6, n_pages=6 * B), seed=B)
    p.step([int(x) for x in p.rng.integers(0, 80, B)])
    new = [int(x) for x in p.rng.integers(0, 3, B)]
    p.step(new)
    q = p.rows(sum(new), 8, 2.0)
    out = p.attend(new, q)
    assert p.status.item() == 0 and torch.isfinite(out).all()
    at = np.concatenate([[0], np.cumsum(new)])
    for b in [b for b in (0, 1, 31, 32, B // 2, B - 2, B - 1) if new[b]]:
        ref, size = R.attend(f64(q[at[b]:at[b + 1]]), p.k[b], p.v[b], 0.125)
        assert (np.abs(f64(out[at[b]:at[b + 1]]) - ref) <= F.tolerance(ref, size, p.lens[b], EPS["bf16"], True)).all(), b


@pytest.mark.parametrize("d,n_q,n_kv,page", [(128, 8, 2, 16), (64, 8, 1, 32), (128, 4, 4, 64), (64, 4, 4, 16)])
def test_items_of_two_tiles(d, n_q, n_kv, page):
    """9 to 16 query rows of an item, one tile and a last one of a few rows, items cut anywhere; row counts up to where chunks begin."""
    g = n_q // n_kv
    new = [n for n in (1, 2, 3, 4, 5, 7, 9, 12, 15, 16, 17, 31, 60) if n * g < CHUNK_ROWS]
    B = len(new)
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=2048 // page, n_pages=B * 2048 // page), seed=d + n_q)
    p.step([int(x) for x in p.rng.integers(0, 1800, B)])
    p.step(new)
    q = p.rows(sum(new), n_q, 2.5)
    for opts in ({}, dict(softcap=20.0, slopes=True, prefix=True)):
        kw = options(opts, n_q, [x // 2 for x in p.lens])
        out = p.attend(new, q, **dict(kw))
        p.check_attention(new, q, out, **kw)
        assert torch.equal(out, p.attend(new, q, **dict(kw)))
    assert p.status.item() == 0


@pytest.mark.parametrize("B,d", [(33, 128), (300, 128), (700, 64)])
def test_many_sequences_with_drafts(B, d):
    p = Program(config(n_q=8, n_kv=2, d=d, page=16, batch=B, pages=6, n_pages=6 * B), seed=B)
    p.step([int(x) for x in p.rng.integers(0, 80, B)])
    new = [int(x) for x in p.rng.integers(0, 6, B)]
    p.step(new)
    q = p.rows(sum(new), 8, 2.0)
    out = p.attend(new, q)
    assert p.status.item() == 0
    p.check_attention(new, q, out)


def test_rows_of_bad_sequences_are_zero_and_other_rows_stay():
    p = Program(config(n_q=4, n_kv=2, d=64, batch=3, pages=4, n_pages=30), seed=2)
    p.step([20, 33, 5])
    q = p.rows(9, 4)
    ref = [R.attend(f64(q[2 * b:2 * b + 2]), p.k[b], p.v[b], 0.125) for b in range(3)]

    def holds(out, *seqs):
        """(Not bit for bit: where the work is cut, and so the order of the sums, depends on the other sequences too.)"""
        return all((np.abs(f64(out[2 * b:2 * b + 2]) - ref[b][0]) <= F.tolerance(*ref[b], p.lens[b], EPS["bf16"], True)).all() for b in seqs)

    def run(slots=None, lens=None, cu=(0, 2, 4, 6), max_new=2):
        st, out = dev([0]), torch.full((9, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        p.cache.attention(q, p.table, dev(lens or p.lens), cu_tokens=dev(cu), max_new=max_new, seq_slots=dev(slots if slots is not None else p.slots),
                          out=out, status=st)
        return st.item(), out
    st, out = run()
    assert st == 0 and holds(out, 0, 1, 2) and (out[6:] == 7).all()
    for kw, code in ((dict(slots=[int(p.slots[0]), 3, int(p.slots[2])]), -8), (dict(slots=[int(p.slots[0]), -1, int(p.slots[2])]), -8),
                     (dict(lens=[20, 1, 5]), -11), (dict(lens=[20, 65, 5]), -11), (dict(lens=[20, -4, 5]), -11)):
        st, out = run(**kw)
        assert st == code and holds(out, 0, 2) and (out[2:4] == 0).all() and (out[6:] == 7).all()
    st, out = run(cu=(0, 2, 5, 6), max_new=2)
    assert st == -11 and holds(out, 0) and (out[2:5] == 0).all()
    for cu in ((0, 2, 1, 3), (0, 2, 11, 12), (0, 2, -3, 2)):
        st, out = run(cu=cu, max_new=9)
        assert st == -11 and (cu[2] == 1 or holds(out, 0))                     # (with 1, rows 1 and 2 are the last sequence's too)
    st, out = run(cu=(0, 0, 0, 0))
    assert st == 0 and (out == 7).all()
    for page in (30, -1, 1 << 30):                                             # a bad page: the other sequences hold
        t = p.table.clone()
        t[int(p.slots[0]), 1] = page
        st = dev([0])
        out = p.cache.attention(q[:6], t, dev(p.lens), cu_tokens=dev([0, 2, 4, 6]), max_new=2, seq_slots=dev(p.slots), status=st)
        assert st.item() == -8 and holds(out, 1, 2)


# ---- the choice of pages ------------------------------------------------------------------------------------------------
def check_select(p, new, q, got, n_select, first, recent):
    P = p.cfg.page_tokens
    seqs, pos = p.tokens(new)
    bnd, scales = p.cache.bounds.cpu().numpy(), p.cache.bound_scales.cpu().numpy()
    qf, got = q.float().cpu().numpy(), got.cpu().numpy()
    for i in range(len(seqs)) if len(seqs) < 40 else sampled(p.rng, len(seqs)):
        pages = p.pages_of(seqs[i])[:pos[i] // P + 1]
        want = F.select(qf[i], bnd[pages], scales[pages], int(pos[i]), P, n_select, first, recent)
        assert np.array_equal(got[i], want), i


@pytest.mark.parametrize("dtype,d,page,n_q,n_kv,lens,new,n_select,first,recent", [
    ("bf16", 128, 16, 8, 2, [300, 20, 1, 700], [1, 1, 1, 1], 8, 1, 2), ("fp32", 64, 16, 4, 4, [500, 90], [7, 3], 5, 0, 1),
    ("bf16", 64, 32, 8, 1, [900, 33, 64], [40, 33, 1], 11, 2, 3), ("fp32", 128, 64, 2, 1, [4000], [9], 60, 1, 1), ("bf16", 64, 16, 16, 8, [800, 600], [100, 130], 20, 1, 1),
    ("bf16", 64, 16, 2, 2, [60, 5000], [60, 300], 1, 0, 1), ("bf16", 128, 128, 32, 4, [2000, 128, 129], [64, 128, 129], 3, 1, 2)])
def test_select_matches_plain_form(dtype, d, page, n_q, n_kv, lens, new, n_select, first, recent):
    """One token to hundreds (blocks of one token and of several), sequences shorter than n_select, drafts whose own pages differ."""
    B = len(lens)
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=-(-max(lens) // page), n_pages=sum(-(-n // page) for n in lens) + 3, dtype=dtype), seed=9)
    p.step(lens)
    q = p.rows(sum(new), n_q, 2.0)
    seqs, pos = p.tokens(new)
    got = p.cache.select_pages(q, p.table, dev(seqs), dev(pos), n_select, n_first=first, n_recent=recent, seq_slots=dev(p.slots), status=p.status)
    check_select(p, new, q, got, n_select, first, recent)
    assert p.status.item() == 0


def bounds_only(pages, n_kv, d, B=1, n_q=None, seed=0, page=16, spread=127):
    """A cache whose bounds are all that matters, pages in any order."""
    rng = np.random.default_rng(seed)
    cfg = config(n_q=n_q or n_kv, n_kv=n_kv, d=d, page=page, batch=B, pages=pages, n_pages=B * pages)
    bnd = np.sort(rng.integers(-spread, spread + 1, (B * pages, n_kv, 2, d)), axis=2)[:, :, ::-1]
    scales = rng.uniform(0.5, 1.5, (B * pages, n_kv)).astype(np.float32)
    blocks = torch.zeros((B * pages, n_kv, page // 16, 18 * d), dtype=torch.uint8, device="cuda")
    cache = binding.Fp4Cache(cfg, blocks=blocks, bounds=dev(bnd.copy(), torch.int8), bound_scales=dev(scales, torch.float32))
    return rng, cfg, cache, bnd, scales, rng.permutation(B * pages).reshape(B, pages)


@pytest.mark.parametrize("pages,n_select,T,n_q,n_kv,spread", [
    (20000, 1024, 1, 4, 1, 127), (20000, 3, 1, 1, 1, 127), (17000, 1000, 2, 8, 8, 127), (5000, 700, 70, 8, 8, 127), (2500, 1024, 200, 16, 8, 2), (6000, 64, 3, 2, 2, 1),
    (1025, 1024, 1, 1, 1, 127)])
def test_select_among_many_pages(pages, n_select, T, n_q, n_kv, spread):
    """More pages than a block has room for, pages in parts, many tokens of one sequence; few different scores (ties everywhere)."""
    rng, cfg, cache, bnd, scales, table = bounds_only(pages, n_kv, 64, n_q=n_q, seed=pages + T, spread=spread)
    if spread < 5:
        scales[:] = 1
        cache.bound_scales.fill_(1)
    q = torch.tensor(rng.standard_normal((T, n_q, 64)), device="cuda").bfloat16()
    if spread == 1:
        q = q.sign()
    pos = np.arange(pages * 16 - T, pages * 16)
    got = cache.select_pages(q, dev(table), dev([0] * T), dev(pos), n_select).cpu().numpy()
    for i in sorted({0, T // 2, T - 1}):
        own = pos[i] // 16 + 1
        want = F.select(q[i].float().cpu().numpy(), bnd[table[0, :own]], scales[table[0, :own]], int(pos[i]), 16, n_select, 1, 1)
        assert np.array_equal(got[i], want), i
    again = cache.select_pages(q, dev(table), dev([0] * T), dev(pos), n_select).cpu().numpy()
    assert np.array_equal(got, again)


def test_select_special_values():
    """Pages with a NaN key come first, rows of the query that are not finite count as zeros, huge and tiny rows keep their order."""
    rng, cfg, cache, bnd, scales, table = bounds_only(100, 2, 64, n_q=4, seed=3)
    for page in (17, 60):
        bnd[table[0, page]], scales[table[0, page]] = 0, np.nan
    cache.bounds.copy_(dev(bnd.copy(), torch.int8))
    cache.bound_scales.copy_(dev(scales, torch.float32))
    q = rng.standard_normal((6, 4, 64)).astype(np.float32)
    q[1] *= 1e38
    q[2] *= 1e-38
    q[3, 0, 5], q[3, 2, 0] = np.inf, np.nan
    q[4] = 0
    q[5, :, 1:] = 0
    qt = torch.tensor(q, device="cuda").bfloat16()
    pos = np.array([1599, 1590, 700, 1599, 1500, 1599])
    got = cache.select_pages(qt, dev(table), dev([0] * 6), dev(pos), 9, n_first=1, n_recent=2).cpu().numpy()
    for i in range(6):
        own = pos[i] // 16 + 1
        want = F.select(qt[i].float().cpu().numpy(), bnd[table[0, :own]], scales[table[0, :own]], int(pos[i]), 16, 9, 1, 2)
        assert np.array_equal(got[i], want), i
    assert 17 in got[0, 0] and 60 in got[0, 1]


def test_select_of_tokens_that_are_not_there():
    rng, cfg, cache, bnd, scales, table = bounds_only(40, 2, 64, B=3, n_q=4, seed=4)
    seqs, pos = [0, 0, -1, 1, 5, 2, 2, 1, -1], [600, 601, 0, 300, 3, 640, -1, 301, 9]
    q = torch.tensor(rng.standard_normal((9, 4, 64)), device="cuda").bfloat16()
    slots = [2, 0, 1]
    st, t = dev([0]), dev(table)
    got = cache.select_pages(q, t, dev(seqs), dev(pos), 6, seq_slots=dev(slots), status=st).cpu().numpy()
    assert st.item() in (binding.ECHOKV_EBADPAGE, binding.ECHOKV_EBADLENGTH)
    for i in range(9):
        if i in (0, 1, 3, 7):
            own = pos[i] // 16 + 1
            rows = table[slots[seqs[i]], :own]
            assert np.array_equal(got[i], F.select(q[i].float().cpu().numpy(), bnd[rows], scales[rows], pos[i], 16, 6, 1, 1)), i
        else:
            assert (got[i] == -1).all()
    t[0, 3] = 1 << 20                                                            # a bad page of sequence 1: the others hold, its pages are its own
    st = dev([0])
    other = cache.select_pages(q[:4], t, dev(seqs[:4]), dev(pos[:4]), 6, seq_slots=dev(slots), status=st).cpu().numpy()
    assert st.item() == binding.ECHOKV_EBADPAGE and np.array_equal(other[:2], got[:2]) and (other[3] <= 300 // 16).all() and (other[3] >= 0).all()


# ---- attention over chosen pages ---------------------------------------------------------------------------------------
def check_sparse(p, seqs, pos, q, pages, out, **kw):
    qf, got = f64(q), f64(out)
    for i in range(len(seqs)) if len(seqs) < 40 else sampled(p.rng, len(seqs)):
        k, v = p.k[seqs[i]], p.v[seqs[i]]
        ref, size = F.attend_pages(qf[i], k, v, int(pos[i]), pages[i], p.cfg.page_tokens, p.cfg.head_dim ** -0.5, **kw)
        tol = F.tolerance(ref[None], size[None], pages.shape[-1] * p.cfg.page_tokens, EPS[p.dtype], p.dtype == "bf16", False, kw.get("softcap", 0.0))
        if kw.get("slopes") is not None:                                         # (the distance, not the number of keys)
            tol = F.tolerance(ref[None], size[None], int(pos[i]) + 1, EPS[p.dtype], p.dtype == "bf16", False, kw.get("softcap", 0.0), kw["slopes"])
        assert (np.abs(got[i] - ref) <= tol[0]).all(), (i, float((np.abs(got[i] - ref) / tol[0]).max()))


@pytest.mark.parametrize("opts", [{}, dict(softcap=10.0), dict(softcap=20.0, slopes=True)])
@pytest.mark.parametrize("dtype,d,page,n_q,n_kv,lens,new,n_select", [
    ("bf16", 128, 16, 8, 2, [300, 20, 1, 700], [1, 1, 1, 1], 8), ("fp32", 64, 16, 4, 4, [500, 90], [7, 3], 5), ("bf16", 64, 32, 8, 1, [900, 33, 64], [40, 33, 1], 4),
    ("fp32", 128, 64, 2, 1, [4000], [9], 40), ("bf16", 64, 128, 16, 8, [800, 600], [100, 130], 2), ("bf16", 128, 16, 4, 4, [40], [40], 64)])
def test_sparse_matches_plain_form(opts, dtype, d, page, n_q, n_kv, lens, new, n_select):
    """Lists in any order with gaps in them, shorter and longer than the sequences."""
    B = len(lens)
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=-(-max(lens) // page), n_pages=sum(-(-n // page) for n in lens) + 3, dtype=dtype), seed=12)
    p.step(lens)
    q = p.rows(sum(new), n_q, 2.5)
    seqs, pos = p.tokens(new)
    pages = np.full((len(seqs), n_kv, n_select), -1)
    for i in range(len(seqs)):
        for h in range(n_kv):
            own = pos[i] // page + 1
            some = p.rng.permutation(own)[:n_select]
            pages[i, h, :len(some)] = np.where(p.rng.random(len(some)) < 0.2, -1, some)
    kw = options(opts, n_q, None)
    extra = dict(kw)
    if "slopes" in extra:
        extra["alibi_slopes"] = dev(extra.pop("slopes"), torch.float32)
    out = p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), dev(pages), seq_slots=dev(p.slots), status=p.status, **extra)
    check_sparse(p, seqs, pos, q, pages, out, **kw)
    assert p.status.item() == 0 and torch.isfinite(out).all()


def test_all_pages_are_the_whole_cache():
    p = Program(config(n_q=8, n_kv=2, d=128, page=32, batch=3, pages=20, n_pages=60), seed=13)
    p.step([600, 32, 33])
    q = p.rows(3, 8, 2.0)
    seqs, pos = p.tokens([1, 1, 1])
    pages = p.cache.select_pages(q, p.table, dev(seqs), dev(pos), 20, seq_slots=dev(p.slots))
    assert pages[0, 0].tolist() == list(range(19)) + [-1] and pages[2, 1].tolist() == [0, 1] + [-1] * 18
    out = p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), pages, seq_slots=dev(p.slots))
    p.check_attention([1, 1, 1], q, out)


def test_sparse_lists_of_all_kinds():
    p = Program(config(n_q=4, n_kv=2, d=64, page=16, batch=3, pages=8, n_pages=30), seed=14)
    p.step([100, 128, 40])
    seqs, pos = np.array([0, 1, 2, -1, 0, 1, 7, 2, 1]), np.array([99, 127, 39, 5, 50, 0, 3, 128, -1])
    q = p.rows(9, 4, 2.0)
    pages = np.full((9, 2, 4), -1)
    pages[0] = [[6, 6, 0, -1], [5, -1, -1, 1]]                                    # twice the same, gaps
    pages[1] = -1                                                                 # nothing
    pages[2] = [[0, 1, 2, 7], [2, 1, 0, 900]]                                     # one behind the token's own: of three pages the fourth is not looked at
    pages[4] = [[3, 1, 6, 0], [0, 0, 0, 0]]                                       # page 6 is behind position 50
    pages[5] = [[0, 5, 5, 5], [-5, 0, 0, 0]]                                      # (one entry is looked at: any below 0 is none)
    st, out = dev([0]), torch.full((9, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), dev(pages), seq_slots=dev(p.slots), out=out, status=st)
    assert st.item() in (binding.ECHOKV_EBADPAGE, binding.ECHOKV_EBADLENGTH)
    assert (out[1] == 0).all() and (out[3] == 7).all() and (out[6:] == 0).all() and (out[5, 2:] == 0).all()
    seen = pages.copy()
    seen[2, :, 3], seen[4, 0, 2], seen[5, 0, 1:], seen[5, 1] = -1, -1, -1, -1
    keep = [0, 2, 4, 5]
    check_sparse(p, seqs[keep], pos[keep], q[keep], seen[keep], out[keep])
    st = dev([0])
    p.cache.sparse_attention(q[:2], p.table, dev(seqs[:2]), dev(pos[:2]), dev(pages[:2]), seq_slots=dev(p.slots), status=st)
    assert st.item() == 0


@pytest.mark.parametrize("T", [33, 500])
def test_sparse_of_many_tokens(T):
    p = Program(config(n_q=4, n_kv=4, d=64, page=16, batch=2, pages=64, n_pages=128), seed=15)
    p.step([T + 300, 40])
    seqs, pos = np.zeros(T, int), np.arange(300, T + 300)
    q = p.rows(T, 4, 2.0)
    pages = p.cache.select_pages(q, p.table, dev(seqs), dev(pos), 6, n_recent=2, seq_slots=dev(p.slots))
    out = p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), pages, seq_slots=dev(p.slots), status=p.status)
    check_sparse(p, seqs, pos, q, pages.cpu().numpy(), out)
    assert p.status.item() == 0


# ---- together ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_run_of_steps(dtype):
    """Prompts, decode steps, a mixed step, a finished request whose pages another one takes: plan, append, choose, attend both ways; at
    the end a sequence is read back into another cache."""
    cfg = config(n_q=8, n_kv=2, d=64, page=16, batch=4, pages=16, n_pages=24, dtype=dtype)
    p = Program(cfg, seed=11)
    dt, r = DT[dtype][1], binding.Rotation(cfg, 10000.0)

    def step(new):
        T, B = sum(new), len(new)
        plan = p.plan(new)
        qkv = torch.tensor(p.rng.standard_normal((T, 12 * 64)), dtype=dt, device="cuda")
        q, k, v = qkv[:, :512].view(T, 8, 64), qkv[:, 512:640].view(T, 2, 64), qkv[:, 640:].view(T, 2, 64)
        q = p.cache.append(k, v, plan.slot_map, q=q, rotation=r, positions=plan.positions, status=p.status)
        slots = dev(p.slots[:B])
        out = p.cache.attention(q, p.table, plan.seq_lens, cu_tokens=plan.cu_tokens, max_new=max(new), seq_slots=slots, softcap=30.0, status=p.status)
        pages = p.cache.select_pages(q, p.table, plan.token_seqs, plan.positions, 3, seq_slots=slots, status=p.status)
        some = p.cache.sparse_attention(q, p.table, plan.token_seqs, plan.positions, pages, seq_slots=slots, softcap=30.0, status=p.status)
        p.note(new, F.turn(k.float().cpu().numpy(), plan.positions.cpu().numpy()[None], 10000.0, [32], 64, False), v.float().cpu().numpy())
        assert plan.seq_lens.tolist() == p.lens and p.status.item() == 0
        p.check_cache()
        p.check_attention(new, q, out, softcap=30.0)
        check_select(p, new, q, pages, 3, 1, 1)
        check_sparse(p, *p.tokens(new), q, pages.cpu().numpy(), some, softcap=30.0)
    step([33, 5, 70, 0])
    for _ in range(3):
        step([1, 1, 1, 0])
    step([1, 40, 1, 90])
    binding.release_pages(cfg, p.table, dev([p.lens[2]]), p.free, p.count, seq_slots=dev(p.slots[2:3]))
    p.lens[2], p.k[2], p.v[2] = 0, p.k[2][:0], p.v[2][:0]
    step([2, 1, 100, 1])
    step([1, 1, 1, 1])
    n = p.lens[1]
    rows = dev(np.concatenate([pg * 16 + np.arange(16) for pg in p.pages_of(1)])[:n], torch.int64)
    k, v = p.cache.read(rows)
    other = binding.Fp4Cache(config(n_q=8, n_kv=2, d=64, page=64, batch=1, pages=2, n_pages=2, dtype=dtype), k_unit=0.25, v_unit=0.0625)
    at = dev(np.arange(n), torch.int64)
    other.append(k, v, at)
    # (what is held in 4 bits is held as it is: a group's largest code is 6, within 2^-4, and its scale comes out the same)
    assert all(torch.equal(got, want) for got, want in zip(other.read(at), (k, v)))


def test_a_captured_step_replays_and_two_graphs_share_a_workspace():
    cfg = config(n_q=8, n_kv=2, d=128, page=16, batch=3, pages=16, n_pages=40)
    p = Program(cfg, seed=12)
    p.step([20, 31, 100])
    slots, new, lens = dev(p.slots), dev([1, 1, 1]), dev(p.lens)
    qkv = torch.zeros(3, 12 * 128, dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv[:, :1024].view(3, 8, 128), qkv[:, 1024:1280].view(3, 2, 128), qkv[:, 1280:].view(3, 2, 128)
    plan = binding.StepPlan(3, 3, "cuda", seq_lens=lens, free_count=p.count)
    layers = [p.cache, binding.Fp4Cache(cfg, k_unit=0.25, v_unit=0.0625, workspace=p.cache.workspace)]
    for name in ("blocks", "bounds", "bound_scales"):
        getattr(layers[1], name).copy_(getattr(layers[0], name))
    r = binding.Rotation(cfg, 10000.0)
    turned, dense, some = ([torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in layers] for _ in range(3))
    pages = [torch.zeros(3, 2, 4, dtype=torch.int32, device="cuda") for _ in layers]

    def layer(i):
        layers[i].append(k, v, plan.slot_map, q=q, rotation=r, positions=plan.positions, q_out=turned[i], status=p.status)
        layers[i].attention(turned[i], p.table, lens, seq_slots=slots, out=dense[i], status=p.status)
        layers[i].select_pages(turned[i], p.table, plan.token_seqs, plan.positions, 4, seq_slots=slots, out=pages[i], status=p.status)
        layers[i].sparse_attention(turned[i], p.table, plan.token_seqs, plan.positions, pages[i], seq_slots=slots, out=some[i], status=p.status)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0], stream=stream):
        binding.plan_tokens(cfg, p.table, lens, new, p.free, p.count, 3, seq_slots=slots, out=plan, status=p.status)
        layer(0)
    with torch.cuda.graph(graphs[1], stream=stream):
        layer(1)
    for i in range(20):
        qkv.copy_(torch.randn(3, 12 * 128, device="cuda", generator=torch.Generator("cuda").manual_seed(i)))
        p.cache.workspace.fill_(0xff)
        graphs[0].replay()
        graphs[1].replay()
        pos = plan.positions.cpu().numpy()
        p.note([1, 1, 1], F.turn(k.float().cpu().numpy(), pos[None], 10000.0, [64], 128, False), v.float().cpu().numpy())
        for pair in (turned, dense, pages, some):
            assert torch.equal(*pair)
        if i in (0, 11, 12, 19):
            p.check_cache()
            p.check_attention([1] * 3, turned[0], dense[0])
            check_select(p, [1] * 3, turned[0], pages[0], 4, 1, 1)
            check_sparse(p, *p.tokens([1] * 3), turned[0], pages[0].cpu().numpy(), some[0])
    assert p.status.item() == 0


def test_on_another_stream_new_tensors_are_that_streams():
    cfg = config(n_q=8, n_kv=2, d=128, page=16, batch=2, pages=16, n_pages=40)
    p = Program(cfg, seed=13)
    plan = p.step([40, 90])
    q, k, v = p.rows(2, 8), p.rows(2, 2), p.rows(2, 2)
    lens, slots, seqs, pos = dev(p.lens), dev(p.slots), dev([0, 1]), dev([39, 89])
    rows, r = plan.slot_map[[0, 100]], binding.Rotation(cfg, 1e4)

    def run(**kw):
        pages = p.cache.select_pages(q, p.table, seqs, pos, 4, seq_slots=slots, **kw)
        return [p.cache.attention(q, p.table, lens, seq_slots=slots, **kw), pages,
                p.cache.sparse_attention(q, p.table, seqs, pos, pages, seq_slots=slots, **kw), *p.cache.read(rows, **kw)]
    want = run()
    want.append(binding.rotate(cfg, q, None, pos, 1e4)[0])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = run(stream=s)
    got.append(p.cache.append(k, v, dev([-1, -1], torch.int64), q=q, rotation=r, positions=pos, stream=s))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[:5], want[:5]))
    assert (got[5].float() - want[5].float()).abs().max() <= 2.0 ** -7 * q.abs().max()      # (cosines of an angle in 64 and in 32 bits: a step apart)
    for t in got:
        assert owner(t) == s.cuda_stream


def test_offsets_beyond_32_bits():
    """Pages near the end of pools of more than 4 GB."""
    n_pages = 60000
    cfg = config(n_q=8, n_kv=8, d=128, page=64, batch=2, pages=8, n_pages=n_pages)
    p = Program(cfg, seed=16, garbage=False)
    assert p.cache.blocks.numel() > 1 << 32
    order = np.concatenate([np.arange(n_pages - 16), n_pages - 1 - p.rng.permutation(16)])
    p.free.copy_(dev(order))
    p.step([300, 500])
    new = [70, 1]
    p.step(new)
    seqs, pos = p.tokens(new)
    q = p.rows(71, 8, 2.0)
    p.check_attention(new, q, p.attend(new, q), only=True)
    pages = p.cache.select_pages(q, p.table, dev(seqs), dev(pos), 3, seq_slots=dev(p.slots), status=p.status)
    check_select(p, new, q, pages, 3, 1, 1)
    out = p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), pages, seq_slots=dev(p.slots), status=p.status)
    check_sparse(p, seqs, pos, q, pages.cpu().numpy(), out)
    last = p.pages_of(1)[:1]
    assert last[0] > n_pages - 17
    k, v = p.cache.read(dev(int(last[0]) * 64 + np.arange(64), torch.int64), status=p.status)
    assert np.array_equal(f64(k), p.k[1][:64]) and np.array_equal(f64(v), p.v[1][:64]) and p.status.item() == 0
