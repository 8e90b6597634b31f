"""The 4-bit cache's operators where a call is unlike the common ones."""
import numpy as np
import pytest
import torch

from paper_2603_22910_b200 import binding
from tests import fp4_ref as F
from tests import serving_ref as R
from tests.test_gpu_fp4 import Program, check_select, check_sparse
from tests.test_gpu_serving import DT, EPS, config, dev, f64

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
PREFIXES = [lambda n: n, lambda n: n + 1, lambda n: -(-n // 16) * 16, lambda n: n + 1000, lambda n: 1 << 30, lambda n: (1 << 31) - 1]


@pytest.mark.parametrize("stale", [0xff, 0x33])            # what lies behind the end: NaN scales, or finite keys (codes 1.5, scales 0.6875)
@pytest.mark.parametrize("dtype,d,page,n_q,n_kv,before,new", [
    ("bf16", 128, 16, 8, 2, [0, 7, 0, 40, 300, 16], [1, 1, 1, 1, 1, 1]),                 # rows in the even columns
    ("bf16", 64, 32, 8, 1, [0, 20, 61, 0], [1, 1, 1, 1]),                                # a whole tile of rows
    ("bf16", 128, 64, 8, 2, [0, 0, 33, 250, 90], [3, 5, 2, 1, 9]),                       # two tiles, one, and few rows
    ("bf16", 64, 16, 4, 4, [5, 0, 130], [11, 30, 9]), ("fp32", 128, 16, 4, 2, [0, 9, 33], [1, 4, 7]),
    ("fp32", 64, 128, 8, 1, [3, 0], [20, 50]), ("bf16", 128, 64, 32, 8, [0, 130], [700, 333])])
def test_a_prefix_longer_than_the_sequence(stale, dtype, d, page, n_q, n_kv, before, new):
    """A bidirectional prefix that comes in pieces: the queries see every key that is there and none behind the end."""
    B = len(new)
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=1024 // page, n_pages=B * 1024 // page, dtype=dtype), seed=d + n_q)
    p.cache.blocks.fill_(stale)
    p.step(before)
    p.step(new)
    assert any(n % 16 for n in p.lens)
    q = p.rows(sum(new), n_q, 2.0)
    for prefix in PREFIXES:
        at = [prefix(n) for n in p.lens]
        p.check_attention(new, q, p.attend(new, q, prefix=at), prefix=at, only=True)
    assert p.status.item() == 0


def test_queries_turned_into_any_place_that_overlaps_no_input():
    """Queries, keys, values and turned queries anywhere in one buffer: between each other's rows is fine, a shared element is refused."""
    cfg = config(n_q=2, n_kv=1, d=64, page=16, batch=1, pages=4, n_pages=4)
    cache, rng = binding.Fp4Cache(cfg, selection=False), np.random.default_rng(23)
    r, counts = binding.Rotation(cfg, 1e4), [0, 0, 0]
    for _ in range(1500):
        T = int(rng.integers(1, 7))
        strides = [128 + 8 * int(x) for x in rng.integers(0, 70, 4)] if rng.random() < 0.6 else [128 + 8 * int(rng.integers(0, 70))] * 4
        at = [8 * int(x) for x in rng.integers(0, rng.choice([60, 300, 900]), 4)]
        if rng.random() < 0.3:
            at[3], strides[3] = at[0], strides[0]                              # in place
        shape = [(T, h, 64) for h in (2, 1, 1, 2)]
        hold = torch.tensor(rng.standard_normal(12000), device="cuda").bfloat16()
        q, k, v, out = (hold.as_strided(s, (n, 64, 1), a) for s, n, a in zip(shape, strides, at))
        used = [{a + i * n + j for i in range(T) for j in range(s[1] * 64)} for s, n, a in zip(shape, strides, at)]
        same = at[0] == at[3] and (strides[0] == strides[3] or T == 1)
        shared = (used[3] & used[0] and not same) or used[3] & (used[1] | used[2])
        pos, rows = dev(rng.integers(0, 5000, T)), dev(rng.permutation(64)[:T], torch.int64)
        before = hold.clone()
        if shared:
            with pytest.raises(binding.EchoKVError) as e:
                cache.append(k, v, rows, q=q, rotation=r, positions=pos, q_out=out)
            assert e.value.status == binding.ECHOKV_EINVAL and torch.equal(hold, before)
            counts[0] += 1
            continue
        want = cache.append(k.clone(), v.clone(), rows, q=q.clone(), rotation=r, positions=pos)
        held = cache.read(rows)
        cache.append(k, v, rows, q=q, rotation=r, positions=pos, q_out=out)
        assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip(cache.read(rows), held))
        out.copy_(before.as_strided(shape[3], (strides[3], 64, 1), at[3]))
        assert torch.equal(hold, before)                                       # nothing else was written
        counts[1 + same] += 1
    assert min(counts) > 100


@pytest.mark.parametrize("softcap", [0.0, 5.0])
@pytest.mark.parametrize("dtype,new", [("bf16", [1, 1, 2]), ("fp32", [1, 1, 2]), ("bf16", [3, 1, 20]), ("bf16", [1, 500, 1])])
def test_queries_that_are_not_finite(dtype, new, softcap):
    """A query row with an infinity or NaN has scores of which none is an ordinary number: its output is NaN, also where every key that
    it sees scores -inf; a cap makes infinite scores finite.  Other rows are left alone."""
    n_q = n_kv = 4
    p = Program(config(n_q=n_q, n_kv=n_kv, d=64, page=16, batch=3, pages=64, n_pages=192, dtype=dtype), seed=17)
    T = sum(new)
    size = torch.tensor(p.rng.uniform(1.0, 1.5, (T, n_kv, 64)), device="cuda").to(DT[dtype][1])         # (no code of it is 0)
    k = torch.where(torch.arange(n_kv, device="cuda")[:, None] % 2 == 0, -size, size)
    p.step(new, k=k)
    q = p.rows(T, n_q)
    first = np.concatenate([[0], np.cumsum(new)[:-1]]).tolist()
    q[first[0], :, 5], q[first[1], :2, 9], q[first[2], 1, 63], q[first[2], 2, 0] = INF, -INF, NAN, INF
    q[first[2], 2, 7] = -1e6                                               # (beyond fp16's range beside the infinity)
    out = f64(p.attend(new, q, softcap=softcap))
    seqs, pos = p.tokens(new)
    pages = np.arange(-(-max(new) // 16))
    pages = np.broadcast_to(np.where(pages <= pos[:, None, None] // 16, pages, -1), (T, n_kv, len(pages))).copy()
    some = f64(p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), dev(pages), seq_slots=dev(p.slots), softcap=softcap, status=p.status))
    assert np.array_equal(np.isnan(some), np.isnan(out))
    pages[:] = -1
    none = p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), dev(pages), seq_slots=dev(p.slots), softcap=softcap)
    assert (none == 0).all()                                                   # (a token that has no key)
    for b, n in enumerate(new):
        with np.errstate(invalid="ignore"):
            ref, s = R.attend(f64(q[first[b]:first[b] + n]), p.k[b], p.v[b], 0.125, softcap, only=sorted({0, n // 2, n - 1}))
        for i in sorted({0, n // 2, n - 1}):
            got = out[first[b] + i]
            assert np.array_equal(np.isnan(got), np.isnan(ref[i])), (b, i)
            fine = ~np.isnan(ref[i]).any(-1) & np.isfinite(f64(q[first[b] + i])).all(-1)
            tol = F.tolerance(ref[i:i + 1], s[i:i + 1], n, EPS[dtype], dtype == "bf16", n >= 64, softcap)[0]
            assert (np.abs(got - ref[i]) <= tol)[fine].all(), (b, i)
    assert p.status.item() == 0


@pytest.mark.parametrize("d,at", [(64, "first"), (128, "last")])
def test_many_small_probabilities_beside_one_large_one_in_fp32(d, at):
    """One key holds nearly everything and 32767 others 2^-e of it each: their sum is part of the result.  Every sequence is the same
    pages, with queries that give e from 20 to 44; there is an item for every warp, so that one pass over the keys holds them all.

    Keys and queries have one feature: a score is one product.  In base-2 units it is below 2^6 and off by less than 2^-18 of that in fp32
    steps and 22-bit operands: 2^-12 of a small weight.  Sums of 32768 / 16 parts in fp32: 2^11 2^-24 = 2^-13, twice.  A probability
    has 22 bits, or is off by at most 2^-43 of the largest."""
    L, B = 32768, 1776
    cfg = config(n_q=1, n_kv=1, d=d, page=128, batch=B, pages=L // 128, n_pages=L // 128, dtype="fp32")
    cache = binding.Fp4Cache(cfg, selection=False)
    k, v = np.zeros((L, 1, d), np.float32), np.full((L, 1, d), 6.0, np.float32)
    v[:, 0, 1::2] = -3.0
    big = 0 if at == "first" else L - 1
    k[big, 0, 0], v[big] = 6.0, 0.0
    cache.append(dev(k, torch.float32), dev(v, torch.float32), dev(np.arange(L), torch.int64))
    table = dev(np.tile(np.arange(L // 128), (B, 1)))
    e = np.linspace(20, 44, B)
    q = np.zeros((B, 1, d), np.float32)
    q[:, 0, 0] = e * np.log(2.0) * np.sqrt(d) / 6.0
    out = f64(cache.attention(dev(q, torch.float32), table, dev([L] * B)))
    w = np.exp(-q[:, :, :1].astype(np.float64) * 6.0 / np.sqrt(d))                             # of a small one
    ref = (L - 1) * w / (1 + (L - 1) * w) * v[L // 2].astype(np.float64)
    tol = np.abs(ref) * (2.0 ** -12 + 2.0 ** -12) + L * 2.0 ** -43 * 6.0
    err = np.abs(out - ref)
    assert (err <= tol).all(), (float(e[np.argmax((err / tol).max((1, 2)))]), float((err / tol).max()))


@pytest.mark.parametrize("T", [1, 40, 600])
def test_the_number_of_sequences_changes_no_choice(T):
    """However many sequences a call says that there are, and so however many tokens a block takes."""
    cfg = config(n_q=8, n_kv=8, d=64, page=16, batch=300, pages=64, n_pages=200)
    p = Program(cfg, seed=24)
    p.step([T + 300, 70])
    p.step([0, 1])
    seqs, pos = (dev(np.append(x, [y, -1])) for x, y in zip(p.tokens([T, 1]), (5, 3)))       # then one of a sequence beyond some counts, one of none
    q, slots = p.rows(T + 3, 8, 2.0), dev(p.slots)
    want = p.cache.select_pages(q[:T + 1], p.table, seqs[:T + 1], pos[:T + 1], 6, seq_slots=slots[:2], status=p.status)
    check_select(p, [T, 1], q, want, 6, 1, 1)
    some = p.cache.sparse_attention(q[:T + 1], p.table, seqs[:T + 1], pos[:T + 1], want, seq_slots=slots[:2], status=p.status)
    for n in (2, 3, 5, 6, 30, 300):
        status = dev([0])
        got = p.cache.select_pages(q, p.table, seqs, pos, 6, seq_slots=slots, status=status, n_seqs=n)
        assert torch.equal(got[:T + 1], want) and (got[T + 2] == -1).all()
        assert status.item() == (binding.ECHOKV_EBADPAGE if n <= 5 else 0) and (n > 5 or (got[T + 1] == -1).all())
        out = p.cache.sparse_attention(q[:T + 1], p.table, seqs[:T + 1], pos[:T + 1], want, seq_slots=slots, status=p.status, n_seqs=n)
        assert torch.equal(out, some)
    assert p.status.item() == 0


def wide(x, extra=32):
    """x [T][heads][d] as a slice of rows that are `extra` heads longer, what is around it NaN."""
    T, heads, d = x.shape
    rows = torch.full((T, (heads + extra) * d), NAN, dtype=x.dtype, device=x.device)
    y = rows[:, 8 * d:(8 + heads) * d].view(T, heads, d)
    y.copy_(x)
    return y


@pytest.mark.parametrize("dtype,d,page,n_q,n_kv,before,new", [
    ("bf16", 128, 16, 8, 2, [30, 0, 200], [1, 1, 1]), ("fp32", 64, 32, 4, 4, [90, 5], [3, 9]), ("bf16", 64, 64, 16, 8, [100, 0], [40, 130]),
    ("bf16", 128, 16, 32, 8, [333], [300]), ("bf16", 128, 64, 8, 1, [700], [1])])
def test_queries_inside_a_wider_tensor_and_results_in_place(dtype, d, page, n_q, n_kv, before, new):
    """The fused projection's queries give what dense ones give, bit for bit, and so does every call that writes over its queries."""
    B = len(new)
    p = Program(config(n_q=n_q, n_kv=n_kv, d=d, page=page, batch=B, pages=1024 // page, n_pages=B * 1024 // page, dtype=dtype), seed=19)
    p.step(before)
    p.step(new)
    q = p.rows(sum(new), n_q, 2.0)
    inside, slots = wide(q), dev(p.slots)
    seqs, pos = (dev(x) for x in p.tokens(new))
    assert len(q) == 1 or inside.stride(0) == (n_q + 32) * d
    assert torch.equal(p.attend(new, inside), p.attend(new, q))
    pages = p.cache.select_pages(q, p.table, seqs, pos, 5, seq_slots=slots)
    check_select(p, new, q, pages, 5, 1, 1)
    assert torch.equal(p.cache.select_pages(inside, p.table, seqs, pos, 5, seq_slots=slots), pages)
    some = p.cache.sparse_attention(q, p.table, seqs, pos, pages, seq_slots=slots)
    check_sparse(p, *p.tokens(new), q, pages.cpu().numpy(), some)
    assert torch.equal(p.cache.sparse_attention(inside, p.table, seqs, pos, pages, seq_slots=slots), some)
    over = q.clone()
    assert p.cache.sparse_attention(over, p.table, seqs, pos, pages, seq_slots=slots, out=over) is over and torch.equal(over, some)
    want, over = p.attend(new, q), q.clone()
    assert p.attend(new, over, out=over) is over and torch.equal(over, want)
    assert p.status.item() == 0


@pytest.mark.parametrize("dtype,new", [("bf16", [1, 1]), ("fp32", [2, 5]), ("bf16", [200, 90])])
def test_the_callers_softmax_scale(dtype, new):
    p = Program(config(n_q=8, n_kv=2, d=64, page=16, batch=2, pages=32, n_pages=64, dtype=dtype, softmax_scale=0.37), seed=20)
    p.step([40, 3])
    p.step(new)
    q = p.rows(sum(new), 8)
    out, (seqs, pos), at = p.attend(new, q), p.tokens(new), 0
    pages = np.arange(-(-max(p.lens) // 16))
    pages = np.broadcast_to(np.where(pages[None, None] <= pos[:, None, None] // 16, pages, -1), (len(pos), 2, len(pages)))
    some = p.cache.sparse_attention(q, p.table, dev(seqs), dev(pos), dev(pages.copy()), seq_slots=dev(p.slots), status=p.status)
    for b, n in enumerate(new):
        rows = sorted({0, n // 2, n - 1})
        ref, size = R.attend(f64(q[at:at + n]), p.k[b], p.v[b], 0.37, only=rows)
        for got, chunk in ((out, dtype == "bf16" and 4 * n >= 64), (some, False)):
            tol = F.tolerance(ref, size, p.lens[b], EPS[dtype], dtype == "bf16", chunk)
            assert (np.abs(f64(got[at:at + n]) - ref)[rows] <= tol[rows]).all(), b
        at += n
    assert p.status.item() == 0


def test_a_graph_whose_streams_fork_and_join():
    """Kernels that may come before the one ahead of them has ended, behind and before events of other streams, in a graph and outside."""
    cfg = config(n_q=8, n_kv=2, d=128, page=16, batch=2, pages=64, n_pages=128)
    a, b = Program(cfg, seed=21), Program(cfg, seed=22)
    for p in (a, b):
        p.step([500, 90])
    q, slots, lens = a.rows(2, 8), [dev(p.slots) for p in (a, b)], dev([501, 91])
    seqs, pos = dev([0, 1]), dev([500, 90])
    k, v = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    plans = [p.plan([1, 1]) for p in (a, b)]
    out = [torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(4)]

    def branch(i, p):
        p.cache.append(k, v, plans[i].slot_map, status=p.status)
        p.cache.attention(q, p.table, lens, seq_slots=slots[i], out=out[i], status=p.status)
        pages = p.cache.select_pages(q, p.table, seqs, pos, 6, seq_slots=slots[i], status=p.status)
        p.cache.sparse_attention(q, p.table, seqs, pos, pages, seq_slots=slots[i], out=out[2 + i], status=p.status)

    def step(main, other):
        other.wait_stream(main)
        with torch.cuda.stream(other):
            branch(1, b)
        branch(0, a)
        main.wait_stream(other)
        return a.cache.attention(out[1], a.table, lens, seq_slots=slots[0])                  # (behind the other stream's last kernel)
    other, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        last = step(stream, other)
    for i in range(10):
        k.copy_(a.rows(2, 2))
        v.copy_(a.rows(2, 2))
        graph.replay()
        got = [x.clone() for x in out] + [last.clone()]
        for x in out:
            x.zero_()
        again = step(torch.cuda.current_stream(), other)
        assert all(torch.equal(x, y) for x, y in zip(got, out + [again])), i
    for i, p in enumerate((a, b)):
        p.note([1, 1], k.float().cpu().numpy(), v.float().cpu().numpy())
        p.check_cache()
        p.check_attention([1, 1], q, got[i])
    assert a.status.item() == 0 and b.status.item() == 0
