"""The 4-bit cache's entry points without a GPU: sizes, refusals (which come before any CUDA call), and the plain forms' own checks."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2603_22910_b200 import binding, build
from tests import fp4_ref as F
from tests.test_serving_host import NoStream, OnGpu, P1, config

EINVAL, ECAP, EUNS = binding.ECHOKV_EINVAL, binding.ECHOKV_ECAPACITY, binding.ECHOKV_EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def cache_struct(**kw):
    f = dict(blocks=P1, bounds=P1, bound_scales=P1, k_unit=1.0, v_unit=1.0)
    f.update(kw)
    return binding.echokv_fourbit_cache(*[f[n] for n, _ in binding.echokv_fourbit_cache._fields_])


def rotation(theta=1e4, sections=None, n_axes=1, interleaved=0, rot_dim=0):
    sec = None if sections is None else (C.c_int32 * len(sections))(*sections)
    return binding.echokv_rotation(theta, sec, n_axes, interleaved, rot_dim, 0)


def ref(x):
    return None if x is None else C.byref(x)


def append_call(lib, cfg=None, cache=None, rot=None, q=None, qs=4096, qo=None, qos=4096, k=P1, ks=1024, v=P1, vs=1024, pos=None, rows=P1, n=4,
                status=None):
    return lib.echokv_fourbit_append(C.byref(cfg or config()), C.byref(cache or cache_struct()), ref(rot), q, qs, qo, qos, k, ks, v, vs, pos, rows, n,
                                 status, None)


def read_call(lib, cfg=None, cache=None, rows=P1, n=4, k=P1, ks=1024, v=P1, vs=1024, status=None):
    return lib.echokv_fourbit_read(C.byref(cfg or config()), C.byref(cache or cache_struct()), rows, n, k, ks, v, vs, status, None)


def attn_call(lib, cfg=None, cache=None, opts=None, q=P1, qs=4096, out=P1, table=P1, slots=None, lens=P1, cu=P1, B=2, n=4, max_new=3, ws=P1,
              ws_bytes=1 << 40, status=None):
    return lib.echokv_fourbit_attention(C.byref(cfg or config()), C.byref(cache or cache_struct()), ref(opts), q, qs, out, table, slots, lens, cu, B, n,
                                    max_new, ws, ws_bytes, status, None)


def select_call(lib, cfg=None, cache=None, q=P1, qs=4096, table=P1, slots=None, seqs=P1, pos=P1, B=2, n=4, sel=8, first=1, recent=1, out=P1, ws=P1,
                ws_bytes=1 << 40, status=None):
    return lib.echokv_fourbit_select(C.byref(cfg or config()), C.byref(cache or cache_struct()), q, qs, table, slots, seqs, pos, B, n, sel, first, recent,
                                 out, ws, ws_bytes, status, None)


def sparse_call(lib, cfg=None, cache=None, opts=None, q=P1, qs=4096, out=P1, table=P1, slots=None, seqs=P1, pos=P1, pages=P1, sel=8, B=2, n=4,
                ws=P1, ws_bytes=1 << 40, status=None):
    return lib.echokv_fourbit_sparse_attention(C.byref(cfg or config()), C.byref(cache or cache_struct()), ref(opts), q, qs, out, table, slots, seqs, pos,
                                           pages, sel, B, n, ws, ws_bytes, status, None)


CALLS = (append_call, read_call, attn_call, select_call, sparse_call)


def test_sizes(lib):
    s = binding.query_fourbit_sizes(config())
    assert s.blocks_bytes == 32 * 8 * 18 * 128 and s.bounds_bytes == 32 * 8 * 2 * 128 and s.bound_scales_bytes == 32 * 8 * 4
    assert s.workspace_bytes % 256 == 0 and s.workspace_bytes > 0
    s = binding.query_fourbit_sizes(config(page_tokens=64, head_dim=64))
    assert s.blocks_bytes == 32 * 8 * 4 * 18 * 64


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=96), EUNS), (dict(page_tokens=24), EUNS), (dict(n_q_heads=48), EUNS), (dict(n_q_heads=12), EINVAL), (dict(dtype=3), EINVAL),
    (dict(n_pages=0), EINVAL), (dict(max_batch=0), EINVAL), (dict(softmax_scale=-1.0), EINVAL), (dict(device=-1), EINVAL),
    (dict(max_pages_per_seq=1 << 27), EINVAL), (dict(n_pages=1 << 31), EINVAL)])
def test_bad_configs(lib, kw, code):
    out = binding.echokv_fourbit_sizes()
    assert lib.echokv_query_fourbit_sizes(C.byref(config(**kw)), C.byref(out)) == code
    assert lib.echokv_query_fourbit_sizes(C.byref(config()), None) == EINVAL
    for call in CALLS:
        assert call(lib, cfg=config(**kw)) == code


def test_bad_caches(lib):
    for kw in (dict(blocks=None), dict(blocks=P1 + 8), dict(bounds=None), dict(bound_scales=None), dict(bounds=P1 + 8), dict(bound_scales=P1 + 4),
               dict(k_unit=0.0), dict(v_unit=-1.0), dict(k_unit=float("nan")), dict(v_unit=float("inf")), dict(k_unit=2.0 ** -61),
               dict(v_unit=2.0 ** 61)):
        for call in CALLS:
            assert call(lib, cache=cache_struct(**kw)) == EINVAL, (call, kw)
    without = cache_struct(bounds=None, bound_scales=None)
    assert select_call(lib, cache=without) == EINVAL
    assert append_call(lib, cache=without, n=0) == 0 and attn_call(lib, cache=without, n=0) == 0


def test_append_and_read_refusals(lib):
    for kw in (dict(k=None), dict(v=None), dict(ks=1023), dict(vs=1028), dict(k=P1 + 2), dict(rows=None), dict(rows=P1 + 4), dict(n=-1),
               dict(n=(1 << 27) + 1), dict(status=P1 + 2), dict(q=P1), dict(qo=P1), dict(q=P1, qo=P1),
               dict(rot=rotation()), dict(rot=rotation(), pos=P1 + 2), dict(rot=rotation(0.5), pos=P1), dict(rot=rotation(float("nan")), pos=P1),
               dict(rot=rotation(n_axes=2), pos=P1), dict(rot=rotation(n_axes=5), pos=P1), dict(rot=rotation(n_axes=0), pos=P1),
               dict(rot=rotation(sections=[30, 33], n_axes=2), pos=P1), dict(rot=rotation(sections=[-1, 65], n_axes=2), pos=P1),
               dict(rot=rotation(), pos=P1, q=P1, qo=P1, qos=8192), dict(rot=rotation(), pos=P1, q=P1 + 8, qo=P1),
               dict(rot=rotation(), pos=P1, q=P1, qo=None), dict(rot=rotation(), pos=P1, q=P1, qs=4000, qo=P1)):
        assert append_call(lib, **kw) == EINVAL, kw
    for rot in (8, 24, 144, -16):
        assert append_call(lib, rot=rotation(rot_dim=rot), pos=P1) == EUNS, rot
    assert append_call(lib, n=0, k=None, v=None, rows=None) == 0
    for kw in (dict(k=None, v=None), dict(rows=None), dict(rows=P1 + 4), dict(ks=1000), dict(vs=1027), dict(k=P1 + 4), dict(n=-1), dict(n=(1 << 27) + 1),
               dict(status=P1 + 2)):
        assert read_call(lib, **kw) == EINVAL, kw
    assert read_call(lib, n=0) == 0


def test_attention_refusals(lib):
    need = binding.query_fourbit_sizes(config()).workspace_bytes
    opt = binding.echokv_score_options
    both = (dict(q=None), dict(out=None), dict(out=P1 + 8), dict(table=None), dict(qs=4000), dict(B=0), dict(n=-1), dict(n=(1 << 27) + 1),
            dict(ws=None), dict(ws=P1 + 128), dict(opts=opt(-1.0, 0, None, None)), dict(opts=opt(1e-33, 0, None, None)),
            dict(opts=opt(float("nan"), 0, None, None)), dict(opts=opt(0.0, 0, P1 + 2, None)), dict(table=P1 + 2), dict(slots=P1 + 2),
            dict(status=P1 + 2), dict(out=P1 + 16), dict(q=P1, qs=8192, out=P1))
    for call in (attn_call, sparse_call):
        for kw in both:
            assert call(lib, **kw) == EINVAL, (call, kw)
        assert call(lib, ws_bytes=need - 1) == ECAP and call(lib, B=5) == ECAP
        assert call(lib, n=0, q=None, out=None) == 0
    for kw in (dict(lens=None), dict(lens=P1 + 2), dict(cu=P1 + 2), dict(max_new=0), dict(cu=None, n=4, B=2), dict(cu=None, n=2, max_new=2),
               dict(opts=opt(0.0, 0, None, P1 + 2))):
        assert attn_call(lib, **kw) == EINVAL, kw
    for kw in (dict(seqs=None), dict(pos=None), dict(pages=None), dict(seqs=P1 + 2), dict(pos=P1 + 1), dict(pages=P1 + 2), dict(sel=0), dict(sel=1025),
               dict(opts=opt(0.0, 0, None, P1))):
        assert sparse_call(lib, **kw) == EINVAL, kw


def test_select_refusals(lib):
    need = binding.query_fourbit_sizes(config()).workspace_bytes
    for kw in (dict(q=None), dict(q=P1 + 8), dict(qs=4000), dict(table=None), dict(seqs=None), dict(pos=None), dict(out=None), dict(out=P1 + 2),
               dict(seqs=P1 + 2), dict(pos=P1 + 2), dict(table=P1 + 2), dict(slots=P1 + 2), dict(status=P1 + 2), dict(B=0), dict(n=-1),
               dict(n=(1 << 27) + 1), dict(sel=0), dict(sel=1025), dict(first=-1), dict(recent=0), dict(first=7, recent=2), dict(first=8),
               dict(first=0x7fffffff, recent=0x7fffffff), dict(ws=None), dict(ws=P1 + 128)):
        assert select_call(lib, **kw) == EINVAL, kw
    assert select_call(lib, cfg=config(n_q_heads=128, n_kv_heads=128), qs=1 << 14, n=1 << 27) == EINVAL      # a block for each token and head
    assert select_call(lib, ws_bytes=need - 1) == ECAP and select_call(lib, B=5) == ECAP
    assert select_call(lib, n=0, q=None) == 0


BF, I32 = torch.bfloat16, torch.int32
HELD = dict(blocks=(torch.uint8, 32, 8, 1, 18 * 128), bounds=(torch.int8, 32, 8, 2, 128), bound_scales=(torch.float32, 32, 8), workspace=(torch.uint8, 1 << 30))


def fake_cache(**kw):
    return binding.Fp4Cache(config(), **{n: OnGpu(*t, index=0) for n, t in HELD.items()}, **kw)


def test_binding_refuses_wrong_tensors():
    cfg = config()
    for name in HELD:
        with pytest.raises(ValueError, match=name):
            binding.Fp4Cache(cfg, **{n: OnGpu(*t, index=1 if n == name else 0) for n, t in HELD.items()})
    with pytest.raises(ValueError, match="unit"):
        fake_cache(k_unit=0.0)
    with pytest.raises(ValueError, match="together"):
        binding.Fp4Cache(cfg, blocks=OnGpu(*HELD["blocks"], index=0), bounds=OnGpu(*HELD["bounds"], index=0))
    for kw in (dict(n_axes=2), dict(rot_dim=24), dict(rot_dim=256), dict(n_axes=2, sections=[10, 10]), dict(n_axes=3, sections=[32, 32])):
        with pytest.raises(ValueError, match="Rotation"):
            binding.Rotation(cfg, 1e4, **kw)
    cache = fake_cache()

    def refused(fn, tensors, wrong, **kw):
        args = {n: OnGpu(*t, index=1 if n == wrong else 0) for n, t in tensors.items()}
        with pytest.raises(ValueError, match=wrong):
            fn(**args, stream=NoStream(), **kw)
    new = dict(k_new=(BF, 4, 8, 128), v_new=(BF, 4, 8, 128), slot_map=(torch.int64, 4), q=(BF, 4, 32, 128), positions=(I32, 4), q_out=(BF, 4, 32, 128),
               status=(I32, 1))
    for name in new:
        refused(cache.append, new, name, rotation=binding.Rotation(cfg, 1e4))
    with pytest.raises(ValueError, match="rotation"):
        cache.append(OnGpu(BF, 4, 8, 128, index=0), OnGpu(BF, 4, 8, 128, index=0), OnGpu(torch.int64, 4, index=0), q=OnGpu(BF, 4, 32, 128, index=0))
    with pytest.raises(ValueError, match="positions"):
        cache.append(OnGpu(BF, 4, 8, 128, index=0), OnGpu(BF, 4, 8, 128, index=0), OnGpu(torch.int64, 4, index=0),
                     rotation=binding.Rotation(cfg, 1e4, n_axes=2, sections=[32, 32]), positions=OnGpu(I32, 4, index=0))
    back = dict(slot_map=(torch.int64, 4), k_out=(BF, 4, 8, 128), v_out=(BF, 4, 8, 128), status=(I32, 1))
    for name in back:
        refused(cache.read, back, name)
    common = dict(q=(BF, 4, 32, 128), block_table=(I32, 4, 8), seq_slots=(I32, 2), status=(I32, 1))
    dense = dict(common, seq_lens=(I32, 2), cu_tokens=(I32, 3), alibi_slopes=(torch.float32, 32), prefix_lens=(I32, 2), out=(BF, 4, 32, 128))
    for name in dense:
        refused(cache.attention, dense, name, max_new=3)
    choice = dict(common, token_seqs=(I32, 4), positions=(I32, 4), out=(I32, 4, 8, 16))
    for name in choice:
        refused(cache.select_pages, choice, name, n_select=16)
    sparse = dict(common, token_seqs=(I32, 4), positions=(I32, 4), pages=(I32, 4, 8, 16), alibi_slopes=(torch.float32, 32), out=(BF, 4, 32, 128))
    for name in sparse:
        refused(cache.sparse_attention, sparse, name)
    with pytest.raises(ValueError, match="pages"):
        cache.sparse_attention(OnGpu(BF, 4, 32, 128, index=0), OnGpu(I32, 4, 8, index=0), OnGpu(I32, 4, index=0), OnGpu(I32, 4, index=0),
                               OnGpu(I32, 4, 4, 16, index=0))
    plain = binding.Fp4Cache(cfg, blocks=OnGpu(*HELD["blocks"], index=0), workspace=OnGpu(*HELD["workspace"], index=0), selection=False)
    assert plain.bounds is None
    with pytest.raises(ValueError, match="selection"):
        plain.select_pages(OnGpu(BF, 4, 32, 128, index=0), None, None, None, 16)


def test_what_the_library_holds_stays():
    cache = fake_cache(k_unit=0.5)
    for name in ("cfg", "blocks", "bounds", "bound_scales", "k_unit", "v_unit"):
        before = getattr(cache, name)
        with pytest.raises(AttributeError, match=name):
            setattr(cache, name, None)
        assert getattr(cache, name) is before
    cache.workspace = OnGpu(*HELD["workspace"], index=0)


# ---- the plain forms themselves -----------------------------------------------------------------------------------
def test_codes_ref_by_hand():
    y = np.array([0, 0.2, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 2.6, 3.5, 5, 5.1, 7, -0.25, -0.3, -5.0], dtype=np.float32)
    assert F.e2m1_value(F.e2m1(y)).tolist() == [0, 0, 0, 0.5, 1, 1, 2, 2, 3, 4, 4, 6, 6, 0, -0.5, -4]
    x = np.zeros(16, np.float32)
    x[3], x[4] = 12.0, -5.0
    k, v = F.token(x[None], x[None], 1.0, 0.25)
    assert k[0, 3] == 12 and k[0, 4] == -4 and v[0, 3] == 12 and v[0, 4] == -4                # (5 / 2 is a tie: to the even code)


def test_held_values_are_near():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 128)).astype(np.float32)
    k, v = F.token(x, x * 1e-3, 0.25, 2.0 ** -12)
    a = np.abs(x).reshape(50, 8, 16).max(-1).repeat(16, -1).reshape(50, 128)
    # half the widest step, 2 of 6, and the scale's rounding (2^-4 of it) on a value of up to 6
    assert (np.abs(k - x) <= a * (1 / 6 + 2.0 ** -4)).all() and (np.abs(v / 1e-3 - x) <= a * (1 / 6 + 2.0 ** -4)).all()
    k, v = F.token(np.where(np.arange(128) == 5, np.inf, x).astype(np.float32), x, 1.0, 1.0)
    assert np.isnan(k).all() and (v == 0).all()


def test_bounds_hold_the_keys():
    rng = np.random.default_rng(1)
    k = rng.standard_normal((20, 64))
    b, s = F.bounds(k)
    assert (b[0] * float(s) >= k.max(0) - 0.51 * s).all() and (b[1] * float(s) <= k.min(0) + 0.51 * s).all()
    b, s = F.bounds(np.zeros((3, 64)))
    assert s == np.float32(2.0 ** -60) and (b == 0).all()


def test_select_ref_takes_the_best_and_the_first_of_equals():
    bnd = np.zeros((6, 1, 2, 64), np.int8)
    bnd[:, 0, 0, 0] = [1, 9, 3, 9, 3, 2]
    q = np.zeros((2, 64), np.float32)
    q[1, 0] = 2.0
    got = lambda n, **kw: F.select(q, bnd, np.ones((6, 1), np.float32), 5 * 16, 16, n, **kw)[0].tolist()  # noqa: E731
    assert got(3, n_first=0, n_recent=1) == [1, 3, 5] and got(4, n_first=0, n_recent=1) == [1, 2, 3, 5]
    assert got(3, n_first=1, n_recent=1) == [0, 1, 5] and got(8, n_first=0, n_recent=2) == [0, 1, 2, 3, 4, 5, -1, -1]


def test_attend_pages_of_all_pages_is_attention():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((1, 4, 64)), rng.standard_normal((40, 2, 64)), rng.standard_normal((40, 2, 64))
    a, sa = F.R.attend(q, k, v, 0.125, 5.0, [0.1, 0.2, 0.3, 0.4])
    b, sb = F.attend_pages(q[0], k, v, 39, [[2, 0, 1]] * 2, 16, 0.125, 5.0, [0.1, 0.2, 0.3, 0.4])
    assert np.allclose(a[0], b, atol=1e-13) and np.allclose(sa[0], sb)
