"""The serving-step entry points without a GPU: sizes, refusals (which come before any CUDA call), and the plain forms' own
checks."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2603_22910_b200 import binding, build
from tests import serving_ref as R

EINVAL, ECAP, EUNS = binding.ECHOKV_EINVAL, binding.ECHOKV_ECAPACITY, binding.ECHOKV_EUNSUPPORTED
P1 = 0x10000          # an address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def config(**kw):
    base = dict(n_layers=1, n_q_heads=32, n_kv_heads=8, head_dim=128, group_size=1, n_retained_heads=0, page_tokens=16, max_batch=4,
                max_pages_per_seq=8, n_pages=32, dtype=binding.ECHOKV_BF16)
    base.update(kw)
    return binding.make_config(**base)


def test_quant_sizes(lib):
    s = binding.query_quant_sizes(config())
    assert s.codes_bytes == 32 * 16 * 8 * 128
    assert s.scales_bytes == 32 * 8 * 4
    assert s.tail_bytes == 4 * 8 * 16 * 128 * 2
    assert s.workspace_bytes % 256 == 0 and s.workspace_bytes > 0
    assert binding.query_quant_sizes(config(dtype=binding.ECHOKV_FP32)).tail_bytes == 4 * 8 * 16 * 128 * 4


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=96), EUNS), (dict(page_tokens=24), EUNS), (dict(n_q_heads=48), EUNS), (dict(n_q_heads=12), EINVAL),
    (dict(dtype=3), EINVAL), (dict(n_pages=0), EINVAL), (dict(max_batch=0), EINVAL), (dict(softmax_scale=-1.0), EINVAL),
    (dict(device=-1), EINVAL), (dict(max_pages_per_seq=1 << 27), EINVAL), (dict(n_pages=1 << 31), EINVAL),
])
def test_bad_configs(lib, kw, code):
    out = binding.echokv_quant_sizes()
    assert lib.echokv_query_quant_sizes(C.byref(config(**kw)), C.byref(out)) == code
    assert lib.echokv_query_quant_sizes(C.byref(config()), None) == EINVAL


def plan_call(lib, cfg=None, table=P1, slots=None, lens=P1, new=P1, pages=P1, count=P1, B=2, n=4, plan="full"):
    cfg = config() if cfg is None else cfg
    p = binding.echokv_step_plan(*([P1] * 6)) if plan == "full" else plan
    return lib.echokv_plan_tokens(C.byref(cfg), table, slots, lens, new, pages, count, B, n, None if p is None else C.byref(p), None, None)


def test_plan_refusals(lib):
    for kw in (dict(table=None), dict(lens=None), dict(new=None), dict(pages=None), dict(count=None), dict(plan=None), dict(B=0),
               dict(n=-1), dict(plan=binding.echokv_step_plan(P1, P1, P1, None, P1, P1)),
               dict(plan=binding.echokv_step_plan(None, P1, P1, P1, P1, P1))):
        assert plan_call(lib, **kw) == EINVAL, kw
    assert plan_call(lib, B=5) == ECAP
    assert plan_call(lib, cfg=config(max_batch=9000), B=8193) == ECAP
    assert plan_call(lib, cfg=config(page_tokens=8)) == EUNS
    cfg = config()
    assert lib.echokv_release_pages(C.byref(cfg), P1, None, None, 1, P1, P1, None, None) == EINVAL
    assert lib.echokv_release_pages(C.byref(cfg), P1, None, P1, 0, P1, P1, None, None) == EINVAL
    assert lib.echokv_release_pages(C.byref(cfg), P1, None, P1, 5, P1, P1, None, None) == ECAP
    assert lib.echokv_release_pages(None, P1, None, P1, 1, P1, P1, None, None) == EINVAL


def rotate_call(lib, cfg=None, q=P1, qs=4096, k=P1, ks=1024, qo=P1, qos=4096, ko=P1, kos=1024, pos=P1, axes=1, sec=None, inter=0, rot=0,
                theta=1e4, n=4):
    cfg = config() if cfg is None else cfg
    sec = None if sec is None else (C.c_int32 * len(sec))(*sec)
    return lib.echokv_rotate(C.byref(cfg), q, qs, k, ks, qo, qos, ko, kos, pos, axes, sec, inter, rot, theta, 0, n, None)


def test_rotate_refusals(lib):
    for kw in (dict(q=None), dict(qo=None), dict(q=None, qo=None, k=None, ko=None), dict(qs=4095), dict(qs=4100), dict(q=P1 + 8),
               dict(qo=P1, qos=8192), dict(pos=None), dict(axes=0), dict(axes=5, sec=[64, 0, 0, 0, 0]), dict(axes=2),
               dict(axes=2, sec=[32, 31]), dict(axes=2, sec=[65, -1]), dict(theta=0.5), dict(theta=float("nan")),
               dict(theta=float("inf")), dict(n=-1)):
        assert rotate_call(lib, **kw) == EINVAL, kw
    for rot in (8, 24, 130, 144, -16):
        assert rotate_call(lib, rot=rot) == EUNS, rot
    assert rotate_call(lib, n=0, q=None, pos=None) == 0                # nothing to do


def quant_struct(**kw):
    base = dict(k_codes=P1, v_codes=P1, k_scales=P1, v_scales=P1, k_tail=P1, v_tail=P1, format=0, reserved=0)
    base.update(kw)
    return binding.echokv_quant_cache(**base)


def append_call(lib, cfg=None, cache=None, k=P1, ks=1024, v=P1, vs=1024, rows=P1, seqs=P1, cu=P1, B=2, n=4):
    cfg, cache = cfg or config(), cache or quant_struct()
    return lib.echokv_quant_append(C.byref(cfg), C.byref(cache), k, ks, v, vs, rows, seqs, cu, None, B, n, None, None)


def attn_call(lib, cfg=None, cache=None, opts=None, q=P1, qs=4096, out=P1, table=P1, lens=P1, cu=P1, B=2, n=4, max_new=3, ws=P1,
              ws_bytes=1 << 30):
    cfg, cache = cfg or config(), cache or quant_struct()
    return lib.echokv_quant_attention(C.byref(cfg), C.byref(cache), None if opts is None else C.byref(opts), q, qs, out, table, None,
                                      lens, cu, B, n, max_new, ws, ws_bytes, None, None)


@pytest.mark.parametrize("field", ["k_codes", "v_codes", "k_scales", "v_scales", "k_tail", "v_tail"])
def test_quant_cache_pointers(lib, field):
    for bad in (None, P1 + 4):
        assert append_call(lib, cache=quant_struct(**{field: bad})) == EINVAL
        assert attn_call(lib, cache=quant_struct(**{field: bad})) == EINVAL


def test_quant_refusals(lib):
    assert append_call(lib, cache=quant_struct(format=2)) == EINVAL
    for kw in (dict(k=None), dict(v=None), dict(ks=1023), dict(vs=1028), dict(k=P1 + 2), dict(rows=None), dict(seqs=None), dict(cu=None),
               dict(B=0), dict(n=-1), dict(n=(1 << 27) + 1)):
        assert append_call(lib, **kw) == EINVAL, kw
    assert append_call(lib, B=5) == ECAP
    assert append_call(lib, n=0, k=None) == 0
    for kw in (dict(q=None), dict(out=None), dict(out=P1 + 8), dict(table=None), dict(lens=None), dict(qs=4000), dict(max_new=0), dict(B=0),
               dict(cu=None, n=4, B=2), dict(cu=None, n=2, max_new=2), dict(ws=None), dict(ws=P1 + 128),
               dict(opts=binding.echokv_score_options(-1.0, 0, None, None)), dict(opts=binding.echokv_score_options(1e-33, 0, None, None)),
               dict(n=(1 << 27) + 1),
               dict(opts=binding.echokv_score_options(float("nan"), 0, None, None))):
        assert attn_call(lib, **kw) == EINVAL, kw
    need = binding.query_quant_sizes(config()).workspace_bytes
    assert attn_call(lib, ws_bytes=need - 1) == ECAP
    assert attn_call(lib, B=5) == ECAP
    assert attn_call(lib, n=0, q=None, out=None) == 0


def test_binding_refuses_wrong_tensors():
    cfg = config()
    with pytest.raises(ValueError, match="device tensor"):
        binding.plan_tokens(cfg, torch.zeros(4, 8, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                            torch.zeros(32, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 4)
    with pytest.raises(ValueError, match="format"):
        binding.QuantCache(cfg, "int4")
    with pytest.raises(ValueError, match="neither"):
        binding.rotate(cfg, None, None, torch.zeros(1, dtype=torch.int32), 1e4)
    with pytest.raises(ValueError, match="number of tokens"):
        binding.rotate(cfg, torch.zeros(3, 32, 128, dtype=torch.bfloat16), None, torch.zeros(2, dtype=torch.int32), 1e4)


# ---- the plain forms themselves -------------------------------------------------------------------------------
def test_plan_ref_by_hand():
    r = R.plan([[9, 0, 0], [7, 8, 0]], [1, 0], [17, 16], [15, 3], [5, 6, 4], 3, 20, 16, 2, 32)
    assert r["table"] == [[9, 4, 0], [7, 8, 0]] and r["count"] == 2 and r["cu"] == [0, 15, 18] and r["lens"] == [32, 19]
    assert r["rows"][:2] == [8 * 16 + 1, 8 * 16 + 2] and r["rows"][15:] == [4 * 16, 4 * 16 + 1, 4 * 16 + 2, -1, -1] and r["status"] == 0
    # no page left for the second sequence, the third needs none
    r = R.plan([[0, 0], [0, 0], [1, 0]], [0, 1, 2], [0, 0, 3], [17, 1, 2], [3, 2], 2, 32, 16, 3, 8)
    assert r["cu"] == [0, 17, 17, 19] and r["lens"] == [17, 0, 5] and r["count"] == 0 and r["status"] == -4


def test_quantise_ref_is_within_half_a_step():
    rng = np.random.default_rng(3)
    for fmt in ("int8", "e4m3"):
        x = rng.standard_normal((16, 64)).astype(np.float32)
        scale, codes = R.quantise_block(x, fmt)
        got = codes.astype(np.float64) * float(scale)
        # int8: half a step of the scale; e4m3: half a step of three mantissa bits (2^-4), or of its smallest step 2^-9;
        # both and the division's and product's roundings of 2^-22
        half = 0.5 * scale if fmt == "int8" else np.maximum(2.0 ** -4 * np.abs(x), 0.5 * 2.0 ** -9 * scale)
        assert (np.abs(got - x) <= half * (1 + 2.0 ** -14) + 2.0 ** -20 * np.abs(x)).all()
        assert np.abs(codes).max() == R.QMAX[fmt]


def test_rotate_ref_turns_back_and_keeps_lengths():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((5, 2, 64))
    pos = rng.integers(-100, 100000, (3, 5))
    for inter in (False, True):
        y = R.rotate(x, pos, 1e4, [8, 12, 12], 64, inter, False)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        assert np.allclose(R.rotate(y, pos, 1e4, [8, 12, 12], 64, inter, True), x)


def test_attend_ref_is_plain_softmax():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((2, 4, 64)), rng.standard_normal((7, 2, 64)), rng.standard_normal((7, 2, 64))
    out, _ = R.attend(q, k, v, 0.125)
    t = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q).permute(1, 0, 2), torch.from_numpy(k).permute(1, 0, 2).repeat_interleave(2, 0),
        torch.from_numpy(v).permute(1, 0, 2).repeat_interleave(2, 0),
        attn_mask=torch.ones(2, 7, dtype=torch.bool).tril(5), scale=0.125)
    assert np.allclose(out, t.permute(1, 0, 2).numpy())
    full, _ = R.attend(q, k, v, 0.125, prefix=7)
    last, _ = R.attend(q[:1], k, v, 0.125)
    assert np.allclose(full[:1], last)


# ---- pointers and buffers that a kernel could not use ------------------------------------------------------------
def test_misaligned_small_arrays_are_refused(lib):
    """Every int32, fp32 and int64 array: an address off its type's would end the kernel with a misaligned access."""
    bad = P1 + 2
    for kw in (dict(table=bad), dict(slots=bad), dict(lens=bad), dict(new=bad), dict(pages=bad), dict(count=bad)):
        assert plan_call(lib, **kw) == EINVAL, kw
    for i in range(6):
        p = [P1] * 6
        p[i] = P1 + (4 if i == 3 else 2)                                # (slot_map is int64)
        assert plan_call(lib, plan=binding.echokv_step_plan(*p)) == EINVAL, i
    cfg, s = config(), binding.echokv_step_plan(*([P1] * 6))
    assert lib.echokv_plan_tokens(C.byref(cfg), P1, None, P1, P1, P1, P1, 2, 4, C.byref(s), bad, None) == EINVAL
    for i in range(6):
        p = [P1] * 6
        p[i] = bad
        table, slots, lens, pages, count, status = p
        assert lib.echokv_release_pages(C.byref(cfg), table, slots, lens, 1, pages, count, status, None) == EINVAL, i
    assert rotate_call(lib, pos=bad) == EINVAL
    for kw in (dict(rows=P1 + 4), dict(seqs=bad), dict(cu=bad)):
        assert append_call(lib, **kw) == EINVAL, kw
    cache = quant_struct()
    for slots, status in ((bad, None), (None, bad)):
        assert lib.echokv_quant_append(C.byref(cfg), C.byref(cache), P1, 1024, P1, 1024, P1, P1, P1, slots, 2, 4, status, None) == EINVAL
        need = binding.query_quant_sizes(cfg).workspace_bytes
        assert lib.echokv_quant_attention(C.byref(cfg), C.byref(cache), None, P1, 4096, P1, P1, slots, P1, P1, 2, 4, 3, P1, need, status,
                                          None) == EINVAL
    for kw in (dict(table=bad), dict(lens=bad), dict(cu=bad), dict(opts=binding.echokv_score_options(0.0, 0, bad, None)),
               dict(opts=binding.echokv_score_options(0.0, 0, None, bad))):
        assert attn_call(lib, **kw) == EINVAL, kw


def test_outputs_that_partly_overlap_the_queries_are_refused(lib):
    """out may be q itself where that is dense; 4 rows of 8192 bytes each otherwise lie beside it, between its rows or behind it."""
    row = 32 * 128 * 2
    need = binding.query_quant_sizes(config()).workspace_bytes
    q = P1 + 16 * row
    call = lambda out, qs=4096, n=4: attn_call(lib, q=q, qs=qs, out=out, n=n, ws_bytes=need - 1)  # noqa: E731  (ECAP: nothing else is wrong)
    for out, qs in ((q, 4096), (q - 4 * row, 4096), (q + 4 * row, 4096), (q + row, 6 * 4096), (q + 2 * row, 6 * 4096), (q - 4 * row, 5 * 4096)):
        assert call(out, qs) == ECAP, (out - q, qs)
    for out, qs in ((q + 16, 4096), (q - 16, 4096), (q + row, 4096), (q - row, 4096), (q + 4 * row - 16, 4096), (q, 2 * 4096), (q + 3 * row, 6 * 4096),
                    (q - 3 * row, 6 * 4096), (q + row, 3 * 4096), (q + 18 * row, 6 * 4096)):
        assert call(out, qs) == EINVAL, (out - q, qs)


class OnGpu:
    """What the binding asks of a tensor, without a GPU: `shape` elements on device `index`."""
    is_cuda = True

    def __init__(self, dtype, *shape, index=1):
        self.dtype, self.shape, self.index = dtype, torch.Size(shape), index
        self.device = torch.device("cuda", index)

    def get_device(self):
        return self.index

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P1


class NoStream:
    cuda_stream = 0


def test_tensors_of_another_device_are_refused():
    """The kernels run on cfg.device: an address of another GPU's memory would fault there."""
    cfg, i32, bf16 = config(), torch.int32, torch.bfloat16
    small = dict(block_table=(i32, 4, 8), seq_lens=(i32, 2), new_lens=(i32, 2), free_pages=(i32, 32), free_count=(i32, 1), seq_slots=(i32, 2),
                 status=(i32, 1))
    plan = object.__new__(binding.StepPlan)
    plan._batch, plan._tokens, plan._device, plan._c = 2, 4, 0, binding.echokv_step_plan(*([P1] * 6))

    def refused(fn, tensors, wrong, **kw):
        args = {n: OnGpu(*t, index=1 if n == wrong else 0) for n, t in tensors.items()}
        with pytest.raises(ValueError, match=wrong):
            fn(**args, stream=NoStream(), **kw)
    for name in small:
        refused(lambda **kw: binding.plan_tokens(cfg, n_tokens=4, out=plan, **kw), small, name)
    plan._device = 1
    with pytest.raises(ValueError, match="out"):
        binding.plan_tokens(cfg, n_tokens=4, out=plan, stream=NoStream(), **{n: OnGpu(*t, index=0) for n, t in small.items()})
    free = {n: t for n, t in small.items() if n != "new_lens"}
    for name in free:
        refused(lambda **kw: binding.release_pages(cfg, **kw), free, name)
    turn = dict(q=(bf16, 4, 32, 128), k=(bf16, 4, 8, 128), positions=(i32, 4), q_out=(bf16, 4, 32, 128), k_out=(bf16, 4, 8, 128))
    for name in turn:
        refused(lambda **kw: binding.rotate(cfg, theta=1e4, **kw), turn, name)
    held = dict(k_codes=(torch.int8, 32, 8, 16, 128), v_codes=(torch.int8, 32, 8, 16, 128), k_scales=(torch.float32, 32, 8, 1),
                v_scales=(torch.float32, 32, 8, 1), k_tail=(bf16, 4, 8, 16, 128), v_tail=(bf16, 4, 8, 16, 128),
                workspace=(torch.uint8, 1 << 30))
    for name in held:
        with pytest.raises(ValueError, match=name):
            binding.QuantCache(cfg, "int8", **{n: OnGpu(*t, index=1 if n == name else 0) for n, t in held.items()})
    cache = binding.QuantCache(cfg, "int8", **{n: OnGpu(*t, index=0) for n, t in held.items()})
    new = dict(k_new=(bf16, 4, 8, 128), v_new=(bf16, 4, 8, 128), slot_map=(torch.int64, 4), token_seqs=(i32, 4), cu_tokens=(i32, 3),
               seq_slots=(i32, 2), status=(i32, 1))
    for name in new:
        refused(cache.append, new, name)
    attend = dict(q=(bf16, 4, 32, 128), block_table=(i32, 4, 8), seq_lens=(i32, 2), cu_tokens=(i32, 3), seq_slots=(i32, 2),
                  alibi_slopes=(torch.float32, 32), prefix_lens=(i32, 2), out=(bf16, 4, 32, 128), status=(i32, 1))
    for name in attend:
        refused(cache.attention, attend, name, max_new=3)


def test_the_tensors_whose_addresses_a_cache_and_a_plan_hold_stay():
    """An attribute that is set anew would leave the library with the address of freed memory."""
    cfg, bf16 = config(), torch.bfloat16
    held = dict(k_codes=(torch.int8, 32, 8, 16, 128), v_codes=(torch.int8, 32, 8, 16, 128), k_scales=(torch.float32, 32, 8, 1),
                v_scales=(torch.float32, 32, 8, 1), k_tail=(bf16, 4, 8, 16, 128), v_tail=(bf16, 4, 8, 16, 128),
                workspace=(torch.uint8, 1 << 30))
    cache = binding.QuantCache(cfg, "int8", **{n: OnGpu(*t, index=0) for n, t in held.items()})
    for name in list(held)[:6] + ["cfg"]:
        before = getattr(cache, name)
        with pytest.raises(AttributeError, match=name):
            setattr(cache, name, None)
        assert getattr(cache, name) is before
    cache.workspace = OnGpu(torch.uint8, 1 << 30, index=0)                # (checked at every call)
    lens, count = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    p = binding.StepPlan(2, 4, "cpu", seq_lens=lens, free_count=count)
    q = p._beginning(1, 2)
    addresses = [t.data_ptr() for t in (p.slot_map, lens, count)]
    p.slot_map = p.seq_lens = p.free_count = None
    q.slot_map = q.seq_lens = q.free_count = None
    for plan in (p, q):
        assert [t.data_ptr() for t in plan._held[1:]] == addresses
