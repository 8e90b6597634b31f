"""New tensors of calls that are given a stream belong to that stream: memory that work queued on the current one still uses is not
handed to them."""
import pytest
import torch

from paper_2603_22910_b200 import binding
from tests.test_gpu_serving import Program, config, dev

pytestmark = pytest.mark.gpu


def owner(t):
    """The stream that the memory behind t was allocated for."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's")


def test_new_outputs_of_serving_calls_belong_to_the_given_stream():
    cfg = config(n_q=8, n_kv=2, d=128, page=16, batch=2, pages=16, n_pages=40)
    p = Program(cfg, "e4m3", seed=14)
    p.step([40, 90])
    q, k, pos = p.rows(2, 8), p.rows(2, 2), dev([5, 6])
    lens, new, slots = dev(p.lens), dev([1, 1]), dev(p.slots)
    want = [p.cache.attention(q, p.table, lens, seq_slots=slots), *binding.rotate(cfg, q, k, pos, 1e4)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [p.cache.attention(q, p.table, lens, seq_slots=slots, stream=s), *binding.rotate(cfg, q, k, pos, 1e4, stream=s)]
    plan = binding.plan_tokens(cfg, p.table, lens, new, p.free, p.count, 2, seq_slots=slots, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and plan.positions.tolist() == [40, 90]
    for t in got + [plan.cu_tokens, plan.positions, plan.slot_map, plan.seq_lens, plan.free_count]:
        assert owner(t) == s.cuda_stream
    assert owner(want[0]) != s.cuda_stream and torch.cuda.current_stream() != s


def test_new_outputs_of_a_context_belong_to_the_given_stream():
    cfg = binding.make_config(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, group_size=2, n_retained_heads=1, page_tokens=16,
                              max_batch=2, max_pages_per_seq=4, n_pages=8, dtype=binding.ECHOKV_BF16)
    ctx = binding.Context(cfg, zero_pools=True)
    ctx.set_block_table(torch.arange(8, dtype=torch.int32).view(2, 4))
    q, lens = torch.randn(2, 8, 128, device="cuda").bfloat16(), dev([30, 50])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = ctx.full_attention(0, q, lens, stream=s)
    s.synchronize()
    assert owner(out) == s.cuda_stream and (out == 0).all()
    ctx.close()
