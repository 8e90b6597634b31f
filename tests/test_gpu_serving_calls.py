"""Forms of the serving calls that their documentation allows: outputs over inputs, plans used again for smaller steps."""
import pytest
import torch

from paper_2603_22910_b200 import binding
from tests.test_gpu_serving import Program, attend, check_attention, config, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,n_q,n_kv,before,new", [
    ("bf16", 8, 2, [3000, 5, 40], [1, 1, 1]), ("fp32", 8, 8, [700, 0, 900], [9, 30, 1]), ("bf16", 32, 32, [600, 1500, 0], [300, 700, 1]),
    ("bf16", 8, 1, [6000, 0, 20], [70, 3, 0])])
def test_attention_in_place(dtype, n_q, n_kv, before, new):
    """Whole items and items cut between CTAs, of both kernels; a sequence with a bad slot."""
    cfg = config(n_q=n_q, n_kv=n_kv, d=64, page=64, batch=3, pages=100, n_pages=300, dtype=dtype)
    p = Program(cfg, "int8", seed=n_q, dtype=dtype)
    p.step(before)
    p.step(new)
    q = p.rows(sum(new), n_q, 2.0)
    want = attend(p, new, q)
    for _ in range(3):
        buf = q.clone()
        got = attend(p, new, buf, out=buf)
        assert got is buf and torch.equal(got, want)
    p.slots[1] = -1
    want, buf = attend(p, new, q), q.clone()
    attend(p, new, buf, out=buf)
    assert torch.equal(buf, want) and (buf[new[0]: new[0] + new[1]] == 0).all() and p.status.item() == -8


def test_a_plan_used_again_for_a_smaller_step():
    """What a larger step left behind in the buffers is not part of the returned plan."""
    cfg = config(n_q=4, n_kv=2, d=64, page=16, batch=4, pages=16, n_pages=60)
    p = Program(cfg, "int8", seed=3)
    out = binding.StepPlan(4, 64, "cuda")

    def step(new, n_tokens):
        B = len(new)
        plan = binding.plan_tokens(cfg, p.table, dev(p.lens[:B]), dev(new), p.free, p.count, n_tokens, seq_slots=dev(p.slots[:B]), out=out,
                                   status=p.status)
        p.count.copy_(plan.free_count)
        T, T0 = len(plan.slot_map), sum(new)
        qkv = p.rows(T, 8)
        k, v, q = qkv[:, :2].contiguous(), qkv[:, 2:4].contiguous(), qkv[:, 4:].contiguous()
        p.cache.append(k, v, plan.slot_map, plan.token_seqs, plan.cu_tokens, seq_slots=dev(p.slots[:B]), status=p.status)
        for b, n in enumerate(new):
            at = sum(new[:b])
            if n:
                p.ref.append(b, k[at:at + n].float().cpu().numpy(), v[at:at + n].float().cpu().numpy())
            p.lens[b] += n
        p.check_cache()
        res = p.cache.attention(q, p.table, plan.seq_lens, cu_tokens=plan.cu_tokens, max_new=16, seq_slots=dev(p.slots[:B]), status=p.status)
        check_attention(p, new, q[:T0], res[:T0])
        assert p.status.item() == 0
        return plan
    assert step([10, 16, 15, 16], 64) is out
    plan = step([3, 2], 7)
    assert plan.cu_tokens.tolist() == [0, 3, 5] and plan.seq_lens.tolist() == [13, 18] and plan.token_seqs.tolist() == [0, 0, 0, 1, 1, -1, -1]
    assert plan.slot_map.tolist()[5:] == [-1, -1] and len(plan.positions) == 7
    assert plan.cu_tokens.data_ptr() == out.cu_tokens.data_ptr() and plan.slot_map.data_ptr() == out.slot_map.data_ptr()
    step([1, 1, 1], 3)
    assert step([1, 1, 1, 1], 64) is out
