"""Forms of the serving calls that their documentation allows: outputs over inputs, plans used again for smaller steps."""
import pytest
import torch

from tests.test_gpu_serving import Program, attend, config

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
