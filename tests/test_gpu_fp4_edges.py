"""The 4-bit cache's operators where a call is unlike the common ones."""
import pytest

from tests.test_gpu_fp4 import Program
from tests.test_gpu_serving import config

pytestmark = pytest.mark.gpu
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
