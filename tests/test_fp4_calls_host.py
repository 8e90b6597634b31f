"""Calls of the 4-bit cache's entry points that are refused before any CUDA call, or that the binding passes on, without a GPU."""
import numpy as np
import pytest

from paper_2603_22910_b200 import binding, build
from tests import fp4_ref as F
from tests.test_fp4_host import BF, EINVAL, I32, append_call, fake_cache, rotation
from tests.test_serving_host import NoStream, OnGpu, P1


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_queries_that_are_written_over_an_input_are_refused(lib):
    """32 heads of 128 and 8: query rows of 8192 bytes, keys and values of 2048, 4 tokens."""
    far = P1 + (1 << 20)
    apart = dict(rot=rotation(), pos=far, rows=far + 4096, k=far + 8192, v=far + 32768)
    for kw in (dict(q=P1, qo=P1 + 16), dict(q=P1 + 16, qo=P1), dict(q=P1, qo=P1 + 3 * 8192 + 8176), dict(q=P1 + 3 * 8192 + 8176, qo=P1),     # a part of a row
               dict(q=P1, qs=6144, qo=P1 + 12288), dict(q=P1, qo=P1 + 8192, qos=6144), dict(q=P1, qs=6144, qo=P1 + 4 * 12288 - 8192, qos=4104),
               dict(q=P1, qo=P1, k=P1 + 8192), dict(q=P1, qo=P1, k=P1 + 8176), dict(q=P1, qo=P1, v=P1 - 2032), dict(q=P1, qo=P1, v=P1 - 3 * 2048 - 2032),
               dict(q=P1, qs=6144, qo=P1, qos=6144, k=P1 + 8192, ks=6144, v=P1 + 8176, vs=6144), dict(q=P1, qo=P1, pos=P1 + 8192),
               dict(q=P1, qo=P1, pos=P1 - 12), dict(q=P1, qo=P1, rows=P1 + 4 * 8192 - 8), dict(q=far + (1 << 20), qo=far + 8192)):
        assert append_call(lib, **dict(apart, **kw)) == EINVAL, kw


def test_the_number_of_sequences_is_passed_on(monkeypatch):
    """A bound on the ids is all that the table gives; who knows how many sequences the tokens are of can say so."""
    cache, calls = fake_cache(), {}

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.__setitem__(name, a) or 0
    monkeypatch.setattr(binding, "lib", lambda: Library())
    table, q, ids, pages = OnGpu(I32, 4, 8, index=0), OnGpu(BF, 6, 32, 128, index=0), OnGpu(I32, 6, index=0), OnGpu(I32, 6, 8, 16, index=0)
    slots = OnGpu(I32, 3, index=0)
    for kw, B in ((dict(), 4), (dict(seq_slots=slots), 3), (dict(n_seqs=1), 1), (dict(n_seqs=2, seq_slots=slots), 2)):
        cache.select_pages(q, table, ids, ids, 16, out=pages, stream=NoStream(), **kw)
        assert calls["echokv_fourbit_select"][8:11] == (B, 6, 16)
        cache.sparse_attention(q, table, ids, ids, pages, out=q, stream=NoStream(), **kw)
        assert calls["echokv_fourbit_sparse_attention"][11:14] == (16, B, 6)
    with pytest.raises(ValueError, match="seq_slots"):
        cache.select_pages(q, table, ids, ids, 16, out=pages, stream=NoStream(), n_seqs=4, seq_slots=slots)


@pytest.mark.parametrize("d", [64, 128])
def test_how_far_a_pages_score_may_lie_below_its_best_key(d):
    """q . k <= sum_c max(q_c top_c, q_c low_c), of which each factor is rounded to the nearest of 127 steps of its largest magnitude: a term is
    off by a_q a_k (1 / 127 + 1 / (2 127)^2) at most, less than 1 / 126 of that, d of them in all (fp32 products: 2^-22 of the score)."""
    rng = np.random.default_rng(d)
    below = 0
    for i in range(200):
        k, q = rng.standard_normal((16, d)) * rng.uniform(0.1, 3, d), rng.standard_normal(d).astype(np.float32)
        if i % 3 == 0:
            k, q = k[:1], np.sign(q) * (1 + 0.49 / 127) * (np.arange(d) > 0) + (np.arange(d) == 0) * np.float32(127)      # one key, rounded down nearly everywhere
        b, scale = F.bounds(k)
        s_q = np.abs(q).max() / 127
        code = np.rint(q / s_q)
        score = s_q * float(scale) * np.maximum(code * b[0], code * b[1].astype(float)).sum()
        best = (k @ q).max()
        below += score < best
        assert score >= best * (1 - 2.0 ** -22) - d / 126 * np.abs(q).max() * np.abs(k).max()
    assert below > 0
