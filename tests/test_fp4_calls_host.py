"""Calls of the 4-bit cache's entry points that are refused before any CUDA call, or that the binding passes on, without a GPU."""
import pytest

from paper_2603_22910_b200 import binding, build
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
