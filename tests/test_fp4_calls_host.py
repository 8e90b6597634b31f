"""Calls of the 4-bit cache's entry points that are refused before any CUDA call, or that the binding passes on, without a GPU."""
import pytest

from paper_2603_22910_b200 import binding, build
from tests.test_fp4_host import EINVAL, append_call, rotation
from tests.test_serving_host import P1


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
