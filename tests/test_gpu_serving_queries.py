"""Query rows that are not finite, over the 8-bit cache."""
import numpy as np
import pytest
import torch

from tests import serving_ref as R
from tests.test_gpu_serving import DT, EPS, Program, attend, config, f64

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("softcap", [0.0, 5.0])
@pytest.mark.parametrize("fmt,dtype,new", [("int8", "bf16", [1, 1, 2]), ("e4m3", "fp32", [1, 1, 2]), ("e4m3", "bf16", [3, 1, 20]), ("int8", "fp32", [3, 1, 20]),
                                           ("int8", "bf16", [1, 500, 1])])
def test_queries_that_are_not_finite(fmt, dtype, new, softcap):
    """A query row with an infinity or NaN has scores of which none is an ordinary number: its output is NaN, also where every key that
    it sees scores -inf; a cap makes infinite scores finite.  Other rows are left alone."""
    n_q = n_kv = 4
    p = Program(config(n_q=n_q, n_kv=n_kv, d=64, page=16, batch=3, pages=64, n_pages=192, dtype=dtype), fmt, seed=17, dtype=dtype)
    T = sum(new)
    size = torch.tensor(p.rng.uniform(1.0, 1.5, (T, n_kv, 64)), device="cuda").to(DT[dtype][1])         # (no code of it is 0)
    p.step(new, k=torch.where(torch.arange(n_kv, device="cuda")[:, None] % 2 == 0, -size, size))
    q = p.rows(T, n_q)
    first = np.concatenate([[0], np.cumsum(new)[:-1]]).tolist()
    q[first[0], :, 5], q[first[1], :2, 9], q[first[2], 1, 63], q[first[2], 2, 0] = INF, -INF, NAN, INF
    q[first[2], 2, 7] = -1e6                                               # (beyond fp16's range beside the infinity)
    out = f64(attend(p, new, q, softcap=softcap))
    for b, n in enumerate(new):
        rows = sorted({0, n // 2, n - 1})
        with np.errstate(invalid="ignore"):
            ref, s = R.attend(f64(q[first[b]:first[b] + n]), p.ref.values(p.ref.k[b]), p.ref.values(p.ref.v[b]), 0.125, softcap, only=rows)
        tol = R.tolerance(ref, s, n, EPS[dtype], dtype == "bf16", n >= 64, softcap)
        for i in rows:
            got = out[first[b] + i]
            assert np.array_equal(np.isnan(got), np.isnan(ref[i])), (b, i)
            fine = np.isfinite(f64(q[first[b] + i])).all(-1)
            assert (np.abs(got - ref[i]) <= tol[i])[fine].all(), (b, i)
    assert p.status.item() == 0
