"""The 4-bit cache at its documented limits, against the same definitions: large queries, rows in numbers that make the kernels go round
their loops, evictions in which the weights decide."""
import pytest
import torch

import q4_reference as R
import test_gpu_q4_cache as T
from paper_2508_15806_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = T.DEV


# ---- large queries ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_queries_of_one_sign_up_to_the_documented_bound(d, dtype, sign):
    # from 2^66 to just below 2^67: a group's sum is over 2^71
    lens, hkv, G = [300, 40, 5, 1000], 2, 4
    t = R.random_cache(81 + d, lens, d, hkv, device=DEV)
    u = torch.rand(2, 2, hkv * G, d, generator=torch.Generator().manual_seed(82))
    q = (sign * (1.0 + 0.99 * u) * 2.0 ** 66).to(dtype)
    assert float(q.abs().max()) < 2.0 ** 67
    q_pos = torch.tensor([[100, 400], [3, 5000]], dtype=torch.int32, device=DEV)
    for kw in (dict(), dict(q_pos=q_pos), dict(q_pos=q_pos, softcap=5.0)):
        out, lse = T.check(t, hkv, q, accumulate=True, scale=2.0 ** -66 / d, **kw)
        assert torch.isfinite(out).all()
