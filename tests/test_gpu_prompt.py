"""slkv_prompt_attend against its definition in 64 bits."""
import pytest
import torch

import attend_reference as R
from paper_2508_15806_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(nq, nk, hkv, G, d, dtype, seed=0, behind=3, heads_first=False):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rows(n, heads):
        x = torch.randn(n, heads, d, device="cuda", generator=g)
        if heads_first:
            return x.to(DT[dtype]).transpose(0, 1).contiguous().transpose(0, 1)
        return x.to(DT[dtype])
    q, k, v = rows(sum(nq) + behind, hkv * G), rows(sum(nk) + behind, hkv), rows(sum(nk) + behind, hkv)
    return q, k, v


def cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def attend(q, k, v, nq, nk=None, window=32, scale=None, log2=False, out=None, stream=None):
    cu_q, cu_k = cu(nq), None if nk is None else cu(nk)
    dev = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    if out is None:
        out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    before = out.clone()
    lse = torch.full((len(nq), q.shape[1], window), 5.0, device="cuda")
    p = B.make_prompt(q, k, v, out, len(nq), window=window, scale=scale, lse_units=B.SLKV_LSE_LOG2 if log2 else B.SLKV_LSE_LN)
    ws = B.new_prompt_workspace(p, cu_q, cu_k)
    ws.fill_(0xff)                                                # nobody clears a workspace
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.slkv_prompt_attend(p, q, k, v, dev(cu_q), cu_q, out, ws, cu_k=dev(cu_k), cu_k_host=cu_k, lse=lse, status=status, stream=stream)
    torch.cuda.synchronize()
    assert int(status) == 0
    return out, lse, before


def run(nq, nk=None, hkv=2, G=4, d=128, dtype="bf16", window=32, scale=None, log2=False, seed=0, **kw):
    q, k, v = inputs(nq, nq if nk is None else nk, hkv, G, d, dtype, seed, **kw)
    out, lse, before = attend(q, k, v, nq, nk, window, scale, log2)
    R.check_prompt(q, k, v, cu(nq), cu(nq if nk is None else nk), out, lse, window, d ** -0.5 if scale is None else scale, before,
                   torch.full_like(lse, 5.0), log2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq", [[1], [5], [32], [33], [64], [65], [129], [300], [1, 0, 64, 129, 0, 31]])
def test_lengths(nq, d, dtype):
    run(nq, d=d, dtype=dtype)
