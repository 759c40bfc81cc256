"""Attention of prompts and over paged caches in 64 bits, row by row of its definition, and the bounds that the kernels are held to."""
import math

import torch


def rows(q, k, v, visible, scale):
    """q [n, d], k, v [m, d], visible [n, m] -> out [n, d], lse [n], weight of |v| [n, d], sum of |products| of the largest score [n]."""
    q, k, v = q.double(), k.double(), v.double()
    if k.shape[0] == 0:
        z = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        return z, torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device), z, z[:, 0]
    kk = torch.where(visible.any(0)[:, None], k, torch.zeros_like(k))
    x = torch.where(visible, q @ kk.T * scale, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    p = torch.where(visible, p, torch.zeros_like(p))
    size = (q.abs() @ kk.abs().T * scale).masked_fill(~visible, 0).amax(1)
    fine = torch.isfinite(v)
    clean = torch.where(fine, v, torch.zeros_like(v))
    out, weight = p @ clean, p @ clean.abs()
    for j in torch.nonzero(~fine.all(1)).flatten().tolist():           # values that are not finite reach the rows that see them
        odd = torch.where(fine[j], torch.zeros_like(v[j]), v[j])
        out = out + torch.where(visible[:, j:j + 1], odd[None], torch.zeros_like(odd)[None])
    return out, lse, weight, size


def check(got, lse, ref, bf16, d):
    """|error| of an output, all roundings counted.  A score is a sum of d products in fp32 (d + 2 roundings of 2^-24, relative to the sum of their
    magnitudes) and its exponential is off by 2^-22; a weight is so off by e in relation, twice that with the sum it is divided by.
    bf16: probabilities are rounded to bf16 (2^-8), and the output."""
    out, want_lse, weight, size = ref
    e = ((d + 8) * 2.0 ** -24 * size + 2.0 ** -20)[:, None]
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    tol = (2 * e + (half if bf16 else 0.0)) * weight * 1.01 + half * out.abs() + 1e-30
    got, out = got.double(), out
    fine = torch.isfinite(out)
    assert torch.equal(torch.isfinite(got), fine), "values that are not finite in other places"
    assert torch.equal(torch.isnan(got), torch.isnan(out))
    assert torch.equal(got[~fine].nan_to_num(0.0, 1.0, -1.0), out[~fine].nan_to_num(0.0, 1.0, -1.0))
    worst = ((got - out).abs() / tol)[fine]
    assert worst.numel() == 0 or worst.max() <= 1.0, f"off by {float(worst.max())} of the bound"
    if lse is not None:
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(lse), empty) and (lse[empty] < 0).all()
        bad = ((lse.double() - want_lse).abs() / (e[:, 0] + 2.0 ** -23 * want_lse.abs()))[~empty]
        assert bad.numel() == 0 or bad.max() <= 1.0, f"log-sum-exp off by {float(bad.max())} of the bound"


def causal(nq, nk, device):
    return torch.arange(nk, device=device)[None] <= torch.arange(nq, device=device)[:, None] + nk - nq


def check_prompt(q, k, v, cu_q, cu_k, out, lse, window, scale, before, lse_before, log2=False):
    """out, lse against the definition; rows that are not to be written as `before`."""
    d, G = q.shape[2], q.shape[1] // k.shape[1]
    for s in range(len(cu_q) - 1):
        a, b, c, e = cu_q[s], cu_q[s + 1], cu_k[s], cu_k[s + 1]
        nq, nk = b - a, e - c
        seen = causal(nq, nk, q.device)
        for h in range(q.shape[1]):
            ref = rows(q[a:b, h], k[c:e, h // G], v[c:e, h // G], seen, scale)
            check(out[a:b, h], None, ref, q.dtype == torch.bfloat16, d)
            if lse is not None:
                n = min(nq, window)
                got = lse[s, h, window - n:] * (math.log(2.0) if log2 else 1.0)
                if n:
                    check(out[b - n:b, h], got, tuple(x[nq - n:] for x in ref), q.dtype == torch.bfloat16, d)
                assert torch.equal(lse[s, h, :window - n], lse_before[s, h, :window - n]), "rows before the first query are written"
    assert torch.equal(out[cu_q[-1]:], before[cu_q[-1]:]), "rows behind the last sequence are written"
