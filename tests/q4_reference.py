"""The 4-bit cache in plain 64-bit arithmetic, written from its definition (include/slkv.h): test infrastructure only."""
import math

import numpy as np
import torch

U_BF16 = 2.0 ** -8          # half a step of bf16 relative to the value


def bf16_towards(x: float, up: bool) -> float:
    """The bf16 next to x in one direction (x itself where it is one)."""
    if x == 0.0 or not math.isfinite(x):
        return x
    _, e = math.frexp(x)
    step = 2.0 ** max(e - 8, -133)
    return (math.ceil(x / step) if up else math.floor(x / step)) * step


def quantise_row(x):
    """x: float64 array [d] -> codes [d], scale [d/32], zero [d/32] (NaN for groups that stand for NaN)."""
    d = x.shape[0]
    codes, scale, zero = np.zeros(d, np.int64), np.zeros(d // 32), np.zeros(d // 32)
    for j in range(d // 32):
        g = x[32 * j:32 * j + 32]
        if not np.all(np.isfinite(g)):
            scale[j] = zero[j] = math.nan
            continue
        z = bf16_towards(float(g.min()), up=False) + 0.0                 # -0 is 0
        with np.errstate(over="ignore"):
            span = float(np.float32(np.float32(g.max()) - np.float32(z)))
        if not math.isfinite(span):
            scale[j] = zero[j] = math.nan
            continue
        s = bf16_towards(float(np.float32(span) / np.float32(15.0)), up=True)
        scale[j], zero[j] = s, z
        if s > 0:
            codes[32 * j:32 * j + 32] = np.rint((g.astype(np.float32) - np.float32(z)) / np.float32(s))
    return codes, scale, zero


def decode(records, d):
    """records uint8 tensor [n, bytes] -> (K, V, V's share of the codes' centre) float64 [n, d]: value by value, as the layout is described."""
    rec = records.cpu().numpy()
    n, ng = rec.shape[0], d // 32
    kw = np.ascontiguousarray(rec[:, :d // 2]).view("<u4")
    vu = np.ascontiguousarray(rec[:, d // 2:d]).view("<u2").astype(np.int64)
    s = (np.ascontiguousarray(rec[:, d:]).view("<u2").astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    K, V, A = (np.zeros((n, d)) for _ in range(3))
    for j in range(ng):
        for t in range(4):
            for e in range(8):
                K[:, 32 * j + 8 * t + e] = s[:, ng + j] + s[:, j] * ((kw[:, t * ng + j].astype(np.int64) >> (4 * e)) & 15)
        for g in range(8):
            for e in range(4):
                c = (vu[:, g * ng + j] >> (4 * e)) & 15
                V[:, 32 * j + 4 * g + e] = s[:, 3 * ng + j] + s[:, 2 * ng + j] * c
                A[:, 32 * j + 4 * g + e] = np.abs(s[:, 2 * ng + j] * (c - 8))
    return K, V, A


def attend(records, pos, weight, starts, lens, q, n_kv_heads, scale, softcap=0.0, q_pos=None, slopes=None, decay=1.0):
    """All in float64.  q [n_seqs, n_tokens, n_q_heads, d].  Returns out, lse, new weights and the bounds on a kernel's differences:
    score_err per query (fp32 sums of up to d products and their conversion), out_err parts."""
    ns, nt, hq, d = q.shape
    G = hq // n_kv_heads
    q = q.double().cpu().numpy()
    pos, starts, lens = pos.cpu().numpy(), starts.cpu().numpy(), lens.cpu().numpy()
    w = weight.double().cpu().numpy().copy() if weight is not None else None
    out, lse = np.zeros(q.shape), np.full((ns, hq, nt), -np.inf)
    spread, mass, eta = np.zeros(q.shape), np.zeros(q.shape), np.zeros((ns, hq, nt))
    w_eta = np.zeros_like(w) if w is not None else None
    for seg in range(ns * n_kv_heads):
        s, h = divmod(seg, n_kv_heads)
        b, n = int(starts[seg]), int(lens[seg])
        if n == 0:
            continue
        K, V, A = decode(records[b:b + n], d)
        seen_w, seen_e = np.zeros(n), np.zeros(n)
        for i in range(nt):
            for hh in range(G):
                qq = q[s, i, h * G + hh]
                vis = np.ones(n, bool) if q_pos is None else pos[b:b + n] <= int(q_pos[s, i])
                if not vis.any():
                    continue
                x = scale * (K[vis] @ qq)
                size = abs(scale) * (np.abs(K[vis]) @ np.abs(qq))
                if softcap:
                    x = softcap * np.tanh(x / softcap)
                capped = float(np.max(np.abs(x)))
                if slopes is not None:
                    x = x + float(slopes[h * G + hh]) * (pos[b:b + n][vis] - int(q_pos[s, i]))
                m = x.max()
                p = np.exp(x - m)
                z = p.sum()
                p = p / z
                out[s, i, h * G + hh] = p @ V[vis]
                lse[s, h * G + hh, i] = m + math.log(z)
                # a score is a chain of about 32 fp32 additions of products whose magnitudes add up to `size` (zero and code
                # parts: twice that), converted, exponentiated (2^-22) and summed
                e = 2.0 ** -19 * (1.0 + float(np.max(size))) + 2.0 ** -22 * float(np.max(np.abs(x)))
                # a capped score is cap (1 - 2 t), t = 1 / (1 + 2^y): 2^y off by 2^-22 of itself moves t by t (1 - t) 2^-22 <= 2^-24, the
                # reciprocal by 2^-23; twice both times the cap, and the sum's rounding: under 2^-21 caps.  Scores under a quarter of
                # the cap (x = cap tanh y, |y| < 0.25) come from a series of eight roundings at most, of which all but the last
                # are of terms of y^2 / 3 < 2^-5: under 2^-22 |x|; those above have a cap of under 4.1 |x|: under 2^-18 |x|
                e += min(2.0 ** -21 * softcap, 2.0 ** -18 * capped)
                eta[s, h * G + hh, i] = e
                spread[s, i, h * G + hh] = p @ A[vis]
                mass[s, i, h * G + hh] = p @ np.abs(V[vis]) + p @ A[vis]
                seen_w[vis] += p / G
                seen_e[vis] += 2 * e * p / G
        if w is not None:
            w[b:b + n] = decay * w[b:b + n] + seen_w
            w_eta[b:b + n] = seen_e + 2.0 ** -21 * np.abs(w[b:b + n]) + 1e-30
    return dict(out=out, lse=lse, weight=w, spread=spread, mass=mass, eta=eta, w_eta=w_eta)


def check_attend(got_out, got_lse, ref, bf16, lse_unit=1.0, got_weight=None):
    o, e = got_out.double().cpu().numpy(), np.swapaxes(ref["eta"], 1, 2)[..., None]
    # probabilities are off by 2 eta relative; with bf16 rows p * scale is rounded once, and the result
    tol = 2 * e * ref["mass"] + 2.0 ** -20 * ref["mass"]
    if bf16:
        tol = tol + U_BF16 * (ref["spread"] + np.abs(ref["out"])) * (1 + U_BF16) + U_BF16 * tol
    assert np.array_equal(np.isnan(o), np.isnan(ref["out"]))
    bad = np.abs(o - ref["out"]) > tol
    assert not bad.any(), (np.abs(o - ref["out"])[bad].max(), tol[bad].min(), np.argwhere(bad)[:5])
    if got_lse is not None:
        x, y = got_lse.double().cpu().numpy() * lse_unit, ref["lse"]
        assert np.array_equal(np.isneginf(x), np.isneginf(y)) and np.array_equal(np.isnan(x), np.isnan(y))
        f = np.isfinite(y)
        assert np.all(np.abs(x[f] - y[f]) <= ref["eta"][f] + 2.0 ** -20 * (1 + np.abs(y[f])))
    if got_weight is not None:
        x = got_weight.double().cpu().numpy()
        assert np.all(np.abs(x - ref["weight"]) <= ref["w_eta"])


def evict_order(weight, pos, newest, window, kept):
    """Per kept slot the row it holds: the definition, row by row."""
    n = len(pos)

    def rank(i):
        if pos[i] > newest - window:
            return (0, 0.0, i)
        return (2, 0.0, i) if math.isnan(weight[i]) else (1, -weight[i] + 0.0, i)
    keep = set(sorted(range(n), key=rank)[:kept])
    later = iter([i for i in range(kept, n) if i in keep])
    return [i if i in keep else next(later) for i in range(kept)]


def random_cache(seed, lens, d, n_kv_heads, slack=3, noise=True, device="cpu"):
    """Records of random rows built from the definition (codes and scales drawn, not quantised), positions with gaps, weights; the slots
    behind the filled ones hold NaN scales, large weights and positions: none of it may matter."""
    g = torch.Generator().manual_seed(seed)
    n_seg, ng, rb = len(lens), d // 32, d + d // 4
    starts = [0]
    for i, n in enumerate(lens):
        starts.append(starts[-1] + n + (slack + i % 2 if slack else 0))
    rows = max(starts[-1], 1)
    rec = torch.randint(0, 256, (rows, rb), generator=g, dtype=torch.uint8)
    scale = torch.exp(0.5 * torch.randn(rows, 4, ng, generator=g)) * 0.2
    scale[:, 1], scale[:, 3] = -7.5 * scale[:, 0] + 0.3 * torch.randn(rows, ng, generator=g), -7.5 * scale[:, 2]
    pos = torch.zeros(rows, dtype=torch.int32)
    weight = torch.exp(2 * torch.randn(rows, generator=g))
    filled = torch.zeros(rows, dtype=torch.bool)
    for seg, n in enumerate(lens):
        filled[starts[seg]:starts[seg] + n] = True
        pos[starts[seg]:starts[seg] + n] = torch.cumsum(torch.randint(1, 5, (n,), generator=g), 0).int()
    if noise:
        scale[~filled] = float("nan")
        pos[~filled] = -1
    rec[:, d:] = scale.bfloat16().view(torch.uint8).reshape(rows, -1)
    return dict(records=rec.to(device), pos=pos.to(device), weight=weight.to(device),
                starts=torch.tensor(starts, dtype=torch.int32, device=device), lens=torch.tensor(lens, dtype=torch.int32, device=device))
