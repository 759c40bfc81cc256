"""The 4-bit cache on the GPU against its definition in 64 bits: packing, appending, unpacking, attention, eviction, and a run of them."""
import math

import numpy as np
import pytest
import torch

import q4_reference as R
from paper_2508_15806_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0") if torch.cuda.is_available() else torch.device("cpu")


def cache_of(c, n_kv_heads, **kw):
    c = {**c, **kw}
    return B.make_q4_cache(c["records"], c["pos"], c["weight"], c["starts"], c["lens"], n_kv_heads)


def empty_cache(rooms, d, n_kv_heads, fill=0xAB):
    starts = [0]
    for r in rooms:
        starts.append(starts[-1] + r)
    n = max(starts[-1], 1)
    t = dict(records=torch.full((n, d + d // 4), fill, dtype=torch.uint8, device=DEV), pos=torch.full((n,), -7, dtype=torch.int32, device=DEV),
             weight=torch.full((n,), 5.0, device=DEV), starts=torch.tensor(starts, dtype=torch.int32, device=DEV),
             lens=torch.full((len(rooms),), 12345, dtype=torch.int32, device=DEV))
    return t, cache_of(t, n_kv_heads)


def expected_record(k, v):
    """Bytes of the records of rows k, v (float64 arrays [n, d])."""
    n, d = k.shape
    ng = d // 32
    out = np.zeros((n, d + d // 4), np.uint8)
    for r in range(n):
        parts = []
        for x, lanes, per in ((k[r], 4, 8), (v[r], 8, 4)):
            code, scale, zero = R.quantise_row(x)
            c = code.reshape(ng, lanes, per).transpose(1, 0, 2).reshape(-1)
            parts.append(((c[0::2] | (c[1::2] << 4)).astype(np.uint8), scale, zero))
        s = np.concatenate([parts[0][1], parts[0][2], parts[1][1], parts[1][2]]).astype(np.float32)
        bits = (s.view(np.uint32) >> 16).astype(np.uint16)
        bits[np.isnan(s)] = 0x7FFF
        out[r] = np.concatenate([parts[0][0], parts[1][0], bits.view(np.uint8)])
    return out


def rows(seed, n, d, dtype):
    g = torch.Generator().manual_seed(seed)
    k, v = torch.randn(n, d, generator=g) * 1.5 + torch.randn(d, generator=g), torch.randn(n, d, generator=g)
    return k.to(dtype), v.to(dtype)


# ---- rows in and out -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,hkv,slack", [([1], 1, 0), ([0, 5, 0, 33, 1, 0], 2, 3), ([7, 130, 64], 3, 0), ([0, 0], 1, 2)])
def test_pack_writes_the_defined_records(d, dtype, lens, hkv, slack):
    n = sum(lens)
    k, v = rows(n + d, max(n, 1), d, dtype)
    offsets = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=DEV)
    kept = torch.arange(max(n, 1), dtype=torch.int32, device=DEV) * 3 + 1
    t, c = empty_cache([x + slack for x in lens], d, hkv)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.slkv_q4_pack(c, k.to(DEV), v.to(DEV), offsets, kept, status)
    assert status.item() == 0 and t["lens"].tolist() == lens
    want = expected_record(k.double().numpy(), v.double().numpy())
    slots = [int(t["starts"][s]) + i for s, m in enumerate(lens) for i in range(m)]
    got = t["records"].cpu().numpy()
    assert np.array_equal(got[slots], want[:n])
    assert np.array_equal(t["pos"].cpu().numpy()[slots], kept.cpu().numpy()[:n]) and np.all(t["weight"].cpu().numpy()[slots] == 0)
    rest = np.setdiff1d(np.arange(got.shape[0]), slots)              # slots behind the rows stay as they were
    assert np.all(got[rest] == 0xAB) and np.all(t["pos"].cpu().numpy()[rest] == -7) and np.all(t["weight"].cpu().numpy()[rest] == 5.0)

    # and back: every filled slot, then some slots with padding between them
    K, V, _ = R.decode(t["records"][slots], d)
    for out_dtype in (torch.float32, torch.bfloat16):
        ko, vo = (torch.full((got.shape[0], d), 77.0, dtype=out_dtype, device=DEV) for _ in range(2))
        B.slkv_q4_unpack(c, ko, vo)
        for o, x in ((ko, K), (vo, V)):
            assert torch.equal(o.cpu()[slots], torch.from_numpy(x).float().to(out_dtype)) and torch.all(o.cpu()[rest] == 77.0)
    pick = torch.tensor(slots[::-1][:5] + [-1, got.shape[0], 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    ko, vo = (torch.full((pick.numel(), d), 77.0, device=DEV) for _ in range(2))
    B.slkv_q4_unpack(c, ko, vo, slots=pick)
    m = pick.numel() - 3
    assert torch.equal(ko.cpu()[:m], torch.from_numpy(K[::-1][:m].copy()).float()) and torch.all(ko[m:] == 77.0)
    assert torch.equal(vo.cpu()[:m], torch.from_numpy(V[::-1][:m].copy()).float()) and torch.all(vo[m:] == 77.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_groups_that_are_not_ordinary(dtype):
    big, inf, nan = 3.0e38, float("inf"), float("nan")
    k, v = rows(3, 16, 128, torch.float32)
    k[0, :32] = 0.75                                   # one value
    k[1, 32:64] = 0.0
    k[1, 40] = -0.0
    k[2, 5], k[3, 70], k[4, 127] = nan, inf, -inf
    k[5, 3], k[5, 9] = -big, big                       # a range over fp32's
    k[6, 64:96] = big                                  # large, but one value
    k[7, :32] = torch.arange(32) * 1e-40               # subnormal
    k[8, :32] = torch.arange(32) * 2.0 ** -125
    k[9, :32] = 1000.0 + torch.arange(32) / 64         # small steps far from zero
    k[10, :32] = torch.arange(32) % 16                 # exact codes, and ties between them
    k[11, :32] = (torch.arange(32) % 31) / 2
    k[12, :32] = -torch.arange(32) * 3.7e36
    k[13, 0], k[13, 1] = 2.0 ** -130, -2.0 ** -133
    k, v = k.to(dtype), v.to(dtype)
    t, c = empty_cache([16], 128, 1)
    B.slkv_q4_pack(c, k.to(DEV), v.to(DEV), torch.tensor([0, 16], dtype=torch.int32, device=DEV), torch.zeros(16, dtype=torch.int32, device=DEV))
    want = expected_record(k.double().numpy(), v.double().numpy())
    assert [r for r in range(16) if not np.array_equal(t["records"][r].cpu().numpy(), want[r])] == []
    ko, vo = (torch.zeros(16, 128, device=DEV) for _ in range(2))
    B.slkv_q4_unpack(c, ko, vo)
    x, y = k.double().numpy().reshape(16, 4, 32), ko.double().cpu().numpy().reshape(16, 4, 32)
    poisoned = {(2, 0), (3, 2), (4, 3), (5, 0)}
    for r in range(16):
        for j in range(4):
            if (r, j) in poisoned:
                assert np.all(np.isnan(y[r, j]))
            else:                                      # half a step, the fp32 roundings of x - zero and of the value
                step = R.quantise_row(x[r].reshape(-1))[1][j]
                assert np.all(np.abs(x[r, j] - y[r, j]) <= step / 2 + 2.0 ** -22 * np.abs(x[r, j]).max() + 2.0 ** -148), (r, j)


def test_pack_stops_at_the_segments_ends_and_says_so():
    k, v = rows(5, 30, 128, torch.bfloat16)
    t, c = empty_cache([4, 12, 9], 128, 1)
    off = torch.tensor([0, 10, 22, 30], dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.slkv_q4_pack(c, k.to(DEV), v.to(DEV), off, torch.arange(30, dtype=torch.int32, device=DEV), status)
    assert status.item() == B.ERR["CAPACITY"] and t["lens"].tolist() == [4, 12, 8]
    want = expected_record(k.double().numpy(), v.double().numpy())
    assert np.array_equal(t["records"].cpu().numpy()[:24], want[[0, 1, 2, 3] + list(range(10, 30))]) and torch.all(t["records"][24] == 0xAB)
    # offsets past the rows that are there
    status.zero_()
    t, c = empty_cache([10, 12, 9], 128, 1)
    B.slkv_q4_pack(c, k[:25].contiguous().to(DEV), v[:25].contiguous().to(DEV), off, torch.arange(25, dtype=torch.int32, device=DEV), status)
    assert status.item() == B.ERR["CAPACITY"] and t["lens"].tolist() == [10, 12, 3] and torch.all(t["records"][25:] == 0xAB)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_tokens", [1, 2, 21])
def test_append_behind_the_filled_slots(d, dtype, n_tokens):
    ns, hkv = 3, 2
    lens = [0, 4, 50, 1, 7, 30]
    t, c = empty_cache([x + n_tokens + i % 2 for i, x in enumerate(lens)], d, hkv)
    t["lens"].copy_(torch.tensor(lens))
    k, v = rows(d + n_tokens, ns * n_tokens * hkv, d, dtype)
    # K from a wider tensor, V with its heads outside the tokens
    kt = torch.zeros(ns, n_tokens, hkv + 1, d + 32, dtype=dtype, device=DEV)[:, :, :hkv, :d]
    kt.copy_(k.view(ns, n_tokens, hkv, d))
    vt = torch.zeros(ns, hkv, n_tokens, d, dtype=dtype, device=DEV).transpose(1, 2)
    vt.copy_(v.view(ns, n_tokens, hkv, d))
    pos = torch.arange(ns * n_tokens, dtype=torch.int32, device=DEV).view(ns, n_tokens) + 1000
    after_lens = torch.zeros(6, dtype=torch.int32, device=DEV)
    before = t["records"].clone()
    B.slkv_q4_append(c, kt, vt, pos, after=cache_of(t, hkv, lens=after_lens))
    assert t["lens"].tolist() == lens and after_lens.tolist() == [x + n_tokens for x in lens]
    want = expected_record(k.double().numpy(), v.double().numpy()).reshape(ns, n_tokens, hkv, -1)
    for seg, n in enumerate(lens):
        s, h = divmod(seg, hkv)
        b = int(t["starts"][seg]) + n
        assert np.array_equal(t["records"][b:b + n_tokens].cpu().numpy(), want[s, :, h])
        assert t["pos"][b:b + n_tokens].tolist() == pos[s].tolist() and torch.all(t["weight"][b:b + n_tokens] == 0)
        before[b:b + n_tokens] = t["records"][b:b + n_tokens]
    assert torch.equal(before, t["records"])
    # the lengths themselves move on; a second time not everything fits
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.slkv_q4_append(c, kt, vt, pos, status=status)
    assert t["lens"].tolist() == after_lens.tolist() and status.item() == 0 and torch.equal(before, t["records"])
    B.slkv_q4_append(c, kt, vt, pos, status=status)
    assert status.item() == B.ERR["CAPACITY"] and t["lens"].tolist() == [x + n_tokens + i % 2 for i, x in enumerate(lens)]


# ---- attention -------------------------------------------------------------------------------------------------------
def attend(t, hkv, q, accumulate=False, q_pos=None, slopes=None, units=B.SLKV_LSE_LN, out=None, **kw):
    q = q.to(DEV) if not q.is_cuda else q
    c = cache_of(t, hkv)
    out = torch.full_like(q, 9.0) if out is None else out
    lse = torch.full((q.size(0), q.size(2), q.size(1)), 9.0, device=DEV)
    p = B.make_q4_attend(c, q, out, lse_units=units, **kw)
    ws = B.new_q4_workspace(c, p, accumulate)
    ws.fill_(0xFF)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.slkv_q4_attend(c, p, q, out, ws, q_pos=q_pos, slopes=slopes, lse=lse, accumulate=accumulate, status=status)
    assert status.item() == 0
    return out, lse


def check(t, hkv, q, accumulate=False, q_pos=None, slopes=None, units=B.SLKV_LSE_LN, **kw):
    ref = R.attend(t["records"], t["pos"], t["weight"], t["starts"], t["lens"], q, hkv, kw.get("scale", q.size(3) ** -0.5),
                   kw.get("softcap", 0.0), None if q_pos is None else q_pos.cpu().numpy(), None if slopes is None else slopes.cpu().numpy(),
                   kw.get("weight_decay", 1.0))
    out, lse = attend(t, hkv, q, accumulate, q_pos, slopes, units, **kw)
    R.check_attend(out, lse, ref, q.dtype == torch.bfloat16, math.log(2.0) if units == B.SLKV_LSE_LOG2 else 1.0, t["weight"] if accumulate else None)
    return out, lse


def queries(seed, ns, nt, hq, d, dtype, size=1.0):
    return (size * torch.randn(ns, nt, hq, d, generator=torch.Generator().manual_seed(seed))).to(dtype)


LENS = [[1], [0, 31, 32, 33], [0, 0, 128, 129], [300, 5, 64, 1000, 2, 17]]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,hkv", [(LENS[0], 1), (LENS[1], 2), (LENS[2], 4), (LENS[3], 2)])
@pytest.mark.parametrize("G,nt", [(1, 1), (4, 1), (8, 1), (3, 3), (5, 7)])
def test_attention_over_any_lengths_and_columns(d, dtype, lens, hkv, G, nt):
    t = R.random_cache(sum(lens) + d, lens, d, hkv, device=DEV)
    check(t, hkv, queries(d + G, len(lens) // hkv, nt, hkv * G, d, dtype), accumulate=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kw", [dict(softcap=5.0), dict(softcap=30.0, weight_decay=0.9, scale=0.3), dict(slopes=True), dict(slopes=True, softcap=20.0),
                                dict(units=B.SLKV_LSE_LOG2, weight_decay=0.0), dict(scale=-0.05), dict(softcap=1e6), dict(softcap=3e38), dict(softcap=0.25),
                                dict(slopes=True, softcap=1000.0)])
def test_caps_biases_and_masks_by_position(d, dtype, kw):
    kw = dict(kw)
    hkv, G, nt = 2, 4, 3
    lens = [70, 257, 0, 3, 1000, 33]
    t = R.random_cache(11 + d, lens, d, hkv, device=DEV)
    # tokens between the rows, before all of them (nothing to see), behind all of them
    q_pos = torch.tensor([[0, 90, 500], [4, 5, 1], [10 ** 6, 1200, 17]], dtype=torch.int32, device=DEV)
    slopes = torch.exp2(-torch.arange(hkv * G, device=DEV, dtype=torch.float32)) if kw.pop("slopes", False) else None
    out, lse = check(t, hkv, queries(d, 3, nt, hkv * G, d, dtype), accumulate=True, q_pos=q_pos, slopes=slopes, **kw)
    assert torch.all(out[0, 0] == 0) and torch.all(torch.isneginf(lse[0, :, 0]))
    assert torch.all(out[1, :, :G] == 0)                    # an empty segment


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,hkv,short", [([700, 1, 0, 1300], 2, True), ([2000, 1500, 3000, 0], 4, False), ([5, 6000], 1, False),
                                            ([511, 520, 530, 0, 1023, 1], 3, True), ([900, 1200, 40, 1700], 2, True)])
@pytest.mark.parametrize("G,nt", [(4, 1), (1, 1), (8, 1), (2, 3), (3, 4)])
def test_few_short_units_and_their_clusters(d, dtype, lens, hkv, short, G, nt):
    t = R.random_cache(sum(lens) + d + G, lens, d, hkv, device=DEV)
    q = queries(d + G, len(lens) // hkv, nt, hkv * G, d, dtype)
    check(t, hkv, q, accumulate=True)
    assert B.slkv_last_launch_count() == (1 if short and G * nt <= 8 else 2)      # several blocks of columns: weights need a second one
    q_pos = (torch.arange(len(lens) // hkv * nt, device=DEV, dtype=torch.int32).view(-1, nt) * 397 + 100).contiguous()
    slopes = torch.exp2(-torch.arange(hkv * G, device=DEV, dtype=torch.float32))
    check(t, hkv, q, accumulate=True, q_pos=q_pos, slopes=slopes, softcap=10.0)
    check(t, hkv, q, q_pos=q_pos)
    assert B.slkv_last_launch_count() == (1 if short else 2)


@pytest.mark.parametrize("d,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_long_segments_in_many_pieces(d, dtype):
    lens = [40001, 12, 0, 33000]
    t = R.random_cache(5, lens, d, 4, device=DEV)
    check(t, 4, queries(1, 1, 2, 24, d, dtype, 2.0), accumulate=True, q_pos=torch.tensor([[60000, 200000]], dtype=torch.int32, device=DEV))


def test_many_short_segments():
    lens = [(i * 37) % 90 for i in range(3000)]
    t = R.random_cache(6, lens, 64, 6, slack=0, device=DEV)
    check(t, 6, queries(2, 500, 1, 6, 64, torch.bfloat16), accumulate=True)


def test_as_many_columns_as_are_taken():
    t = R.random_cache(61, [40, 300], 64, 1, device=DEV)
    q_pos = torch.arange(32, dtype=torch.int32, device=DEV).view(2, 16) * 40
    check(t, 1, queries(62, 2, 16, 16, 64, torch.bfloat16), accumulate=True, q_pos=q_pos)


@pytest.mark.parametrize("d", [64, 128])
def test_as_many_segments_as_are_taken(d):
    # one row each: the output is that row's values
    n, hkv = 16384, 8
    t = R.random_cache(63, [1] * n, d, hkv, slack=1, device=DEV)
    q = queries(64, n // hkv, 1, hkv, d, torch.float32).to(DEV)
    t["weight"].zero_()
    out, lse = attend(t, hkv, q, accumulate=True)
    K, V, _ = R.decode(t["records"][t["starts"][:-1].long()], d)
    x = (K * q.view(n, d).double().cpu().numpy()).sum(1) * d ** -0.5
    size = (np.abs(K) * np.abs(q.view(n, d).double().cpu().numpy())).sum(1) * d ** -0.5
    assert np.all(np.abs(lse.view(n).double().cpu().numpy() - x) <= 2.0 ** -19 * (1 + size))
    # one probability of 1: three parts of bf16, a sum of two fp32 products
    assert np.all(np.abs(out.view(n, d).double().cpu().numpy() - V) <= 2.0 ** -20 * (np.abs(V) + 16 * np.abs(V).max(1, keepdims=True)))
    assert torch.all((t["weight"][t["starts"][:-1].long()] - 1).abs() <= 2.0 ** -21)


def test_a_cache_beyond_32_bits():
    d, rows_ = 128, 14_000_100                            # 2.24e9 bytes of records; 160 columns: 2.24e9 scores
    small = R.random_cache(65, [100, 33], d, 1, slack=0, device=DEV)
    big = dict(records=torch.zeros(rows_, 160, dtype=torch.uint8, device=DEV), pos=torch.zeros(rows_, dtype=torch.int32, device=DEV),
               weight=torch.zeros(rows_, device=DEV), starts=torch.tensor([0, 100, rows_], dtype=torch.int32, device=DEV),
               lens=torch.tensor([100, 0], dtype=torch.int32, device=DEV))
    far = dict(big, starts=torch.tensor([0, rows_ - 100, rows_], dtype=torch.int32, device=DEV), lens=torch.tensor([0, 100], dtype=torch.int32, device=DEV))
    here = dict(small, starts=small["starts"].clone(), lens=torch.tensor([100, 0], dtype=torch.int32, device=DEV))
    for x in ("records", "pos", "weight"):
        far[x][-100:] = small[x][:100]
    q = queries(66, 2, 10, 16, d, torch.bfloat16)
    want, lse = attend(here, 1, q, accumulate=True)
    got, lse2 = attend(far, 1, torch.flip(q, [0]), accumulate=True)
    assert torch.equal(got[1], want[0]) and torch.equal(lse2[1], lse[0]) and torch.equal(far["weight"][-100:], small["weight"][:100])
    c = cache_of(far, 1)
    k, v = rows(67, 2, d, torch.bfloat16)
    far["lens"][1] = 99
    B.slkv_q4_append(c, k.view(2, 1, 1, d).to(DEV), v.view(2, 1, 1, d).to(DEV), torch.full((2, 1), 7, dtype=torch.int32, device=DEV))
    want_rec = expected_record(k.double().numpy(), v.double().numpy())
    assert np.array_equal(far["records"][-1].cpu().numpy(), want_rec[1]) and far["lens"].tolist() == [1, 100]
    ko, vo = (torch.zeros(1, d, device=DEV) for _ in range(2))
    B.slkv_q4_unpack(c, ko, vo, slots=torch.tensor([rows_ - 1], dtype=torch.int32, device=DEV))
    assert torch.equal(ko.cpu(), torch.from_numpy(R.decode(far["records"][-1:], d)[0]).float())
    before = {x: far[x][-100:].cpu().clone() for x in ("records", "pos", "weight")}
    before["starts"] = torch.tensor([0, 100])
    assert run_evict(far, 1, [60], 1, [-1, -1]) == 0
    src = R.evict_order(before["weight"].tolist(), before["pos"].tolist(), -1, 1, 60)
    assert torch.equal(far["records"][-100:-40].cpu(), before["records"][src])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scores_far_apart_and_large_queries(dtype):
    t = R.random_cache(8, [500, 90], 128, 1, device=DEV)
    check(t, 1, queries(3, 2, 1, 4, 128, dtype, 40.0))
    check(t, 1, queries(4, 2, 1, 4, 128, dtype, 1e-3))
    check(t, 1, queries(4, 2, 1, 4, 128, dtype, 0.0))


def test_rows_that_are_not_seen_give_nothing_whatever_they_hold():
    lens, d, hkv = [100, 37], 128, 1
    t = R.random_cache(9, lens, d, hkv, device=DEV)
    q = queries(5, 2, 2, 4, d, torch.bfloat16)
    hidden = [40, 41, int(t["starts"][1]) + 36]
    t["pos"][hidden] = 5000
    q_pos = torch.tensor([[1000, 2000], [1000, 4000]], dtype=torch.int32, device=DEV)
    want = attend(t, hkv, q, q_pos=q_pos)
    for bad in (float("nan"), float("inf"), -float("inf"), 3e38):
        s = t["records"][hidden][:, d:].contiguous().view(torch.bfloat16)
        t["records"][hidden, d:] = torch.full_like(s, bad).view(torch.uint8)
        got = attend(t, hkv, q, q_pos=q_pos)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # a row that is seen by the second token alone is that token's
    q_pos[0, 1] = 6000
    t["records"][hidden, d:] = torch.full_like(s, float("nan")).view(torch.uint8)
    got = attend(t, hkv, q, q_pos=q_pos)
    assert torch.all(torch.isnan(got[0][0, 1])) and torch.equal(got[0][0, 0], want[0][0, 0]) and torch.equal(got[0][1], want[0][1])


def test_a_poisoned_value_group_and_a_poisoned_key():
    d = 128
    t = R.random_cache(10, [50], d, 1, device=DEV)
    q = queries(6, 1, 1, 4, d, torch.float32)
    want, lse0 = attend(t, 1, q)
    s = t["records"][:, d:].view(torch.bfloat16).view(-1, 4, 4)
    keep = s.clone()
    s[7, 2:, 1] = float("nan")                             # V, channels 32 .. 63
    got, lse = attend(t, 1, q)
    assert torch.all(torch.isnan(got[..., 32:64])) and torch.equal(lse, lse0)
    rest = torch.cat([got[..., :32], got[..., 64:]], -1)
    assert torch.equal(rest, torch.cat([want[..., :32], want[..., 64:]], -1))
    s.copy_(keep)
    s[7, :2, 1] = float("nan")                             # K
    got, lse = attend(t, 1, q)
    assert torch.all(torch.isnan(got)) and torch.all(torch.isnan(lse))
    s.copy_(keep)
    s[:50, 1, 0] = float("nan")                            # every key
    got, lse = attend(t, 1, q)
    assert torch.all(torch.isnan(got)) and torch.all(torch.isnan(lse))


def test_strided_queries_and_outputs():
    lens, d, hkv, G = [60, 400, 9, 77], 64, 2, 3
    t = R.random_cache(12, lens, d, hkv, device=DEV)
    q = queries(7, 2, 2, hkv * G, d, torch.bfloat16)
    want, _ = attend(t, hkv, q)
    wide = torch.zeros(2, hkv * G + 2, 2, d + 8, dtype=q.dtype, device=DEV)
    qs = wide.transpose(1, 2)[:, :, 1:1 + hkv * G, :d]
    qs.copy_(q)
    o = torch.full((2, hkv * G, 2, 2 * d), 3.0, dtype=q.dtype, device=DEV)
    os_ = o.transpose(1, 2)[..., :d]
    got, _ = attend(t, hkv, qs, out=os_)
    assert torch.equal(got, want) and torch.all(o[..., d:] == 3.0)


def test_lengths_and_starts_that_do_not_fit_are_cut():
    t = R.random_cache(13, [40, 50, 60], 128, 1, slack=2, device=DEV)
    t["records"][:, 128:] = t["records"][0, 128:]            # every slot holds something
    q = queries(8, 3, 1, 4, 128, torch.bfloat16)
    rows_ = t["records"].size(0)
    bad = dict(t, lens=torch.tensor([10 ** 6, -5, 10 ** 9], dtype=torch.int32, device=DEV))
    room = (t["starts"][1:] - t["starts"][:-1]).tolist()
    fit = dict(t, lens=torch.tensor([room[0], 0, room[2]], dtype=torch.int32, device=DEV))
    assert torch.equal(attend(bad, 1, q)[0], attend(fit, 1, q)[0])
    bad = dict(t, starts=torch.tensor([0, 40, rows_ - 5, rows_ + 10 ** 6], dtype=torch.int32, device=DEV),
               lens=torch.tensor([40, 20, 60], dtype=torch.int32, device=DEV))
    fit = dict(bad, starts=torch.tensor([0, 40, rows_ - 5, rows_], dtype=torch.int32, device=DEV), lens=torch.tensor([40, 20, 5], dtype=torch.int32, device=DEV))
    assert torch.equal(attend(bad, 1, q)[0], attend(fit, 1, q)[0])


# ---- eviction --------------------------------------------------------------------------------------------------------
def run_evict(t, hkv, budgets, window, newest, to=None, to_lens=None):
    c = cache_of(t, hkv)
    dst = c if to is None and to_lens is None else cache_of(t, hkv, lens=to_lens) if to is None else cache_of(to, hkv)
    ws = B.new_q4_evict_workspace(c, dst)
    ws.fill_(0xFF)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.slkv_q4_evict(c, dst, torch.tensor(budgets, dtype=torch.int32, device=DEV), window, torch.tensor(newest, dtype=torch.int32, device=DEV), ws, status)
    return status.item()


def expect_evicted(before, lens, hkv, budgets, window, newest, starts_to, room_to, after):
    """`after` (tensors on the CPU) holds what the definition says, and is elsewhere as it was."""
    for seg, n in enumerate(lens):
        b, dst = int(before["starts"][seg]), starts_to[seg]
        kept = min(n, max(budgets[seg % hkv], window))
        src = R.evict_order(before["weight"][b:b + n].tolist(), before["pos"][b:b + n].tolist(), newest[seg // hkv], window, kept)[:room_to[seg]]
        idx = [b + i for i in src]
        for name in ("records", "pos", "weight"):
            got, want = after[name][dst:dst + len(src)], before[name][idx]
            if name == "weight":
                got, want = got.view(torch.int32), want.view(torch.int32)
            assert torch.equal(got, want), (seg, name)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,hkv,budgets,window", [
    ([1], 1, [1], 1), ([0, 5, 3, 9], 2, [2, 4], 1), ([40, 41, 200, 100, 33, 1], 3, [33, 40, 100], 32), ([1000, 2500, 2049, 10], 2, [999, 1], 16),
    ([90, 80], 1, [-3], 64), ([300, 400], 2, [10 ** 6, 400], 8), ([70000, 17000, 50000, 49153], 2, [30000, 100], 64)])
@pytest.mark.parametrize("in_place", [True, False])
def test_eviction_keeps_what_the_definition_says(d, lens, hkv, budgets, window, in_place):
    t = R.random_cache(sum(lens), lens, d, hkv, device=DEV)
    g = torch.Generator().manual_seed(1)
    t["weight"].copy_(torch.where(torch.rand(t["weight"].shape, generator=g) < 0.3, torch.tensor(0.0), t["weight"].cpu()))       # many ties
    special = [float("nan"), float("inf"), -float("inf"), -0.0, 0.0, -1.5, 1e-42, float("nan")]
    for i, x in enumerate(special):
        if t["weight"].numel() > 3 * i:
            t["weight"][3 * i] = x
    newest = [int(t["pos"].max())] * (len(lens) // hkv)
    if len(newest) > 1:
        newest[1] = 20                                   # its rows count as new, most of them
    before = {k: v.cpu().clone() for k, v in t.items()}
    kept = [min(n, max(budgets[s % hkv], window)) for s, n in enumerate(lens)]
    if in_place:
        other = torch.full_like(t["lens"], -1)
        assert run_evict(t, hkv, budgets, window, newest, to_lens=other) == 0
        assert other.tolist() == kept and t["lens"].tolist() == lens
        t2 = {k: v.clone().to(DEV) for k, v in before.items()}
        assert run_evict(t2, hkv, budgets, window, newest) == 0          # the lengths in place too
        assert t2["lens"].tolist() == kept and torch.equal(t2["records"], t["records"])
        after = {k: v.cpu() for k, v in t.items()}
        expect_evicted(before, lens, hkv, budgets, window, newest, before["starts"].tolist(), kept, after)
        for seg in range(len(lens)):                     # behind the kept rows nothing changes
            b, e = int(before["starts"][seg]) + kept[seg], int(before["starts"][seg + 1])
            assert torch.equal(after["records"][b:e], before["records"][b:e]) and torch.equal(after["pos"][b:e], before["pos"][b:e])
    else:
        to, _ = empty_cache([x + 2 for x in kept], d, hkv)
        assert run_evict(t, hkv, budgets, window, newest, to=to) == 0
        assert to["lens"].tolist() == kept and t["lens"].tolist() == lens and torch.equal(t["records"].cpu(), before["records"])
        after = {k: v.cpu() for k, v in to.items()}
        expect_evicted(before, lens, hkv, budgets, window, newest, after["starts"].tolist(), kept, after)
        for seg in range(len(lens)):
            b, e = int(after["starts"][seg]) + kept[seg], int(after["starts"][seg + 1])
            assert torch.all(after["records"][b:e] == 0xAB) and torch.all(after["pos"][b:e] == -7)


@pytest.mark.parametrize("kind", ["equal", "zero", "narrow", "huge", "tiny", "negative", "inf", "nan", "two values"])
@pytest.mark.parametrize("lens,hkv", [([900, 3000], 1), ([20000, 9000, 30001], 3)])
def test_eviction_by_weights_of_any_size(kind, lens, hkv):
    t = R.random_cache(71, lens, 64, hkv, device=DEV)
    n = t["weight"].numel()
    g = torch.Generator().manual_seed(72)
    u = torch.rand(n, generator=g)
    w = {"equal": torch.full((n,), 1.25), "zero": torch.zeros(n), "narrow": 1 + u * 1e-4, "huge": u * 1e38, "tiny": u * 1e-38, "negative": -u * 1e3,
         "inf": torch.where(u < 0.6, float("inf"), u), "nan": torch.where(u < 0.6, float("nan"), u),
         "two values": torch.where(u < 0.4, 0.5, 0.25)}[kind]
    t["weight"].copy_(w)
    before = {k: v.cpu().clone() for k, v in t.items()}
    budgets, newest = [len_ // 2 for len_ in lens[:hkv]], [-10 ** 6] * (len(lens) // hkv)          # no row is among the newest
    assert run_evict(t, hkv, budgets, 1, newest) == 0
    kept = [min(n_, budgets[s % hkv]) for s, n_ in enumerate(lens)]
    assert t["lens"].tolist() == kept
    expect_evicted(before, lens, hkv, budgets, 1, newest, before["starts"].tolist(), kept, {k: v.cpu() for k, v in t.items()})


@pytest.mark.parametrize("lens", [[60000] + [10] * 23, [200001, 5, 0, 77]])
@pytest.mark.parametrize("in_place", [True, False])
def test_eviction_where_one_segment_is_far_longer_than_the_others(lens, in_place):
    t = R.random_cache(73, lens, 64, 1, device=DEV)
    before = {k: v.cpu().clone() for k, v in t.items()}
    budgets, newest = [31000], [10 ** 6] * len(lens)
    kept = [min(n, 31000) for n in lens]
    to = None if in_place else empty_cache([x + 1 for x in kept], 64, 1)[0]
    assert run_evict(t, 1, budgets, 16, newest, to=to) == 0
    after = {k: v.cpu() for k, v in (to or t).items()}
    expect_evicted(before, lens, 1, budgets, 16, newest, after["starts"].tolist(), kept, after)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,launches", [([9000, 4000, 12001], 2), ([33000], 2), ([5000, 30, 9001, 8192] * 6, 1)])
def test_eviction_of_long_segments_into_another_cache(d, lens, launches):
    t = R.random_cache(74, lens, d, 1, device=DEV)
    before = {k: v.cpu().clone() for k, v in t.items()}
    newest = [10 ** 6] * len(lens)
    kept = [min(n, 4444) for n in lens]                     # some stay whole
    rooms = [k + (7 * s) % 100 if s % 3 else k - 5 for s, k in enumerate(kept)]          # some too small, some with slack
    to, _ = empty_cache(rooms, d, 1)
    assert run_evict(t, 1, [4444], 16, newest, to=to) == B.ERR["CAPACITY"]
    assert B.slkv_last_launch_count() == launches
    n = [min(k, r) for k, r in zip(kept, rooms)]
    assert to["lens"].tolist() == n and torch.equal(t["records"].cpu(), before["records"])
    after = {k: v.cpu() for k, v in to.items()}
    expect_evicted(before, lens, 1, [4444], 16, newest, after["starts"].tolist(), rooms, after)
    for seg in range(len(lens)):
        b, e = int(after["starts"][seg]) + n[seg], int(after["starts"][seg + 1])
        assert torch.all(after["records"][b:e] == 0xAB) and torch.all(after["pos"][b:e] == -7) and torch.all(after["weight"][b:e] == 5.0)


def test_eviction_into_a_cache_that_is_too_small():
    lens = [50, 60]
    t = R.random_cache(3, lens, 128, 1, device=DEV)
    before = {k: v.cpu().clone() for k, v in t.items()}
    to, _ = empty_cache([10, 40], 128, 1)
    assert run_evict(t, 1, [30], 4, [10 ** 6] * 2, to=to) == B.ERR["CAPACITY"]
    assert to["lens"].tolist() == [10, 30]
    after = {k: v.cpu() for k, v in to.items()}
    expect_evicted(before, lens, 1, [30], 4, [10 ** 6] * 2, [0, 10], [10, 40], after)
    assert torch.all(after["records"][40:] == 0xAB)


# ---- together --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_a_compressed_prefill_decoded_at_its_budget(dtype, d):
    ns, hkv, G, w, steps = 2, 2, 4, 16, 12
    hq, cu = hkv * G, [0, 700, 1000]
    g = torch.Generator().manual_seed(d)
    T = cu[-1]
    k, v = (torch.randn(T, hkv, d, generator=g).to(dtype).to(DEV) for _ in range(2))
    q_win = torch.randn(ns, w, hq, d, generator=g).to(dtype).to(DEV)
    p = B.make_params(q_win, k, v, w, 5)
    cu_dev = torch.tensor(cu, dtype=torch.int32, device=DEV)
    budgets = B.slkv_alloc_budgets(torch.tensor([[0.4, 0.9]], device=DEV), 32, 300)[0]
    cap = B.slkv_packed_rows_upper_bound(p, cu)
    ko, vo = (torch.empty(cap, d, dtype=dtype, device=DEV) for _ in range(2))
    off, kept = torch.empty(ns * hkv + 1, dtype=torch.int32, device=DEV), torch.empty(cap, dtype=torch.int32, device=DEV)
    B.slkv_compress(p, q_win, k, v, cu_dev, cu, budgets, ko, vo, off, kept, B.new_workspace(p, cu, DEV))
    t, c = empty_cache([int(x) + 4 for x in budgets] * ns, d, hkv)
    B.slkv_q4_pack(c, ko, vo, off, kept)
    assert torch.equal(t["lens"], off[1:] - off[:-1])

    out, lse = torch.empty(ns, 2, hq, d, dtype=dtype, device=DEV), torch.empty(ns, hq, 2, device=DEV)
    params = B.make_q4_attend(c, out, out, weight_decay=0.95)
    ws, ews = B.new_q4_workspace(c, params, True), B.new_q4_evict_workspace(c)
    for step in range(steps):
        newest = torch.tensor([cu[1] + 2 * step + 1, cu[2] - cu[1] + 2 * step + 1], dtype=torch.int32, device=DEV)
        q_pos = torch.stack([newest - 1, newest], 1).contiguous()
        kn, vn = (torch.randn(ns, 2, hkv, d, generator=g).to(dtype).to(DEV) for _ in range(2))
        q = torch.randn(ns, 2, hq, d, generator=g).to(dtype).to(DEV)
        B.slkv_q4_append(c, kn, vn, q_pos)
        before = {x: y.cpu().clone() for x, y in t.items()}
        ref = R.attend(before["records"], before["pos"], before["weight"], before["starts"], before["lens"], q, hkv, d ** -0.5,
                       q_pos=q_pos.cpu().numpy(), decay=float(np.float32(0.95)))
        B.slkv_q4_attend(c, params, q, out, ws, q_pos=q_pos, lse=lse, accumulate=True)
        R.check_attend(out, lse, ref, dtype == torch.bfloat16, got_weight=t["weight"])
        before = {x: y.cpu().clone() for x, y in t.items()}
        B.slkv_q4_evict(c, c, budgets, w, newest, ews)
        n = before["lens"].tolist()
        expect_evicted(before, n, hkv, budgets.tolist(), w, newest.tolist(), before["starts"].tolist(), n, {x: y.cpu() for x, y in t.items()})
        assert t["lens"].tolist() == [min(x, max(int(b), w)) for x, b in zip(n, budgets.tolist() * ns)]


def test_the_same_bits_every_time_on_two_streams_and_in_a_graph():
    lens, d, hkv, G = [3000, 200, 900, 4100], 128, 2, 4
    base = R.random_cache(21, lens, d, hkv, device=DEV)
    q = queries(9, 2, 1, hkv * G, d, torch.bfloat16).to(DEV)
    k, v = (queries(10 + i, 2, 1, hkv, d, torch.bfloat16).to(DEV) for i in range(2))
    newest = torch.tensor([20000, 20000], dtype=torch.int32, device=DEV)
    budgets = torch.tensor([700, 1500], dtype=torch.int32, device=DEV)

    def prepare():
        t = {x: y.clone() for x, y in base.items()}
        c = cache_of(t, hkv)
        out, lse = torch.empty_like(q), torch.empty(2, hkv * G, 1, device=DEV)
        p = B.make_q4_attend(c, q, out)
        return t, c, out, lse, p, B.new_q4_workspace(c, p, True).fill_(0xEE), B.new_q4_evict_workspace(c).fill_(0xEE)

    def step(s):
        t, c, out, lse, p, ws, ews = s
        B.slkv_q4_append(c, k, v, newest.view(2, 1))
        B.slkv_q4_attend(c, p, q, out, ws, lse=lse, accumulate=True)
        B.slkv_q4_evict(c, c, budgets, 8, newest, ews)
    one = prepare()
    step(one)
    step(one)
    torch.cuda.synchronize()
    runs = [prepare(), prepare()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(2):
        for s, r in zip(streams, runs):
            with torch.cuda.stream(s):
                step(r)
    torch.cuda.synchronize()
    graphed = prepare()
    step(graphed)                                          # sets every kernel up
    graphed[0]["lens"].copy_(base["lens"])
    for x in ("records", "pos", "weight"):
        graphed[0][x].copy_(base[x])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for r in runs + [graphed]:
        assert torch.equal(r[2], one[2]) and torch.equal(r[3], one[3])
        for x in ("lens", "records", "pos"):
            assert torch.equal(r[0][x], one[0][x]), x
        assert torch.equal(r[0]["weight"].view(torch.int32), one[0]["weight"].view(torch.int32))


def test_the_first_calls_of_a_process_can_be_captured():
    import os
    import subprocess
    import sys
    program = """
import sys
sys.path[:0] = [%r, %r]
import torch
import q4_reference as R
import test_gpu_q4_cache as T
from paper_2508_15806_b200 import binding as B
B.lib()
lens = [3000, 5000, 100, 4100]
t = R.random_cache(5, lens, 128, 2, device=T.DEV)
few = R.random_cache(6, [300, 700], 64, 1, device=T.DEV)
q = T.queries(1, 2, 1, 8, 128, torch.bfloat16).to(T.DEV)
qf = T.queries(2, 2, 1, 4, 64, torch.float32).to(T.DEV)
k, v = (T.queries(3 + i, 2, 1, 2, 128, torch.bfloat16).to(T.DEV) for i in range(2))
newest = torch.full((2,), 50000, dtype=torch.int32, device=T.DEV)
budgets = torch.tensor([700, 1500], dtype=torch.int32, device=T.DEV)
ko, vo = (torch.zeros(t["records"].size(0), 128, device=T.DEV) for _ in range(2))
c, cf = T.cache_of(t, 2), T.cache_of(few, 1)
out, outf = torch.empty_like(q), torch.empty_like(qf)
p, pf = B.make_q4_attend(c, q, out), B.make_q4_attend(cf, qf, outf)
ws, wsf, ews = B.new_q4_workspace(c, p, True), B.new_q4_workspace(cf, pf), B.new_q4_evict_workspace(c)
def step():
    B.slkv_q4_append(c, k, v, newest.view(2, 1))
    B.slkv_q4_attend(c, p, q, out, ws, accumulate=True)
    B.slkv_q4_attend(cf, pf, qf, outf, wsf)
    B.slkv_q4_evict(c, c, budgets, 8, newest, ews)
    B.slkv_q4_unpack(c, ko, vo)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step()
start = {x: y.clone() for x, y in t.items()}
g.replay()
torch.cuda.synchronize()
first = [x.clone() for x in (out, outf, ko, vo, t["lens"], t["records"])]
for x, y in start.items():
    t[x].copy_(y)
step()
torch.cuda.synchronize()
assert all(torch.equal(x, y) for x, y in zip(first, (out, outf, ko, vo, t["lens"], t["records"])))
print("captured")
""" % (os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout + r.stderr
