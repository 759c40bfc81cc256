"""The 4-bit cache at its documented limits, against the same definitions: large queries, rows in numbers that make the kernels go round
their loops, evictions in which the weights decide."""
import math

import numpy as np
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


# ---- large keys, values and scores --------------------------------------------------------------------------------------
def times_power(t, d, parts, power):
    """The cache with the scales and zeros of K (parts 0, 1) or V (2, 3) times 2^power."""
    s = t["records"][:, d:].contiguous().view(torch.bfloat16).view(-1, 4, d // 32).float()
    s[:, parts] *= 2.0 ** power
    return dict(t, records=torch.cat([t["records"][:, :d], s.bfloat16().view(t["records"].size(0), -1).view(torch.uint8)], 1).contiguous())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k_power,q_power,v_power", [(0, 0, 105), (100, 60, 0), (100, 20, 0), (120, 0, -60), (-60, 60, 0), (60, -30, 40)])
def test_keys_and_values_within_the_documented_bounds(d, dtype, k_power, q_power, v_power):
    lens, hkv, G = [300, 40, 5, 1000], 2, 4
    t = R.random_cache(91 + d, lens, d, hkv, device=DEV)
    t = times_power(times_power(t, d, slice(0, 2), k_power), d, slice(2, 4), v_power)
    q = T.queries(92, 2, 2, hkv * G, d, torch.float32, 2.0 ** q_power).to(dtype)
    scale = float(np.float32(2.0 ** -(k_power + q_power) * 0.125))          # as it is passed: 2^-163 is 0 in fp32
    q_pos = torch.tensor([[100, 400], [3, 5000]], dtype=torch.int32, device=DEV)
    for kw in (dict(), dict(q_pos=q_pos), dict(q_pos=q_pos, softcap=3.0)):
        out, lse = T.check(t, hkv, q, accumulate=True, scale=scale, **kw)
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("softcap", [0.0, 2.0 ** 110, 2.0 ** 124, 3e38])
def test_scores_up_to_the_documented_bound(dtype, softcap):
    # powers of two apart, so that one row takes everything whatever is rounded: its values come out, its score is the log-sum-exp
    d, n = 64, 40
    t = R.random_cache(93, [n], d, 1, slack=2, device=DEV)
    s = t["records"][:, d:].contiguous().view(torch.bfloat16).view(-1, 4, 2)
    s[:, 0], s[:, 1] = 0.0, (2.0 ** torch.arange(s.size(0), device=DEV).remainder(n).float())[:, None].bfloat16()      # K row r: 2^r throughout
    t["records"][:, d:] = s.view(s.size(0), -1).view(torch.uint8)
    q = torch.ones(1, 1, 2, d, dtype=dtype, device=DEV)
    q[0, 0, 1] = -1.0
    scale = 2.0 ** 50                                         # 64 channels: the largest score is 2^(50 + 6 + 39)
    q = q * 2.0 ** 28                                         # .. now 2^123
    out, lse = T.attend(t, 1, q, scale=scale, softcap=softcap)
    _, V, _ = R.decode(t["records"][:n], d)
    for head, row in ((0, n - 1), (1, 0)):
        x = 2.0 ** (84 + row) * (1 if head == 0 else -1)
        if softcap:
            x = softcap * math.tanh(x / softcap)
        if softcap == 2.0 ** 110 and head == 0:              # several scores at the cap: some mixture of those rows
            assert torch.isfinite(out[0, 0, head]).all()
        else:
            # three parts of bf16 at least hold the value; the bf16 way rounds p * scale, then the output
            tol = 2.0 ** -19 * np.abs(V).max() if dtype == torch.float32 else 2.0 ** -6 * np.abs(V).max()
            assert np.all(np.abs(out[0, 0, head].double().cpu().numpy() - V[row]) <= tol)
        assert abs(float(lse[0, head, 0]) - x) <= 2.0 ** -17 * abs(x)


# ---- packing behind overlapped compressions ----------------------------------------------------------------------------
def test_packing_sends_out_what_its_stream_has_queued():
    # no join between the compression and the packing
    from test_gpu_streams_threads import Job
    job = Job([900, 1300], 2, 200, 0)
    hkv, d = job.wl.n_kv_heads, 128
    want = job.reference()
    torch.cuda.synchronize()
    got = []
    outs = job.outputs()
    for o in outs:
        o["off"].zero_()                                     # rows that are not there yet: none
    torch.cuda.synchronize()
    rooms = (want[0]["off"][1:] - want[0]["off"][:-1]).tolist()
    other = torch.cuda.Stream()
    for way in ("same stream", "another stream"):
        tables = [T.empty_cache([x + 400 for x in rooms], d, hkv) for _ in outs]
        torch.cuda.synchronize()
        for layer, o in enumerate(outs):
            job.call(B.slkv_compress_overlapped, layer, o, None)
        if way == "same stream":
            for o, (t, c) in zip(outs, tables):
                B.slkv_q4_pack(c, o["k"], o["v"], o["off"], o["kept"])
            got = [t for t, _ in tables]
            B.slkv_join()
        else:                                                # whose calls are no other stream's: what is queued waits for its join
            with torch.cuda.stream(other):
                B.slkv_q4_pack(tables[0][1], want[0]["k"], want[0]["v"], want[0]["off"], want[0]["kept"])
            assert B.slkv_last_launch_count() == 1
            B.slkv_join()
            assert B.slkv_last_launch_count() > 0
            torch.cuda.synchronize()
            assert torch.equal(tables[0][0]["records"], got[0]["records"])
        torch.cuda.synchronize()
    for t, o, w in zip(got, outs, want):
        assert torch.equal(o["off"], w["off"]) and torch.equal(o["kept"], w["kept"])
        t2, c2 = T.empty_cache([x + 400 for x in rooms], d, hkv)
        B.slkv_q4_pack(c2, w["k"], w["v"], w["off"], w["kept"])
        for name in ("lens", "pos", "records", "weight"):
            assert torch.equal(t[name], t2[name]), name
        assert t["lens"].tolist() == (w["off"][1:] - w["off"][:-1]).tolist()


# ---- a wait that runs out ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("lens,hkv,launches", [([700, 1, 0, 1300], 2, 1), ([5000, 90, 9000, 1], 4, 2), ([300] * 600, 8, 2)])
def test_a_wait_that_runs_out_is_told_by_the_status_and_by_nan(dtype, d, lens, hkv, launches):
    base = R.random_cache(83, lens, d, hkv, device=DEV)
    q = T.queries(84, len(lens) // hkv, 1, 4 * hkv, d, dtype).to(DEV)
    c0 = T.cache_of(base, hkv)
    out, lse = torch.full_like(q, 9.0), torch.full((q.size(0), q.size(2), 1), 9.0, device=DEV)
    p = B.make_q4_attend(c0, q, out)
    ws, status = B.new_q4_workspace(c0, p, True).fill_(0xFF), torch.zeros(1, dtype=torch.int32, device=DEV)

    def call():
        t = {x: y.clone() for x, y in base.items()}
        status.zero_()
        B.slkv_q4_attend(T.cache_of(t, hkv), p, q, out, ws, lse=lse, accumulate=True, status=status)
        assert B.slkv_last_launch_count() == launches
        torch.cuda.synchronize()
        return int(status), out.clone(), lse.clone(), t
    ok, want, want_lse, want_t = call()
    assert ok == 0
    B.slkv_debug_expire_next_wait(5)
    try:
        lost, got, got_lse, got_t = call()
    finally:
        B.slkv_debug_expire_next_wait(0)
    assert lost == B.ERR["DEVICE_TIMEOUT"]
    # the segments whose rows were not waited for are NaN throughout, the others as ever
    gone = torch.isnan(got_lse).view(len(lens), 4)
    assert torch.equal(gone.any(1), gone.all(1)) and 0 < int(gone[:, 0].sum()) < len(lens)
    for seg in range(len(lens)):
        s, h = divmod(seg, hkv)
        b, n = int(base["starts"][seg]), lens[seg]
        mine, w = got[s, 0, 4 * h:4 * h + 4], got_t["weight"][b:b + n]
        if bool(gone[seg, 0]):
            assert n > 0 and torch.isnan(mine).all() and torch.isnan(w).all()
        else:
            assert torch.equal(mine, want[s, 0, 4 * h:4 * h + 4]) and torch.equal(got_lse[s, 4 * h:4 * h + 4], want_lse[s, 4 * h:4 * h + 4])
            assert torch.equal(w, want_t["weight"][b:b + n])
    for name in ("records", "pos", "lens"):
        assert torch.equal(got_t[name], base[name])
    ok, again, again_lse, again_t = call()
    assert ok == 0 and torch.equal(again, want) and torch.equal(again_lse, want_lse) and torch.equal(again_t["weight"], want_t["weight"])


# ---- rows in numbers -------------------------------------------------------------------------------------------------
def many_rows(seed, n, d, dtype):
    """n rows that repeat some hundred different ones in a random order, and their records by the definition."""
    k, v = T.rows(seed, 251, d, dtype)
    pick = torch.randint(0, 251, (n,), generator=torch.Generator().manual_seed(seed + 1))
    rec = torch.from_numpy(T.expected_record(k.double().numpy(), v.double().numpy()))
    return k[pick], v[pick], rec[pick]


@pytest.mark.parametrize("d,dtype", [(128, torch.bfloat16), (64, torch.float32), (64, torch.bfloat16), (128, torch.float32)])
@pytest.mark.parametrize("n_tokens", [33, 65, 130])
def test_more_appended_tokens_than_one_round_takes(d, dtype, n_tokens):
    ns, hkv = 2, 2
    lens, room = [0, 7, 300, 1], [n_tokens, n_tokens + 2, n_tokens - 1, 0]          # slots behind the filled ones
    t, _ = T.empty_cache([a + b for a, b in zip(lens, room)], d, hkv)
    t["lens"].copy_(torch.tensor(lens))
    k, v, rec = many_rows(85, ns * n_tokens * hkv, d, dtype)
    k, v = (x.view(ns, n_tokens, hkv, d).to(DEV) for x in (k, v))
    rec = rec.view(ns, n_tokens, hkv, -1).to(DEV)
    pos = torch.arange(ns * n_tokens, dtype=torch.int32, device=DEV).view(ns, n_tokens) + 50
    want = {x: t[x].clone() for x in ("records", "pos", "weight")}
    for seg, n in enumerate(lens):
        s, h = divmod(seg, hkv)
        m = min(n_tokens, room[seg])
        b = int(t["starts"][seg]) + n
        want["records"][b:b + m], want["pos"][b:b + m], want["weight"][b:b + m] = rec[s, :m, h], pos[s, :m], 0.0
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.slkv_q4_append(T.cache_of(t, hkv), k, v, pos, status=status)
    assert status.item() == B.ERR["CAPACITY"]
    assert t["lens"].tolist() == [n + min(n_tokens, r) for n, r in zip(lens, room)]
    for x, y in want.items():
        assert torch.equal(t[x], y), x


@pytest.mark.parametrize("d,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_more_rows_packed_and_unpacked_than_the_device_takes_at_once(d, dtype):
    lens = [120001, 0, 7, 33, 89999, 1, 99990, 0]
    n = sum(lens)
    k, v, rec = many_rows(86, n, d, dtype)
    offsets = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=DEV)
    kept = torch.randint(0, 1 << 30, (n,), generator=torch.Generator().manual_seed(87)).int().to(DEV)
    t, c = T.empty_cache([x + 3 for x in lens], d, 4)
    rows = t["records"].size(0)
    assert n > 148 * 8 * 32 * 2 and rows > 148 * 8 * 64 * 2           # several rounds each
    B.slkv_q4_pack(c, k.to(DEV), v.to(DEV), offsets, kept)
    assert t["lens"].tolist() == lens
    slots = torch.cat([int(t["starts"][s]) + torch.arange(m) for s, m in enumerate(lens)]).to(DEV)
    want = torch.full((rows, rec.size(1)), 0xAB, dtype=torch.uint8, device=DEV)
    want[slots] = rec.to(DEV)
    assert torch.equal(t["records"], want)
    assert torch.equal(t["pos"][slots], kept) and torch.all(t["weight"][slots] == 0)
    assert int((t["pos"] == -7).sum()) == rows - n and int((t["weight"] == 5.0).sum()) == rows - n

    different, at = torch.unique(rec, dim=0, return_inverse=True)
    K, V, _ = (torch.from_numpy(x).float() for x in R.decode(different, d))
    K, V = K[at].to(DEV), V[at].to(DEV)                      # of row i
    of_slot = torch.full((rows,), -1, dtype=torch.int64, device=DEV)
    of_slot[slots] = torch.arange(n, device=DEV)
    for out_dtype in (torch.float32, torch.bfloat16):
        ko, vo = (torch.full((rows, d), 77.0, dtype=out_dtype, device=DEV) for _ in range(2))
        B.slkv_q4_unpack(c, ko, vo)
        for o, x in ((ko, K), (vo, V)):
            assert torch.equal(o[slots], x.to(out_dtype)) and bool((o[of_slot < 0] == 77.0).all())
        pick = slots[torch.randperm(n, generator=torch.Generator().manual_seed(88)).to(DEV)].int()
        pick[5::7] = torch.tensor([-1, rows, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV).repeat(n // 28 + 1)[:pick[5::7].numel()]
        ko, vo = (torch.full((n, d), 77.0, dtype=out_dtype, device=DEV) for _ in range(2))
        B.slkv_q4_unpack(c, ko, vo, slots=pick)
        given = (pick >= 0) & (pick < rows)
        row = of_slot[pick[given].long()]
        for o, x in ((ko, K), (vo, V)):
            assert torch.equal(o[given], x[row].to(out_dtype)) and bool((o[~given] == 77.0).all())


# ---- nothing asked for ------------------------------------------------------------------------------------------------
def test_an_empty_list_of_slots_unpacks_nothing():
    t = R.random_cache(89, [40], 128, 1, device=DEV)
    c = T.cache_of(t, 1)
    ko, vo = (torch.full((50, 128), 77.0, device=DEV) for _ in range(2))
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    B.slkv_q4_unpack(c, ko[:0], vo[:0], slots=none)
    B.slkv_q4_unpack(c, torch.empty(0, 128, device=DEV), torch.empty(0, 128, device=DEV), slots=none)
    torch.cuda.synchronize()
    assert torch.all(ko == 77.0) and torch.all(vo == 77.0)


def test_a_layer_without_rows_empties_the_segments():
    t, c = T.empty_cache([3, 0, 5], 64, 1)
    none = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.slkv_q4_pack(c, none, none, torch.zeros(4, dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), status)
    assert status.item() == 0 and t["lens"].tolist() == [0, 0, 0] and torch.all(t["records"] == 0xAB)


# ---- evictions in which the weights decide -----------------------------------------------------------------------------
def orders(before, lens, hkv, budgets, window, newest):
    """Per segment the rows that stay, in their slots' order."""
    for seg, n in enumerate(lens):
        b = int(before["starts"][seg])
        yield seg, R.evict_order(before["weight"][b:b + n].tolist(), before["pos"][b:b + n].tolist(), newest[seg // hkv], window,
                                 min(n, max(budgets[seg % hkv], window)))


@pytest.mark.parametrize("kind", ["equal", "zero", "narrow", "huge", "tiny", "negative", "inf", "-inf", "nan", "two values", "one bit apart"])
@pytest.mark.parametrize("lens,hkv", [([900, 3000], 1), ([20000, 9000, 30001], 3)])
@pytest.mark.parametrize("in_place", [True, False])
def test_weights_of_any_size_decide(kind, lens, hkv, in_place):
    t = R.random_cache(71, lens, 64, hkv, device=DEV)
    n = t["weight"].numel()
    u = torch.rand(n, generator=torch.Generator().manual_seed(72))
    w = {"equal": torch.full((n,), 1.25), "zero": torch.zeros(n), "narrow": 1 + u * 1e-4, "huge": u * 1e38, "tiny": u * 1e-38, "negative": -u * 1e3,
         "inf": torch.where(u < 0.6, float("inf"), u), "-inf": torch.where(u < 0.6, -float("inf"), u), "nan": torch.where(u < 0.6, float("nan"), u),
         "two values": torch.where(u < 0.4, 0.5, 0.25), "one bit apart": torch.where(u < 0.4, 1.0 + 2.0 ** -23, 1.0)}[kind]
    t["weight"].copy_(w)
    before = {k: v.cpu().clone() for k, v in t.items()}
    budgets, newest = [x // 2 for x in lens[:hkv]], [10 ** 7] * (len(lens) // hkv)          # beyond all positions: no row is new
    kept = [min(n_, budgets[s % hkv]) for s, n_ in enumerate(lens)]
    for seg, src in orders(before, lens, hkv, budgets, 1, newest):
        assert (src == list(range(kept[seg]))) == (kind in ("equal", "zero")), seg          # else the weights would decide nothing
    to = None if in_place else T.empty_cache([x + 1 for x in kept], 64, hkv)[0]
    assert T.run_evict(t, hkv, budgets, 1, newest, to=to) == 0
    after = {k: v.cpu() for k, v in (t if in_place else to).items()}
    assert after["lens"].tolist() == kept
    T.expect_evicted(before, lens, hkv, budgets, 1, newest, after["starts"].tolist(), kept, after)


@pytest.mark.parametrize("lens,room", [([500001], 310007), ([400003, 5, 130000], 250001)])
def test_more_rows_moved_than_the_device_takes_at_once(lens, room):
    d = 64
    t = R.random_cache(90, lens, d, 1, device=DEV)
    before = {k: v.cpu().clone() for k, v in t.items()}
    budgets, newest = [room], [10 ** 8] * len(lens)
    kept = [min(n, room) for n in lens]
    to, _ = T.empty_cache([k + 11 for k in kept], d, 1)
    assert to["records"].size(0) > 6 * 148 * 256             # slots of one round
    assert T.run_evict(t, 1, budgets, 16, newest, to=to) == 0
    assert B.slkv_last_launch_count() == 2
    after = {k: v.cpu() for k, v in to.items()}
    assert after["lens"].tolist() == kept
    assert torch.equal(t["records"].cpu(), before["records"])
    for seg, src in orders(before, lens, 1, budgets, 16, newest):
        b, dst = int(before["starts"][seg]), int(after["starts"][seg])
        assert (src == list(range(kept[seg]))) == (kept[seg] == lens[seg])
        at = b + torch.tensor(src)
        for name in ("records", "pos"):
            assert torch.equal(after[name][dst:dst + kept[seg]], before[name][at]), (seg, name)
        assert torch.equal(after["weight"][dst:dst + kept[seg]], before["weight"][at])
        e = int(after["starts"][seg + 1])
        assert torch.all(after["records"][dst + kept[seg]:e] == 0xAB) and torch.all(after["pos"][dst + kept[seg]:e] == -7)


@pytest.mark.parametrize("in_place", [True, False])
def test_rows_beyond_32_bits_move(in_place):
    d, rows, n, keep = 128, 14_000_100, 100, 60              # 2.24e9 bytes of records
    small = R.random_cache(65, [n, 33], d, 1, slack=0, device=DEV)
    far = dict(records=torch.zeros(rows, 160, dtype=torch.uint8, device=DEV), pos=torch.zeros(rows, dtype=torch.int32, device=DEV),
               weight=torch.zeros(rows, device=DEV), starts=torch.tensor([0, rows - n, rows], dtype=torch.int32, device=DEV),
               lens=torch.tensor([0, n], dtype=torch.int32, device=DEV))
    for x in ("records", "pos", "weight"):
        far[x][-n:] = small[x][:n]
    newest = 10 ** 8
    src = R.evict_order(small["weight"][:n].tolist(), small["pos"][:n].tolist(), newest, 1, keep)
    assert src != list(range(keep))
    to = None if in_place else T.empty_cache([rows - n, n], d, 1)[0]
    assert T.run_evict(far, 1, [keep], 1, [newest, newest], to=to) == 0
    got = far if in_place else to
    assert got["lens"].tolist() == [0, keep]
    for x in ("records", "pos", "weight"):
        assert torch.equal(got[x][rows - n:rows - n + keep], small[x][src]), x
        if in_place:
            assert torch.equal(got[x][rows - n + keep:], small[x][keep:n]) and not bool(got[x][:rows - n].any())
    if not in_place:
        assert bool((got["records"][:rows - n] == 0xAB).all()) and torch.equal(far["records"][-n:], small["records"][:n])
