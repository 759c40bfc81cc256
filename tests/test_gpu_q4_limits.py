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
