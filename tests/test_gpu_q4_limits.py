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
