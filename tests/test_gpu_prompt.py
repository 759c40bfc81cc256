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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 3, 5, 8, 16, 48, 64])
def test_groups(G, dtype):
    run([70, 3, 140], hkv=2, G=G, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [([1], [1000]), ([1, 40, 100], [700, 41, 100]), ([200], [1500]), ([7, 64], [2500, 65])])
def test_chunks(nq, nk, dtype):
    """Queries behind keys that were there already; few units, whose tiles several CTAs share."""
    run(nq, nk, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [([50], [0]), ([50], [20]), ([300, 10, 300], [150, 0, 5])])
def test_queries_that_see_nothing(nq, nk, dtype):
    run(nq, nk, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_units(dtype):
    """Whole units dealt out, the longest first, several of one CTA."""
    run([1500, 1, 700, 0, 2300, 64], hkv=8, G=8 if dtype == "bf16" else 4, d=64, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    run([1 + 7 * i % 90 for i in range(150)], hkv=2, G=2, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_before_tokens(dtype):
    """[heads, tokens, head_dim] in memory: strides in the other order."""
    run([130, 33], dtype=dtype, heads_first=True)
    run([9], [600], dtype=dtype, heads_first=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_inside_wider_ones(dtype):
    """q, k, v are parts of one projection's output, out of a wider buffer."""
    g = torch.Generator(device="cuda").manual_seed(3)
    n, hkv, G, d = 77, 2, 3, 64
    qkv = torch.randn(n, hkv * (G + 2), d, device="cuda", generator=g).to(DT[dtype])
    q, k, v = qkv[:, :hkv * G], qkv[:, hkv * G:hkv * (G + 1)], qkv[:, hkv * (G + 1):]
    wide = torch.full((n, hkv * G, 2 * d), 7.0, dtype=q.dtype, device="cuda")
    out, lse, before = attend(q, k, v, [n], out=wide[:, :, :d])
    R.check_prompt(q, k, v, [0, n], [0, n], out, lse, 32, d ** -0.5, before, torch.full_like(lse, 5.0))
    assert (wide[:, :, d:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite(bad, dtype):
    """K and V at a position reach the queries from there on and no other, in every sequence; what lies behind the last sequence
    reaches nobody."""
    nq = [200, 70, 333]
    q, k, v = inputs(nq, nq, 2, 4, 128, dtype, seed=5)
    for pos in (0 + 150, 200 + 69, 270 + 40, 270 + 41, 270 + 300):
        v[pos, 0, 5] = bad
        v[pos, 1, 100] = -bad
    k[sum(nq):], v[sum(nq):] = bad, bad
    k[270 + 332, 1] = float("nan")                                # the last key of a sequence: only its last query sees it
    out, lse, before = attend(q, k, v, nq)
    kk = k.clone()
    kk[270 + 332, 1] = 0.0
    for s, (a, n) in enumerate(zip(cu(nq), nq)):
        for h in range(8):
            upto = n - 1 if s == 2 and h >= 4 else n
            ref = R.rows(q[a:a + n, h], kk[a:a + n, h // 4], v[a:a + n, h // 4], R.causal(n, n, "cuda"), 128 ** -0.5)
            R.check(out[a:a + upto, h], None, tuple(x[:upto] for x in ref), dtype == "bf16", 128)
            assert upto == n or torch.isnan(out[a + upto, h]).all()
    assert torch.equal(out[sum(nq):], before[sum(nq):])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite_in_shared_units(dtype):
    """The same where several CTAs share a unit, and where two warpgroups share its tiles."""
    for nq, nk in (([60], [1400]), ([20], [900]), ([3], [700])):
        q, k, v = inputs(nq, nk, 1, 4, 128, dtype, seed=6)
        for back in (1, 3, 19):
            if back <= nq[0]:
                v[nk[0] - back, 0, 7] = float("inf")
        v[100, 0, 9] = float("nan")
        out, lse, before = attend(q, k, v, nq, nk)
        R.check_prompt(q, k, v, cu(nq), cu(nk), out, lse, 32, 128 ** -0.5, before, torch.full_like(lse, 5.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_rise_and_fall(dtype):
    """Maxima that come late, early and far apart: the running reference is raised again and again, or never."""
    for order in (1, -1):
        nq = [700]
        q, k, v = inputs(nq, nq, 1, 4, 64, dtype, seed=7)
        q.copy_(torch.ones_like(q))
        ramp = torch.linspace(-3.0, 3.0, k.shape[0], device="cuda") * order
        k.copy_(ramp[:, None, None].expand(k.shape).to(k.dtype))
        out, lse, before = attend(q, k, v, nq, scale=1.0)
        R.check_prompt(q, k, v, cu(nq), cu(nq), out, lse, 32, 1.0, before, torch.full_like(lse, 5.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_at_the_limits(dtype):
    """Scores of 2^120 and differences that leave one key per row; scale at its ends."""
    nq = [150]
    for factor, scale in ((2.0 ** 60, 1.0), (2.0 ** 40, 2.0 ** 40), (1.0, 2.0 ** -54), (2.0 ** 30, 2.0 ** -54), (2.0 ** 10, 2.0 ** 54)):
        q, k, v = inputs(nq, nq, 1, 2, 64, dtype, seed=8)
        q.zero_(), k.zero_()
        i = torch.arange(k.shape[0], device="cuda")
        q[:, :, 0] = factor
        k[:, 0, 0] = (factor * (1 + (i * 37) % 101)).to(k.dtype) if factor < 2.0 ** 50 else factor * (2.0 ** (i % 4).float()).to(k.dtype)
        out, lse, before = attend(q, k, v, nq, scale=scale)
        R.check_prompt(q, k, v, cu(nq), cu(nq), out, lse, 32, scale, before, torch.full_like(lse, 5.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_and_units(dtype):
    for window in (1, 33, 200):
        run([150, 20], window=window, dtype=dtype, log2=window == 33)


def test_the_same_again_and_without_lse():
    nq, nk = [33, 500], [1200, 500]
    q, k, v = inputs(nq, nk, 2, 4, 128, "bf16", seed=9)
    first = attend(q, k, v, nq, nk)
    for _ in range(3):
        again = attend(q, k, v, nq, nk)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    p = B.make_prompt(q, k, v, first[0], 2)
    c_q, c_k = cu(nq), cu(nk)
    out = torch.zeros_like(q)
    ws = B.new_prompt_workspace(p, c_q, c_k)
    B.slkv_prompt_attend(p, q, k, v, torch.tensor(c_q, dtype=torch.int32, device="cuda"), tuple(c_q), out, ws,
                         cu_k=torch.tensor(c_k, dtype=torch.int32, device="cuda"), cu_k_host=tuple(c_k))
    assert torch.equal(out[:sum(nq)], first[0][:sum(nq)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_on_another_stream(dtype):
    nq, nk = [40, 100], [900, 100]
    q, k, v = inputs(nq, nk, 2, 4, 128, dtype, seed=10)
    want = attend(q, k, v, nq, nk)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = attend(q, k, v, nq, nk)
    torch.cuda.synchronize()
    got_too = attend(q, k, v, nq, nk, stream=torch.cuda.current_stream())
    assert torch.equal(got_too[0], want[0])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c_q, c_k = cu(nq), cu(nk)
    dq, dk = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (c_q, c_k))
    out, lse = torch.zeros_like(q), torch.full_like(want[1], 5.0)
    p = B.make_prompt(q, k, v, out, 2, window=32)
    ws = B.new_prompt_workspace(p, c_q, c_k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.slkv_prompt_attend(p, q, k, v, dq, c_q, out, ws, cu_k=dk, cu_k_host=c_k, lse=lse)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:sum(nq)], want[0][:sum(nq)]) and torch.equal(lse, want[1])


def test_compression_takes_the_log_sum_exp():
    """prompt -> its window rows' log-sum-exp -> slkv_score: the scores that slkv_score computes by itself over the same softmax."""
    nq, hkv, G, d, w = [900, 1300], 4, 4, 128, 32
    q, k, v = inputs(nq, nq, hkv, G, d, "bf16", seed=11, behind=0)
    out, lse, _ = attend(q, k, v, nq, window=w)
    c = cu(nq)
    q_win = torch.stack([q[e - w:e] for e in c[1:]])
    params = B.make_params(q_win, k, v, w, 7, softmax_domain=B.SLKV_ALL_CAUSAL)
    dev = torch.tensor(c, dtype=torch.int32, device="cuda")
    pooled = []
    for given in (None, lse):
        x = torch.zeros(B.slkv_pooled_elems(params, c), device="cuda")
        ws = torch.empty(B.slkv_workspace_bytes(params, c), dtype=torch.uint8, device="cuda")
        B.slkv_score(params, q_win, k, dev, c, x, ws, lse=given)
        pooled.append(x)
    # slkv_score's own bound (10^-3 of the value), and the log-sum-exp's 2^-20
    assert ((pooled[0] - pooled[1]).abs() <= 2e-3 * pooled[0].abs() + 1e-30).all()


def test_a_wait_that_runs_out():
    q, k, v = inputs([300], [300], 1, 4, 128, "bf16", seed=12)
    p = B.make_prompt(q, k, v, torch.zeros_like(q), 1)
    out, status = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    c = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    ws = B.new_prompt_workspace(p, [0, 300])
    B.slkv_debug_expire_next_wait(5)
    B.slkv_prompt_attend(p, q, k, v, c, [0, 300], out, ws, status=status)
    torch.cuda.synchronize()
    assert int(status) == B.ERR["DEVICE_TIMEOUT"]
    good, _, _ = attend(q, k, v, [300])
    got = out[:300]
    fine = (got == good[:300]) | (got == 7.0) | torch.isnan(got)      # computed, left as it was, or NaN
    assert fine.all() and not torch.equal(got, good[:300])
    status.zero_()
    B.slkv_prompt_attend(p, q, k, v, c, [0, 300], out, ws, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(out[:300], good[:300])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_thousands_of_sequences(dtype):
    run([1 + i % 3 if i % 7 else 0 for i in range(3001)], hkv=1, G=2, d=64, dtype=dtype, window=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite_in_many_short_sequences(d, dtype):
    """Units of one tile, many of one CTA: what is noted of one while others are loaded ahead of its results."""
    nq = [1 + 11 * i % 60 for i in range(400)]
    q, k, v = inputs(nq, nq, 2, 2, d, dtype, seed=9)
    at = cu(nq)
    for s in range(0, len(nq), 3):
        v[at[s] + nq[s] // 2, s % 2, s % d] = float("inf") if s % 2 else float("nan")
    out, lse, before = attend(q, k, v, nq)
    R.check_prompt(q, k, v, at, at, out, lse, 32, d ** -0.5, before, torch.full_like(lse, 5.0))


def test_a_wait_that_runs_out_in_fp32():
    q, k, v = inputs([40], [900], 1, 4, 64, "f32", seed=13)           # units shared by several CTAs
    good, _, before = attend(q, k, v, [40], [900])
    out, status = before.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    c, ck = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (40, 900))
    p = B.make_prompt(q, k, v, out, 1)
    ws = B.new_prompt_workspace(p, [0, 40], [0, 900])
    for expire in (True, False):
        status.zero_()
        if expire:
            B.slkv_debug_expire_next_wait(5)
        B.slkv_prompt_attend(p, q, k, v, c, [0, 40], out, ws, cu_k=ck, cu_k_host=[0, 900], status=status)
        torch.cuda.synchronize()
        if expire:
            assert int(status) == B.ERR["DEVICE_TIMEOUT"]
            fine = (out == good) | (out == 7.0) | torch.isnan(out)
            assert fine[:40].all() and not torch.equal(out[:40], good[:40])
        else:
            assert int(status) == 0 and torch.equal(out, good)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_side_by_side(dtype):
    """Two streams with a workspace each, several calls of both under way."""
    shapes = [([300, 5], [1700, 5]), ([64], [2000])]
    made = []
    for i, (nq, nk) in enumerate(shapes):
        q, k, v = inputs(nq, nk, 2, 4, 128, dtype, seed=14 + i)
        want = attend(q, k, v, nq, nk)[0]
        c, ck = (torch.tensor(cu(x), dtype=torch.int32, device="cuda") for x in (nq, nk))
        outs = [torch.full_like(q, 7.0) for _ in range(6)]
        p = B.make_prompt(q, k, v, outs[0], len(nq))
        made.append((p, q, k, v, c, cu(nq), ck, cu(nk), outs, B.new_prompt_workspace(p, cu(nq), cu(nk)), want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for turn in range(6):
        for p, q, k, v, c, cq, ck, chk, outs, ws, _, stream in made:
            B.slkv_prompt_attend(p, q, k, v, c, cq, outs[turn], ws, cu_k=ck, cu_k_host=chk, stream=stream)
    torch.cuda.synchronize()
    for *_, outs, _, want, _ in made:
        for out in outs:
            assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graphs_that_share_a_workspace(dtype):
    """Two captured calls of different shape in one workspace, replayed in turn on one stream."""
    shapes = [([30], [1500]), ([1, 90], [800, 900])]
    made, ws = [], torch.empty(0, dtype=torch.uint8, device="cuda")
    for i, (nq, nk) in enumerate(shapes):
        q, k, v = inputs(nq, nk, 2, 4, 64, dtype, seed=16 + i)
        want = attend(q, k, v, nq, nk)[0]
        c, ck = (torch.tensor(cu(x), dtype=torch.int32, device="cuda") for x in (nq, nk))
        out = torch.full_like(q, 7.0)
        p = B.make_prompt(q, k, v, out, len(nq))
        made.append([p, q, k, v, c, cu(nq), ck, cu(nk), out, want])
        one = B.new_prompt_workspace(p, cu(nq), cu(nk))
        ws = one if one.numel() > ws.numel() else ws
    graphs = []
    for p, q, k, v, c, cq, ck, chk, out, _ in made:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            B.slkv_prompt_attend(p, q, k, v, c, cq, out, ws, cu_k=ck, cu_k_host=chk)
    for _ in range(3):
        for x in made:
            x[8].fill_(7.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x in made:
            assert torch.equal(x[8], x[9])
