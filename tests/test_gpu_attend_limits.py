"""Prompt attention and the paged cache at what their documentation allows: workspaces, queued layers, drafted rows of several blocks, large tables."""
import random

import pytest
import torch

import test_gpu_paged as G
import test_gpu_prompt as T
from paper_2508_15806_b200 import binding as B

pytestmark = pytest.mark.gpu


# ---- workspaces ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("offset", [16, 32, 48, 240])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_workspaces_from_any_16_byte_boundary(dtype, offset):
    """Of the size asked for and no more, in units that several CTAs share; what lies around them stays as it is."""
    def carve(n):
        buf = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        assert buf.data_ptr() % 256 == 0
        return buf, buf[offset:offset + n]

    def untouched(buf, ws):
        assert (buf[:offset] == 0xA5).all() and (buf[offset + ws.numel():] == 0xA5).all()

    nq, nk = [33, 5], [1900, 700]
    q, k, v = T.inputs(nq, nk, 2, 4, 128, dtype, seed=21)
    want, want_lse, _ = T.attend(q, k, v, nq, nk)
    c_q, c_k = T.cu(nq), T.cu(nk)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    out, lse = torch.full_like(q, 7.0), torch.full_like(want_lse, 5.0)
    p = B.make_prompt(q, k, v, out, len(nq), window=32)
    buf, ws = carve(B.slkv_prompt_attend_workspace_bytes(p, c_q, c_k))
    B.slkv_prompt_attend(p, q, k, v, dev(c_q), c_q, out, ws, cu_k=dev(c_k), cu_k_host=c_k, lse=lse)
    torch.cuda.synchronize()
    assert B.slkv_last_launch_count() == 2                                 # pieces and the launch that joins them
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    untouched(buf, ws)

    c = G.Cache([3000, 200, 1700, 900], 2, 2, 64, dtype, 32)
    for n in (3, 64):                                                        # one block of query rows, more
        q, k, v, want, _, _ = G.attend(c, 4, n)
        out = torch.full_like(q, 7.0)
        p = B.make_paged_attend(c.c, q, out, k, v)
        buf, ws = carve(B.slkv_paged_attend_workspace_bytes(c.c, p))
        B.slkv_paged_attend(c.c, p, q, out, ws, k, v)
        torch.cuda.synchronize()
        assert B.slkv_last_launch_count() == 2
        assert torch.equal(out, want)
        untouched(buf, ws)


# ---- the same bit for bit --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads,n", [(4, 1), (4, 3), (3, 40), (5, 64)])
def test_results_do_not_depend_on_what_ran_before(heads, n):
    """Blocks with rows that no query has: whatever an earlier launch left in shared memory there, results are the same bit for bit."""
    c = G.Cache([3000, 200, 1700, 900], 2, 2, 128, "bf16", 32)
    q, k, v = T.inputs([3000], [3000], 8, 4, 128, "bf16", seed=22, behind=0)
    got = []
    for factor in (0.0, 1.0, 2.0 ** 30, 2.0 ** 60):
        T.attend(q * factor, k, v, [3000])                                # queries of this size in every CTA's buffers
        got.append(G.attend(c, heads, n)[3:5])
        nq, nk = [20, 5], [900, 5]
        x = T.inputs(nq, nk, 2, heads, 128, "bf16", seed=23)
        T.attend(q * factor, k, v, [3000])
        got[-1] = got[-1] + T.attend(*x, nq, nk)[:2]
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert torch.equal(x, y)


# ---- drafted rows ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads,n", [(4, 33), (4, 40), (4, 64), (16, 8), (16, 24), (5, 61), (1, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_drafted_values_that_are_not_finite_in_two_blocks(dtype, heads, n):
    """Both blocks of a unit see the same drafted rows: values that are not finite reach every token that sees them, in both, and no other."""
    c = G.Cache([200, 300, 0, 128], 2, 2, 128, dtype, 32, junk=float("nan"), seed=4)
    counts = [n - 1, n]

    def edit(q, k, v):
        inf = float("inf")
        v[0, 1, :, 4], v[0, n // 2, :, 64], v[0, n - 2, :, 127], v[1, 0, :, 0], v[1, n - 1, :, 100] = float("nan"), inf, -inf, inf, -inf
        k[0, n - 1], v[0, n - 1] = float("nan"), float("nan")              # padding
    for seed in range(3):
        masks = G.tree_masks(2, n, seed)
        for s in range(2):
            for i in range(seed, n):
                masks[s][i] |= 1 << (n // 2) if i % 3 == 0 else 1          # seen from both blocks
        G.check_attend(c, heads, n, masks, counts=counts, edit=edit, seed=seed)
    first = G.attend(c, heads, n, masks, counts, edit=edit)[3]
    for _ in range(20):
        again = G.attend(c, heads, n, masks, counts, edit=edit)[3]
        assert torch.equal(torch.isfinite(again), torch.isfinite(first)) and torch.equal(again.nan_to_num(), first.nan_to_num())


# ---- many sequences ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences_behind_keys_of_their_own(dtype):
    nq = [1 + i % 4 if i % 9 else 0 for i in range(700)]
    T.run(nq, [n + i % 5 * 31 for i, n in enumerate(nq)], hkv=1, G=2, d=64, dtype=dtype, window=2)


# ---- beside overlapped compressions --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shared", ["nothing", "lse", "workspace", "both"])
def test_prompts_between_overlapped_compressions(shared):
    """Layer by layer, prompt attention and the compression that takes its log-sum-exps, which may stay queued.  One buffer of log-sum-exps for all
    layers, one workspace for everything: the results are those of calls without overlap.  With buffers of their own, layers stay queued."""
    nq, nk, hkv, g, d, w = [40, 20], [900, 700], 4, 4, 128, 16
    c_q, c_k = T.cu(nq), T.cu(nk)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    dq, dk, budgets = dev(c_q), dev(c_k), dev([60, 100, 33, 250])
    layers, ws, lse = [], None, torch.zeros(2, hkv * g, w, device="cuda")
    for i in range(3):
        q, k, v = T.inputs(nq, nk, hkv, g, d, "bf16", seed=40 + i, behind=0)
        q_win = torch.stack([q[e - w:e] for e in c_q[1:]])
        pp, pc = B.make_prompt(q, k, v, torch.empty_like(q), 2, window=w), B.make_params(q_win, k, v, w, 5, softmax_domain=B.SLKV_ALL_CAUSAL)
        sizes = B.slkv_workspace_bytes_overlapped(pc, c_k), B.slkv_prompt_attend_workspace_bytes(pp, c_q, c_k)
        if ws is None:
            ws = [torch.full((max(sizes),), 0xff, dtype=torch.uint8, device="cuda") for _ in range(2)]
        cap = B.slkv_packed_rows_upper_bound(pc, c_k)

        def outs():
            return (*(torch.zeros(cap, d, dtype=k.dtype, device="cuda") for _ in range(2)), torch.zeros(2 * hkv + 1, dtype=torch.int32, device="cuda"),
                    torch.zeros(cap, dtype=torch.int32, device="cuda"))
        layers.append((q, k, v, q_win, pp, pc, torch.empty_like(q), lse if shared in ("lse", "both") else torch.zeros_like(lse), outs(), outs()))
    own, wants = [], []
    for q, k, v, q_win, pp, pc, out, _, _, want in layers:                 # one behind the other
        x = torch.zeros_like(lse)
        B.slkv_prompt_attend(pp, q, k, v, dq, c_q, out, ws[0], cu_k=dk, cu_k_host=c_k, lse=x)
        own.append(B.slkv_last_launch_count())
        B.slkv_compress(pc, q_win, k, v, dk, c_k, budgets, *want, ws[1], lse=x)
        wants.append(out.clone())
    torch.cuda.synchronize()
    counts = []
    for q, k, v, q_win, pp, pc, out, x, got, _ in layers:
        out.zero_()
        B.slkv_prompt_attend(pp, q, k, v, dq, c_q, out, ws[0], cu_k=dk, cu_k_host=c_k, lse=x)
        counts.append(B.slkv_last_launch_count())
        B.slkv_compress_overlapped(pc, q_win, k, v, dk, c_k, budgets, *got, ws[0 if shared in ("workspace", "both") else 1], lse=x)
        assert B.slkv_last_launch_count() == 0                              # queued
    B.slkv_join()
    torch.cuda.synchronize()
    for (_, _, _, _, _, _, out, _, got, want), o in zip(layers, wants):
        assert torch.equal(out, o)
        n = int(want[2][-1])
        assert torch.equal(got[2], want[2]) and all(torch.equal(got[i][:n], want[i][:n]) for i in (0, 1, 3))
    assert counts[0] == own[0] and all(n == m if shared == "nothing" else n > m for n, m in zip(counts[1:], own[1:])), (counts, own)


# ---- plans of many segments ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layers,ns,hkv", [(33, 32, 8), (32, 64, 8), (3, 2048, 8), (40, 300, 1)])
def test_plan_more_segments_than_threads(layers, ns, hkv):
    """Several segments a thread, in rounds that write lengths in place: by lengths up and down, ragged and wide slots, by rows added, there and back."""
    r = random.Random(layers + ns)
    n = layers * ns * hkv
    assert n > 8192
    c = G.Cache([r.choice([0, 1, 16, 17, 32, r.randint(0, 70)]) for _ in range(n)], ns, hkv, 64, "bf16", 16, spare=3 * n, room=4)
    before = [list(t) for t in c.host_tables], list(c.host_lens), list(c.host_free)
    up = [x + r.choice([0, 0, 1, 5, 40]) for x in c.host_lens]
    G.check_plan(c, B.SLKV_PAGED_LENGTHS, up, up)
    G.check_plan(c, B.SLKV_PAGED_LENGTHS, before[1], before[1], width=3)
    assert (c.host_lens, c.host_free) == before[1:]
    want = [r.choice([x, 0, x + 1, max(0, x - 20), r.randint(0, 70)]) for x in c.host_lens]
    G.check_plan(c, B.SLKV_PAGED_LENGTHS, want, want)
    add = [r.randint(-1, 4) for _ in range(ns)]
    lengths = [x + max(add[i // hkv % ns], 0) for i, x in enumerate(c.host_lens)]
    after = B.make_paged_cache(c.k, c.v, c.tables, torch.zeros_like(c.lens), c.free, torch.zeros_like(c.n_free), ns, hkv)
    first = G.check_plan(c, B.SLKV_PAGED_ADD, add, lengths, width=4, after=after)
    assert torch.equal(first, G.check_plan(c, B.SLKV_PAGED_ADD, add, lengths, width=4))


def test_plan_many_segments_run_out():
    """Pages that run out in a later round, in the middle of a CTA's segments."""
    r = random.Random(9)
    n, ns = 9000, 9000 // 8
    for spare in (100, 6000, 15000):
        c = G.Cache([r.randint(0, 20) for _ in range(n)], ns, 8, 64, "f32", 16, spare=spare, room=5)
        want = [x + r.randint(0, 60) for x in c.host_lens]
        G.check_plan(c, B.SLKV_PAGED_LENGTHS, want, want)


@pytest.mark.parametrize("layers,ns,hkv", [(32, 16, 8), (32, 512, 1), (2, 300, 8)])
def test_plan_few_that_grow_among_many(layers, ns, hkv):
    """One sequence comes in and another goes while the others stay: new rows of a layer and of the next lie far apart, long runs of segments without."""
    r = random.Random(ns)
    n, per = layers * ns * hkv, ns * hkv
    c = G.Cache([r.randint(1, 40) for _ in range(n)], ns, hkv, 64, "bf16", 32, spare=12 * layers * hkv, room=12)
    comes, goes = r.sample(range(ns), 2)
    want = [r.randint(200, 380) if i % per // hkv == comes else 0 if i % per // hkv == goes else x for i, x in enumerate(c.host_lens)]
    G.check_plan(c, B.SLKV_PAGED_LENGTHS, want, want)
    last = [x + (i in (0, n - 1)) * 50 for i, x in enumerate(c.host_lens)]                # the first and the last one only
    G.check_plan(c, B.SLKV_PAGED_LENGTHS, last, last)
    G.check_plan(c, B.SLKV_PAGED_LENGTHS, last, last)                                      # nothing comes in at all


@pytest.mark.parametrize("grows", [False, True])
def test_plan_without_room_for_a_slot(grows):
    """An empty tensor of slots, as many as no row needs: offsets are written all the same, and the status tells where rows do come in."""
    c = G.Cache([3, 0, 40, 16], 2, 2, 64, "bf16", 16, spare=9, room=3)
    want = [3, 0, 41, 16] if grows else [3, 0, 20, 0]
    G.check_plan(c, B.SLKV_PAGED_LENGTHS, want, want, n_slots=0)
