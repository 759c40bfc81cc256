"""The paged cache: plans against lists, rows written through slots, attention of trees over it against its definition in 64 bits."""
import random

import pytest
import torch

import attend_reference as R
import paged_reference as P
from paper_2508_15806_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(x, t=torch.int32):
    return torch.tensor(x, dtype=t, device="cuda")


class Cache:
    """A cache with segments of the lengths given, in pages taken at random; rows behind the last one, and pages that nobody has, hold `junk`."""

    def __init__(self, lens, n_seqs, hkv, d, dtype, page_rows, spare=5, room=2, seed=0, junk=None):
        r = random.Random(seed)
        have = [-(-n // page_rows) for n in lens]
        self.n_pages, self.page_rows, self.max_pages = sum(have) + spare, page_rows, max(have) + room
        pages = list(range(self.n_pages))
        r.shuffle(pages)
        at, rows = 0, []
        for h in have:
            rows.append(pages[at:at + h] + [r.randrange(self.n_pages) for _ in range(self.max_pages - h)])
            at += h
        self.host_tables, self.host_lens, self.host_free = rows, list(lens), pages[at:]
        g = torch.Generator(device="cuda").manual_seed(seed)
        shape = (self.n_pages, page_rows, d)
        self.k, self.v = (torch.randn(shape, device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
        if junk is not None:
            keep = torch.zeros(self.n_pages, page_rows, dtype=torch.bool)
            for t, n in zip(rows, lens):
                for i in range(-(-n // page_rows)):
                    keep[t[i], :min(page_rows, n - i * page_rows)] = True
            self.k[~keep.cuda()] = junk
            self.v[~keep.cuda()] = junk
        self.tables, self.lens = dev(rows), dev(lens)
        self.free, self.n_free = dev(self.host_free + [-7] * (self.n_pages - len(self.host_free))), dev([len(self.host_free)])
        self.c = B.make_paged_cache(self.k, self.v, self.tables, self.lens, self.free, self.n_free, n_seqs, hkv)
        self.n_seqs, self.hkv, self.d, self.dtype = n_seqs, hkv, d, dtype

    def rows(self, seg):
        n = max(0, min(self.lens[seg].item(), self.max_pages * self.page_rows))
        pages = self.tables[seg, :-(-n // self.page_rows)].long()
        return self.k[pages].reshape(-1, self.d)[:n], self.v[pages].reshape(-1, self.d)[:n]


def slots_of(cache, tables, rows):
    return [tables[s][r // cache.page_rows] * cache.page_rows + r % cache.page_rows for s, r in rows]


def check_plan(cache, mode, want, lengths, width=None, after=None, n_slots=None, stream=None):
    """Plans and compares everything; lengths: what `want` comes to."""
    tables, lens, free, rows, fits = P.plan(cache.host_tables, cache.host_lens, cache.host_free, cache.page_rows, lengths)
    n_seg = len(lens)
    status = dev([0])
    if width is None:
        n = len(rows) + 9 if n_slots is None else n_slots
        slots, offsets = torch.full((n,), 99, dtype=torch.int32, device="cuda"), dev([0] * (n_seg + 1))
    else:
        slots, offsets = torch.full((n_seg, width), 99, dtype=torch.int32, device="cuda"), None
    B.slkv_paged_plan(cache.c, mode, dev(want), slots=slots, slot_offsets=offsets, after=after, status=status, stream=stream)
    torch.cuda.synchronize()
    got = after.tensors if after is not None else cache.c.tensors
    assert got[3].tolist() == lens and int(got[5]) == len(free)
    assert cache.free[:len(free)].tolist() == free
    for s in range(n_seg):
        used = -(-lens[s] // cache.page_rows)
        assert cache.tables[s, :used].tolist() == tables[s][:used], s
    if after is not None:
        assert cache.lens.tolist() == cache.host_lens and int(cache.n_free) == len(cache.host_free)
    named = slots_of(cache, tables, rows)
    if width is None:
        count = [0] * (n_seg + 1)
        for s, _ in rows:
            count[s + 1] += 1
        for s in range(n_seg):
            count[s + 1] += count[s]
        assert offsets.tolist() == count
        named = (named + [-1] * n)[:n]
        assert slots.tolist() == named
        fits &= len(rows) <= n
    else:
        by = [[] for _ in range(n_seg)]
        for (s, _), x in zip(rows, named):
            by[s].append(x)
        fits &= max(len(x) for x in by) <= width
        assert slots.tolist() == [(x + [-1] * width)[:width] for x in by]
    assert int(status) == (0 if fits else B.ERR["CAPACITY"])
    if after is None:
        cache.host_tables, cache.host_lens, cache.host_free = tables, lens, free
    return slots


SHAPES = [(1, 1, 1), (1, 3, 2), (2, 5, 7), (3, 40, 8), (32, 16, 8), (70, 33, 3)]


@pytest.mark.parametrize("layers,ns,hkv", SHAPES)
@pytest.mark.parametrize("page_rows", [16, 128])
def test_plan_lengths(layers, ns, hkv, page_rows):
    """Up and down at random, segments that end and begin, there and back."""
    r = random.Random(layers * 100 + ns)
    n = layers * ns * hkv
    size = 400 if n < 300 else 60
    c = Cache([r.choice([0, r.randint(1, size), page_rows, 2 * page_rows]) for _ in range(n)], ns, hkv, 64, "bf16", page_rows,
              spare=n * (size // page_rows + 1), room=6)
    for step in range(4):
        before = [list(t) for t in c.host_tables], list(c.host_lens), list(c.host_free)
        want = [r.choice([x, 0, x + 1, max(0, x - 1), r.randint(0, size)]) for x in c.host_lens]
        if step == 2:
            want = [x + r.randint(0, 5) for x in c.host_lens]         # only up, then back: everything is as it was
        check_plan(c, B.SLKV_PAGED_LENGTHS, want, want, width=None if step % 2 else 8 if step == 0 else 5)
        if step == 2:
            check_plan(c, B.SLKV_PAGED_LENGTHS, before[1], before[1])
            assert (c.host_lens, c.host_free) == before[1:]


@pytest.mark.parametrize("layers,ns,hkv", SHAPES[:5])
def test_plan_added_and_by_offsets(layers, ns, hkv):
    r = random.Random(ns)
    n, per = layers * ns * hkv, ns * hkv
    c = Cache([0] * n, ns, hkv, 64, "f32", 32, spare=n * 6, room=8)
    offsets, lengths = [], []
    for _ in range(layers):
        o = [0]
        for _ in range(per):
            lengths.append(r.choice([0, 1, 32, r.randint(0, 120)]))
            o.append(o[-1] + lengths[-1])
        offsets.append(o)
    check_plan(c, B.SLKV_PAGED_OFFSETS, offsets, lengths)
    add = [r.randint(-1, 6) for _ in range(ns)]
    lengths = [x + max(add[i // hkv % ns], 0) for i, x in enumerate(c.host_lens)]
    lens2, free2 = dev([0] * n), dev([0])
    after = B.make_paged_cache(c.k, c.v, c.tables, lens2, c.free, free2, ns, hkv)
    first = check_plan(c, B.SLKV_PAGED_ADD, add, lengths, width=6, after=after)
    again = check_plan(c, B.SLKV_PAGED_ADD, add, lengths, width=6)     # drafted, then in earnest: the same pages
    assert torch.equal(first, again)


def test_plan_many_rows():
    """More ragged slots than the planning launch writes itself; pages of a long segment."""
    c = Cache([0] * 6, 3, 2, 64, "bf16", 16, spare=9000, room=7000)
    want = [30000, 0, 17, 60001, 1, 20000]
    check_plan(c, B.SLKV_PAGED_LENGTHS, want, want)
    check_plan(c, B.SLKV_PAGED_LENGTHS, [5, 70000, 17, 60000, 0, 0], [5, 70000, 17, 60000, 0, 0])


def test_plan_runs_out():
    """Pages that run out in the middle of a segment, tables that are too narrow, slots that are too few, lengths that mean nothing."""
    c = Cache([40, 0, 10, 33], 2, 2, 64, "bf16", 16, spare=4, room=2)
    check_plan(c, B.SLKV_PAGED_LENGTHS, [40, 35, 60, 64], [40, 35, 60, 64])
    c = Cache([40, 0, 10, 33], 2, 2, 64, "bf16", 16, spare=40, room=2)
    check_plan(c, B.SLKV_PAGED_LENGTHS, [1000, 7, -5, 33], [1000, 7, -5, 33])
    c = Cache([40, 0, 10, 33], 2, 2, 64, "bf16", 16, spare=40, room=2)
    check_plan(c, B.SLKV_PAGED_LENGTHS, [45, 20, 12, 60], [45, 20, 12, 60], n_slots=11)
    c = Cache([40, 0, 10, 33], 2, 2, 64, "bf16", 16, spare=40, room=2)
    check_plan(c, B.SLKV_PAGED_ADD, [9, 3], [49, 9, 13, 36], width=4)
    c = Cache([40, 0, 10, 33], 2, 2, 64, "bf16", 16, spare=40, room=2)
    check_plan(c, B.SLKV_PAGED_LENGTHS, [2 ** 31 - 1, -2 ** 31, 0, 1], [2 ** 31 - 1, -2 ** 31, 0, 1])
    c = Cache([40, 0, 10, 33], 2, 2, 64, "bf16", 16, spare=0, room=2)
    check_plan(c, B.SLKV_PAGED_ADD, [10, 10], [50, 10, 20, 43])


def test_plan_captured():
    """A replay takes the lengths that are there then."""
    c = Cache([5, 70, 16, 0], 2, 2, 64, "bf16", 16, spare=30, room=6)
    slots = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    add = dev([3, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.slkv_paged_plan(c.c, B.SLKV_PAGED_ADD, add, slots=slots)
    for _ in range(9):
        tables, lens, free, rows, fits = P.plan(c.host_tables, c.host_lens, c.host_free, 16, [
            x + (3 if i < 2 else 1) for i, x in enumerate(c.host_lens)])
        graph.replay()
        torch.cuda.synchronize()
        assert fits and c.lens.tolist() == lens and int(c.n_free) == len(free)
        assert [x for x in slots.flatten().tolist() if x >= 0] == slots_of(c, tables, rows)
        c.host_tables, c.host_lens, c.host_free = tables, lens, free


# ---- rows -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_write(d, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    c = Cache([10, 20, 0, 33, 16, 1], 3, 2, d, dtype, 16, spare=20, room=3)
    # a packed layer: padding and slots outside the pool are passed over
    k, v = (torch.randn(50, d, device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
    free = [p * 16 + i for p in c.host_free for i in range(16)]
    slots = free[:50]
    slots[7], slots[20], slots[21] = -1, c.n_pages * 16, 2 ** 31 - 1
    want = c.k.clone(), c.v.clone()
    for x, rows in zip(want, (k, v)):
        for i, s in enumerate(slots):
            if 0 <= s < c.n_pages * 16:
                x.view(-1, d)[s] = rows[i]
    B.slkv_paged_write(c.c, k, v, dev(slots + [-1, 3]))              # more slots than rows: those behind are padding
    assert torch.equal(c.k, want[0]) and torch.equal(c.v, want[1])
    # tokens by index, from strided rows
    wide = torch.randn(3, 2, 5, 2 * d, device="cuda", generator=g).to(DT[dtype])
    k, v = wide[..., :d].transpose(1, 2), wide[..., d:].transpose(1, 2)       # [3, 5, 2, d]
    take = [[4, 0, 2], [1, 1, 9], [-1, 3, 0]]
    slots = torch.tensor(free[60:78]).view(3, 2, 3)
    slots[0, 1, 2] = -1
    for s in range(3):
        for h in range(2):
            for r in range(3):
                t, at = take[s][r], int(slots[s, h, r])
                if 0 <= t < 5 and at >= 0:
                    want[0].view(-1, d)[at], want[1].view(-1, d)[at] = k[s, t, h], v[s, t, h]
    B.slkv_paged_write(c.c, k, v, slots.int().cuda(), take=dev(take))
    assert torch.equal(c.k, want[0]) and torch.equal(c.v, want[1])
    B.slkv_paged_write(c.c, k[:, :0], v[:, :0], slots.int().cuda())           # no tokens: nothing happens
    assert torch.equal(c.k, want[0])


def test_write_far_rows():
    """A pool whose rows pass 2^31 bytes and elements, and a token whose offset does."""
    n_pages = (1 << 31) // (128 * 128) + 3
    k_pages = torch.zeros(n_pages, 128, 128, dtype=torch.bfloat16, device="cuda")
    v_pages = torch.zeros_like(k_pages)
    c = B.make_paged_cache(k_pages, v_pages, dev([[0]]), dev([0]), torch.zeros(n_pages, dtype=torch.int32, device="cuda"), dev([0]), 1, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(3, 128, device="cuda", generator=g).bfloat16() for _ in range(2))
    slots = [n_pages * 128 - 1, 5, (1 << 31) // 128 + 1]
    B.slkv_paged_write(c, k, v, dev(slots))
    for i, s in enumerate(slots):
        assert torch.equal(k_pages.view(-1, 128)[s], k[i]) and torch.equal(v_pages.view(-1, 128)[s], v[i])
    assert int((k_pages.view(-1, 128).abs().amax(1) > 0).sum()) == 3
    far = k_pages.view(1, -1, 1, 128)                                   # tokens of one sequence, 2^24 + 384 of them
    take = dev([[n_pages * 128 - 1, 5]])
    dst = torch.zeros(1, 16, 128, dtype=torch.bfloat16, device="cuda")
    c2 = B.make_paged_cache(dst, torch.zeros_like(dst), dev([[0]]), dev([0]), dev([0]), dev([0]), 1, 1)
    B.slkv_paged_write(c2, far, far, dev([2, 3]), take=take)
    assert torch.equal(dst[0, 2], k[0]) and torch.equal(dst[0, 3], k[1])
    # attention over the far pages
    q = torch.randn(1, 1, 4, 128, device="cuda", generator=g).bfloat16()
    out = torch.zeros_like(q)
    c3 = B.make_paged_cache(k_pages, v_pages, dev([[n_pages - 1]]), dev([128]), torch.zeros(n_pages, dtype=torch.int32, device="cuda"), dev([0]), 1, 1)
    p = B.make_paged_attend(c3, q, out)
    B.slkv_paged_attend(c3, p, q, out, B.new_paged_workspace(c3, p))
    for h in range(4):
        R.check(out[0, :, h], None, R.rows(q[0, :, h], k_pages[-1], v_pages[-1], torch.ones(1, 128, dtype=torch.bool, device="cuda"), 128 ** -0.5), True, 128)


# ---- attention ----------------------------------------------------------------------------------------------------------------
def tree_masks(n_seqs, n, seed):
    r = random.Random(seed)
    out = []
    for _ in range(n_seqs):
        m = []
        for i in range(n):
            parent = r.randint(-1, i - 1)
            m.append((m[parent] if parent >= 0 else 0) | 1 << i)
        out.append(m)
    return out


def signed(masks):
    return dev([[x - (1 << 64) if x >> 63 else x for x in m] for m in masks], torch.int64)


def attend(c, G, n, masks=None, counts=None, new=True, layer=0, seed=0, heads_first=False, scale=None, edit=None, log2=False):
    g = torch.Generator(device="cuda").manual_seed(seed + 1)

    def rows(heads):
        x = torch.randn(c.n_seqs, n, heads, c.d, device="cuda", generator=g).to(DT[c.dtype])
        return x.transpose(1, 2).contiguous().transpose(1, 2) if heads_first else x
    q, k, v = rows(c.hkv * G), rows(c.hkv), rows(c.hkv)
    if edit is not None:
        edit(q, k, v)
    out = torch.full_like(q, 7.0)
    lse = torch.full((c.n_seqs, c.hkv * G, n), 5.0, device="cuda")
    p = B.make_paged_attend(c.c, q, out, *((k, v) if new else ()), layer=layer, scale=scale,
                            lse_units=B.SLKV_LSE_LOG2 if log2 else B.SLKV_LSE_LN)
    ws = B.new_paged_workspace(c.c, p)
    ws.fill_(0xff)
    status = dev([0])
    B.slkv_paged_attend(c.c, p, q, out, ws, *((k, v) if new else ()), tree=None if masks is None else signed(masks),
                        n_new=None if counts is None else dev(counts), lse=lse, status=status)
    torch.cuda.synchronize()
    return q, k, v, out, lse, status


def check_attend(c, G, n, masks=None, counts=None, new=True, layer=0, scale=None, log2=False, **kw):
    q, k, v, out, lse, status = attend(c, G, n, masks, counts, new, layer, scale=scale, log2=log2, **kw)
    assert int(status) == 0
    if log2:
        lse = lse * 0.6931471805599453
    for s in range(c.n_seqs):
        t = n if counts is None else max(0, min(counts[s], n))
        drafted = torch.tensor([[bool(masks[s][i] >> j & 1) if masks is not None else j <= i for j in range(t)] for i in range(t)],
                               dtype=torch.bool, device="cuda").view(t, t)
        for h in range(c.hkv):
            rk, rv = c.rows((layer * c.n_seqs + s) * c.hkv + h)
            see = torch.ones(t, rk.shape[0], dtype=torch.bool, device="cuda")
            if new:
                rk, rv, see = torch.cat([rk, k[s, :t, h]]), torch.cat([rv, v[s, :t, h]]), torch.cat([see, drafted], 1)
            for qh in range(h * G, h * G + G):
                ref = R.rows(q[s, :t, qh], rk, rv, see, c.d ** -0.5 if scale is None else scale)
                R.check(out[s, :t, qh], lse[s, qh, :t], ref, c.dtype == "bf16", c.d)
        assert (out[s, t:] == 7.0).all() and (lse[s, :, t:] == (5.0 * 0.6931471805599453 if log2 else 5.0)).all()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page_rows", [16, 32, 64, 128])
def test_attend_lengths(d, dtype, page_rows):
    """Segments without rows, of one, ends inside pages and tiles, several tiles."""
    lens = [0, 1, 15, 16, 17, 127, 128, 129, 300, 64, 700, 255]
    c = Cache(lens, 6, 2, d, dtype, page_rows, junk=float("nan"))
    check_attend(c, 4, 1)
    check_attend(c, 4, 1, new=False)
    check_attend(c, 4, 5, tree_masks(6, 5, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,n", [(1, 64), (2, 33), (3, 7), (4, 32), (4, 33), (8, 64), (16, 3), (64, 2), (5, 64), (1, 1)])
def test_attend_groups_and_trees(G, n, dtype):
    """One block of query rows, two, several units; masks of 64 bits."""
    c = Cache([200, 0, 513, 90], 2, 2, 128, dtype, 32, junk=float("inf"))
    check_attend(c, G, n, tree_masks(2, n, G))
    check_attend(c, G, n, counts=[n // 2 + 1, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_masks_of_any_kind(dtype):
    """Tokens that see nothing at all, later tokens, not themselves; bits behind the last token; counts out of range."""
    c = Cache([0, 0, 40, 0, 0, 130], 3, 2, 64, dtype, 16, junk=float("nan"))
    masks = [[0, 1 << 5, 0b111111, 0, 1 << 63 | 1, 2], [0] * 6, [(1 << 64) - 1] * 6]
    check_attend(c, 4, 6, masks)
    check_attend(c, 4, 6, masks, counts=[4, 9, -3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_values_that_are_not_finite(dtype):
    """In the cache they reach every token, in drafted rows those that see them, in padding nobody."""
    c = Cache([200, 300, 0, 128], 2, 2, 128, dtype, 32, junk=float("nan"), seed=3)
    c.v.view(-1, 128)[c.host_tables[1][3] * 32 + 5, 9] = float("inf")

    def edit(q, k, v):
        v[0, 2, :, 4], v[0, 5, :, 4], v[1, 3, :, 100] = float("nan"), float("inf"), -float("inf")
        k[0, 6:], v[0, 6:] = float("nan"), float("nan")
    check_attend(c, 4, 8, tree_masks(2, 8, 4), counts=[6, 8], edit=edit)
    check_attend(c, 16, 8, tree_masks(2, 8, 5), counts=[6, 8])

    def hidden(q, k, v):                                                # a drafted key that is NaN, seen by itself alone
        k[:, 4] = float("nan")
    masks = [[1 << i for i in range(8)]] * 2
    q, k, v, out, lse, _ = attend(c, 4, 8, masks, edit=hidden)
    assert torch.isnan(out[:, 4]).all() and not torch.isnan(out[1, [0, 1, 2, 3, 5, 6, 7]]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_layers_and_strides(dtype):
    r = random.Random(5)
    c = Cache([r.randint(0, 400) for _ in range(3 * 4 * 2)], 4, 2, 64, dtype, 32)
    for layer in (0, 2):
        check_attend(c, 4, 3, layer=layer, heads_first=layer == 2, log2=layer == 2, scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_many_pieces(dtype):
    """Long segments over many CTAs, and more segments than CTAs."""
    check_attend(Cache([9001, 5000], 1, 2, 128, dtype, 64), 4, 2)
    check_attend(Cache([30001], 1, 1, 64, dtype, 128), 8, 1)
    r = random.Random(6)
    check_attend(Cache([r.randint(0, 300) for _ in range(150 * 3)], 150, 3, 64, dtype, 16), 2, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_bad_pages_and_lengths(dtype):
    """Pages outside the pool are pages of zeros, and the status says so; lengths beyond the tables are cut."""
    c = Cache([100, 50], 1, 2, 64, dtype, 16, room=0)
    good = c.tables.clone()
    c.tables[0, 3], c.tables[0, 5] = c.n_pages, -5
    c.lens[0] = 2 ** 31 - 1
    c.lens[1] = -4
    q, k, v, out, lse, status = attend(c, 4, 1, new=False)
    assert int(status) == B.ERR["BAD_SHAPE"]
    c.tables.copy_(good)
    rk, rv = c.rows(0)
    assert rk.shape[0] == c.max_pages * 16
    rk, rv = rk.clone(), rv.clone()
    for i in (3, 5):
        rk[16 * i:16 * i + 16], rv[16 * i:16 * i + 16] = 0, 0
    for h in range(4):
        see = torch.ones(1, rk.shape[0], dtype=torch.bool, device="cuda")
        R.check(out[0, :, h], lse[0, h], R.rows(q[0, :, h], rk, rv, see, 0.125), dtype == "bf16", 64)
    assert (out[0, :, 4:] == 0).all() and torch.isinf(lse[0, 4:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_captured_and_repeated(dtype):
    c = Cache([900, 400, 77, 0], 2, 2, 128, dtype, 32)
    q, k, v, want, lse, _ = attend(c, 4, 3)
    for _ in range(2):
        assert torch.equal(attend(c, 4, 3)[3], want)
    out = torch.zeros_like(want)
    p = B.make_paged_attend(c.c, q, out, k, v)
    ws = B.new_paged_workspace(c.c, p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.slkv_paged_attend(c.c, p, q, out, ws, k, v)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    c.lens.copy_(dev([100, 0, 70, 0]))                                   # a replay takes the lengths that are there then
    graph.replay()
    torch.cuda.synchronize()
    c2 = attend(c, 4, 3)[3]
    assert torch.equal(out, c2)


# ---- the whole way ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_to_accepted_tokens(dtype):
    """prompt attention -> compression with its log-sum-exps -> pages -> a tree of drafted tokens -> the accepted ones into the pages,
    against the same rows attended to in 64 bits."""
    ns, hkv, G, d, w, nq = 2, 4, 4, 128, 16, [300, 150]
    g = torch.Generator(device="cuda").manual_seed(20)
    t = sum(nq)
    q, k, v = (torch.randn(t, h, d, device="cuda", generator=g).to(DT[dtype]) for h in (hkv * G, hkv, hkv))
    cu = [0, nq[0], t]
    cu_dev = dev(cu)
    out, lse = torch.zeros_like(q), torch.zeros(ns, hkv * G, w, device="cuda")
    p = B.make_prompt(q, k, v, out, ns, window=w)
    B.slkv_prompt_attend(p, q, k, v, cu_dev, cu, out, B.new_prompt_workspace(p, cu), lse=lse)
    q_win = torch.stack([q[e - w:e] for e in cu[1:]])
    params = B.make_params(q_win, k, v, w, 5, softmax_domain=B.SLKV_ALL_CAUSAL)
    cap = B.slkv_packed_rows_upper_bound(params, cu)
    ko, vo = (torch.zeros(cap, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    offsets, kept = torch.zeros(ns * hkv + 1, dtype=torch.int32, device="cuda"), torch.zeros(cap, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.slkv_workspace_bytes_overlapped(params, cu), dtype=torch.uint8, device="cuda")
    # queued: planning and writing send it out
    B.slkv_compress_overlapped(params, q_win, k, v, cu_dev, cu, dev([60, 100, 33, 250]), ko, vo, offsets, kept, ws, None, None, lse=lse)
    c = Cache([0] * (ns * hkv), ns, hkv, d, dtype, 16, spare=200, room=40)
    slots, so = torch.full((cap,), -1, dtype=torch.int32, device="cuda"), torch.zeros(ns * hkv + 1, dtype=torch.int32, device="cuda")
    B.slkv_paged_plan(c.c, B.SLKV_PAGED_OFFSETS, offsets, slots=slots, slot_offsets=so)
    B.slkv_paged_write(c.c, ko, vo, slots)
    torch.cuda.synchronize()
    assert torch.equal(so, offsets)
    for seg in range(ns * hkv):
        a, b = offsets[seg].item(), offsets[seg + 1].item()
        s, h = divmod(seg, hkv)
        rows = cu[s] + kept[a:b].long()
        rk, rv = c.rows(seg)
        assert torch.equal(rk, k[rows, h]) and torch.equal(rv, v[rows, h])
    # a tree, then what was accepted of it
    masks = tree_masks(ns, 6, 2)
    check_attend(c, G, 6, masks, seed=30)
    _, kn, vn, _, _, _ = attend(c, G, 6, masks, seed=30)
    take, accepted = dev([[0, 2, 5, 0], [1, 3, 0, 0]]), dev([3, 2])
    slots = torch.zeros(ns * hkv, 4, dtype=torch.int32, device="cuda")
    old = [c.rows(seg) for seg in range(ns * hkv)]
    B.slkv_paged_plan(c.c, B.SLKV_PAGED_ADD, accepted, slots=slots)
    B.slkv_paged_write(c.c, kn, vn, slots, take=take)
    for seg in range(ns * hkv):
        s, h = divmod(seg, hkv)
        idx = take[s, :accepted[s]].long()
        rk, rv = c.rows(seg)
        assert torch.equal(rk, torch.cat([old[seg][0], kn[s, idx, h]])) and torch.equal(rv, torch.cat([old[seg][1], vn[s, idx, h]]))
    check_attend(c, G, 1, seed=31)


def test_attend_far_rows_in_fp32():
    """Pages whose offsets pass 2^31 elements and 2^33 bytes."""
    n_pages = (1 << 31) // (128 * 64) + 3
    k_pages = torch.zeros(n_pages, 128, 64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    k_pages[-2:] = torch.randn(2, 128, 64, device="cuda", generator=g)
    c = B.make_paged_cache(k_pages, k_pages, dev([[n_pages - 1, 0, n_pages - 2]]), dev([384]), torch.zeros(n_pages, dtype=torch.int32, device="cuda"),
                           dev([0]), 1, 1)
    q = torch.randn(1, 1, 4, 64, device="cuda", generator=g)
    out = torch.zeros_like(q)
    p = B.make_paged_attend(c, q, out)
    B.slkv_paged_attend(c, p, q, out, B.new_paged_workspace(c, p))
    rows = torch.cat([k_pages[-1], k_pages[0], k_pages[-2]])
    for h in range(4):
        R.check(out[0, :, h], None, R.rows(q[0, :, h], rows, rows, torch.ones(1, 384, dtype=torch.bool, device="cuda"), 0.125), False, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_a_wait_that_runs_out(dtype):
    c = Cache([3000, 200, 1700, 900], 2, 2, 64, dtype, 32)
    q, k, v, good, lse, _ = attend(c, 4, 3)
    out, status = torch.full_like(good, 7.0), dev([0])
    p = B.make_paged_attend(c.c, q, out, k, v)
    ws = B.new_paged_workspace(c.c, p)
    B.slkv_debug_expire_next_wait(5)
    B.slkv_paged_attend(c.c, p, q, out, ws, k, v, status=status)
    torch.cuda.synchronize()
    assert int(status) == B.ERR["DEVICE_TIMEOUT"]
    fine = (out == good) | (out == 7.0) | torch.isnan(out)
    assert fine.all() and not torch.equal(out, good)
    status.zero_()
    B.slkv_paged_attend(c.c, p, q, out, ws, k, v, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(out, good)


@pytest.mark.parametrize("sizes", [(1, 5, 700), (3, 11, 300), (8, 8, 64), (1, 40, 33)])
def test_plan_few_segments_of_many_pages(sizes):
    """Warps that share the pages of few segments; clusters where whole segments come and go; back again, and in part."""
    ns, hkv, most = sizes
    r = random.Random(sum(sizes))
    n_seg = ns * hkv
    pages = 16
    full = [r.randint(0, most * pages) for _ in range(n_seg)]
    c = Cache([0] * n_seg, ns, hkv, 64, "bf16", pages, spare=n_seg * most, room=most)
    before = c.tables.clone(), c.free.clone(), c.n_free.clone()
    slots, so = torch.full((sum(full) + 5,), 9, dtype=torch.int32, device="cuda"), torch.zeros(n_seg + 1, dtype=torch.int32, device="cuda")
    status = dev([0])
    B.slkv_paged_plan(c.c, B.SLKV_PAGED_LENGTHS, dev(full), slots=slots, slot_offsets=so, status=status)
    assert int(status) == 0 and c.lens.tolist() == full
    tables, got, taken = c.tables.cpu(), slots.tolist(), []
    for s, n in enumerate(full):
        need = -(-n // pages)
        taken += tables[s, :need].tolist()
        assert got[int(so[s]):int(so[s]) + n] == [int(tables[s, i // pages]) * pages + i % pages for i in range(n)]
    assert got[sum(full):] == [-1] * 5
    stack = before[1].tolist()[:int(before[2])]
    assert taken == stack[::-1][:len(taken)]                              # from the top, in order
    assert int(c.n_free) == len(stack) - len(taken)
    half = [n // 2 for n in full]
    B.slkv_paged_plan(c.c, B.SLKV_PAGED_LENGTHS, dev(half))
    assert c.lens.tolist() == half
    B.slkv_paged_plan(c.c, B.SLKV_PAGED_LENGTHS, dev(full))
    assert torch.equal(c.tables.cpu(), tables)                            # taking and returning are each other's inverse
    B.slkv_paged_plan(c.c, B.SLKV_PAGED_LENGTHS, dev([0] * n_seg))
    assert torch.equal(c.free, before[1]) and torch.equal(c.n_free, before[2])
