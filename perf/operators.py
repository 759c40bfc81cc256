"""What happens to a compressed cache in decoding, as cases that can be timed: packing rows into 4 bits, attention over
the packed rows, eviction by accumulated attention weight.  Each case has a plain form in elementary torch operations and
the calls a user makes of this library.

A cache: segment seg = sequence * n_kv_heads + KV head owns the slots starts[seg] .. starts[seg + 1] - 1, the first lens[seg]
of them filled.  A slot has a record (both rows in 4 bits), a position in its sequence and an accumulated weight.  A record
holds d/2 bytes of K codes, d/2 bytes of V codes, then d/32 bf16 each of K scales, K zeros, V scales and V zeros; channel
32 j + i of a row has value zero[j] + scale[j] * code.
  K codes  32-bit word t * (d/32) + j: channels 32 j + 8 t + e, e = 0 .. 7, in the word's nibbles, lowest first (t < 4)
  V codes  16-bit unit g * (d/32) + j: channels 32 j + 4 g + e, e = 0 .. 3, likewise (g < 8)
"""
import math
import random

import torch

own = False
DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DENSE_TAIL = 32            # the newest rows of a segment are always kept: their positions have no gaps


# ---- the cases ---------------------------------------------------------------------------------------------------
def _case(kind, **kw):
    """Defaults: a Llama-3-8B / Mistral-7B layer (32 query heads, 8 KV heads, head_dim 128, bf16)."""
    c = dict(kind=kind, n_seqs=1, n_kv_heads=8, group=4, head_dim=128, dtype="bf16", n_tokens=1, len_min=512, len_max=512,
             idle=False, masked=False, softcap=0.0, slopes=False, accumulate=False, decay=1.0, budget=512, window=32)
    c.update(kw)
    return c


def listed():
    return [
        # one decode step's new rows of a batch go into the cache
        _case("append", name="append-16", n_seqs=16, len_min=200, len_max=1024),
        # a short prompt's compressed layer, packed once behind the prefill
        _case("pack", name="pack-512", len_min=129, len_max=1031),
        # the same in fp32 with narrow heads, odd lengths, one token's draft behind it
        _case("pack", name="pack-f32-d64", n_seqs=3, n_kv_heads=6, head_dim=64, dtype="f32", len_min=77, len_max=4001),
        # a batch of long prompts that kept much
        _case("pack", name="pack-batch", n_seqs=16, len_min=2000, len_max=12000),
        # one user's decode step over a compressed cache: latency counts
        _case("attend", name="attend-512", len_min=129, len_max=1031),
        # an ordinary serving batch: budgets that differ per head, one sequence idle, weights accumulated for the eviction
        _case("attend", name="attend-batch", n_seqs=32, len_min=256, len_max=4096, idle=True, accumulate=True),
        # four drafted tokens verified at once, fp32, narrow heads, every head with keys of its own
        _case("attend", name="attend-draft-f32", n_seqs=5, n_kv_heads=12, group=1, head_dim=64, dtype="f32", n_tokens=4,
              len_min=33, len_max=3001, masked=True),
        # capped scores with a bias by distance (positions of kept rows are far apart), decaying weights
        _case("attend", name="attend-biased", n_seqs=8, group=8, len_min=700, len_max=6000, masked=True, softcap=30.0,
              slopes=True, accumulate=True, decay=0.97),
        # the largest: long contexts kept whole in 4 bits
        _case("attend", name="attend-long", n_seqs=8, len_min=20000, len_max=65536),
        # a decode step's update of a cache that stands at its budget: one row in, one row out, in place
        _case("step", name="evict-step", n_seqs=16, len_min=480, len_max=2048),
        # after a prompt's second turn: down to two thirds, into a cache with other room per head
        _case("evict", name="evict-batch", n_seqs=32, len_min=600, len_max=2400, budget=1024),
        # a long conversation down to a fixed budget
        _case("evict", name="evict-long", n_seqs=4, len_min=20000, len_max=65000, budget=16384, window=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "pack", "pack", "attend", "attend", "attend", "attend", "step", "evict", "evict"])
    n_kv = rng.choice([1, 2, 4, 8, 8, 12])
    n_seqs = _log_int(rng, 1, 48)
    most = {"append": 1 << 18, "pack": 700000, "attend": 1500000, "step": 1 << 18, "evict": 600000}[kind]
    top = max(40, min(_log_int(rng, 64, 65536), most // (n_seqs * n_kv)))
    c = _case(kind, n_seqs=n_seqs, n_kv_heads=n_kv, group=rng.choice([1, 2, 4, 4, 6, 8, 16]), head_dim=rng.choice([64, 128, 128]),
              dtype=rng.choice(["bf16", "bf16", "f32"]), len_max=top, len_min=max(1, top // rng.choice([1, 2, 8, 40])),
              n_tokens=rng.choice([1, 1, 1, 2, 5, 8]))
    if kind == "attend":
        c.update(idle=rng.random() < 0.2, masked=rng.random() < 0.4 or c["n_tokens"] > 1, accumulate=rng.random() < 0.4,
                 softcap=rng.choice([0.0, 0.0, 20.0, 50.0]), decay=rng.choice([1.0, 0.9]))
        c["slopes"] = c["masked"] and rng.random() < 0.4
    if kind in ("evict", "step"):
        c.update(window=rng.choice([1, 16, 32, 64]), budget=max(1, int(top * rng.uniform(0.1, 0.9))), dtype="bf16")
    if kind == "step":
        c.update(len_min=max(c["len_min"], c["window"]), len_max=max(c["len_max"], c["window"]), n_tokens=1)
    return c


# ---- sizes that follow from a case ---------------------------------------------------------------------------------
def _lens(c):
    """Filled slots per segment: from len_min to len_max over their logarithm, both among them; an idle batch has one
    sequence without any."""
    r = random.Random(c["n_seqs"] * 7919 + c["n_kv_heads"] * 31 + c["len_max"])
    n = c["n_seqs"] * c["n_kv_heads"]
    lens = [_log_int(r, c["len_min"], c["len_max"]) for _ in range(n)]
    lens[0] = c["len_max"]
    if n > 1:
        lens[1] = c["len_min"]
    if c["idle"] and c["n_seqs"] > 1:
        lens[-c["n_kv_heads"]:] = [0] * c["n_kv_heads"]
    return lens


def _record_bytes(d):
    return d + d // 4


def _starts(lens, room):
    """Every segment has `room` slots more than it fills, some one more or two."""
    s = [0]
    for i, n in enumerate(lens):
        s.append(s[-1] + n + room + i % 3)
    return s


def _kept(c, lens):
    return [min(n, max(b, c["window"])) for n, b in zip(lens, [b for _ in range(c["n_seqs"]) for b in _budgets(c, lens)])]


def _budgets(c, lens):
    """Per KV head: around the case's budget; of a step, what the first sequence's heads hold."""
    if c["kind"] == "step":
        return [max(lens[h::c["n_kv_heads"]]) for h in range(c["n_kv_heads"])]
    r = random.Random(c["budget"])
    return [max(1, int(c["budget"] * r.uniform(0.5, 1.5))) for _ in range(c["n_kv_heads"])]


def work(case):
    c = case
    d, e, lens = c["head_dim"], 4 if c["dtype"] == "f32" else 2, _lens(c)
    if c["kind"] == "step":
        lens = _step_lens(c)
    rows, rec, n_seg = sum(lens), _record_bytes(d), len(lens)
    slot = rec + 8                                                   # record, position, weight
    if c["kind"] == "append":
        new = n_seg * c["n_tokens"]
        return {"bytes": new * (2 * d * e + slot + rec + 4 * d) + 8 * n_seg, "flops": new * 2 * d * 8}
    if c["kind"] == "pack":
        return {"bytes": rows * (2 * d * e + 4 + slot + rec + 4 * d) + 12 * n_seg, "flops": rows * 2 * d * 8}
    if c["kind"] == "attend":
        r = c["group"] * c["n_tokens"]
        moved = rows * (rec + (4 if c["masked"] else 0) + (8 if c["accumulate"] else 0)) + n_seg * r * (2 * d * e + 4)
        return {"bytes": moved, "flops": rows * r * d * 4 + rows * 2 * d * 2}
    if c["kind"] == "step":
        return {"bytes": rows * 8 + n_seg * (2 * d * e + 3 * slot), "flops": rows * 4}
    return {"bytes": rows * 8 + sum(_kept(c, lens)) * 2 * slot, "flops": rows * 4}


# ---- the 4-bit format in torch -------------------------------------------------------------------------------------
def _up(x):
    """Non-negative fp32 -> the next bf16 not below it, as fp32."""
    return ((x.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)


def _down(x):
    """fp32 -> the next bf16 not above it, as fp32."""
    b = x.view(torch.int32)
    return torch.where(b < 0, (b + 0xFFFF) & -65536, b & -65536).view(torch.float32)


def _quantise(x):
    """[rows, d] -> codes [rows, d/32, 32] as fp32, scale and zero [rows, d/32] as fp32 (bf16 values)."""
    g = x.float().unflatten(1, (-1, 32))
    zero = _down(g.amin(2))
    span = g.amax(2) - zero
    fine = torch.isfinite(span)
    span, zero = torch.where(fine, span, 0.0), torch.where(fine, zero, 0.0)
    scale = _up(span / torch.full_like(span, 15.0))                  # divided, not multiplied by 1/15: exact shares stay exact
    code = torch.round((g - zero[:, :, None]) / torch.where(scale > 0, scale, 1.0)[:, :, None]).clamp(0.0, 15.0)
    code = torch.where((fine & (scale > 0))[:, :, None], code, 0.0)
    nan = torch.tensor(float("nan"), device=x.device)
    return code, torch.where(fine, scale, nan), torch.where(fine, zero, nan)


def _encode(k, v):
    """Rows [rows, d] -> records [rows, record bytes]."""
    n, d = k.shape
    ng = d // 32
    parts = []
    (ck, sk, zk), (cv, sv, zv) = _quantise(k), _quantise(v)
    ck = ck.to(torch.uint8).view(n, ng, 4, 8).permute(0, 2, 1, 3).reshape(n, d)            # channel order t, j, e
    cv = cv.to(torch.uint8).view(n, ng, 8, 4).permute(0, 2, 1, 3).reshape(n, d)            # channel order g, j, e
    for c in (ck, cv):
        parts.append(c[:, 0::2] | (c[:, 1::2] << 4))
    for s in (sk, zk, sv, zv):
        parts.append(s.bfloat16().view(torch.uint8))
    return torch.cat(parts, 1)


def _decode(rec, d):
    """Records [..., record bytes] -> the K and V rows they stand for, fp32 [..., d]."""
    ng, lead = d // 32, rec.shape[:-1]
    s = rec[..., d:].contiguous().view(torch.bfloat16).float().unflatten(-1, (4, ng))
    out = []
    for at, units, lane in ((0, 4, 8), (d // 2, 8, 4)):
        b = rec[..., at:at + d // 2]
        code = torch.stack([b & 15, b >> 4], -1).reshape(*lead, units, ng, lane).transpose(-3, -2).float()
        i = 0 if at == 0 else 2
        x = code * s[..., i, :, None, None] + s[..., i + 1, :, None, None]
        out.append(x.reshape(*lead, d))
    return out


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _step_lens(c):
    """A cache at its budget: every segment of a head holds what the head may hold."""
    return _budgets(c, _lens(c)) * c["n_seqs"]


def _rows(g, seg, slot, u, d):
    """K and V rows: channels with offsets of their own, a sink and some needles along the direction u that the segment's
    queries share."""
    n = seg.numel()
    k = torch.randn(n, d, device=DEVICE, generator=g)
    k += 2.0 * torch.sin(torch.arange(d, device=DEVICE) * 1.7)
    hit = (slot == 0) | (torch.rand(n, device=DEVICE, generator=g) < 0.01)
    k += torch.where(hit, 1.0, 0.0)[:, None] * u[seg]
    return k, torch.randn(n, d, device=DEVICE, generator=g)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    d, hkv, ns, dt, nt = c["head_dim"], c["n_kv_heads"], c["n_seqs"], DTYPES[c["dtype"]], c["n_tokens"]
    lens = _step_lens(c) if c["kind"] == "step" else _lens(c)
    n_seg, width = len(lens), max(lens) + nt
    starts = _starts(lens, nt)
    total = starts[-1]
    dev = lambda v, t=torch.int32: torch.tensor(v, dtype=t, device=DEVICE)      # noqa: E731
    st = dict(case=c, width=width, total=total, starts=dev(starts), lens=dev(lens))
    u = torch.randn(n_seg, d, device=DEVICE, generator=g)

    # positions: the newest of a sequence's rows is at newest[s] in every head, gaps of 1 to 7 before the last rows
    newest = 8 * width + 100 + torch.randint(0, 50, (ns,), device=DEVICE, generator=g)
    st["newest"] = newest.int()
    seg = torch.repeat_interleave(torch.arange(n_seg, device=DEVICE), dev(lens, torch.int64))
    slot = torch.arange(seg.numel(), device=DEVICE) - torch.repeat_interleave(
        torch.cumsum(dev(lens, torch.int64), 0) - dev(lens, torch.int64), dev(lens, torch.int64))
    back = dev(lens, torch.int64)[seg] - 1 - slot                    # rows behind this one
    jump = torch.randint(0, 7, (seg.numel(),), device=DEVICE, generator=g)
    pos = newest[seg // hkv] - back - torch.where(back >= DENSE_TAIL, 6 * (back - DENSE_TAIL) + jump, 0)
    at = dev(starts, torch.int64)[seg] + slot

    # one slot more than the cache has: where the plain forms put what goes nowhere
    st["records"] = torch.zeros(total + 1, _record_bytes(d), dtype=torch.uint8, device=DEVICE)
    st["pos"] = torch.zeros(total + 1, dtype=torch.int32, device=DEVICE)
    st["weight"] = torch.zeros(total + 1, dtype=torch.float32, device=DEVICE)
    if c["kind"] == "pack":
        k, v = _rows(g, seg, slot, u, d)
        st.update(k=k.to(dt), v=v.to(dt), kept_idx=pos.int(), offsets=dev([0] + torch.tensor(lens).cumsum(0).tolist()),
                  slots=at.int())
        st["lens"] = torch.zeros(n_seg, dtype=torch.int32, device=DEVICE)
    else:
        for i in range(0, seg.numel(), 1 << 18):
            part = slice(i, i + (1 << 18))
            st["records"][at[part]] = _encode(*_rows(g, seg[part], slot[part], u, d))
        st["pos"][at] = pos.int()
        # what heads that look at few rows leave behind: most weights small, some large
        st["weight"][at] = torch.exp(2.0 * torch.randn(seg.numel(), device=DEVICE, generator=g))
    if c["kind"] in ("append", "step"):
        new = [x.reshape(ns, hkv, nt, d).transpose(1, 2).contiguous().to(dt) for x in _rows(
            g, torch.arange(n_seg, device=DEVICE).repeat_interleave(nt), torch.ones(n_seg * nt, device=DEVICE), u, d)]
        st.update(k=new[0], v=new[1], new_pos=(newest[:, None] + 1 + torch.arange(nt, device=DEVICE)).int())
        st["slots"] = (dev(starts)[:-1, None] + dev(lens)[:, None] + dev(list(range(nt)))).reshape(-1).int()
        st["lens_out"] = torch.zeros(n_seg, dtype=torch.int32, device=DEVICE)
    if c["kind"] in ("append", "pack"):
        st["k_out"], st["v_out"] = (torch.empty(st["slots"].numel(), d, dtype=torch.bfloat16, device=DEVICE) for _ in range(2))
    if c["kind"] == "attend":
        hq = hkv * c["group"]
        q = 0.7 * u.view(ns, 1, hkv, 1, d) + 0.7 * torch.randn(ns, nt, hkv, c["group"], d, device=DEVICE, generator=g)
        st["q"] = q.reshape(ns, nt, hq, d).to(dt)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(ns, hq, nt, dtype=torch.float32, device=DEVICE)
        st["q_pos"] = (newest[:, None] - (nt - 1) + torch.arange(nt, device=DEVICE)).int()
        st["slopes"] = torch.exp2(-8.0 * (torch.arange(hq, device=DEVICE) + 1) / hq)
    if c["kind"] in ("evict", "step"):
        st["budgets"] = dev(_budgets(c, lens))
        if c["kind"] == "step":
            st["newest"] = st["newest"] + 1
        else:
            kept = _kept(c, lens)
            to = _starts(kept, 5)
            st["to"] = dict(starts=dev(to), lens=torch.zeros(n_seg, dtype=torch.int32, device=DEVICE), total=to[-1])
            for name in ("records", "pos", "weight"):
                st["to"][name] = torch.zeros(to[-1] + 1, *st[name].shape[1:], dtype=st[name].dtype, device=DEVICE)
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _padded(st, lens):
    """Slot indices [segments, width], and which of them are filled."""
    n = torch.arange(st["width"], device=DEVICE)
    idx = st["starts"][:-1, None].long() + n
    return idx.clamp(max=st["total"]), n < lens[:, None]


def _plain_append(st, lens, lens_out):
    nt, d = st["case"]["n_tokens"], st["case"]["head_dim"]
    rows = [st[x].transpose(1, 2).reshape(-1, d) for x in ("k", "v")]
    at = (st["starts"][:-1, None].long() + lens[:, None] + torch.arange(nt, device=DEVICE)).reshape(-1)
    st["records"][at] = _encode(*rows)
    st["pos"][at] = st["new_pos"][:, None].expand(-1, st["case"]["n_kv_heads"], -1).reshape(-1)
    st["weight"][at] = 0.0
    lens_out.copy_(lens + nt)


def _plain_pack(st):
    n = st["offsets"][1:] - st["offsets"][:-1]
    i = torch.arange(st["k"].shape[0], device=DEVICE)
    seg = torch.bucketize(i, st["offsets"][1:].long(), right=True)
    at = st["starts"][seg].long() + i - st["offsets"][seg]
    st["records"][at] = _encode(st["k"], st["v"])
    st["pos"][at] = st["kept_idx"]
    st["weight"][at] = 0.0
    st["lens"].copy_(n)


def _plain_attend(st):
    c = st["case"]
    ns, hkv, G, nt, d = c["n_seqs"], c["n_kv_heads"], c["group"], c["n_tokens"], c["head_dim"]
    idx, filled = _padded(st, st["lens"])
    k, v = _decode(st["records"][idx], d)
    q = st["q"].float().view(ns, nt, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(ns * hkv, G * nt, d)
    s = torch.matmul(q, k.transpose(1, 2)).view(ns, hkv, G, nt, -1) * (1.0 / math.sqrt(d))
    if c["softcap"]:
        s = c["softcap"] * torch.tanh(s / c["softcap"])
    visible = filled.view(ns, hkv, 1, 1, -1)
    if c["masked"]:
        away = st["pos"][idx].view(ns, hkv, 1, 1, -1) - st["q_pos"].view(ns, 1, 1, nt, 1)
        if c["slopes"]:
            s = s + st["slopes"].view(1, hkv, G, 1, 1) * away
        visible = visible & (away <= 0)
    s = torch.where(visible, s, -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    p = p / torch.where(z > 0, z, 1.0)
    st["lse"].copy_((m + torch.log(z)).reshape(ns, hkv * G, nt))
    o = torch.matmul(p.reshape(ns * hkv, G * nt, -1), v)
    st["out"].copy_(o.view(ns, hkv, G, nt, d).permute(0, 3, 1, 2, 4).reshape(ns, nt, hkv * G, d))
    got = {"out": st["out"], "lse": st["lse"]}
    if c["accumulate"]:
        seen = p.sum((2, 3)).view(ns * hkv, -1) / G
        new = c["decay"] * st["weight"][idx] + seen
        st["weight"][torch.where(filled, idx, st["total"])] = new
        got["weight"] = st["weight"][:-1]
    return got


def _plain_evict(st, to, hkv, window, lens):
    idx, filled = _padded(st, lens)
    n_seg, width = idx.shape
    slot = torch.arange(width, device=DEVICE)
    w, pos = st["weight"][idx] + 0.0, st["pos"][idx]
    bits = w.view(torch.int32).long()
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
    key = torch.where(torch.isnan(w), -(1 << 33), key)
    newest = st["newest"].repeat_interleave(hkv)
    key = torch.where(pos > newest[:, None] - window, 1 << 33, key)
    key = torch.where(filled, key, -(1 << 40))
    rank = torch.empty_like(idx).scatter_(1, torch.argsort(key, dim=1, descending=True, stable=True), slot.expand(n_seg, -1))
    budget = st["budgets"].repeat(n_seg // hkv)
    kept = torch.minimum(lens, budget.clamp(min=window))
    keep, inside = rank < kept[:, None], slot < kept[:, None]
    hole, mover = inside & ~keep, keep & ~inside
    table = torch.zeros(n_seg, width + 1, dtype=torch.long, device=DEVICE)
    table.scatter_(1, torch.where(mover, mover.cumsum(1) - 1, width), slot.expand(n_seg, -1))
    source = torch.where(hole, table.gather(1, (hole.cumsum(1) - 1).clamp(min=0)), slot)
    src = (st["starts"][:-1, None].long() + source).clamp(max=st["total"]).reshape(-1)
    dst = torch.where(inside, to["starts"][:-1, None].long() + slot, to["total"]).reshape(-1)
    for name in ("records", "pos", "weight"):
        to[name][dst] = st[name][src]
    to["lens"].copy_(kept)
    return {"lens": to["lens"], "pos": to["pos"][:-1], "weight": to["weight"][:-1], "records": to["records"][:-1]}


# ---- the library's calls --------------------------------------------------------------------------------------------
def _cache(st):
    from paper_2508_15806_b200 import binding as B
    return B.make_q4_cache(st["records"][:-1], st["pos"][:-1], st["weight"][:-1], st["starts"], st["lens"],
                           st.get("n_kv_heads") or st["case"]["n_kv_heads"])


def _own(st):
    """The handles a program keeps (made on the first pass), then the calls of one pass."""
    from paper_2508_15806_b200 import binding as B
    c = st["case"]
    h = st.get("handles")
    if h is None:
        h = st["handles"] = dict(cache=_cache(st))
        if c["kind"] == "append":
            h["after"] = B.make_q4_cache(st["records"][:-1], st["pos"][:-1], st["weight"][:-1], st["starts"], st["lens_out"],
                                         c["n_kv_heads"])
        if c["kind"] == "attend":
            h["params"] = B.make_q4_attend(h["cache"], st["q"], st["out"], softcap=c["softcap"], weight_decay=c["decay"])
            h["workspace"] = B.new_q4_workspace(h["cache"], h["params"], accumulate=c["accumulate"])
        if c["kind"] in ("evict", "step"):
            h["to"] = h["cache"] if c["kind"] == "step" else _cache(dict(st["to"], n_kv_heads=c["n_kv_heads"]))
            h["workspace"] = B.new_q4_evict_workspace(h["cache"], h["to"])
    cache = h["cache"]
    if c["kind"] == "append":
        B.slkv_q4_append(cache, st["k"], st["v"], st["new_pos"], after=h["after"])
    elif c["kind"] == "pack":
        B.slkv_q4_pack(cache, st["k"], st["v"], st["offsets"], st["kept_idx"])
    elif c["kind"] == "attend":
        B.slkv_q4_attend(cache, h["params"], st["q"], st["out"], h["workspace"], lse=st["lse"],
                         q_pos=st["q_pos"] if c["masked"] else None, slopes=st["slopes"] if c["slopes"] else None,
                         accumulate=c["accumulate"])
        got = {"out": st["out"], "lse": st["lse"]}
        return dict(got, weight=st["weight"][:-1]) if c["accumulate"] else got
    else:
        if c["kind"] == "step":
            B.slkv_q4_append(cache, st["k"], st["v"], st["new_pos"])
        B.slkv_q4_evict(cache, h["to"], st["budgets"], c["window"], st["newest"], h["workspace"])
        to = st if c["kind"] == "step" else st["to"]
        return {"lens": to["lens"], "pos": to["pos"][:-1], "weight": to["weight"][:-1], "records": to["records"][:-1]}
    B.slkv_q4_unpack(cache, st["k_out"], st["v_out"], slots=st["slots"])
    return {"k": st["k_out"], "v": st["v_out"], "lens": st["lens_out"] if c["kind"] == "append" else st["lens"],
            "pos": st["pos"][:-1]}


def run(state):
    st = state
    c = st["case"]
    if own:
        return _own(st)
    if c["kind"] == "attend":
        return _plain_attend(st)
    if c["kind"] == "evict":
        return _plain_evict(st, st["to"], c["n_kv_heads"], c["window"], st["lens"])
    if c["kind"] == "step":
        _plain_append(st, st["lens"], st["lens"])
        return _plain_evict(st, st, c["n_kv_heads"], c["window"], st["lens"])
    if c["kind"] == "append":
        _plain_append(st, st["lens"], st["lens_out"])
    else:
        _plain_pack(st)
    k, v = _decode(st["records"][st["slots"].long()], c["head_dim"])
    return {"k": k.bfloat16(), "v": v.bfloat16(), "lens": st["lens_out"] if c["kind"] == "append" else st["lens"],
            "pos": st["pos"][:-1]}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------
def _exact_values(x):
    """What a row's channels stand for once packed: the definition, group by group, in 64 bits."""
    x = x.double()
    out = torch.empty_like(x)
    for j in range(x.shape[1] // 32):
        g = x[:, 32 * j:32 * j + 32]
        low = g.min(1, keepdim=True).values
        zero = _bf16_towards(low, -math.inf)
        scale = _bf16_towards((g.max(1, keepdim=True).values - zero) / 15.0, math.inf)
        code = torch.where(scale > 0, torch.round((g - zero) / scale), torch.zeros_like(g)).clamp(0, 15)
        out[:, 32 * j:32 * j + 32] = zero + scale * code
    return out


def _bf16_towards(x, way):
    """The bf16 values next to x in one direction (normal range), as 64-bit numbers."""
    m, e = torch.frexp(x)                                             # |m| in [1/2, 1): 8 bits of it
    m = torch.floor(m * 256.0) if way < 0 else torch.ceil(m * 256.0)
    return torch.ldexp(m / 256.0, e)


def _exact_decode(rec, d):
    """Records [rows, bytes] -> 64-bit K and V rows, word by word."""
    ng = d // 32
    words, units = rec[:, :d // 2].contiguous().view(torch.int32), rec[:, d // 2:d].contiguous().view(torch.int16).int()
    s = rec[:, d:].contiguous().view(torch.bfloat16).double()
    k, v = (torch.empty(rec.shape[0], d, dtype=torch.float64, device=rec.device) for _ in range(2))
    for j in range(ng):
        for t in range(4):
            for e in range(8):
                k[:, 32 * j + 8 * t + e] = ((words[:, t * ng + j] >> (4 * e)) & 15) * s[:, j] + s[:, ng + j]
        for g in range(8):
            for e in range(4):
                v[:, 32 * j + 4 * g + e] = ((units[:, g * ng + j] >> (4 * e)) & 15) * s[:, 2 * ng + j] + s[:, 3 * ng + j]
    return k, v


def _exact_attend(st):
    c = st["case"]
    ns, hkv, G, nt, d = c["n_seqs"], c["n_kv_heads"], c["group"], c["n_tokens"], c["head_dim"]
    out = torch.zeros(ns, nt, hkv * G, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((ns, hkv * G, nt), -math.inf, dtype=torch.float64, device=DEVICE)
    weight = st["weight"][:-1].double()
    starts, lens = st["starts"].tolist(), st["lens"].tolist()
    for seg in range(ns * hkv):
        s, h = divmod(seg, hkv)
        rows = slice(starts[seg], starts[seg] + lens[seg])
        if lens[seg] == 0:
            continue
        k, v = _exact_decode(st["records"][rows], d)
        q = st["q"][s, :, h * G:h * G + G].double()                   # [tokens, G, d]
        x = torch.einsum("igd,nd->gin", q, k) / math.sqrt(d)
        if c["softcap"]:
            x = torch.tanh(x / c["softcap"]) * c["softcap"]
        if c["masked"]:
            away = st["pos"][rows].double()[None, None, :] - st["q_pos"][s].double()[None, :, None]
            if c["slopes"]:
                x = x + st["slopes"][h * G:h * G + G].double()[:, None, None] * away
            x = x.masked_fill((away > 0).expand_as(x), -math.inf)
        z = torch.logsumexp(x, -1)
        p = torch.where(torch.isinf(z)[..., None], torch.zeros_like(x), torch.exp(x - z[..., None]))
        out[s, :, h * G:h * G + G] = torch.einsum("gin,nd->igd", p, v)
        lse[s, h * G:h * G + G] = z
        weight[rows] = c["decay"] * weight[rows] + p.sum((0, 1)) / G
    got = {"out": out, "lse": lse}
    return dict(got, weight=weight) if c["accumulate"] else got


def _exact_evict(st, lens, to_starts, to_weight):
    """The weights that are left, segment by segment; all else is whole numbers."""
    c = st["case"]
    hkv, starts, weight = c["n_kv_heads"], st["starts"].tolist(), st["weight"].double().cpu().tolist()
    pos, newest, budgets, out = st["pos"].tolist(), st["newest"].tolist(), st["budgets"].tolist(), to_weight.double().cpu().tolist()
    for seg, n in enumerate(lens):
        w, p = weight[starts[seg]:starts[seg] + n], pos[starts[seg]:starts[seg] + n]
        first = newest[seg // hkv] - c["window"]
        order = sorted(range(n), key=lambda i: (p[i] <= first, 0.0 if p[i] > first else -w[i], i))
        kept = min(n, max(budgets[seg % hkv], c["window"]))
        keep = set(order[:kept])
        later = iter(sorted(i for i in keep if i >= kept))
        for i in range(kept):
            out[to_starts[seg] + i] = w[i if i in keep else next(later)]
    return torch.tensor(out, dtype=torch.float64)


def exact(case, seed):
    st = prepare(case, seed)
    c = st["case"]
    if c["kind"] == "attend":
        return _exact_attend(st)
    if c["kind"] in ("append", "pack"):
        rows = [(st[x].transpose(1, 2) if c["kind"] == "append" else st[x]).reshape(-1, c["head_dim"]) for x in ("k", "v")]
        return {"k": _exact_values(rows[0]), "v": _exact_values(rows[1]), "lens": None, "pos": None}
    lens = st["lens"].tolist()
    if c["kind"] == "step":
        at = st["slots"].long()
        st["weight"][at], st["pos"][at] = 0.0, st["new_pos"][:, :1].expand(-1, c["n_kv_heads"]).reshape(-1)
        lens = [n + 1 for n in lens]
        to = st
    else:
        to = st["to"]
    return {"lens": None, "pos": None, "weight": _exact_evict(st, lens, to["starts"].tolist(), to["weight"][:-1]), "records": None}
