"""From a prompt to drafted tokens over what is kept of it, as cases that can be timed: causal attention of whole prompts (with the
window rows' log-sum-exps that the compression takes), pages planned for segments of any length, rows written into them, and
attention of trees of drafted tokens over the pages.  Each case has a plain form in elementary torch operations and the calls a
user makes of this library.

A paged cache: segment seg = (layer * n_seqs + sequence) * n_kv_heads + KV head has lens[seg] rows; row r lies in row r % page_rows
of page tables[seg][r / page_rows].  A slot is page * page_rows + row.  free_pages[0 .. n_free) is a stack of the pages that nobody
has.  A plan gives every segment a new length: first the pages that are no longer needed are returned, so that in the end the first
segment's lie on top (of a segment's, its first), then the segments take theirs from the top, in order.
"""
import math
import random

import torch

own = False
DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases ---------------------------------------------------------------------------------------------------
def _case(kind, **kw):
    """Defaults: a Llama-3-8B / Mistral-7B layer (32 query heads, 8 KV heads, head_dim 128, bf16)."""
    c = dict(kind=kind, n_layers=1, n_seqs=1, n_kv_heads=8, group=4, head_dim=128, dtype="bf16", n_tokens=1, len_min=512, len_max=512,
             prefix=0, idle=False, window=32, page_rows=32, ragged=False)
    c.update(kw)
    return c


def listed():
    return [
        # one short prompt: latency counts
        _case("prompt", name="prompt-129", len_min=129, len_max=129),
        # a batch of packed prompts of mixed length, one of them empty
        _case("prompt", name="prompt-batch", n_seqs=12, len_min=90, len_max=4001, idle=True),
        # fp32, narrow heads, keys shared by three query heads, other window
        _case("prompt", name="prompt-f32-d64", n_seqs=3, n_kv_heads=4, group=3, head_dim=64, dtype="f32", len_min=333, len_max=2000,
              window=16),
        # chunked prefill: a few hundred new tokens each behind what is there already, one sequence that decodes (a single token)
        _case("prompt", name="prompt-chunk", n_seqs=4, len_min=1, len_max=512, prefix=24000),
        # the largest: one long context
        _case("prompt", name="prompt-32k", len_min=32000, len_max=32000),
        # a decode step's accepted tokens of a batch: slots, then the rows of one layer
        _case("step", name="step-16", n_seqs=16, len_min=200, len_max=1024, n_tokens=8, ragged=True),
        # the same for the tables of all layers of a larger batch, fp32 rows
        _case("step", name="step-layers-f32", n_layers=32, n_seqs=16, head_dim=64, dtype="f32", len_min=64, len_max=512, n_tokens=4,
              page_rows=16, ragged=True),
        # a batch of long prompts' compressed layer into pages
        _case("fill", name="fill-batch", n_seqs=16, len_min=2000, len_max=12000, page_rows=64),
        # one user's decode step over a compressed cache: latency counts
        _case("tree", name="tree-one", len_min=129, len_max=1031),
        # an ordinary serving batch: trees of different size, budgets that differ per head, one sequence without any rows yet
        _case("tree", name="tree-batch", n_seqs=32, len_min=256, len_max=4096, n_tokens=16, idle=True, ragged=True),
        # fp32, narrow heads, every head with keys of its own
        _case("tree", name="tree-f32-d64", n_seqs=5, n_kv_heads=12, group=1, head_dim=64, dtype="f32", n_tokens=7, len_min=33,
              len_max=3001, page_rows=16),
        # long contexts kept whole
        _case("tree", name="tree-long", n_seqs=8, len_min=20000, len_max=65536, n_tokens=32, page_rows=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "prompt", "step", "fill", "tree", "tree", "tree", "tree"])
    n_kv, group = rng.choice([1, 2, 4, 8, 8, 12]), rng.choice([1, 2, 3, 4, 4, 6, 8, 16])
    dtype, n_seqs = rng.choice(["bf16", "bf16", "f32"]), _log_int(rng, 1, 48)
    c = _case(kind, n_seqs=n_seqs, n_kv_heads=n_kv, group=group, head_dim=rng.choice([64, 128, 128]), dtype=dtype,
              page_rows=rng.choice([16, 32, 64, 128]), n_tokens=rng.choice([1, 1, 2, 5, 8, 16, 33, 64]), idle=rng.random() < 0.2,
              ragged=rng.random() < 0.5, window=rng.choice([1, 16, 32, 64]))
    if kind == "prompt":
        # the work of all sequences, in pairs of a query and a key times query heads, is bounded
        prefix = rng.choice([0, 0, 0, min(_log_int(rng, 100, 40000), 200000 // n_seqs)])
        pairs = (3e10 if dtype == "bf16" else 6e9) / (n_seqs * n_kv * group)
        top = max(1, min(_log_int(rng, 1, 32000), int(math.sqrt(prefix * prefix + pairs) - prefix), 200000 // n_seqs))
        c.update(prefix=prefix, len_max=top, len_min=max(1, top // rng.choice([1, 2, 8, 40])))
        return c
    most = {"step": 1 << 18, "fill": 700000, "tree": 1500000}[kind]
    if kind == "step":
        c.update(n_tokens=rng.choice([1, 2, 4, 8]), n_layers=rng.choice([1, 2, 8, 32]) if n_seqs * n_kv <= 128 else 1, idle=False)
    top = max(40, min(_log_int(rng, 64, 65536), most // (c["n_layers"] * n_seqs * n_kv)))
    if kind == "tree":
        top = max(40, min(top, int(3e8 / (n_seqs * n_kv * group * c["n_tokens"]))))
    c.update(len_max=top, len_min=max(1, top // rng.choice([1, 2, 8, 40])))
    return c


# ---- sizes that follow from a case ---------------------------------------------------------------------------------
def _spread(c, n, salt):
    """n lengths from len_min to len_max over their logarithm, both among them."""
    r = random.Random(n * 7919 + c["n_kv_heads"] * 31 + c["len_max"] + salt)
    lens = [_log_int(r, c["len_min"], c["len_max"]) for _ in range(n)]
    lens[0] = c["len_max"]
    if n > 1:
        lens[1] = c["len_min"]
    return lens


def _lens(c):
    """Rows per segment of a layer, the same in every layer but for one more or two; an idle batch has one sequence without any."""
    lens = _spread(c, c["n_seqs"] * c["n_kv_heads"], 0)
    if c["idle"] and c["n_seqs"] > 1:
        lens[-c["n_kv_heads"]:] = [0] * c["n_kv_heads"]
    return [n + layer % 3 if n else 0 for layer in range(c["n_layers"]) for n in lens]


def _prompt_lens(c):
    """Queries and keys per sequence: a prefix of about the case's length lies before the queries."""
    nq = _spread(c, c["n_seqs"], 1)
    if c["idle"] and c["n_seqs"] > 1:
        nq[-1] = 0
    r = random.Random(c["prefix"])
    return nq, [n + int(c["prefix"] * r.uniform(0.5, 1.0)) if c["prefix"] and n else n for n in nq]


def _counts(c):
    """Tokens of each sequence's tree (step: accepted ones), n_tokens of them at most."""
    r = random.Random(c["n_tokens"] * 101 + c["n_seqs"])
    return [r.randint(1, c["n_tokens"]) if c["ragged"] and s else c["n_tokens"] for s in range(c["n_seqs"])]


def _pages(c, lens):
    return [-(-n // c["page_rows"]) for n in lens]


def work(case):
    c = case
    d, e, hkv, G = c["head_dim"], 4 if c["dtype"] == "f32" else 2, c["n_kv_heads"], c["group"]
    if c["kind"] == "prompt":
        nq, nk = _prompt_lens(c)
        pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(nq, nk))
        rows = 2 * sum(nq) * hkv * G + 2 * sum(nk) * hkv
        return {"bytes": rows * d * e + sum(min(n, c["window"]) for n in nq) * hkv * G * 4, "flops": pairs * hkv * G * d * 4}
    lens, counts = _lens(c), _counts(c)
    if c["kind"] == "tree":
        new = sum(counts) * hkv
        pairs = sum(n * counts[i // hkv] for i, n in enumerate(lens)) * G + sum(t * (t + 1) // 2 for t in counts) * hkv * G
        moved = (sum(lens) + new) * 2 * d * e + new * G * (2 * d * e + 4) + 4 * sum(_pages(c, lens))
        return {"bytes": moved, "flops": pairs * d * 4}
    if c["kind"] == "fill":
        rows, pages = sum(lens), sum(_pages(c, lens))
        return {"bytes": rows * (4 * d * e + 8) + pages * 8 + 12 * len(lens), "flops": rows}
    added = [counts[i // hkv % c["n_seqs"]] for i in range(len(lens))]
    taken = sum(_pages(c, [n + a for n, a in zip(lens, added)])) - sum(_pages(c, lens))
    rows = sum(counts) * hkv
    return {"bytes": len(lens) * (8 + 4 * c["n_tokens"]) + taken * 8 + rows * (4 * d * e + 4), "flops": len(lens) * 8}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _dev(v, t=torch.int32):
    return torch.tensor(v, dtype=t, device=DEVICE)


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _rows(g, n, d, u, hits):
    """K rows [n, ...heads, d]: channels with offsets of their own, some needles along the direction u that the queries share."""
    k = torch.randn(n, *u.shape[-2:-1], d, device=DEVICE, generator=g)
    k += 2.0 * torch.sin(torch.arange(d, device=DEVICE) * 1.7)
    hit = torch.rand(k.shape[:-1], device=DEVICE, generator=g) < hits
    return k + torch.where(hit, 1.0, 0.0)[..., None] * u


def _prepare_prompt(c, g):
    d, hkv, G, dt = c["head_dim"], c["n_kv_heads"], c["group"], DTYPES[c["dtype"]]
    nq, nk = _prompt_lens(c)
    u = torch.randn(hkv, d, device=DEVICE, generator=g)
    q = torch.randn(max(1, sum(nq)), hkv, G, d, device=DEVICE, generator=g).mul_(0.7).add_(0.7 * u[:, None])
    st = dict(case=c, q=q.view(-1, hkv * G, d).to(dt), k=_rows(g, max(1, sum(nk)), d, u, 0.01).to(dt))
    st["v"] = torch.randn(st["k"].shape, device=DEVICE, generator=g).to(dt)
    st.update(cu_q=_cu(nq), cu_k=_cu(nk), out=torch.zeros_like(st["q"]),
              lse=torch.zeros(c["n_seqs"], hkv * G, c["window"], dtype=torch.float32, device=DEVICE))
    st.update(cu_q_dev=_dev(st["cu_q"]), cu_k_dev=_dev(st["cu_k"]))
    return st


def _tree_masks(c, counts, seed):
    """Bit j of token i's mask: token j is i or one of its ancestors.  Parents are drawn among the last few tokens."""
    r = random.Random(seed)
    masks = []
    for n in counts:
        m = []
        for i in range(c["n_tokens"]):
            parent = r.randint(max(-1, i - 4), i - 1)
            m.append((m[parent] if parent >= 0 else 0) | 1 << i)
        masks.append([x - (1 << 64) if x >> 63 else x for x in m])
    return _dev(masks, torch.int64)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    if c["kind"] == "prompt":
        return _prepare_prompt(c, g)
    d, hkv, ns, dt, nt, rows = c["head_dim"], c["n_kv_heads"], c["n_seqs"], DTYPES[c["dtype"]], c["n_tokens"], c["page_rows"]
    lens, counts = _lens(c), _counts(c)
    n_seg, n_layer_seg = len(lens), ns * hkv
    have = [0] * n_seg if c["kind"] == "fill" else _pages(c, lens)
    most = max(_pages(c, [n + nt for n in lens])) + 1
    n_pages = sum(_pages(c, [n + nt for n in lens])) + 7
    perm = torch.randperm(n_pages, device=DEVICE, generator=g).int()
    used = sum(have)
    st = dict(case=c, counts=_dev(counts), width=most * rows)
    # the pages in use in the tables, the others on the stack; entries behind a segment's pages are left from earlier
    seg = torch.repeat_interleave(torch.arange(n_seg, device=DEVICE), _dev(have, torch.int64))
    first = torch.cumsum(_dev(have, torch.int64), 0) - _dev(have, torch.int64)
    at = torch.arange(used, device=DEVICE) - first[seg]
    st["tables"] = torch.randint(0, n_pages, (n_seg, most), device=DEVICE, generator=g).int()
    st["tables"][seg, at] = perm[:used]
    st["free_pages"] = torch.zeros(n_pages, dtype=torch.int32, device=DEVICE)
    st["free_pages"][:n_pages - used] = perm[used:]
    st["n_free"], st["n_free_out"] = _dev([n_pages - used]), _dev([0])
    st["lens"] = _dev([0] * n_seg if c["kind"] == "fill" else lens)
    st["lens_out"] = torch.zeros(n_seg, dtype=torch.int32, device=DEVICE)
    # recycled pages: rows behind a segment's last are somebody's old ones
    u = torch.randn(hkv, d, device=DEVICE, generator=g)
    one = u[0].expand(1, d)
    st["k_pages"] = torch.empty(n_pages, rows, d, dtype=dt, device=DEVICE)
    for i in range(0, n_pages, 8192):
        part = st["k_pages"][i:i + 8192]
        part.copy_(_rows(g, part.shape[0] * rows, d, one, 0.01).view(part.shape))
    st["v_pages"] = torch.empty_like(st["k_pages"]).normal_(generator=g)
    if c["kind"] == "fill":
        n = sum(lens)
        st["k"], st["v"] = _rows(g, n, d, one, 0.01).view(n, d).to(dt), torch.randn(n, d, device=DEVICE, generator=g).to(dt)
        st["offsets"] = _dev(_cu(lens))
        st["slots"] = torch.full((n + 5,), -1, dtype=torch.int32, device=DEVICE)
        st["slot_offsets"] = torch.zeros(n_seg + 1, dtype=torch.int32, device=DEVICE)
        return st
    st["k"] = _rows(g, ns * nt, d, u, 0.2).view(ns, nt, hkv, d).to(dt)
    st["v"] = torch.randn(ns, nt, hkv, d, device=DEVICE, generator=g).to(dt)
    if c["kind"] == "step":
        st["slots"] = torch.full((n_seg, nt), -1, dtype=torch.int32, device=DEVICE)
        st["take"] = torch.argsort(torch.rand(ns, nt, device=DEVICE, generator=g), dim=1).int()
        st["n_layer_seg"] = n_layer_seg
        return st
    q = 0.7 * u[:, None] + 0.7 * torch.randn(ns, nt, hkv, c["group"], d, device=DEVICE, generator=g)
    st["q"] = q.reshape(ns, nt, hkv * c["group"], d).to(dt)
    st["tree"] = _tree_masks(c, counts, seed)
    st["out"] = torch.zeros_like(st["q"])
    st["lse"] = torch.zeros(ns, hkv * c["group"], nt, dtype=torch.float32, device=DEVICE)
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _softmax(s):
    """exp(s - max) over its sum and the log-sum-exp; rows without anything give zeros and -infinity."""
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    return p / torch.where(z > 0, z, 1.0), (m + torch.log(z)).squeeze(-1)


def _plain_prompt(st):
    c = st["case"]
    d, hkv, G, w = c["head_dim"], c["n_kv_heads"], c["group"], c["window"]
    for s in range(c["n_seqs"]):
        q0, nq, k0 = st["cu_q"][s], st["cu_q"][s + 1] - st["cu_q"][s], st["cu_k"][s]
        nk = st["cu_k"][s + 1] - k0
        k = st["k"][k0:k0 + nk].float().permute(1, 2, 0)
        v = st["v"][k0:k0 + nk].float().transpose(0, 1)
        step = max(1, min(2048, (1 << 31) // max(1, nk * hkv * G)))                # queries at a time: scores of 8 GB at most
        for i in range(0, nq, step):
            n = min(step, nq - i)
            q = st["q"][q0 + i:q0 + i + n].float().view(n, hkv, G, d).permute(1, 2, 0, 3).reshape(hkv, G * n, d)
            seen = nk - nq + i + n                                                  # keys that the last of these queries sees
            x = (torch.matmul(q, k[:, :, :seen]) * (1.0 / math.sqrt(d))).view(hkv, G, n, seen)
            row = torch.arange(n, device=DEVICE) + nk - nq + i
            x = torch.where(torch.arange(seen, device=DEVICE) <= row[:, None], x, -math.inf)
            p, z = _softmax(x)
            del x
            o = torch.matmul(p.view(hkv, G * n, seen), v[:, :seen]).view(hkv, G, n, d)
            st["out"][q0 + i:q0 + i + n] = o.permute(2, 0, 1, 3).reshape(n, hkv * G, d)
            begin = max(i, nq - w)                                                  # the window rows among these
            if begin < i + n:
                at = begin - (nq - w)
                st["lse"][s, :, at:at + i + n - begin] = z.reshape(hkv * G, n)[:, begin - i:]
    return {"out": st["out"], "lse": st["lse"]}


def _plain_plan(st, want):
    """New lengths want [n_seg]: pages returned, pages taken, the slots of new rows."""
    rows, most = st["case"]["page_rows"], st["tables"].shape[1]
    tables, free = st["tables"], st["free_pages"]
    lens, n_pages = st["lens"].long(), free.numel()
    want = want.long().clamp(0, most * rows)
    have, need = -(-lens // rows), -(-want // rows)
    col = torch.arange(most, device=DEVICE)
    gone = (col >= need[:, None]) & (col < have[:, None])
    more = (col >= have[:, None]) & (col < need[:, None])
    n_gone, n_more = gone.sum(), more.sum()
    base = st["n_free"].long()
    place = base + n_gone - gone.view(-1).cumsum(0)                  # the first returned page lies on top
    n_free = base + n_gone
    padded = torch.cat([free, free.new_zeros(1)])
    padded.scatter_(0, torch.where(gone.view(-1), place, n_pages), tables.view(-1))
    rank = more.view(-1).cumsum(0) - 1
    there = more.view(-1) & (rank < n_free)
    taken = padded[torch.where(there, n_free - 1 - rank, n_pages)]
    free.copy_(padded[:-1])
    tables.copy_(torch.where(there, taken, tables.view(-1)).view(tables.shape))
    got = have.minimum(need) + there.view(more.shape).sum(1)
    new = torch.minimum(want, got * rows)
    st["lens_out"].copy_(new)
    st["n_free_out"].copy_(n_free - there.sum())
    return lens, new


def _slot(st, seg, row):
    rows = st["case"]["page_rows"]
    return st["tables"][seg, row // rows] * rows + (row % rows).int()


def _plain_fill(st):
    want = st["offsets"][1:] - st["offsets"][:-1]
    lens, new = _plain_plan(st, want)
    add = new - lens
    offsets = torch.cat([add.new_zeros(1), add.cumsum(0)])
    st["slot_offsets"].copy_(offsets)
    i = torch.arange(st["slots"].numel(), device=DEVICE)
    seg = torch.bucketize(i, offsets[1:], right=True)
    inside = i < offsets[-1]
    seg = torch.where(inside, seg, 0)
    slots = torch.where(inside, _slot(st, seg, torch.where(inside, lens[seg] + i - offsets[seg], 0)), -1)
    st["slots"].copy_(slots)
    at = slots[:st["k"].shape[0]].long()
    for name in ("k", "v"):
        st[name + "_pages"].view(-1, st["case"]["head_dim"])[at] = st[name]
    return _state(st)


def _plain_step(st):
    c = st["case"]
    hkv, ns, nt, d = c["n_kv_heads"], c["n_seqs"], c["n_tokens"], c["head_dim"]
    add = st["counts"].repeat_interleave(hkv).repeat(c["n_layers"])
    lens, new = _plain_plan(st, st["lens"] + add)
    row = lens[:, None] + torch.arange(nt, device=DEVICE)
    inside = row < new[:, None]
    seg = torch.arange(lens.numel(), device=DEVICE)[:, None].expand(row.shape)
    st["slots"].copy_(torch.where(inside, _slot(st, seg, torch.where(inside, row, 0)), -1))
    slots = st["slots"][:ns * hkv].view(ns, hkv, nt)
    put = slots >= 0
    source = st["take"].long()[:, None, :].expand(ns, hkv, nt)
    s, h = torch.arange(ns, device=DEVICE)[:, None, None], torch.arange(hkv, device=DEVICE)[None, :, None]
    for name in ("k", "v"):
        st[name + "_pages"].view(-1, d)[slots[put].long()] = st[name][s, source, h][put]
    return _state(st)


def _state(st):
    """What planning and writing leave; of the stack the part in use."""
    return {x: st[x] for x in ("tables", "lens_out", "n_free_out", "free_pages", "slots", "k_pages", "v_pages")}


def _plain_tree(st):
    c = st["case"]
    ns, hkv, G, nt, d, rows = c["n_seqs"], c["n_kv_heads"], c["group"], c["n_tokens"], c["head_dim"], c["page_rows"]
    step = max(1, (1 << 31) // (hkv * st["width"] * max(d, G * nt) * 4))            # sequences at a time
    for s in range(0, ns, step):
        n = min(step, ns - s)
        lens = st["lens"].view(ns, hkv)[s:s + n].long()
        pages = st["tables"].view(ns, hkv, -1)[s:s + n].long()
        width = st["width"] + nt
        col = torch.arange(width, device=DEVICE)
        filled = col[:st["width"]] < lens[..., None]
        visible = torch.zeros(n, hkv, 1, nt, width, dtype=torch.bool, device=DEVICE)
        visible[..., :st["width"]] = filled[:, :, None, None]
        j = torch.arange(nt, device=DEVICE)
        seen = (st["tree"][s:s + n, :, None] >> j & 1 > 0) & (j < st["counts"][s:s + n, None, None])
        visible[..., st["width"]:] = seen[:, None, None]
        kv = [torch.cat([st[x + "_pages"][pages].view(n, hkv, -1, d).float(), st[x][s:s + n].float().transpose(1, 2)], 2)
              for x in ("k", "v")]
        q = st["q"][s:s + n].float().view(n, nt, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * nt, d)
        x = (torch.matmul(q, kv[0].transpose(2, 3)) * (1.0 / math.sqrt(d))).view(n, hkv, G, nt, width)
        p, z = _softmax(torch.where(visible, x, -math.inf))
        o = torch.matmul(p.view(n, hkv, G * nt, width), kv[1]).view(n, hkv, G, nt, d)
        there = j < st["counts"][s:s + n, None]                                     # rows of padding stay as they are
        out = o.permute(0, 3, 1, 2, 4).reshape(n, nt, hkv * G, d)
        st["out"][s:s + n] = torch.where(there[..., None, None], out, st["out"][s:s + n])
        st["lse"][s:s + n] = torch.where(there[:, None], z.reshape(n, hkv * G, nt), st["lse"][s:s + n])
    return {"out": st["out"], "lse": st["lse"]}


# ---- the library's calls --------------------------------------------------------------------------------------------
def _own(st):
    """The handles a program keeps (made on the first pass), then the calls of one pass."""
    from paper_2508_15806_b200 import binding as B
    c = st["case"]
    h = st.get("handles")
    if h is None:
        h = st["handles"] = {}
        if c["kind"] == "prompt":
            h["params"] = B.make_prompt(st["q"], st["k"], st["v"], st["out"], c["n_seqs"], window=c["window"])
            h["workspace"] = B.new_prompt_workspace(h["params"], st["cu_q"], st["cu_k"])
        else:
            for name, lens, n_free in (("cache", "lens", "n_free"), ("after", "lens_out", "n_free_out")):
                h[name] = B.make_paged_cache(st["k_pages"], st["v_pages"], st["tables"], st[lens], st["free_pages"], st[n_free],
                                             c["n_seqs"], c["n_kv_heads"])
        if c["kind"] == "step":
            h["slots"] = st["slots"][:st["n_layer_seg"]]
        if c["kind"] == "tree":
            h["params"] = B.make_paged_attend(h["cache"], st["q"], st["out"], st["k"], st["v"])
            h["workspace"] = B.new_paged_workspace(h["cache"], h["params"])
    if c["kind"] == "prompt":
        B.slkv_prompt_attend(h["params"], st["q"], st["k"], st["v"], st["cu_q_dev"], st["cu_q"], st["out"], h["workspace"],
                             cu_k=st["cu_k_dev"], cu_k_host=st["cu_k"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if c["kind"] == "tree":
        B.slkv_paged_attend(h["cache"], h["params"], st["q"], st["out"], h["workspace"], k_new=st["k"], v_new=st["v"],
                            tree=st["tree"], n_new=st["counts"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if c["kind"] == "fill":
        B.slkv_paged_plan(h["cache"], B.SLKV_PAGED_OFFSETS, st["offsets"], slots=st["slots"], slot_offsets=st["slot_offsets"],
                          after=h["after"])
        B.slkv_paged_write(h["cache"], st["k"], st["v"], st["slots"])
    else:
        B.slkv_paged_plan(h["cache"], B.SLKV_PAGED_ADD, st["counts"], slots=st["slots"], after=h["after"])
        B.slkv_paged_write(h["cache"], st["k"], st["v"], h["slots"], take=st["take"])
    return _state(st)


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_prompt, "fill": _plain_fill, "step": _plain_step, "tree": _plain_tree}[state["case"]["kind"]](state)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------
def _exact_rows(q, k, v, visible):
    """q [n, d], k, v [m, d] in 64 bits, visible [n, m] -> outputs and log-sum-exps."""
    x = (q @ k.T / math.sqrt(q.shape[1])).masked_fill(~visible, -math.inf)
    z = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
    return p @ v, z


def _exact_prompt(st):
    c = st["case"]
    G, w = c["group"], c["window"]
    out, lse = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEVICE), st["lse"].double()
    for s in range(c["n_seqs"]):
        q0, q1, k0, k1 = st["cu_q"][s], st["cu_q"][s + 1], st["cu_k"][s], st["cu_k"][s + 1]
        for h in range(c["n_kv_heads"] * G):
            k, v = st["k"][k0:k1, h // G].double(), st["v"][k0:k1, h // G].double()
            for i in range(q0, q1, 4096):
                j = min(q1, i + 4096)
                at = torch.arange(i, j, device=DEVICE) - q1 + (k1 - k0)             # the last key that each query sees
                m = (k1 - k0) - (q1 - j)
                o, z = _exact_rows(st["q"][i:j, h].double(), k[:m], v[:m], torch.arange(m, device=DEVICE)[None] <= at[:, None])
                out[i:j, h] = o
                a = max(i, q1 - w)
                if a < j:
                    lse[s, h, a - (q1 - w):j - (q1 - w)] = z[a - i:]
    return {"out": out, "lse": lse}


def _exact_tree(st):
    c = st["case"]
    hkv, G, nt, d, rows = c["n_kv_heads"], c["group"], c["n_tokens"], c["head_dim"], c["page_rows"]
    out, lse = st["out"].double(), st["lse"].double()
    lens, counts, tree = st["lens"].tolist(), st["counts"].tolist(), st["tree"].tolist()
    for s in range(c["n_seqs"]):
        t = counts[s]
        drafted = torch.tensor([[bool(tree[s][i] >> j & 1) for j in range(t)] for i in range(t)], device=DEVICE)
        for h in range(hkv):
            n = lens[s * hkv + h]
            pages = st["tables"][s * hkv + h, :-(-n // rows)].long()
            k, v = (torch.cat([st[x + "_pages"][pages].reshape(-1, d)[:n], st[x][s, :t, h]]).double() for x in ("k", "v"))
            visible = torch.cat([torch.ones(t, n, dtype=torch.bool, device=DEVICE), drafted], 1)
            for g in range(h * G, h * G + G):
                out[s, :t, g], lse[s, g, :t] = _exact_rows(st["q"][s, :t, g].double(), k, v, visible)
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["kind"] not in ("prompt", "tree"):                       # whole numbers and copies
        return None
    st = prepare(case, seed)
    return _exact_prompt(st) if case["kind"] == "prompt" else _exact_tree(st)
