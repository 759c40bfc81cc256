"""The 4-bit cache's entry points without a GPU: argument checks come before anything is enqueued; sizes."""
import ctypes as C

import pytest
import torch

from paper_2508_15806_b200 import binding as B
from paper_2508_15806_b200 import build as builder

FAKE = 1 << 20           # an aligned address that is never dereferenced


@pytest.fixture(scope="module")
def L():
    builder.build()
    return B.lib()


def cache(**kw):
    d = dict(n_seqs=2, n_kv_heads=4, head_dim=128, reserved=0, capacity_rows=1000, records=FAKE, pos=2 * FAKE, weight=3 * FAKE,
             starts=4 * FAKE, lens=5 * FAKE)
    d.update(kw)
    return B.SlkvQ4Cache(**d)


def attend_params(**kw):
    d = dict(n_q_heads=16, n_tokens=1, dtype=B.SLKV_BF16, lse_units=B.SLKV_LSE_LN, scale=0.1, softcap=0.0, weight_decay=1.0, reserved=0,
             q_stride_seq=2048, q_stride_tok=2048, q_stride_head=128, o_stride_seq=2048, o_stride_tok=2048, o_stride_head=128)
    d.update(kw)
    return B.SlkvQ4AttendParams(**d)


BAD_CACHES = [(dict(records=None), "NULL_PTR"), (dict(pos=None), "NULL_PTR"), (dict(starts=None), "NULL_PTR"), (dict(lens=None), "NULL_PTR"),
              (dict(n_seqs=0), "BAD_SHAPE"), (dict(n_kv_heads=0), "BAD_SHAPE"), (dict(n_seqs=4097), "BAD_SHAPE"),
              (dict(n_seqs=1 << 30, n_kv_heads=1 << 30), "BAD_SHAPE"), (dict(head_dim=96), "BAD_SHAPE"), (dict(capacity_rows=0), "BAD_SHAPE"),
              (dict(capacity_rows=1 << 31), "BAD_SHAPE"), (dict(records=FAKE + 8), "BAD_ALIGN")]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(L, kw, code):
    c, p, good = C.byref(cache(**kw)), C.byref(attend_params()), C.byref(cache())
    f, code = C.c_void_p(FAKE), B.ERR[code]
    assert L.slkv_q4_pack(c, 1, f, f, 10, f, f, None, None) == code
    assert L.slkv_q4_append(c, 1, f, f, 1, 512, 512, 128, 512, 512, 128, f, None, None, None) == code
    assert L.slkv_q4_unpack(c, 1, None, 0, f, f, None) == code
    assert L.slkv_q4_attend(c, p, f, None, None, f, None, 0, None, f, 1 << 40, None) == code
    assert L.slkv_q4_attend_workspace_bytes(c, p, 0) == 0
    assert L.slkv_q4_evict(c, good, f, 1, f, None, f, 1 << 40, None) == code
    assert L.slkv_q4_evict(good, c, f, 1, f, None, f, 1 << 40, None) == code
    assert L.slkv_q4_evict_workspace_bytes(c) == 0


def test_rows_in_and_out(L):
    c, f, odd = C.byref(cache()), C.c_void_p(FAKE), C.c_void_p(FAKE + 4)
    E = B.ERR
    for args, code in [((7, f, f, 10, f, f), "BAD_DTYPE"), ((1, f, f, 10, None, f), "NULL_PTR"), ((1, None, f, 10, f, f), "NULL_PTR"),
                       ((1, f, None, 10, f, f), "NULL_PTR"), ((1, f, f, 10, f, None), "NULL_PTR"), ((1, f, f, -1, f, f), "BAD_SHAPE"),
                       ((1, f, f, 1 << 31, f, f), "BAD_SHAPE"), ((1, odd, f, 10, f, f), "BAD_ALIGN"), ((1, f, odd, 10, f, f), "BAD_ALIGN")]:
        assert L.slkv_q4_pack(c, *args, None, None) == E[code], args
    st = (512, 512, 128, 512, 512, 128)
    for args, code in [((1, None, f, 1, *st, f), "NULL_PTR"), ((1, f, None, 1, *st, f), "NULL_PTR"), ((1, f, f, 1, *st, None), "NULL_PTR"),
                       ((2, f, f, 1, *st, f), "BAD_DTYPE"), ((1, f, f, 0, *st, f), "BAD_SHAPE"), ((1, f, f, 65537, *st, f), "BAD_SHAPE"),
                       ((1, f, f, 1, 512, 512, 64, 512, 512, 128, f), "BAD_SHAPE"), ((1, f, f, 1, 512, 513, 128, 512, 512, 128, f), "BAD_ALIGN"),
                       ((1, f, f, 1, 512, 512, 128, 512, 512, 132, f), "BAD_ALIGN"), ((1, odd, f, 1, *st, f), "BAD_ALIGN")]:
        assert L.slkv_q4_append(c, *args, None, None, None) == E[code], args
    # new lengths that lie half across the old ones
    assert L.slkv_q4_append(c, 1, f, f, 1, *st, f, C.c_void_p(5 * FAKE + 4), None, None) == E["BAD_SHAPE"]
    for args, code in [((3, None, 0, f, f), "BAD_DTYPE"), ((1, f, -1, f, f), "BAD_SHAPE"), ((1, f, 1 << 31, f, f), "BAD_SHAPE"),
                       ((1, None, 0, None, f), "NULL_PTR"), ((1, f, 5, f, None), "NULL_PTR"), ((1, f, 5, odd, f), "BAD_ALIGN")]:
        assert L.slkv_q4_unpack(c, *args, None) == E[code], args
    assert L.slkv_q4_unpack(c, 1, f, 0, None, None, None) == 0          # nothing asked for
    assert [L.slkv_q4_record_bytes(d) for d in (64, 128, 96, 0)] == [80, 160, 0, 0]


def test_attention_arguments(L):
    f, odd = C.c_void_p(FAKE), C.c_void_p(FAKE + 8)
    E, c = B.ERR, C.byref(cache())
    for kw, code in [(dict(dtype=2), "BAD_DTYPE"), (dict(lse_units=5), "BAD_DTYPE"), (dict(n_tokens=0), "BAD_SHAPE"), (dict(n_q_heads=2), "BAD_SHAPE"),
                     (dict(n_q_heads=18), "BAD_SHAPE"), (dict(n_tokens=65), "BAD_SHAPE"), (dict(scale=float("nan")), "BAD_SHAPE"),
                     (dict(softcap=-1.0), "BAD_SHAPE"), (dict(softcap=1e-30), "BAD_SHAPE"), (dict(softcap=float("inf")), "BAD_SHAPE"), (dict(weight_decay=float("inf")), "BAD_SHAPE"),
                     (dict(q_stride_head=64), "BAD_SHAPE"), (dict(o_stride_tok=2052), "BAD_ALIGN")]:
        p = C.byref(attend_params(**kw))
        assert L.slkv_q4_attend(c, p, f, None, None, f, None, 0, None, f, 1 << 40, None) == E[code], kw
        assert L.slkv_q4_attend_workspace_bytes(c, p, 0) == 0
    p = C.byref(attend_params())
    need = L.slkv_q4_attend_workspace_bytes(c, p, 0)
    assert need > 0 and L.slkv_q4_attend_workspace_bytes(c, p, 1) >= need + 1000 * 4 * 4      # a score per slot and query head
    call = lambda *a: L.slkv_q4_attend(*a, None)            # noqa: E731
    assert call(c, None, f, None, None, f, None, 0, None, f, need) == E["NULL_PTR"]
    assert call(c, p, None, None, None, f, None, 0, None, f, need) == E["NULL_PTR"]
    assert call(c, p, f, None, None, None, None, 0, None, f, need) == E["NULL_PTR"]
    assert call(c, p, f, None, f, f, None, 0, None, f, need) == E["NULL_PTR"]                 # slopes need positions
    assert call(C.byref(cache(weight=None)), p, f, None, None, f, None, 1, None, f, 1 << 40) == E["NULL_PTR"]
    assert call(c, p, odd, None, None, f, None, 0, None, f, need) == E["BAD_ALIGN"]
    assert call(c, p, f, None, None, odd, None, 0, None, f, need) == E["BAD_ALIGN"]
    assert call(c, p, f, None, None, f, None, 0, None, odd, need) == E["BAD_ALIGN"]
    assert call(c, p, f, None, None, f, None, 0, None, None, need) == E["WORKSPACE"]
    assert call(c, p, f, None, None, f, None, 0, None, f, need - 1) == E["WORKSPACE"]
    assert call(c, p, f, None, None, f, None, 1, None, f, need) == E["WORKSPACE"]             # accumulating needs more
    # more tiles than are counted in 32 bits
    big = C.byref(cache(capacity_rows=(1 << 31) - 1))
    assert L.slkv_q4_attend_workspace_bytes(big, C.byref(attend_params(n_tokens=64)), 0) == 0
    assert L.slkv_q4_attend_workspace_bytes(big, p, 0) > 0


def test_eviction_arguments(L):
    f, E = C.c_void_p(FAKE), B.ERR
    a, other = cache(), cache(records=10 * FAKE, pos=12 * FAKE, weight=13 * FAKE, starts=14 * FAKE, lens=15 * FAKE)
    need = L.slkv_q4_evict_workspace_bytes(C.byref(a))

    def call(x, y, budgets=f, window=1, newest=f, ws=f, n=need):
        return L.slkv_q4_evict(C.byref(x), C.byref(y), budgets, window, newest, None, ws, n, None)
    assert call(a, other, budgets=None) == call(a, other, newest=None) == E["NULL_PTR"]
    assert call(cache(weight=None), other) == call(a, cache(records=10 * FAKE, weight=None)) == E["NULL_PTR"]
    assert call(a, other, window=0) == E["BAD_SHAPE"]
    for kw in (dict(n_seqs=3), dict(n_kv_heads=2), dict(head_dim=64)):
        assert call(a, cache(**{**dict(records=10 * FAKE, pos=12 * FAKE, weight=13 * FAKE, lens=15 * FAKE), **kw})) == E["BAD_SHAPE"]
    # half in place: the same records but another of something else; or arrays that share memory
    for kw in (dict(pos=7 * FAKE), dict(weight=7 * FAKE), dict(starts=7 * FAKE), dict(capacity_rows=999), dict(lens=5 * FAKE + 4)):
        assert call(a, cache(**kw)) == E["BAD_SHAPE"], kw
    base = dict(records=10 * FAKE, pos=12 * FAKE, weight=13 * FAKE, starts=14 * FAKE, lens=15 * FAKE)
    for kw in (dict(records=FAKE + 160), dict(pos=2 * FAKE + 400), dict(weight=3 * FAKE), dict(lens=5 * FAKE + 8)):
        assert call(a, cache(**{**base, **kw})) == E["BAD_SHAPE"], kw
    assert call(a, other, ws=None) == call(a, other, n=need - 1) == E["WORKSPACE"]
    assert call(a, other, ws=C.c_void_p(FAKE + 4)) == E["BAD_ALIGN"]


def test_python_layer_refuses_what_the_library_cannot_see(L):
    t = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt)        # noqa: E731
    rec, pos, w, starts, lens = t(10, 160, dt=torch.uint8), t(10), t(10, dt=torch.float32), t(9), t(8)
    c = B.make_q4_cache(rec, pos, w, starts, lens, 4)
    assert (c.n_seqs, c.n_kv_heads, c.head_dim, c.capacity_rows) == (2, 4, 128, 10)
    for bad in [(rec, pos[:9], w, starts, lens, 4), (rec, pos, w[:9], starts, lens, 4), (rec, pos, w, starts[:8], lens, 4),
                (rec, pos, w, starts, lens, 3), (rec, pos.long(), w, starts, lens, 4), (rec, pos, w.double(), starts, lens, 4),
                (rec[:, :], pos, w, starts[::2], lens[::2], 4)]:
        with pytest.raises(AssertionError):
            B.make_q4_cache(*bad)
    with pytest.raises(KeyError):
        B.make_q4_cache(t(10, 96, dt=torch.uint8), pos, w, starts, lens, 4)
    q = torch.zeros(2, 1, 16, 128)
    B.make_q4_attend(c, q, q)
    with pytest.raises(AssertionError):
        B.make_q4_attend(c, q[:1], q[:1])
    with pytest.raises(AssertionError):                              # not on a GPU
        B.slkv_q4_attend(c, B.make_q4_attend(c, q, q), q, q, rec)


def test_python_layer_refuses_arguments_made_for_another_cache(monkeypatch):
    # the library and the device taken away: a call that is not refused is seen
    calls = []
    monkeypatch.setattr(B, "_current_device", lambda: -1)
    monkeypatch.setattr(B, "_fn", {n: lambda *a: calls.append(a) or B.SLKV_OK for n in ("slkv_q4_attend", "slkv_q4_append")})
    t = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt)        # noqa: E731
    rec, pos, w, starts, lens = t(10, 160, dt=torch.uint8), t(10), t(10, dt=torch.float32), t(9), t(8)

    def make(rec, n_seg, n_kv_heads):
        c = B.make_q4_cache(rec, pos, w, starts[:n_seg + 1], lens[:n_seg], n_kv_heads)
        c.index = -1
        return c
    c = make(rec, 8, 4)
    q, new, at = torch.zeros(2, 1, 16, 128), torch.zeros(2, 1, 4, 128), t(2, 1)
    p = B.make_q4_attend(c, q, q)
    B.slkv_q4_attend(c, p, q, q, rec)
    B.slkv_q4_append(c, new, new, at, c)
    assert len(calls) == 2
    for other in (make(rec, 4, 4), make(rec, 4, 2), make(t(10, 80, dt=torch.uint8), 8, 4)):
        if (other.n_seqs, other.head_dim) != (2, 128):               # else: 16 query heads go with two KV heads as well
            with pytest.raises(AssertionError):
                B.slkv_q4_attend(other, p, q, q, rec)
        with pytest.raises(AssertionError):                          # lengths for fewer segments than are written
            B.slkv_q4_append(c, new, new, at, other)
    with pytest.raises(AssertionError):
        B.slkv_q4_append(c, new, new, at, make(rec, 8, 2))
    assert len(calls) == 2
