"""What the prompt attention and the paged cache refuse before anything is enqueued (no GPU)."""
import ctypes as C

import pytest

from paper_2508_15806_b200 import binding as B

P = 1 << 20                                                          # an aligned address that nobody follows
E = B.ERR


def cu(*lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return (C.c_int32 * len(out))(*out)


def prompt(**kw):
    f = dict(n_seqs=2, n_q_heads=8, n_kv_heads=2, head_dim=128, window=32, dtype=B.SLKV_BF16, lse_units=0, scale=0.1,
             q_stride_tok=1024, q_stride_head=128, k_stride_tok=256, k_stride_head=128, v_stride_tok=256, v_stride_head=128,
             o_stride_tok=1024, o_stride_head=128)
    f.update(kw)
    return B.SlkvPromptParams(**f)


def call_prompt(p, q=P, k=P, v=P, cu_dev=P, host=None, cu_k_dev=None, k_host=None, out=P, lse=None, ws=P, ws_bytes=1 << 40):
    return B.lib().slkv_prompt_attend(p, q, k, v, cu_dev, cu(5, 9) if host is None else host, cu_k_dev, k_host, out, lse, None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_seqs=0), "BAD_SHAPE"), (dict(n_seqs=1 << 30), "BAD_SHAPE"), (dict(n_q_heads=9), "BAD_SHAPE"), (dict(n_q_heads=0), "BAD_SHAPE"), (dict(n_kv_heads=0), "BAD_SHAPE"),
    (dict(n_q_heads=130), "BAD_SHAPE"), (dict(head_dim=96), "BAD_SHAPE"), (dict(window=0), "BAD_SHAPE"), (dict(dtype=2), "BAD_DTYPE"),
    (dict(lse_units=2), "BAD_DTYPE"), (dict(scale=0.0), "BAD_SHAPE"), (dict(scale=-1.0), "BAD_SHAPE"), (dict(scale=float("nan")), "BAD_SHAPE"),
    (dict(scale=float("inf")), "BAD_SHAPE"), (dict(scale=2.0 ** 55), "BAD_SHAPE"), (dict(scale=2.0 ** -55), "BAD_SHAPE"),
    (dict(q_stride_tok=64), "BAD_SHAPE"), (dict(k_stride_head=0), "BAD_SHAPE"), (dict(v_stride_tok=-256), "BAD_SHAPE"),
    (dict(o_stride_tok=1 << 38), "BAD_SHAPE"), (dict(q_stride_tok=1028), "BAD_ALIGN"), (dict(v_stride_head=132), "BAD_ALIGN"),
    (dict(o_stride_head=129), "BAD_ALIGN")])
def test_prompt_parameters(kw, code):
    p = prompt(**kw)
    assert call_prompt(p) == E[code]
    assert B.lib().slkv_prompt_attend_workspace_bytes(p, cu(5, 9), None) == 0


def test_prompt_arguments():
    p = prompt()
    assert B.lib().slkv_prompt_attend_workspace_bytes(p, cu(5, 9), None) >= 256
    assert B.lib().slkv_prompt_attend_workspace_bytes(p, cu(5, 9), cu(500, 9000)) > 256
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(cu_dev=None), dict(cu_k_dev=P), dict(k_host=cu(5, 9))):
        assert call_prompt(p, **kw) == E["NULL_PTR"], kw
    for kw in (dict(q=P + 8), dict(k=P + 8), dict(v=P + 2), dict(out=P + 4), dict(ws=P + 8)):
        assert call_prompt(p, **kw) == E["BAD_ALIGN"], kw
    assert call_prompt(p, ws=None) == E["WORKSPACE"] and call_prompt(p, ws_bytes=16) == E["WORKSPACE"]
    bad = cu(5, 9)
    bad[0] = 1
    assert call_prompt(p, host=bad) == E["BAD_SHAPE"]
    bad = cu(9, 5)
    bad[1] = 15
    assert call_prompt(p, host=bad) == E["BAD_SHAPE"]
    assert call_prompt(p, host=cu(2 ** 30, 2 ** 30 - 100)) == E["BAD_SHAPE"]
    assert call_prompt(p, cu_k_dev=P, k_host=cu(2 ** 30, 2 ** 30 - 100)) == E["BAD_SHAPE"]
    assert call_prompt(p, host=cu(0, 0), q=None, out=None) == 0       # no query: nothing to do
    assert B.lib().slkv_prompt_attend(None, P, P, P, P, cu(5), None, None, P, None, None, P, 1 << 40, None) == E["NULL_PTR"]


def cache(**kw):
    f = dict(n_layers=2, n_seqs=3, n_kv_heads=2, head_dim=128, dtype=B.SLKV_BF16, page_rows=32, n_pages=100, max_pages=10, k_pages=P, v_pages=P,
             tables=P, lens=P, free_pages=P, n_free=P)
    f.update(kw)
    return B.SlkvPagedCache(**f)


CACHES = [(dict(n_layers=0), "BAD_SHAPE"), (dict(n_seqs=0), "BAD_SHAPE"), (dict(n_kv_heads=0), "BAD_SHAPE"), (dict(n_seqs=8193), "BAD_SHAPE"),
          (dict(n_layers=1 << 18, n_seqs=8), "BAD_SHAPE"), (dict(head_dim=32), "BAD_SHAPE"), (dict(dtype=7), "BAD_DTYPE"),
          (dict(page_rows=8), "BAD_SHAPE"), (dict(page_rows=48), "BAD_SHAPE"), (dict(page_rows=256), "BAD_SHAPE"), (dict(n_pages=0), "BAD_SHAPE"),
          (dict(n_pages=1 << 27), "BAD_SHAPE"), (dict(max_pages=0), "BAD_SHAPE"), (dict(max_pages=1 << 27), "BAD_SHAPE"),
          (dict(n_seqs=4096, n_layers=60, max_pages=1 << 13), "BAD_SHAPE"), (dict(k_pages=None), "NULL_PTR"), (dict(v_pages=None), "NULL_PTR"),
          (dict(tables=None), "NULL_PTR"), (dict(lens=None), "NULL_PTR"), (dict(free_pages=None), "NULL_PTR"), (dict(n_free=None), "NULL_PTR"),
          (dict(k_pages=P + 8), "BAD_ALIGN"), (dict(v_pages=P + 8), "BAD_ALIGN")]


def plan(c, mode=0, want=P, slots=None, n_slots=0, width=0, offsets=None, lens_out=None, n_free_out=None):
    return B.lib().slkv_paged_plan(c, mode, want, slots, n_slots, width, offsets, lens_out, n_free_out, None, None)


def write(c, k=P, v=P, n_seqs=3, n_heads=2, n_tokens=4, strides=(1024, 256, 128) * 2, slots=P, n_slots=4, take=None):
    return B.lib().slkv_paged_write(c, k, v, n_seqs, n_heads, n_tokens, *strides, slots, n_slots, take, None)


def tree(**kw):
    f = dict(n_q_heads=8, n_tokens=4, layer=1, has_new=1, lse_units=0, scale=0.1)
    f.update({f"{x}_stride_{y}": z for x in "qokv" for y, z in (("seq", 4096), ("tok", 1024), ("head", 128))})
    f.update(kw)
    return B.SlkvPagedAttendParams(**f)


def attend(c, p, q=P, k=P, v=P, out=P, ws=P, ws_bytes=1 << 40):
    return B.lib().slkv_paged_attend(c, p, q, k, v, None, None, out, None, None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", CACHES)
def test_caches(kw, code):
    c = cache(**kw)
    assert plan(c) == write(c) == attend(c, tree()) == E[code]
    assert B.lib().slkv_paged_attend_workspace_bytes(c, tree()) == 0


def test_plan_arguments():
    c = cache()
    assert plan(c, mode=3) == E["BAD_DTYPE"] and plan(c, want=None) == E["NULL_PTR"]
    assert plan(c, slots=P, n_slots=5, width=0) == E["NULL_PTR"]      # ragged slots without offsets
    assert plan(c, slots=P, n_slots=47, width=4) == E["BAD_SHAPE"]
    assert plan(c, slots=P, n_slots=-1, offsets=P) == E["BAD_SHAPE"] and plan(c, slots=P, n_slots=1 << 31, offsets=P) == E["BAD_SHAPE"]
    assert plan(c, slots=P, n_slots=48, width=-1) == E["BAD_SHAPE"]
    assert plan(c, lens_out=2 * P) == E["NULL_PTR"] and plan(c, n_free_out=2 * P) == E["NULL_PTR"]
    assert plan(c, lens_out=P + 4, n_free_out=2 * P) == E["BAD_SHAPE"]
    assert plan(None) == E["NULL_PTR"]


def test_write_arguments():
    c = cache()
    for kw in (dict(k=None), dict(v=None), dict(slots=None)):
        assert write(c, **kw) == E["NULL_PTR"]
    for kw in (dict(n_seqs=0), dict(n_heads=0), dict(n_tokens=-1), dict(n_slots=-1), dict(n_slots=1 << 30), dict(strides=(1024, 256, 64) * 2),
               dict(strides=(1024, 256, 128, 1024, -256, 128))):
        assert write(c, **kw) == E["BAD_SHAPE"], kw
    assert write(c, strides=(1024, 260, 128) * 2) == E["BAD_ALIGN"] and write(c, k=P + 8) == E["BAD_ALIGN"]
    assert write(c, n_slots=0) == 0 and write(c, n_tokens=0, k=None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(n_q_heads=7), "BAD_SHAPE"), (dict(n_q_heads=130), "BAD_SHAPE"), (dict(n_tokens=0), "BAD_SHAPE"), (dict(n_tokens=65), "BAD_SHAPE"),
    (dict(layer=-1), "BAD_SHAPE"), (dict(layer=2), "BAD_SHAPE"), (dict(lse_units=5), "BAD_DTYPE"), (dict(scale=0.0), "BAD_SHAPE"),
    (dict(q_stride_tok=1), "BAD_SHAPE"), (dict(o_stride_seq=4100), "BAD_ALIGN"), (dict(k_stride_head=1 << 39), "BAD_SHAPE"),
    (dict(v_stride_seq=64), "BAD_SHAPE")])
def test_attend_parameters(kw, code):
    c, p = cache(), tree(**kw)
    assert attend(c, p) == E[code] and B.lib().slkv_paged_attend_workspace_bytes(c, p) == 0


def test_attend_arguments():
    c, p = cache(), tree()
    n = B.lib().slkv_paged_attend_workspace_bytes(c, p)
    assert n > 0
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None)):
        assert attend(c, p, **kw) == E["NULL_PTR"]
    for kw in (dict(q=P + 8), dict(k=P + 8), dict(v=P + 8), dict(out=P + 8), dict(ws=P + 8)):
        assert attend(c, p, **kw) == E["BAD_ALIGN"]
    assert attend(c, p, ws=None) == E["WORKSPACE"] and attend(c, p, ws_bytes=n - 1) == E["WORKSPACE"]
    assert attend(c, None) == E["NULL_PTR"]
    # strides of axes of length one say nothing; without drafted rows theirs are not looked at
    one = cache(n_seqs=1, n_kv_heads=1)
    assert B.lib().slkv_paged_attend_workspace_bytes(one, tree(n_tokens=1, k_stride_head=0, k_stride_tok=3, q_stride_seq=-5)) > 0
    assert B.lib().slkv_paged_attend_workspace_bytes(c, tree(has_new=0, k_stride_head=0, v_stride_tok=3)) > 0
