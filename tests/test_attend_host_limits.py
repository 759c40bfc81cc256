"""Prompt attention and paged attention at what their documentation allows: what can be seen of it on the host (no GPU)."""
import pytest

import test_attend_host as T
from paper_2508_15806_b200 import binding as B


def up256(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("paged", [False, True])
def test_workspaces_have_room_from_any_16_byte_boundary(paged):
    """Pieces are written 32 bytes at a time.  A workspace may begin 16 bytes off such a boundary, so it has to have room for the way to the next one."""
    def size(d):
        if paged:
            return B.lib().slkv_paged_attend_workspace_bytes(T.cache(head_dim=d, max_pages=1000), T.tree())
        return B.lib().slkv_prompt_attend_workspace_bytes(T.prompt(head_dim=d), T.cu(5, 9), T.cu(500, 9000))

    places, rest = divmod(size(128) - size(64), 64 * 4)              # rows of pieces: a row of head_dim floats, a reference and a sum each
    assert places > 0 and rest == 0
    n_pieces = places // 128                                           # of 128 rows: few tokens; 32 bytes each for what it belongs to
    for d in (64, 128):
        assert size(d) >= up256(places * d * 4) + up256(places * 8) + up256(n_pieces * 32) + 16


class Stream:
    cuda_stream = 0


@pytest.mark.parametrize("n", [3, 255, 256, 511, 512, 600, 5000])
def test_two_lists_of_any_length(n):
    """The binding hands over host offsets of queries and of keys, both as long as there are sequences."""
    p = T.prompt(n_seqs=n)
    call = B._fn["slkv_prompt_attend"]

    def status(cu_q, cu_k):
        return call(Stream, p, None, T.P, T.P, T.P, cu_q, T.P, cu_k, None, None, None, T.P, 1 << 40)

    none, keys = [0] * (n + 1), list(range(0, 3 * (n + 1), 3))
    assert status(none, keys) == status(tuple(none), tuple(keys)) == B.SLKV_OK      # no query: nothing to do, but both lists are looked through
    for i in (1, n // 2 + 1, n):
        bad = list(keys)
        bad[i] = -1
        assert status(none, bad) == B.ERR["BAD_SHAPE"], i
        bad = list(none)
        bad[i - 1] = 7
        assert status(bad, keys) == B.ERR["BAD_SHAPE"], i


@pytest.mark.parametrize("dtype,tile,blocks", [(B.SLKV_BF16, 128, 2), (B.SLKV_F32, 64, 1)])
@pytest.mark.parametrize("n_q_heads,n_tokens", [(8, 64), (8, 5), (24, 64), (128, 3)])
def test_tiles_of_a_layer_are_counted_in_32_bits(dtype, tile, blocks, n_q_heads, n_tokens):
    """Where the documentation draws the line, whatever the dimensions: the longest tables that are taken, and one page more."""
    G = n_q_heads // 2
    per = -(-n_tokens // (blocks * (128 // G)))
    segments = 1 << 14
    for new in (0, 1):
        most = ((1 << 31) - 1) // (segments * per) - 3 - new           # tiles of a table
        pages = most * tile // 64
        p = T.tree(n_q_heads=n_q_heads, n_tokens=n_tokens, layer=0, has_new=new)
        for n, good in ((pages, True), (pages + 1 + tile // 64, False)):
            c = T.cache(n_layers=1, n_seqs=segments // 2, page_rows=64, max_pages=n, dtype=dtype)
            if segments * n >= 1 << 31:                                  # the cache itself is refused
                continue
            assert (B.lib().slkv_paged_attend_workspace_bytes(c, p) > 0) == good
            assert T.attend(c, p, ws=None) == B.ERR["WORKSPACE" if good else "BAD_SHAPE"]
