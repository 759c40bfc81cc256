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
