"""The grids of the row operators' launches (host side, nothing is launched)."""
import ctypes

import pytest

import paper_2502_04507_amd as sta

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("per", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("heads", [1, 3, 24, 196608])
def test_grids_hold_all_tokens_and_less_than_2_to_the_32_lanes(per, heads):
    grid = (ctypes.c_uint32 * 3)()
    sizes = {1, per, per + 1, 1000, MOST, MOST - per} | {min(MOST, (n + d) * per) for n in (2 ** 23, 2 ** 24, 2 ** 25) for d in (-1, 0, 1)}
    for tokens in sorted(sizes):
        sta.load_library().sta_rows_grid(ctypes.c_uint32(tokens), per, heads, grid)
        x, y, z = grid
        groups = -(-tokens // per)
        assert x * 256 < 2 ** 32 and y <= 65535 and z <= 65535 and y >= 1, tokens
        # workgroup (x, z) has the group of tokens z * 2^23 + x: all of them, each once
        assert x == min(groups, 2 ** 23) and z == -(-groups // 2 ** 23), tokens
        assert ((z - 1) * 2 ** 23 + x - 1) * per < 2 ** 32 - 64, tokens
        assert y == 1 or groups * y <= 1024 + groups, tokens
