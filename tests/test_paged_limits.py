"""Sizes at which launches of the operators on a cache in pages end: host side, nothing is launched (what is not refused for its size has an argument that is refused next)."""
import pytest

from tests.test_paged_refusals import ALIAS, M, SHAPE, both, evict, into, pool, rows, weights

S20 = 1 << 20


def many(S, max_q, D=64, width=64, **kw):
    """2 key heads of four heads each; keys for `width` pages of 16; numbers that are written over the bounds."""
    return weights(S=S, max_q=max_q, max_k=16 * width, D=D, q=rows(100 * M, token=512, head=64) if D == 64 else rows(100 * M),
                   cache=both_of(D, width), weights=502 * M, **kw)


def both_of(D, width):
    c = both(token=128, head=64, page=2048) if D == 64 else both()
    c.table_row = c.table_pages = width
    return c


@pytest.mark.parametrize("max_q", [1, 8, 100, 200, 5000])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_of_up_to_2_to_the_24_groups_of_256_keys(D, max_q):
    """Few rows, up to 512 and more: one workgroup for 256 keys of every sequence and key head where the launch is large."""
    assert many(S20 * 2 - 1, max_q, D) == ALIAS                             # 4 groups of 256 keys, 2 heads
    assert many(S20 * 2, max_q, D) == SHAPE
    assert many(S20, max_q, D) == ALIAS
    assert many(S20 * 8 - 1, max_q, D, width=16) == ALIAS and many(S20 * 8, max_q, D, width=16) == SHAPE


def test_numbers_beside_the_pages_of_two_pools():
    """One array may be the numbers of both caches where the pool is the same; page 3 of another pool as large would write the number that is read of page 3 of this one."""
    assert evict(into=into(pages=1000), into_weights=700 * M) == ALIAS
    assert evict(into=into(k=pool(200 * M), pages=1000), into_weights=700 * M) == ALIAS                 # keys in the same, values in another
    assert evict(into=into(k=pool(200 * M), v=pool(300 * M), pages=500), into_weights=700 * M) == ALIAS  # half of the same
