"""What the operators on a cache in pages refuse of numbers by sequence: host side, nothing is launched."""
import pytest

from tests.test_paged_refusals import ALIAS, M, SHAPE, UNSUPPORTED, append, cache, evict, forward, into, weights


def shared(c, value=1):
    c.numbers_by_sequence = value
    return c


@pytest.mark.parametrize("call", [append, forward, weights, evict])
@pytest.mark.parametrize("value", [2, -1, 256])
def test_a_layout_of_numbers_that_is_none(call, value):
    assert call(cache=shared(cache(), value)) == UNSUPPORTED


def test_the_extent_of_numbers_follows_their_layout():
    # one page of 16 * 2 numbers for every sequence's row of 640: the last of these lie 15 KB behind their beginning, just behind the first of the bounds
    few, at = dict(pages=1), 502 * M - 3 * 2 * 640 * 4 + 4
    for call in (append, weights):
        assert call(cache=shared(cache(**few)), weights=at) == ALIAS
    assert evict(cache=shared(cache(**few)), kept=700 * M + 3 * 2 * 640 * 4 - 4) == ALIAS
    assert evict(into=shared(into(**few)), kept=1700 * M + 3 * 2 * 640 * 4 - 4) == ALIAS


def test_more_numbers_than_64_bits_count():
    wide = dict(width=2 ** 31 - 1, page_size=2 ** 20, row=2 ** 31)
    for call, S in ((append, 65535), (weights, 65535)):
        assert call(cache=shared(cache(**wide)), S=S) == SHAPE
    assert evict(cache=shared(cache(**wide)), S=65535, keep=0, first=0, recent=0) == SHAPE


def test_numbers_by_sequence_are_not_moved_in_place():
    """They would be written where others of the same row are still to be read; by page they go where none is."""
    one = dict(k=cache().k, v=cache().v, pages=1000)
    assert evict(into=shared(into(**one)), cache=shared(cache()), into_weights=700 * M) == ALIAS
    assert evict(into=into(**one), cache=shared(cache()), into_weights=700 * M) == ALIAS
    assert evict(into=shared(into(**one)), cache=cache(), into_weights=700 * M) == ALIAS
    assert evict(cache=shared(cache()), into=shared(into()), into_weights=700 * M + 3 * 2 * 640 * 4 - 4) == ALIAS
