"""An eviction from about as many keys as a sequence can have, on the GPU."""
import pytest
import torch

import paper_2502_04507_amd as sta
from tests.paged_util import BF, DEV, ints, same
from tests.test_gpu_packed import randn

pytestmark = pytest.mark.gpu


def test_evict_of_two_billion_keys():
    """One page over and over, so that the rows take 128 MB, and numbers by sequence, 8.6 GB: a run of a wave ends less than its own length below 2^31."""
    page, D, keep = 1 << 20, 64, 64
    k, v = (randn((1, page, 1, D), i).to(DEV) for i in (1, 2))
    n, used = 2046, 2045 * page + 12345
    assert used + used // 16 > 2 ** 31
    cache = sta.StaPagedCache(k, v, torch.zeros((1, n), dtype=torch.int32, device=DEV), ints([used]), shared=True)
    w = torch.zeros(cache.weights_shape, device=DEV)
    most = [used - 1, 2 ** 31 - 2 ** 27 + 5, 2 ** 30 + 1, 2 ** 27, 10 ** 9 + 7, 77]
    w[0, 0, torch.tensor(most, device=DEV)] = torch.tensor([1.0, 5.0, 2.0, 1e-30, 3.0, 4.0], device=DEV)
    w[0, 0, used:] = 9.0                                        # places without a key
    into = sta.StaPagedCache(*[torch.zeros((2, 32, 1, D), dtype=BF, device=DEV) for _ in range(2)], ints([[1, 0]]), ints([0]))
    kept, to_w = torch.zeros((1, 1, keep), dtype=torch.int32, device=DEV), torch.zeros(into.weights_shape, device=DEV)
    sta.sta_paged_evict(cache, w, into, to_w, kept)
    want = sorted(list(range(keep - len(most))) + most)         # of equal ones the earlier
    assert kept[0, 0].tolist() == want and into.used.tolist() == [keep]
    at = torch.tensor([j % page for j in want], device=DEV)
    assert same(into.k[[1, 0]].flatten(0, 1), k[0, at]) and same(into.v[[1, 0]].flatten(0, 1), v[0, at])
    assert torch.equal(to_w[[1, 0]].flatten(), w[0, 0, torch.tensor(want, device=DEV)])
