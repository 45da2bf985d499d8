"""The example's conversation on a cache in pages, against the formulas on small sizes."""
import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu
from tests import paged_util as pu
from tests.test_gpu_examples import example

pytestmark = pytest.mark.gpu


def test_conversation_against_64_bits():
    """Queries and keys are rounded to bf16 behind norm and rotation, probabilities and the outputs once more, each with a relative error of at most 2^-8 of what is
    rounded: 2-norms within 2e-2, as the prompt layer's output.  Which keys stay follows the weights, whose sums differ from those in 64 bits by a relative 2^-8 or so through the
    rounded queries and keys: where two are closer than that either may stay, so the keys that stayed are taken from the run, and looked at for being among the greatest."""
    ex = example()
    Hq, Hkv, D, lengths, keep, window = 4, 2, 64, [150, 9, 80], 32, 16
    S, T, steps = len(lengths), sum(lengths), 3
    g = torch.Generator().manual_seed(7)
    qkv, further = (torch.randn(s, generator=g).to(torch.bfloat16) for s in ((1, T, Hq + 2 * Hkv, D), (steps, S, Hq + 2 * Hkv, D)))
    w = [1.0 + 0.2 * torch.randn(D, generator=g) for _ in range(2)]
    o, kept, outs = ex.conversation(qkv.cuda(), further.cuda(), [x.cuda() for x in w], lengths, Hq, Hkv, keep, page=8, window=window)
    turn, magnitude = sta.sta_rope_steps(D, theta=500000.0, scaling=sta.STA_ROPE_YARN, factor=4.0, original_positions=8192)

    def rows(x, positions):
        q, k, v = x.double().split([Hq, Hkv, Hkv], 1)
        angle = lu.angles(turn.tolist(), (D // 2,), torch.tensor(positions).numpy()[:, None])
        q, k = (lu.norm_rope(t[None], ww.double(), 1e-6, lambda y: lu.rotate(y, angle, False, magnitude))[0] for t, ww in ((q, w[0]), (k, w[1])))
        return q, k, v

    def rel(a, b):
        return float((a.cpu().double() - b).norm() / b.norm())

    kept, at = kept.cpu(), 0
    for s, n in enumerate(lengths):
        q, k, v = rows(qkv[0, at:at + n], list(range(n)))
        want, lse = lu.attention(q, k, v, True, D ** -0.5)
        assert rel(o[at:at + n], want) < 2e-2
        at += n
        m = min(n, window)
        weight = pu.weights(q[n - m:], k, lse[:, n - m:], True, D ** -0.5)
        keys, values = [], []
        for h in range(Hkv):
            stay = kept[s, h, :min(n, keep)].tolist()
            assert stay == sorted(set(stay)) and (n <= keep or set(range(4)) | set(range(n - keep // 4, n)) <= set(stay))
            gone = [j for j in range(n) if j not in stay]
            if gone:
                free = [j for j in stay if 4 <= j < n - keep // 4]
                assert float(weight[h][gone].max()) <= 1.05 * float(weight[h][free].min())
            keys.append(k[stay, h])
            values.append(v[stay, h])
        for i in range(steps):
            q1, k1, v1 = rows(further[i, s:s + 1], [n + i])
            keys = [torch.cat((a, k1[:, h])) for h, a in enumerate(keys)]
            values = [torch.cat((a, v1[:, h])) for h, a in enumerate(values)]
            want, _ = lu.attention(q1, torch.stack(keys, 1), torch.stack(values, 1), True, D ** -0.5)
            assert rel(outs[i][s:s + 1], want) < 2e-2
