"""Row operators refuse to write the steps or positions that they read (host side, nothing is launched)."""
import pytest

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import layer_ops as lo
from tests.test_layer_rows_refusals import ALIAS, norm, rope, rotary, rows

OUT, OUT2 = 1 << 30, 1 << 31                                # of [2, 8, 4, 128] bf16: 4096 elements a batch entry
LAST = 2 * (4096 + 7 * 512 + 3 * 128 + 128)                 # bytes of it

WHERE = [
    dict(steps=OUT), dict(steps=OUT + LAST - 8), dict(steps=OUT - 8 * 63), dict(positions=OUT + 64), dict(positions=OUT - 4 * 7),
    dict(positions=OUT - 4 * (7 * 3 + 2), position_token=3, pairs=(32, 16, 16)), dict(positions=OUT - 4 * 1007, position_batch=1000),
]


@pytest.mark.parametrize("kw", WHERE)
def test_outputs(kw):
    assert rope(rot=rotary(**kw)) == ALIAS
    assert norm(rot=rotary(**kw)) == ALIAS


def test_the_second_output():
    moved = [{k: v - OUT + OUT2 if k in ("steps", "positions") else v for k, v in kw.items()} for kw in WHERE]
    assert all(norm(rot=rotary(**kw)) == ALIAS for kw in moved)


@pytest.mark.parametrize("at", [OUT, OUT2, 1 << 42, 1 << 43])
def test_gradients(at):
    """Gradients of rows and of weights, and the workspace."""
    for kw in (dict(steps=at + 128), dict(positions=at + 128)):
        assert lo._lib().sta_qk_norm_rope_backward(rows(), rows(1 << 25), rows(1 << 27), rows(1 << 28), None, rows(OUT), rows(OUT2), None, None, None, 1, 1 << 43, None,
                                                   1e-6, rotary(**kw), 2, 8, 128, None, None, 1 << 42, sta.sta_qk_norm_rope_workspace_bytes(128), None) == ALIAS
