"""What the binding hands to the library: tables of whole numbers that fit, or refused, where a cast would wrap or cut them without a word;
tensors that are missing are refused as the library does it."""
import numpy as np
import pytest
import torch

from paper_2508_21058_b200 import MocCross, MocError, MocRope
from paper_2508_21058_b200.binding import _rows, debug_cross_plan

WRAPS = np.array([0, 2**32 + 5])


@pytest.mark.parametrize("kw", [dict(q_off=WRAPS), dict(k_off=WRAPS), dict(k_len=WRAPS[1:]), dict(q_off=np.array([0, 2**31])), dict(q_off=[0, 5.5]),
                                dict(k_off=torch.tensor([0.0, 7.25])), dict(k_off=[0, float('nan')]), dict(k_off=[0, float('inf')]), dict(k_len=["3"]), dict(q_off=np.array([0, 2**32 + 5], np.uint64))])
def test_offsets_of_a_cross_attention(kw):
    args = dict(n_heads=1, n_kv_heads=1, head_dim=64, q_off=[0, 5], k_off=[0, 7], k_len=[3])
    args.update(kw)
    for call in (MocCross, debug_cross_plan):
        with pytest.raises(MocError) as e:
            call(**args)
        assert e.value.code == -2


def test_offsets_of_any_type():
    want = debug_cross_plan(1, 1, 64, [0, 5], [0, 7], [3])
    for t in (np.int64, np.uint8, np.int32, np.float64):
        assert debug_cross_plan(1, 1, 64, np.array([0, 5], t), np.array([0, 7], t), np.array([3], t)) == want
    assert debug_cross_plan(1, 1, 64, torch.tensor([0, 5]), torch.tensor([0, 7], dtype=torch.int32), (3,)) == want
    assert debug_cross_plan(1, 1, 64, [0], [0])["dq"] == 0 and debug_cross_plan(1, 1, 64, [0], [0], [])["dq"] == 0


def test_axes_of_a_rotation():
    assert MocRope(64, np.array([0, 2**32 + 1]) % 2, [1.0, 2.0]).n_axes == 2
    for axis in ([0, 2**32 + 1], np.array([0, 2**32 + 1]), [0.0, 0.5]):
        with pytest.raises(MocError) as e:
            MocRope(64, axis, [1.0, 2.0])
        assert e.value.code == -2


def test_a_missing_tensor():
    with pytest.raises(MocError) as e:
        _rows(None, 2, 3, 64, torch.bfloat16, "k_out", 0)
    assert e.value.code == -1
    with pytest.raises(MocError) as e:
        MocRope(64)._common(None, None, None, 0)
    assert e.value.code == -1
