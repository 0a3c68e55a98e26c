"""The ends of the scales' range and refusals of 8-bit pools, without a GPU."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from test_paged_rope_window_host import ALL, UNS, _call


def test_oracle_saturates_where_codes_would_be_infinities():
    """240 * 2^120 is 1.875 * 2^127, the next code's value 2^128."""
    p = dict(k=np.zeros((1, 1, 16, 4)), v=np.zeros((1, 1, 16, 4)), pos=np.zeros((1, 1, 16), int), weight=np.ones((1, 1, 16)),
             k_scale=np.ones((1, 1, 1)), v_scale=np.ones((1, 1, 1)))
    most = float(torch.finfo(torch.bfloat16).max)
    x = np.array([[[most, -most, -np.inf, 1.75 * 2.0 ** 127]]])
    small = x / 2.0 ** 20
    p = P.append_scaled(small, x, small, np.array([[7]]), p, dict(table=[[0]], lens=[1], row_start=[0, 1]), 448.0)
    assert p["v_scale"].item() == 2.0 ** 120 and p["v"][0, 0, 0].tolist() == [240.0, -240.0, -240.0, 224.0]
    assert p["k_scale"].item() == 2.0 ** 100 and p["k"][0, 0, 0].tolist() == [256.0, -256.0, -448.0, 224.0]
    assert np.isfinite(np.float32(P.dequantised(p)["v"])).all()
    top = np.array([[[1.75 * 2.0 ** 127, 1.0, 0.0, 0.0]]])        # the largest that 448 codes hold
    p = P.append_scaled(top, top, top, np.array([[7]]), p, dict(table=[[0]], lens=[1], row_start=[0, 1]), 448.0)
    assert p["v_scale"].item() == 2.0 ** 119 and p["v"][0, 0, 0, 0] == 448.0


@pytest.mark.parametrize("change", [dict(dtype="f32"), dict(d=64, section=(8, 12, 12)), dict(dtype="f32", d=64, section=(8, 12, 12))])
def test_8_bit_pools_of_other_layouts_are_refused(change):
    if torch.cuda.is_available():
        pytest.skip("calls that are not refused would run over made-up addresses")
    got = _call(format=1, k_scale=None, v_scale=None, **change)
    assert {got[name] for name in ALL} == {UNS}
