"""Committed lengths and row offsets at the end of 32 bits: the request is skipped and flagged, the others are computed."""
import numpy as np
import pytest

from test_gpu_kv8 import _attend, _attention, _check, sv

pytestmark = pytest.mark.gpu

TOP, LOW = 2 ** 31 - 1, -2 ** 31


@pytest.mark.parametrize("plan", [1, 2])
@pytest.mark.parametrize("n", [1, 12])
def test_quantized_attention_skips_lengths_that_pass_32_bits(plan, n):
    b = _attention(6, [300, 200, 90, 50], [3, 1, 1, 2], 8, 2, "int8")
    lens = b["lens"].copy()
    sv.spec_set_tuning("attn_plan", plan)
    try:
        for far in (TOP, TOP - 1):
            b["lens"] = np.array([300, far, 90, far])
            out, lse, status, _ = _attend(b, max_kv_len=400, n_max=max(3, n))
            b["lens"] = lens
            assert int(status) == sv.FLAG_BAD_LENGTH
            for i in (1, 3):
                assert (out[b["qo"][i]:b["qo"][i + 1]] == 77.0).all() and (lse[b["qo"][i]:b["qo"][i + 1]] == 77.0).all()
            _check(b, out, lse, requests=[0, 2])
    finally:
        sv.spec_set_tuning("attn_plan", 0)


@pytest.mark.parametrize("plan", [1, 2])
@pytest.mark.parametrize("far", [TOP, LOW, LOW + 3])
def test_quantized_attention_skips_offsets_that_pass_32_bits(plan, far):
    """The offset between requests 1 and 2 is far off: neither of them has rows, the others do."""
    b = _attention(9, [300, 200, 90, 50], [3, 1, 1, 2], 8, 2, "e4m3")
    qo = b["qo"].copy()
    sv.spec_set_tuning("attn_plan", plan)
    try:
        b["qo"] = np.array([qo[0], qo[1], far, qo[3], qo[4]], dtype=np.int64).astype(np.int32)
        out, lse, status, _ = _attend(b, max_kv_len=400)
    finally:
        sv.spec_set_tuning("attn_plan", 0)
    b["qo"] = qo
    assert int(status) == sv.FLAG_BAD_LENGTH
    assert (out[qo[1]:qo[3]] == 77.0).all() and (lse[qo[1]:qo[3]] == 77.0).all()
    _check(b, out, lse, requests=[0, 3])
