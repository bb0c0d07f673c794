"""Attention over an 8-bit cache cut into ranges of a given number of keys: from ranges shorter than what a piece costs besides its steps to ones that hold several requests."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import _attend, _attention, _check, sv

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1], ids=["automatic", "ranges"])
def plan(request):
    sv.spec_set_tuning("attn_plan", request.param)
    yield request.param
    sv.spec_set_tuning("attn_plan", 0)
    sv.spec_set_tuning("attn_chunk", 0)


def _is_cut(args):
    """A call of whole requests takes any workspace, one that is cut up asks for its own."""
    with pytest.raises(sv.SpecError) as e:
        sv.spec_verify_attn_quantized(*args[:-1], args[-1][:256])
    return e.value.code == -3


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("chunk", [50, 128, 256, 1000, 8192])
@pytest.mark.parametrize("lens,ns,Hq,Hkv", [
    ([3000], [1], 4, 1), ([0, 3000, 1], [1, 1, 1], 8, 2), ([0, 2900, 1, 700, 128], [3, 3, 1, 2, 3], 16, 2), ([127, 128, 129, 2000], [5, 4, 5, 1], 8, 1), ([1500, 90], [9, 2], 16, 2),
    ([40, 1100], [2, 16], 8, 1)])
def test_ranges_of_a_given_number_of_keys(plan, type_, chunk, lens, ns, Hq, Hkv):
    b = _attention(chunk + sum(lens), lens, ns, Hq, Hkv, type_, sharp=2.0)
    sv.spec_set_tuning("attn_chunk", chunk)
    for bound in (b["L"], 9000):                              # (a loose bound: more ranges than have work)
        out, lse, status, args = _attend(b, max_kv_len=bound)
        assert _is_cut(args)
        assert int(status) == 0
        _check(b, out, lse)
        again = out.clone(), lse.clone()
        sv.spec_verify_attn_quantized(*args)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("chunk", [50, 300])
def test_a_request_that_is_refused_takes_no_range(plan, chunk):
    b = _attention(5, [600, 700, 3, 900], [2, 3, 1, 2], 8, 2, "e4m3")
    sv.spec_set_tuning("attn_chunk", chunk)
    lens = b["lens"].copy()
    b["lens"] = np.array([600, -1, 3, 900])
    out, lse, status, args = _attend(b)
    b["lens"] = lens
    assert _is_cut(args) and int(status) == sv.FLAG_BAD_LENGTH
    assert (out[2:5] == 77.0).all() and (lse[2:5] == 77.0).all()
    _check(b, out, lse, requests=[0, 2, 3])


def test_many_requests_in_short_ranges(plan):
    rng = np.random.default_rng(8)
    b = _attention(8, rng.integers(0, 700, 200), rng.integers(1, 4, 200), 8, 2, "int8")
    sv.spec_set_tuning("attn_chunk", 64)
    out, lse, status, args = _attend(b)
    assert _is_cut(args) and int(status) == 0
    _check(b, out, lse)
