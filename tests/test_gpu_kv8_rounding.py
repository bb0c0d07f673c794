"""How near attention over an 8-bit cache comes to 64 bits, whatever the numbers of query rows of a request and of its neighbours."""
import numpy as np
import pytest

import kv8_plain as plain
from test_gpu_kv8 import D, _attend, _attention

pytestmark = pytest.mark.gpu


def _tolerance(out, size, span, keys):
    """A probability, times V's scale, is the sum of two bf16 numbers: the first is off by at most 2^-8 of it, and the second by 2^-8 of what the first left.  The output is
    rounded to bf16 once.  Scores, their exponentials and all sums are fp32 (as in kv8_plain.tolerance)."""
    score = (D + 4) * 2.0 ** -24 * span + 2.0 ** -22
    sums = (keys + 64) * 2.0 ** -24
    return 2.0 ** -8 * np.abs(out) + (2.0 ** -16 * (1 + 2.0 ** -8) + 4 * score + 2 * sums)[..., None] * size + 1e-30


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,ns,Hq,Hkv", [
    ([777, 30], [1, 1], 8, 1), ([300, 100], [5, 1], 32, 8), ([64, 900, 3], [9, 1, 2], 16, 2), ([1500], [16], 4, 1), ([250, 90], [6, 1], 8, 1), ([40, 2], [128, 1], 2, 2),
    ([2500, 20], [5, 1], 40, 8)])
def test_probabilities_are_rounded_to_two_bf16_numbers(type_, lens, ns, Hq, Hkv):
    for power in (True, False):
        b = _attention(sum(lens) + Hq, lens, ns, Hq, Hkv, type_, sharp=0.5, power=power)
        out, _, status, _ = _attend(b)
        assert int(status) == 0
        want, _, size, span = plain.attend(b["q"].double().numpy(), b["raw"][0], b["raw"][1], b["scale"][0], b["scale"][1], b["table"], b["lens"], b["qo"], 1 / D ** 0.5, type_)
        err = np.abs(out.double().cpu().numpy() - want)
        tol = _tolerance(want, size, span, b["L"])
        assert (err <= tol).all(), float((err / tol).max())
