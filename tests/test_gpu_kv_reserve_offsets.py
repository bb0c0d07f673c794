"""spec_kv_reserve with row offsets that descend: a row would belong to two requests, so nobody is served."""
import numpy as np
import pytest

from test_gpu_kv8 import _qo, _reserve, _tables, sv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P_", [1, 16])
@pytest.mark.parametrize("B,M", [(4, 40), (4, 9000), (700, 5000), (1024, 4000), (1025, 4000), (2500, 9000)])
def test_no_pages_are_taken_where_offsets_descend(B, M, P_):
    rng = np.random.default_rng(B + M)
    lens, ns = rng.integers(0, 60, B), np.full(B, M // B)
    table, num_pages, free, count = _tables(rng, lens, ns, P_, spare=4 * M // P_ + 4)
    table = np.concatenate([table, np.full((B, 3 * (M // B) // P_ + 2), -1, np.int32)], 1)
    good = _qo(ns)
    for at in {1, B // 2, B - 1}:                             # the request before ends behind the start of the one after
        qo = good.copy()
        qo[at] = good[min(at + 2, B)]
        if qo[at] <= qo[at + 1]:
            qo[at] = qo[at + 1] + 1
        dev = _reserve(table, num_pages, lens, qo, free, count, M + 4, P_)
        assert int(dev["status"]) == sv.FLAG_BAD_LENGTH
        assert int(dev["count"]) == count and np.array_equal(dev["table"].cpu().numpy(), table)
        assert (dev["slots"] == -1).all()
    dev = _reserve(table, num_pages, lens, good, free, count, M + 4, P_)
    assert int(dev["status"]) == 0 and (dev["slots"][:int(good[-1])] >= 0).all() and (dev["slots"][int(good[-1]):] == -1).all()
