"""Attention over an 8-bit cache with scores from 2^20 to 2^115 in size: one key has all the weight."""
import numpy as np
import pytest
import torch

import kv8_plain as plain
from test_gpu_kv8 import D, P, TORCH, _i32, _qo, _status, sv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("plan", [0, 1])
@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("ns,Hq,Hkv", [([1], 2, 1), ([5, 1], 8, 2), ([3, 20], 8, 4), ([6], 8, 1)])
@pytest.mark.parametrize("power", [24, 40, 60, 100])
@pytest.mark.parametrize("sign", [1, -1])
def test_the_largest_score_has_all_the_weight(plan, type_, ns, Hq, Hkv, power, sign):
    """K is the same in all of a key's dimensions and no two of a request's keys are alike, so scores are 128 q k scale and their order is that of k: with q < 0 the smallest
    key wins and all scores are negative.  The closest ones are apart by 2^24 * 2^-6 (e4m3: the steps of values from 2^-3 on) * 128 / sqrt(128) > 2^20: the others' weights are 0."""
    rng = np.random.default_rng(len(ns) + power)
    lens = [70, 33][:len(ns)]
    totals = np.array(lens) + np.array(ns)
    pages = -(-totals // P)
    table = np.full((len(ns), int(pages.max())), -1, np.int32)
    perm = rng.permutation(int(pages.sum()) + 2)
    bytes_ = np.arange(0x20, 0x7F) if type_ == "e4m3" else np.arange(1, 127)
    raw = rng.integers(0, 0x70, (2, len(perm), Hkv, P, D)).astype(np.uint8)
    qo = _qo(ns)
    M, G = int(qo[-1]), Hq // Hkv
    want, top = np.zeros((M, Hq, D)), np.zeros((M, Hq))
    v_scale = 0.25
    for i, (c, n, total) in enumerate(zip(lens, ns, totals)):
        table[i, :pages[i]] = perm[pages[:i].sum():pages[:i + 1].sum()]
        at = np.arange(total)
        for h in range(Hkv):
            keys = rng.permutation(bytes_)[:total].astype(np.uint8)
            raw[0, table[i, at // P], h, at % P] = keys[:, None]
            x = sign * plain.values(keys, type_)
            for j in range(n):
                best = int(np.argmax(x[:c + j + 1]))
                r, hs = int(qo[i]) + j, slice(h * G, (h + 1) * G)
                want[r, hs] = plain.values(raw[1, table[i, best // P], h, best % P], type_) * v_scale
                top[r, hs] = x[best] * D * 2.0 ** power / D ** 0.5
    dev = lambda a: torch.from_numpy(a).cuda().view(TORCH[type_])                 # noqa: E731
    scales = [torch.full((len(perm), Hkv), s, device="cuda") for s in (2.0 ** power, v_scale)]
    q = torch.full((M, Hq, D), float(sign), dtype=torch.bfloat16, device="cuda")
    out, lse, status = torch.full_like(q, 77.0), torch.full((M, Hq), 77.0, device="cuda"), _status()
    sv.spec_set_tuning("attn_plan", plan)
    try:
        size = sv.spec_verify_attn_quantized_workspace_bytes(len(ns), M, Hq, Hkv, D, 400, max(ns))
        wide = np.full((len(ns), 25), -1, np.int32)
        wide[:, :table.shape[1]] = table
        sv.spec_verify_attn_quantized(q, dev(raw[0]), dev(raw[1]), *scales, _i32(wide), _i32(lens), _i32(qo), out, lse, 400, max(ns), D ** -0.5, status,
                                      torch.empty(max(256, size), dtype=torch.uint8, device="cuda"))
    finally:
        sv.spec_set_tuning("attn_plan", 0)
    assert int(status) == 0
    assert np.array_equal(out.double().cpu().numpy(), want)                       # (8-bit values times a power of two are bf16 values)
    # lse: products of the score's factors in fp32, 2^-24 each, and its two conversions between logarithms
    assert (np.abs(lse.double().cpu().numpy() - top) <= 8 * 2.0 ** -24 * np.abs(top)).all()
