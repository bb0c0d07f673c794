"""Committed lengths and row offsets at the end of 32 bits: the request is skipped and flagged, the others are computed."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import D, P, _attend, _attention, _check, _i32, sv

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


@pytest.mark.parametrize("far", [TOP, TOP - 1])
@pytest.mark.parametrize("n,G", [(1, 4), (5, 8), (16, 8)])
@pytest.mark.parametrize("chunk,plan,rows", [(0, 0, 0), (256, 2, 0), (0, 1, 0), (256, 2, 1), (256, 2, 2)])
def test_bf16_attention_skips_lengths_that_pass_32_bits(far, n, G, chunk, plan, rows):
    """The same bits as with a negative length in their place: nothing is written for such a request, and the others are cut up alike."""
    rng = np.random.default_rng(n)
    lens, Hkv, pages = [300, far, 700, 90, far], 2, 200
    cache = [torch.from_numpy(rng.normal(0, 1, (pages, Hkv, P, D))).to(torch.bfloat16).cuda() for _ in range(2)]
    q = torch.from_numpy(rng.normal(0, 1, (5 * n, Hkv * G, D))).to(torch.bfloat16).cuda()
    table, qo = _i32(rng.permutation(pages)[:5 * 40].reshape(5, 40)), _i32(np.arange(6) * n)
    table = torch.cat([table, table.flip(0)], 1).contiguous()
    got = []
    for name, value in (("attn_chunk", chunk), ("attn_plan", plan), ("attn_rows", rows)):
        sv.spec_set_tuning(name, value)
    try:
        for far_ in (-1, far):
            status = _i32([0])
            out, lse = torch.full_like(q, 77.0), torch.full((5 * n, Hkv * G), 77.0, device="cuda")
            ws = torch.zeros(max(256, sv.spec_verify_attn_workspace_bytes(5, 5 * n, Hkv * G, Hkv, D, 1000, n)), dtype=torch.uint8, device="cuda")
            sv.spec_verify_attn(q, *cache, table, _i32([far_ if c == far else c for c in lens]), qo, out, lse, 1000, n, 0.09, status, ws)
            assert int(status) == sv.FLAG_BAD_LENGTH
            got.append((out, lse))
    finally:
        for name in ("attn_chunk", "attn_plan", "attn_rows"):
            sv.spec_set_tuning(name, 0)
    for a, b in zip(*got):
        assert torch.equal(a, b)
        for i in range(5):
            assert (b[i * n:(i + 1) * n] == 77.0).all() == (lens[i] == far)
