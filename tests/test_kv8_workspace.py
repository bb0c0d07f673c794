"""The workspace of attention over an 8-bit cache: sized once for a server's largest batch, it serves every smaller one."""
import ctypes
import random

import pytest
import torch

ONE = ctypes.c_void_p(4096)                                   # aligned, never dereferenced on the host


def _sizes(rng):
    Hq, Hkv = rng.choice([(8, 1), (32, 8), (16, 2), (12, 4), (64, 8), (40, 8), (7, 7), (1, 1), (128, 1)])
    return Hq, Hkv, int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 17)), rng.randint(1, 128 // (Hq // Hkv))


@pytest.mark.parametrize("tuning", [{}, {"attn_plan": 1}, {"attn_chunk": 128}, {"attn_plan": 1, "attn_chunk": 1000}, {"attn_plan_waves": 1}])
def test_a_smaller_batch_needs_no_more(tuning):
    from paper_2605_08151_amd import binding as sv
    rng = random.Random(len(tuning))
    size = sv.spec_verify_attn_quantized_workspace_bytes
    try:
        for name, value in tuning.items():
            sv.spec_set_tuning(name, value)
        for _ in range(4000):
            Hq, Hkv, B, keys, n = _sizes(rng)
            b, k, m = rng.choice([B, max(1, B // 2), rng.randint(1, B)]), rng.choice([keys, rng.randint(1, keys)]), rng.choice([n, rng.randint(1, n)])
            assert size(b, b * m, Hq, Hkv, 128, k, m) <= size(B, B * n, Hq, Hkv, 128, keys, n), (Hq, Hkv, B, keys, n, b, k, m)
    finally:
        for name in tuning:
            sv.spec_set_tuning(name, 0)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls have no tensors: without a GPU they end before a launch")
@pytest.mark.parametrize("tuning", [{}, {"attn_plan": 1}, {"attn_chunk": 128}, {"attn_plan": 1, "attn_chunk": 1000}])
def test_every_call_fits_the_answer(tuning):
    from paper_2605_08151_amd import binding as sv
    rng = random.Random(7)
    try:
        for name, value in tuning.items():
            sv.spec_set_tuning(name, value)
        for _ in range(3000):
            Hq, Hkv, B, keys, n = _sizes(rng)
            bytes_ = sv.spec_verify_attn_quantized_workspace_bytes(B, B * n, Hq, Hkv, 128, keys, n)
            rc = sv._lib.spec_verify_attn_quantized(ONE, ONE, ONE, ONE, ONE, ONE, keys // 16 + 1, 100, ONE, ONE, ONE, None, B, B * n, Hq, Hkv, 128, 16, 0, keys, n, 0.1,
                                                    None, ONE, bytes_, None)
            assert rc == -4, (rc, Hq, Hkv, B, keys, n)        # (past all checks: no device)
    finally:
        for name in tuning:
            sv.spec_set_tuning(name, 0)


@pytest.mark.gpu
def test_one_workspace_serves_smaller_batches():
    """Under these bounds 64 requests are taken whole and 32 are cut."""
    import numpy as np
    from test_gpu_kv8 import D, _attend, _attention, _check, sv
    ws = torch.empty(max(256, sv.spec_verify_attn_quantized_workspace_bytes(64, 320, 32, 8, D, 4096, 5)), dtype=torch.uint8, device="cuda")
    for B in (64, 32, 3, 1):
        b = _attention(B, np.random.default_rng(B).integers(0, 120, B), np.full(B, 5), 32, 8, "e4m3")
        out, lse, status, args = _attend(b, max_kv_len=4096)
        out.fill_(77.0)
        sv.spec_verify_attn_quantized(*args[:-1], ws)
        assert int(status) == 0
        _check(b, out, lse)


def test_a_step_without_the_workspace_says_so():
    from paper_2605_08151_amd.step import VerifyStep
    step = VerifyStep(1, 1, 8, 1, 128, 64, 64, 0, 100, device="cpu")
    with pytest.raises(AssertionError, match="quantized_cache=True"):
        step.attn_quantized(*[None] * 9)
