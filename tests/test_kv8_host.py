"""The 8-bit cache without a GPU: what the host refuses, its size arithmetic, and the plain forms that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import kv8_plain as plain
from test_abi import LIB

ONE = ctypes.c_void_p(4096)                                   # aligned, never dereferenced on the host
ODD = ctypes.c_void_p(4100)


@pytest.fixture(scope="module")
def lib():
    from paper_2605_08151_amd import binding
    return binding._lib


def _text(lib):
    return lib.spec_last_error_string().decode()


def test_reserve_refuses(lib):
    def call(table=ONE, width=4, pages=8, lens=ONE, qo=ONE, free=ONE, cap=8, count=ONE, slots=ONE, B=2, M=4, P=16, ws=ONE, size=1 << 20):
        return lib.spec_kv_reserve(table, width, pages, lens, qo, free, cap, count, slots, B, M, P, None, ws, size, None)

    for bad in (dict(B=-1), dict(M=-1), dict(P=0), dict(width=-1), dict(pages=-1), dict(cap=-1)):
        assert call(**bad) == -1 and "size" in _text(lib)
    for bad in ("table", "lens", "qo", "free", "count", "slots"):
        assert call(**{bad: None}) == -1 and "NULL" in _text(lib)
    assert call(pages=1 << 27) == -2 and "32 bits" in _text(lib)
    assert call(ws=None) == -1 and call(ws=ODD) == -1 and "256-byte" in _text(lib)
    assert call(size=100) == -3
    assert call(B=0, M=0, table=None) == 0
    assert lib.spec_kv_reserve_workspace_bytes(0) == 0 and lib.spec_kv_reserve_workspace_bytes(-3) == 0
    assert lib.spec_kv_reserve_workspace_bytes(1) >= 256 + 8 and lib.spec_kv_reserve_workspace_bytes(5000) >= 256 + 40000


@pytest.mark.parametrize("name", ["spec_kv_quantize", "spec_kv_dequantize"])
def test_rows_into_and_out_of_the_cache_are_refused(lib, name):
    def call(k=ONE, v=ONE, stride=256, slots=ONE, kc=ONE, vc=ONE, ks=ONE, vs=ONE, pages=8, M=4, Hkv=2, D=128, P=16, type_=0):
        if name == "spec_kv_quantize":
            return lib.spec_kv_quantize(k, v, stride, slots, kc, vc, ks, vs, pages, M, Hkv, D, P, type_, None, None)
        return lib.spec_kv_dequantize(kc, vc, ks, vs, pages, slots, k, v, stride, M, Hkv, D, P, type_, None, None)

    for bad in (dict(M=-1), dict(Hkv=0), dict(pages=-1), dict(type_=2), dict(type_=-1), dict(stride=128), dict(stride=260)):
        assert call(**bad) == -1, bad
    for bad in ("k", "v", "slots", "kc", "vc", "ks", "vs"):
        assert call(**{bad: None}) == -1 and "NULL" in _text(lib)
    for bad in ("k", "v", "kc", "vc"):
        assert call(**{bad: ODD}) == -1 and "16-byte" in _text(lib)
    for bad in (dict(D=64), dict(P=32), dict(pages=1 << 27), dict(M=1 << 27, Hkv=8, stride=1024)):
        assert call(**bad) == -2, bad
    assert call(M=0, k=None, slots=None) == 0
    assert name in (call(M=-1), _text(lib))[1]


def test_attention_refuses(lib):
    def call(q=ONE, kc=ONE, vc=ONE, ks=ONE, vs=ONE, table=ONE, width=64, pages=100, lens=ONE, qo=ONE, out=ONE, B=2, M=4, Hq=8, Hkv=2, D=128, P=16, type_=0,
             L=1000, n=2, ws=ONE, size=1 << 30):
        return lib.spec_verify_attn_quantized(q, kc, vc, ks, vs, table, width, pages, lens, qo, out, None, B, M, Hq, Hkv, D, P, type_, L, n, 0.1, None, ws, size, None)

    for bad in ("q", "kc", "vc", "ks", "vs", "table", "lens", "qo", "out"):
        assert call(**{bad: None}) == -1 and "NULL" in _text(lib)
    for bad in (dict(B=-1), dict(M=-2), dict(Hq=0), dict(Hkv=-1), dict(width=0), dict(pages=0), dict(L=0), dict(n=0), dict(type_=2), dict(L=1025), dict(q=ODD), dict(kc=ODD), dict(vc=ODD)):
        assert call(**bad) == -1, bad
    for bad in (dict(D=64), dict(P=32), dict(Hq=9), dict(n=33), dict(n=1 << 30, Hq=2), dict(B=65536, M=65536), dict(M=1 << 29)):
        assert call(**bad) == -2, bad
    assert call(ws=None) == -1 and call(ws=ODD) == -1 and "256-byte" in _text(lib)
    long = dict(L=60000, width=4096)                          # (one that is cut up)
    assert call(ws=None, **long) == -1 and call(size=1000, **long) == -3 and "workspace" in _text(lib)
    assert call(B=0, q=None) == 0 and call(M=0, q=None) == 0
    bytes_ = lib.spec_verify_attn_quantized_workspace_bytes
    assert bytes_(0, 4, 8, 2, 128, 1000, 2) == 0 and bytes_(2, 4, 9, 2, 128, 1000, 2) == 0
    assert bytes_(8, 40, 8, 1, 128, 65536, 5) > 0


def test_the_binding_checks_its_tensors():
    from paper_2605_08151_amd import binding as sv
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    cache, scale = torch.zeros((4, 2, 16, 128), dtype=torch.int8), torch.zeros((4, 2))
    slots = torch.zeros(3, dtype=torch.int32)
    for bad in (dict(k=k.float()), dict(k=k[:, :1]), dict(cache=cache.to(torch.uint8)), dict(scale=scale[:3]), dict()):
        a = dict(k=k, cache=cache, scale=scale)
        a.update(bad)
        with pytest.raises(AssertionError):                   # (the last: tensors on the host)
            sv.spec_kv_quantize(a["k"], k, slots, a["cache"], cache, a["scale"], scale, None)
        with pytest.raises(AssertionError):
            sv.spec_kv_dequantize(a["cache"], cache, a["scale"], scale, slots, a["k"], k, None)


def test_plain_e4m3_is_torchs():
    b = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(b).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(plain.E4M3, want, equal_nan=True)
    # every value, every border between two neighbours (a tie), and its surroundings
    v = np.unique(plain.E4M3[~np.isnan(plain.E4M3)])
    ties = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, ties, ties * (1 + 2.0 ** -20), ties * (1 - 2.0 ** -20), np.random.default_rng(0).uniform(-448, 448, 10000), [0.0, -0.0, 1e-9, -1e-9]])
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(plain.to_bytes(x.astype(np.float32).astype(np.float64), "e4m3"), want)


def test_plain_scales_are_the_smallest_powers_of_two():
    for most in (448.0, 127.0):
        for amax in (1e-45, 2.0 ** -126, 1.0, 1.75, 1.7500001, 127.0, 127.5, 448.0, 450.0, 3.3e38):
            s = plain.power_scale(amax, most)
            assert amax <= most * s and (s == 2.0 ** -126 or amax > most * s / 2)
        assert plain.power_scale(0.0, most) == 0.0
