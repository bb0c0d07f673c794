"""The 8-bit paged cache on the GPU, through the binding, against tests/kv8_plain.py (64 bits): pages and slots, writing and reading rows, attention."""
import numpy as np
import pytest
import torch

import kv8_plain as plain

pytestmark = pytest.mark.gpu

from paper_2605_08151_amd import binding as sv  # noqa: E402
from paper_2605_08151_amd.step import VerifyStep  # noqa: E402

D, P = plain.D, plain.P
TORCH = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _cache(raw, type_):
    """uint8 [pages, Hkv, P, D] on the host -> the device's typed cache"""
    return torch.from_numpy(raw).cuda().view(TORCH[type_])


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


def _qo(ns):
    return np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)


# ------------------------------------------------------------------------------------------------------------------
# spec_kv_reserve
# ------------------------------------------------------------------------------------------------------------------
def _reserve(table, num_pages, lens, qo, free, count, M, P_, fill=-7):
    dev = dict(table=_i32(table), free=_i32(free), count=_i32([count]), slots=torch.full((M,), fill, dtype=torch.int32, device="cuda"), status=_status())
    ws = torch.empty(max(256, sv.spec_kv_reserve_workspace_bytes(len(lens))), dtype=torch.uint8, device="cuda")
    sv.spec_kv_reserve(dev["table"], num_pages, _i32(lens), _i32(qo), dev["free"], dev["count"], dev["slots"], P_, dev["status"], ws)
    return dev


def _same_as_plain(table, num_pages, lens, qo, free, count, M, P_):
    want = plain.reserve(table, lens, qo, free, count, M, num_pages, P_)
    dev = _reserve(table, num_pages, lens, qo, free, count, M, P_)
    assert np.array_equal(dev["table"].cpu().numpy(), want[0])
    assert int(dev["count"]) == want[1]
    assert np.array_equal(dev["slots"].cpu().numpy(), want[2])
    assert int(dev["status"]) == want[3]
    assert np.array_equal(dev["free"].cpu().numpy(), free)
    return dev, want


def _tables(rng, lens, ns, P_, spare=5):
    """A page table that maps the committed tokens, and the free list of the other pages."""
    B = len(lens)
    has, wants = -(-lens // P_), -(-(lens + ns) // P_)
    num_pages = int(wants.sum()) + spare
    perm = rng.permutation(num_pages).astype(np.int32)
    table = np.full((B, int(wants.max()) + 1), -1, np.int32)
    first = np.concatenate([[0], np.cumsum(has)])
    for i in range(B):
        table[i, :has[i]] = perm[first[i]:first[i + 1]]
    count = num_pages - int(first[-1])
    free = np.full(num_pages, -1, np.int32)
    free[:count] = perm[first[-1]:]
    return table, num_pages, free, count


@pytest.mark.parametrize("B,ctx,n,P_,pad", [
    (1, 0, 1, 16, 0), (1, 15, 1, 16, 0), (1, 16, 1, 16, 3), (3, 100, 9, 16, 0), (256, 4000, 9, 16, 0), (1000, 60, 3, 16, 1), (1024, 500, 8, 16, 0), (1025, 40, 2, 16, 2),
    (2100, 50, 12, 16, 7), (5, 0, 5000, 16, 0), (64, 300, 300, 16, 100), (3, 7, 9000, 16, 1), (7, 33, 40, 1, 0), (9, 100, 50, 7, 5), (6, 1000, 700, 64, 0), (4, 0, 1, 128, 0)])
def test_reserve_is_the_plain_one(B, ctx, n, P_, pad):
    rng = np.random.default_rng(B * 7 + n)
    lens, ns = rng.integers(0, ctx + 1, B), rng.integers(0, n + 1, B)
    lens[0], ns[0] = ctx, n
    qo = _qo(ns)
    table, num_pages, free, count = _tables(rng, lens, ns, P_)
    dev, want = _same_as_plain(table, num_pages, lens, qo, free, count, int(qo[-1]) + pad, P_)
    assert want[3] == 0 and (want[2][:qo[-1]] >= 0).all() and (want[2][qo[-1]:] == -1).all()
    used = want[2][:qo[-1]]
    assert len(np.unique(used)) == len(used)
    # once more: everything is mapped, nothing is taken
    dev2 = _reserve(want[0], num_pages, lens, qo, free, want[1], len(want[2]), P_)
    assert int(dev2["count"]) == want[1] and np.array_equal(dev2["slots"].cpu().numpy(), want[2])
    # all rows taken back: the free list and the table are as they were
    sv.spec_kv_truncate(dev["table"], _i32(lens + ns), _i32(lens), dev["free"], dev["count"], P_, dev["status"])
    assert int(dev["count"]) == count and int(dev["status"]) == 0
    assert np.array_equal(dev["table"].cpu().numpy(), table)
    assert np.array_equal(dev["free"].cpu().numpy()[:count], free[:count])


@pytest.mark.parametrize("B,n,have", [(4, 40, 0), (4, 40, 5), (300, 9, 37), (1500, 9, 100), (5, 4000, 300), (5, 4000, 1000)])
def test_reserve_serves_as_far_as_the_free_list_goes(B, n, have):
    rng = np.random.default_rng(B + have)
    lens, ns = rng.integers(0, 200, B), rng.integers(1, n + 1, B)
    table, num_pages, free, count = _tables(rng, lens, ns, P)
    keep = min(count, have)
    free[keep:] = -1
    _, want = _same_as_plain(table, num_pages, lens, _qo(ns), free, keep, int(ns.sum()), P)
    wants = int((-(-(lens + ns) // P) - -(-lens // P)).sum())
    assert want[3] == (sv.FLAG_NO_PAGES if wants > keep else 0)


@pytest.mark.parametrize("rows", [1, 9000])
def test_reserve_leaves_out_what_does_not_fit(rows):
    """Lengths that do not fit, holes and foreign ids in the table, a free list with a foreign id, a counter beyond the list: flags, and no other request suffers."""
    rng = np.random.default_rng(3)
    lens = np.array([40, -3, 40, 33, 40, 20, 40, 2 ** 31 - 5, 10])
    ns = np.array([20, 4, 9, 20, 20, 200, 20, 9, rows])
    qo = _qo(ns)
    table, num_pages, free, count = _tables(rng, np.where(np.abs(lens) < 100, np.maximum(lens, 0), 0), ns, P)
    width = table.shape[1]
    table[0, 3] = 1                                           # mapped behind an unmapped entry (40 tokens + 20 rows: pages 2, 3)
    table[0, 2] = -1
    table[2, 2] = num_pages                                   # foreign id
    table[3, 2] = -1                                          # 33 tokens, but no page for the 33rd
    ns[5] = width * P                                         # more pages than the table has
    qo = _qo(ns)
    free[count - 3] = num_pages + 4                           # foreign id in the free list
    _, want = _same_as_plain(table, num_pages, lens, qo, free, count, int(qo[-1]), P)
    assert want[3] & (sv.FLAG_BAD_PAGE | sv.FLAG_BAD_LENGTH) == sv.FLAG_BAD_PAGE | sv.FLAG_BAD_LENGTH
    _same_as_plain(table, num_pages, lens, qo, free, len(free) + 100, int(qo[-1]), P)
    _same_as_plain(table, num_pages, lens, qo, free, -4, int(qo[-1]), P)
    _same_as_plain(table, num_pages, lens, qo, free, count, int(qo[-1]) - 1, P)              # the last request's rows end behind M


def test_reserve_without_requests_marks_all_rows():
    slots = torch.full((70,), 5, dtype=torch.int32, device="cuda")
    sv.spec_kv_reserve(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 8, _i32([]), _i32([0]), _i32(np.arange(8)), _i32([8]), slots, P, _status(),
                       torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert (slots == -1).all()


# ------------------------------------------------------------------------------------------------------------------
# spec_kv_quantize, spec_kv_dequantize
# ------------------------------------------------------------------------------------------------------------------
def _rows(rng, M, Hkv, spread=1.0):
    x = rng.normal(0, 1, (M, Hkv, D)) * np.exp(rng.normal(0, spread, (M, Hkv, 1)))
    return torch.from_numpy(x).to(torch.bfloat16)


def _slots(rng, lens, ns, spare=3):
    table, num_pages, free, count = _tables(rng, lens, ns, P, spare)
    _, _, slots, flags = plain.reserve(table, lens, _qo(ns), free, count, int(ns.sum()), num_pages, P)
    assert flags == 0
    return slots, num_pages


def _quantize_both(k, v, slots, raw, scale, type_, strided=False):
    """Runs the kernel and the plain form on copies of the cache; everything must be the same bit for bit."""
    want = [(raw[0].copy(), scale[0].copy()), (raw[1].copy(), scale[1].copy())]
    flags = 0
    for (c, s), x in zip(want, (k, v)):
        flags |= plain.quantize(x.double().numpy(), slots, c, s, type_)
    dev = [_cache(raw[0], type_), _cache(raw[1], type_), torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda()]
    status = _status()
    if strided:
        M, Hkv, _ = k.shape
        wide = torch.full((M, 2 * Hkv + 3, D), 9.0, dtype=torch.bfloat16, device="cuda")
        wide[:, 1:1 + Hkv], wide[:, 2 + Hkv:2 + 2 * Hkv] = k.cuda(), v.cuda()
        kd, vd = wide[:, 1:1 + Hkv], wide[:, 2 + Hkv:2 + 2 * Hkv]
    else:
        kd, vd = k.cuda(), v.cuda()
    sv.spec_kv_quantize(kd, vd, _i32(slots), *dev, status)
    for which in range(2):
        assert np.array_equal(dev[2 + which].cpu().numpy(), want[which][1], equal_nan=True), which
        assert np.array_equal(_bytes(dev[which]), want[which][0]), which
    assert int(status) == flags
    return dev, want, flags


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("B,ctx,n,Hkv,strided", [
    (1, 0, 1, 1, False), (1, 0, 1, 8, True), (5, 100, 1, 8, False), (7, 50, 9, 3, True), (40, 300, 5, 2, False), (3, 0, 700, 8, True), (30, 60, 400, 8, False), (2, 3, 5000, 7, True)])
def test_quantize_is_the_plain_one(type_, B, ctx, n, Hkv, strided):
    rng = np.random.default_rng(B + n)
    lens, ns = rng.integers(0, ctx + 1, B), rng.integers(1, n + 1, B)
    lens[0], ns[0] = ctx, n
    slots, pages = _slots(rng, lens, ns)
    raw = rng.integers(0, 256, (2, pages, Hkv, P, D)).astype(np.uint8)
    raw[(raw & 0x7F) == 0x7F] = 0x31                          # no NaN among the tokens that are there
    scale = (2.0 ** rng.integers(-12, 3, (2, pages, Hkv))).astype(np.float32)
    k, v = _rows(rng, len(slots), Hkv), _rows(rng, len(slots), Hkv, 3.0)
    _, want, flags = _quantize_both(k, v, slots, raw, scale, type_, strided)
    assert flags == 0
    # what a run does not write stays: the slots behind it, and the other pages
    untouched = np.setdiff1d(np.arange(pages), slots // P)
    assert len(untouched) and np.array_equal(want[0][0][untouched], raw[0][untouched])


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
def test_quantize_at_the_edges(type_):
    """Rows of zeros, of the smallest and the largest values, with infinities and NaN; slots of nobody; scales that a caller set; a fresh page's garbage scale."""
    rng = np.random.default_rng(11)
    Hkv, pages = 2, 40
    M = 24
    k = _rows(rng, M, Hkv)
    k[0] = 0
    k[1] = 2.0 ** -133                                        # a subnormal
    k[2] = torch.finfo(torch.bfloat16).max
    k[3, 0, 5], k[3, 1, 7], k[3, 0, 9] = float("inf"), float("-inf"), float("nan")
    k[4] = float("nan")
    k[5] = 448.0                                              # exactly the largest value at scale 1
    k[6] = 450.0
    k[7] = 127.0
    k[8] = 127.5
    k[9] = -0.0
    v = k.flip(0)
    slots = np.arange(M) * P                                  # a page of its own for every row ...
    slots[10:16] = 30 * P + 7 + np.arange(6)                  # ... a run that ends inside a page
    slots[16] = -1
    slots[17] = pages * P                                     # outside
    slots[18] = -2
    slots[19] = 31 * P + 15                                   # the last slot of a page, then the first of the one behind it in memory: two runs
    slots[20] = 32 * P
    slots[21] = 33 * P + 3                                    # scales that a caller set: larger than needed, no power of two, ...
    slots[22] = 34 * P + 3                                    # ... zero, ...
    slots[23] = 35 * P + 3                                    # ... NaN
    raw = rng.integers(0, 127, (2, pages, Hkv, P, D)).astype(np.uint8)
    scale = np.full((2, pages, Hkv), np.nan, np.float32)
    scale[:, 30:36] = 2.0 ** -9
    scale[:, 33], scale[:, 34], scale[:, 35] = 0.3, 0.0, np.nan
    dev, want, flags = _quantize_both(k, v, slots, raw, scale, type_)
    assert flags == sv.FLAG_BAD_KV | sv.FLAG_BAD_PAGE
    assert float(dev[2][5, 0]) == (1.0 if type_ == "e4m3" else 4.0) and float(dev[2][7, 0]) == (0.5 if type_ == "e4m3" else 1.0)
    assert float(dev[2][33, 0]) == np.float32(0.3)
    # one that is larger than any value needs, and the smallest and largest scales there are
    for s in (2.0 ** 127, 3e38, 2.0 ** -126, 1e-40):
        scale[:, 33] = s
        _quantize_both(k, v, slots, raw, scale, type_)


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
def test_tokens_of_a_page_keep_their_values_when_its_scale_grows(type_):
    """Sixteen calls of one row each, every row larger than the ones before: what the page stands for stays within the roundings that its scales allow."""
    rng = np.random.default_rng(5)
    Hkv = 3
    x = rng.normal(0, 1, (P, Hkv, D)) * 2.0 ** (np.arange(P)[:, None, None] / 2)
    x = torch.from_numpy(x).to(torch.bfloat16)
    dev = [torch.zeros((2, Hkv, P, D), dtype=torch.uint8, device="cuda").view(TORCH[type_]) for _ in range(2)]
    dev += [torch.full((2, Hkv), float("nan"), device="cuda") for _ in range(2)]
    for t in range(P):
        sv.spec_kv_quantize(x[t:t + 1].cuda(), (-x[t:t + 1]).cuda(), _i32([P + t]), *dev, None)
    back = [torch.empty((P, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sv.spec_kv_dequantize(*dev, _i32(P + np.arange(P)), *back, None)
    scale = dev[2][1].double().cpu().numpy()
    want = x.double().numpy()
    got = back[0].double().cpu().numpy()
    assert np.array_equal(got, -back[1].double().cpu().numpy())
    # int8: the steps of the scales that a token met are scale, scale / 2, ...: half of each, at most a whole step in sum; e4m3: half a step of 2^-3 at its
    # size once (scales are powers of two), and the same sum over the steps of its subnormals, 2^-9
    step = scale[None, :, None]
    tol = step if type_ == "int8" else 2.0 ** -4 * np.abs(want) + step * 2.0 ** -9
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("M,Hkv", [(1, 1), (17, 3), (1000, 8)])
def test_dequantize_reads_what_the_elements_stand_for(type_, M, Hkv):
    rng = np.random.default_rng(M)
    pages = M // P + 9
    raw = rng.integers(0, 256, (2, pages, Hkv, P, D)).astype(np.uint8)
    scale = rng.uniform(0.001, 3, (2, pages, Hkv)).astype(np.float32)          # no powers of two: one rounding to bf16
    slots = rng.integers(0, pages * P, M)
    if M > 1:
        slots[1], slots[M // 2], slots[-1] = -1, pages * P, -9
    status = _status()
    for strided in (False, True):
        wide = torch.full((M, 2 * Hkv + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
        k, v = (wide[:, :Hkv], wide[:, Hkv:2 * Hkv]) if strided else (wide[:, :Hkv].clone(), wide[:, Hkv:2 * Hkv].clone())
        sv.spec_kv_dequantize(_cache(raw[0], type_), _cache(raw[1], type_), torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda(), _i32(slots), k, v, status)
        assert int(status) == (sv.FLAG_BAD_PAGE if M > 1 else 0)
        good = (slots >= 0) & (slots < pages * P)
        for which, got in enumerate((k, v)):
            page, at = slots[good] // P, slots[good] % P
            x = plain.values(raw[which][page, :, at], type_).astype(np.float32) * scale[which][page][:, :, None]
            want = torch.full((M, Hkv, D), 7.0, dtype=torch.bfloat16)
            want[torch.from_numpy(good)] = torch.from_numpy(x).to(torch.bfloat16)
            assert torch.equal(torch.nan_to_num(got.cpu().float(), 1e9), torch.nan_to_num(want.float(), 1e9))
        assert (wide[:, 2 * Hkv:] == 7.0).all()


def test_the_binding_refuses_tensors_that_do_not_fit():
    cache, scale, slots = torch.zeros((4, 2, P, D), dtype=torch.int8, device="cuda"), torch.zeros((4, 2), device="cuda"), _i32([0, 1, 2])
    wide = torch.zeros((3, 5, D), dtype=torch.bfloat16, device="cuda")
    k = wide[:, :2].clone()
    heads_apart = k.transpose(0, 1).contiguous().transpose(0, 1)
    for k_, v_ in ((wide[:, :2], k), (heads_apart, heads_apart), (wide[:, ::2][:, :2], wide[:, ::2][:, :2]), (k.float(), k.float()), (k[:, :1], k[:, :1]), (k, k[:2])):
        with pytest.raises(AssertionError):
            sv.spec_kv_quantize(k_, v_, slots, cache, cache, scale, scale, None)
        with pytest.raises(AssertionError):
            sv.spec_kv_dequantize(cache, cache, scale, scale, slots, k_, v_, None)
    for c, v, s in ((cache.view(torch.uint8), cache, scale), (cache, cache.view(torch.float8_e4m3fn), scale), (cache, cache[:3], scale), (cache, cache, scale[:3]),
                    (cache, cache, scale.half()), (cache.transpose(1, 2), cache.transpose(1, 2), scale), (cache, cache, scale.cpu())):
        with pytest.raises(AssertionError):
            sv.spec_kv_quantize(k, k, slots, c, v, s, scale, None)
    with pytest.raises(AssertionError):
        sv.spec_kv_quantize(k, k, slots[:2], cache, cache, scale, scale, None)
    with pytest.raises(sv.SpecError):                         # a row that does not begin at a multiple of 16 bytes
        odd = torch.zeros(3 * 2 * D + 1, dtype=torch.bfloat16, device="cuda")[1:].view(3, 2, D)
        sv.spec_kv_quantize(odd, odd, slots, cache, cache, scale, scale, None)
    sv.spec_kv_quantize(wide[:, :2], wide[:, 2:4], slots, cache, cache.clone(), scale, scale.clone(), None)


# ------------------------------------------------------------------------------------------------------------------
# spec_verify_attn_quantized
# ------------------------------------------------------------------------------------------------------------------
def _attention(seed, lens, ns, Hq, Hkv, type_, sharp=1.0, power=True, slack=3):
    rng = np.random.default_rng(seed)
    lens, ns = np.asarray(lens), np.asarray(ns)
    qo = _qo(ns)
    pages = -(-(lens + ns) // P)
    num_pages = int(pages.sum()) + slack
    perm = rng.permutation(num_pages)
    table = np.full((len(lens), int(pages.max()) + 1), -1, np.int32)
    first = np.concatenate([[0], np.cumsum(pages)])
    for i in range(len(lens)):
        table[i, :pages[i]] = perm[first[i]:first[i + 1]]
    raw = rng.integers(0, 256, (2, num_pages, Hkv, P, D)).astype(np.uint8)
    if type_ == "e4m3":
        raw = plain.to_bytes(np.clip(rng.normal(0, 60, raw.shape), -448, 448), "e4m3")
    scale = (2.0 ** rng.integers(-8, -5, (2, num_pages, Hkv)) if power else rng.uniform(0.003, 0.03, (2, num_pages, Hkv))).astype(np.float32)
    # whatever no request sees may hold anything: NaN bytes behind the last token, NaN scales on pages of nobody
    nan = 0x7F if type_ == "e4m3" else 0x81
    for i in range(len(lens)):
        end = lens[i] + ns[i]
        if end % P:
            raw[:, table[i, end // P], :, end % P:] = nan
    raw[:, perm[first[-1]:]] = nan
    scale[:, perm[first[-1]:]] = np.nan
    q = torch.from_numpy(rng.normal(0, sharp, (int(qo[-1]), Hq, D))).to(torch.bfloat16)
    return dict(q=q, raw=raw, scale=scale, table=table, lens=lens, qo=qo, type=type_, num_pages=num_pages, Hq=Hq, Hkv=Hkv, n_max=int(ns.max()), L=int((lens + ns).max()))


def _attend(b, factor=None, max_kv_len=None, want_lse=True, pad=0, n_max=None, stream=None):
    M = b["q"].shape[0] + pad
    q = torch.zeros((M, b["Hq"], D), dtype=torch.bfloat16, device="cuda")
    q[:b["q"].shape[0]] = b["q"].cuda()
    L, n_max = max_kv_len or b["L"], n_max or b["n_max"]
    size = sv.spec_verify_attn_quantized_workspace_bytes(len(b["lens"]), M, b["Hq"], b["Hkv"], D, L, n_max)
    width = max(b["table"].shape[1], -(-L // P))
    table = np.full((len(b["lens"]), width), -1, np.int32)
    table[:, :b["table"].shape[1]] = b["table"]
    out = torch.full((M, b["Hq"], D), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((M, b["Hq"]), 77.0, device="cuda") if want_lse else None
    status = _status()
    args = (q, _cache(b["raw"][0], b["type"]), _cache(b["raw"][1], b["type"]), torch.from_numpy(b["scale"][0]).cuda(), torch.from_numpy(b["scale"][1]).cuda(),
            _i32(table), _i32(b["lens"]), _i32(b["qo"]), out, lse, L, n_max, 1 / D ** 0.5 if factor is None else factor, status,
            torch.full((max(256, size),), 0xFF, dtype=torch.uint8, device="cuda"))
    sv.spec_verify_attn_quantized(*args)
    return out, lse, status, args


def _check(b, out, lse, factor=None, requests=None):
    want, want_lse, size, span = plain.attend(b["q"].double().numpy(), b["raw"][0], b["raw"][1], b["scale"][0], b["scale"][1], b["table"], b["lens"], b["qo"],
                                              1 / D ** 0.5 if factor is None else np.float64(np.float32(factor)), b["type"], requests)
    tol, tol_lse = plain.tolerance(want, want_lse, size, span, b["L"])
    rows = np.concatenate([np.arange(b["qo"][i], b["qo"][i + 1]) for i in (range(len(b["lens"])) if requests is None else requests)])
    err = np.abs(out.double().cpu().numpy()[:len(want)] - want)[rows]
    assert (err <= tol[rows]).all(), float((err / tol[rows]).max())
    if lse is not None:
        err = np.abs(lse.double().cpu().numpy()[:len(want)] - want_lse)[rows]
        assert (err <= tol_lse[rows]).all(), float((err / tol_lse[rows]).max())


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,ns,Hq,Hkv", [
    ([0], [1], 1, 1), ([0, 1, 15, 16, 17], [1, 1, 1, 1, 2], 4, 2), ([31, 32, 33, 127, 128], [1, 2, 3, 4, 5], 8, 1), ([777], [1], 8, 1), ([300, 5], [1, 1], 7, 7),
    ([100, 200, 1], [5, 1, 3], 12, 4), ([511, 40], [9, 2], 8, 1), ([64, 130, 900], [4, 1, 5], 40, 8), ([250, 90], [6, 1], 16, 2), ([50, 513], [16, 1], 8, 1), ([10, 600], [128, 3], 2, 2),
    ([1300, 20, 4], [2, 2, 2], 64, 1), ([0, 2000], [25, 25], 5, 1)])
def test_attention_is_the_plain_one(type_, lens, ns, Hq, Hkv):
    for power in (True, False):
        b = _attention(sum(lens) + Hq, lens, ns, Hq, Hkv, type_, power=power)
        out, lse, status, _ = _attend(b)
        assert int(status) == 0
        _check(b, out, lse)


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("chunk,plan", [(128, 2), (256, 2), (8192, 2), (0, 1), (0, 2)])
@pytest.mark.parametrize("n,G", [(1, 4), (3, 8), (4, 8), (9, 8), (16, 8)])
def test_attention_of_split_requests(type_, chunk, plan, n, G):
    """Fixed chunks of several lengths, the work list, and every number of row tiles."""
    rng = np.random.default_rng(n * G)
    lens = np.concatenate([[0, 3000, 1], rng.integers(0, 1500, 4)])
    ns = rng.integers(1, n + 1, 7)
    ns[1] = n
    b = _attention(n + G, lens, ns, 2 * G, 2, type_, sharp=2.0)
    sv.spec_set_tuning("attn_chunk", chunk)
    sv.spec_set_tuning("attn_plan", plan)
    try:
        out, lse, status, args = _attend(b)
        assert int(status) == 0
        _check(b, out, lse)
        again = out.clone(), lse.clone()
        sv.spec_verify_attn_quantized(*args)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])       # nothing depends on timing
        # without lse, with bounds that are looser than the batch, and rows behind the last request left as they were
        loose, none, status, _ = _attend(b, max_kv_len=9000, want_lse=False, pad=3, n_max=128 // G)
        assert none is None and int(status) == 0
        _check(b, loose, None)
        assert (loose[-3:] == 77.0).all()
    finally:
        sv.spec_set_tuning("attn_chunk", 0)
        sv.spec_set_tuning("attn_plan", 0)


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
def test_attention_of_long_contexts(type_):
    b = _attention(4, [20000, 70000], [2, 5], 8, 1, type_)
    out, lse, status, _ = _attend(b)
    assert int(status) == 0
    _check(b, out, lse)


def test_attention_with_sharp_and_flat_scores_and_empty_scales():
    b = _attention(8, [500, 200, 40], [3, 1, 2], 8, 2, "e4m3", sharp=30.0)
    for factor in (0.0883, 4.0, 1e-6, 0.0):
        out, lse, status, _ = _attend(b, factor)
        _check(b, out, lse, factor)
    # pages of zeros (scale 0), and scales far apart inside one request
    b["scale"][:, b["table"][0, 3:9]] = 0.0
    b["scale"][:, b["table"][0, 12]] = 2.0 ** -100
    b["scale"][1, b["table"][0, 13]] = 2.0 ** 40
    out, lse, status, _ = _attend(b)
    _check(b, out, lse)
    b["scale"][:] = 0.0
    out, lse, status, _ = _attend(b)
    assert (out == 0).all()
    _check(b, out, lse)


@pytest.mark.parametrize("B,plan", [(300, 0), (300, 1), (1024, 1), (1025, 1), (1100, 0)])
def test_attention_of_many_requests(B, plan):
    """More requests than are ordered by length, as many as ranges are found for, and more."""
    rng = np.random.default_rng(B)
    b = _attention(B, rng.integers(0, 90, B), rng.integers(1, 4, B), 4, 1, "int8")
    sv.spec_set_tuning("attn_plan", plan)
    try:
        out, lse, status, _ = _attend(b)
    finally:
        sv.spec_set_tuning("attn_plan", 0)
    assert int(status) == 0
    _check(b, out, lse)


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("plan,n", [(1, 2), (2, 1), (1, 25)])
def test_attention_of_a_batch_too_large_for_the_cache(type_, shared, plan, n):
    """More than 96 MB of pages, with a prefix that all requests map or without: nontemporal loads or ordinary ones, and requests with more than 48 rows both."""
    rng = np.random.default_rng(n)
    lens = rng.integers(2500, 4500, 14)
    lens[3], lens[9] = lens.max(), lens.max()                 # (ties in the order by length)
    b = _attention(n, lens, np.full(14, n), 32, 8, type_)
    if shared:
        b["table"][:, :100] = b["table"][5, :100]
    sv.spec_set_tuning("attn_plan", plan)
    try:
        out, lse, status, _ = _attend(b)
    finally:
        sv.spec_set_tuning("attn_plan", 0)
    assert int(status) == 0
    _check(b, out, lse, requests=[0, 3, 9, 13])


def test_attention_with_a_negative_factor():
    for G in (4, 24):
        b = _attention(3, [200, 700], [1, 2], 2 * G, 2, "e4m3")
        out, lse, status, _ = _attend(b, -0.25)
        _check(b, out, lse, -0.25)


@pytest.mark.parametrize("plan", [1, 2])
def test_attention_skips_and_flags_what_breaks_a_bound(plan):
    b = _attention(6, [300, 200, 90, 50], [3, 4, 1, 2], 8, 2, "int8")
    sv.spec_set_tuning("attn_plan", plan)
    try:
        lens = b["lens"].copy()
        b["lens"] = np.array([300, -1, 90, 10 ** 6])
        out, lse, status, _ = _attend(b, max_kv_len=400)
        assert int(status) == sv.FLAG_BAD_LENGTH
        b["lens"] = lens
        for i in (1, 3):
            assert (out[b["qo"][i]:b["qo"][i + 1]] == 77.0).all() and (lse[b["qo"][i]:b["qo"][i + 1]] == 77.0).all()
        _check(b, out, lse, requests=[0, 2])
        for bad in (-1, b["num_pages"], 2 ** 31 - 1):
            keep = b["table"].copy()
            b["table"][1, 4] = bad
            out, lse, status, _ = _attend(b)
            b["table"] = keep
            assert int(status) == sv.FLAG_BAD_PAGE
            _check(b, out, lse, requests=[0, 2, 3])
    finally:
        sv.spec_set_tuning("attn_plan", 0)


def test_a_cache_beyond_32_bits_of_bytes():
    """Pages at the far end of a cache of more than 4 GiB each: written, read back, attended to."""
    Hkv = 8
    pages = (1 << 32) // (Hkv * P * D) + 700
    dev = [torch.empty((pages, Hkv, P, D), dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros((pages, Hkv), device="cuda") for _ in range(2)]
    rng = np.random.default_rng(2)
    n = 40
    k, v = _rows(rng, n, Hkv).cuda(), _rows(rng, n, Hkv).cuda()
    far = np.array([pages - 1, pages - 300, pages - 2])
    near = np.array([5, 90, 7])
    got = {}
    for name, ids in (("far", far), ("near", near)):
        slots = _i32(ids[np.arange(n) // P] * P + np.arange(n) % P)
        sv.spec_kv_quantize(k, v, slots, *dev, None)
        back = [torch.empty_like(k), torch.empty_like(k)]
        sv.spec_kv_dequantize(*dev, slots, *back, None)
        q = torch.from_numpy(np.random.default_rng(3).normal(0, 1, (1, 16, D))).to(torch.bfloat16).cuda()
        out, lse = torch.empty_like(q), torch.empty((1, 16), device="cuda")
        ws = torch.empty(max(256, sv.spec_verify_attn_quantized_workspace_bytes(1, 1, 16, Hkv, D, n, 1)), dtype=torch.uint8, device="cuda")
        sv.spec_verify_attn_quantized(q, *dev, _i32(ids[None]), _i32([n - 1]), _i32([0, 1]), out, lse, n, 1, 0.1, None, ws)
        got[name] = (*back, out, lse)
    for a, b in zip(got["far"], got["near"]):
        assert torch.equal(a, b)
    # a byte is off by at most half a step, which is the scale of its page
    half = 0.5 * dev[2][torch.from_numpy(far[np.arange(n) // P]).cuda()][:, :, None]
    assert ((got["far"][0].float() - k.float()).abs() <= half).all()


# ------------------------------------------------------------------------------------------------------------------
# together
# ------------------------------------------------------------------------------------------------------------------
def _round_inputs(rng, B, Hq, Hkv, gamma):
    ns = rng.integers(1, gamma + 2, B)
    qo = _qo(ns)
    M = int(qo[-1])
    return ns, qo, _rows(rng, M, Hkv, 0.5), _rows(rng, M, Hkv, 0.5), torch.from_numpy(rng.normal(0, 1, (M, Hq, D))).to(torch.bfloat16)


@pytest.mark.parametrize("type_", ["e4m3", "int8"])
def test_rounds_of_a_server_on_an_8_bit_cache(type_):
    """Prompts are admitted, then rounds of candidates: pages reserved, rows written, attended to, committed in part, pages of rejected rows returned."""
    rng = np.random.default_rng(21)
    B, Hq, Hkv, gamma, num_pages = 6, 8, 2, 4, 220
    dev = [torch.full((num_pages, Hkv, P, D), 0x7F, dtype=torch.uint8, device="cuda").view(TORCH[type_]) for _ in range(2)]
    dev += [torch.full((num_pages, Hkv), float("nan"), device="cuda") for _ in range(2)]
    raw, scale = np.full((2, num_pages, Hkv, P, D), 0x7F, np.uint8), np.full((2, num_pages, Hkv), np.nan, np.float32)
    table = torch.full((B, 40), -1, dtype=torch.int32, device="cuda")
    free = _i32(rng.permutation(num_pages))
    count, lens = _i32([num_pages]), _i32(np.zeros(B))
    for round_ in range(7):
        ns, qo, k, v, q = _round_inputs(rng, B, Hq, Hkv, 24 if round_ == 0 else gamma)
        M = int(qo[-1])
        step = VerifyStep(B, M, Hq, Hkv, D, 256, 1000, int(ns.max()) - 1, 640, quantized_cache=True)
        before = lens.cpu().numpy()
        step.reserve(table, num_pages, lens, _i32(qo), free, count)
        step.quantize(k.cuda(), v.cuda(), *dev)
        out = step.attn_quantized(q.cuda(), *dev, table, lens, _i32(qo), 0.0883)
        assert int(step.status) == 0
        slots = step.slot_map.cpu().numpy()
        for which, x in enumerate((k, v)):
            plain.quantize(x.double().numpy(), slots, raw[which], scale[which], type_)
            assert np.array_equal(_bytes(dev[which]), raw[which]) and np.array_equal(dev[2 + which].cpu().numpy(), scale[which], equal_nan=True)
        b = dict(q=q, raw=raw, scale=scale, table=table.cpu().numpy(), lens=before, qo=qo, type=type_, L=640)
        _check(b, out, step.lse, 0.0883)
        accepted = ns - 1 if round_ == 0 else rng.integers(0, ns)
        step.accept_len.copy_(_i32(accepted))
        step.commit(table, lens, _i32(qo), free, count)
        assert np.array_equal(lens.cpu().numpy(), before + accepted + 1)
        held = table[table >= 0]
        assert int(count) + held.numel() == num_pages and held.unique().numel() == held.numel()
        assert held.numel() == int((-(-lens // P)).sum())


def test_a_captured_round_is_replayed_like_the_eager_one():
    """Reserve, write and attend in one graph, on a stream of their own; between the replays the lengths move on and eager calls run."""
    rng = np.random.default_rng(31)
    B, Hq, Hkv, num_pages = 5, 8, 1, 120
    ns, qo, k, v, q = _round_inputs(rng, B, Hq, Hkv, 3)
    M = int(qo[-1])
    k, v, q, qo_d = k.cuda(), v.cuda(), q.cuda(), _i32(qo)
    table0 = np.full((B, 20), -1, np.int32)
    lens0 = np.array([0, 40, 100, 15, 16])
    pages = -(-lens0 // P)
    ids = rng.permutation(num_pages)
    for i in range(B):
        table0[i, :pages[i]] = ids[pages[:i].sum():pages[:i + 1].sum()]
    free0 = ids[pages.sum():]

    def state():
        dev = [torch.zeros((num_pages, Hkv, P, D), dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros((num_pages, Hkv), device="cuda") for _ in range(2)]
        return dict(dev=dev, table=_i32(table0), lens=_i32(lens0), free=_i32(free0), count=_i32([len(free0)]), accept=_i32(np.zeros(B)),
                    step=VerifyStep(B, M, Hq, Hkv, D, 256, 1000, int(ns.max()) - 1, 320, quantized_cache=True))

    def once(s):
        s["step"].reserve(s["table"], num_pages, s["lens"], qo_d, s["free"], s["count"])
        s["step"].quantize(k, v, *s["dev"])
        s["step"].attn_quantized(q, *s["dev"], s["table"], s["lens"], qo_d, 0.09)
        sv.spec_kv_commit(s["table"], s["lens"], qo_d, s["accept"], s["free"], s["count"], P, s["step"].status)

    eager, graphed, scratch = state(), state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once(scratch)                                         # (LDS limits and the like are set outside the capture)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once(graphed)
    for replay in range(5):
        graph.replay()
        once(eager)
        torch.cuda.synchronize()
        for name in ("table", "lens", "free", "count"):
            assert torch.equal(eager[name], graphed[name]), (replay, name)
        for a, b in zip(eager["dev"], graphed["dev"]):
            assert torch.equal(a, b), replay
        assert torch.equal(eager["step"].attn_out, graphed["step"].attn_out) and torch.equal(eager["step"].lse, graphed["step"].lse), replay
        assert torch.equal(eager["step"].slot_map, graphed["step"].slot_map) and int(graphed["step"].status) == 0
        once(scratch)


def test_calls_on_a_side_stream():
    """The calls run on torch's current stream."""
    b = _attention(12, [200, 90], [2, 1], 8, 2, "int8")
    want, want_lse, _, _ = _attend(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, lse, _, _ = _attend(b)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
