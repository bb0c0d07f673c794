"""The 8-bit paged cache written plainly: numpy, 64 bits, a loop per request and run.  Test infrastructure only."""
import numpy as np

D, P = 128, 16
MOST = {"e4m3": 448.0, "int8": 127.0}


def e4m3_values():
    """The value of every e4m3 byte (S.EEEE.FFF, bias 7, no infinities, S.1111.111 is NaN)."""
    b = np.arange(256)
    e, f = (b >> 3) & 15, b & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * 2.0 ** (e.astype(np.float64) - 7))
    v = np.where((e == 15) & (f == 7), np.nan, v)
    return np.where(b >> 7, -v, v)


E4M3 = e4m3_values()


def values(raw, type_):
    """uint8 bytes -> what they stand for before the scale."""
    return E4M3[raw] if type_ == "e4m3" else raw.view(np.int8).astype(np.float64)


def to_bytes(x, type_):
    """fp64 -> bytes, to nearest, ties to even; |x| at most the type's largest value."""
    if type_ == "int8":
        return np.rint(x).astype(np.int8).view(np.uint8)
    size = np.abs(x)
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(size > 0, size, 1.0))), -6)
    step = 2.0 ** (e - 3)
    size = np.rint(size / step) * step
    order = E4M3[:127]                                        # 0 .. 448 ascending
    out = np.searchsorted(order, np.where(np.isnan(x), 0.0, size)).astype(np.uint8)
    out = np.where(np.isnan(x), 0x7F, out).astype(np.uint8)
    return (out | (np.signbit(x).astype(np.uint8) << 7)).astype(np.uint8)


def power_scale(amax, most):
    if amax == 0:
        return 0.0
    e = -126
    while amax > most * 2.0 ** e:
        e += 1
    return 2.0 ** e


def reserve(page_table, seq_lens, qo, free_list, free_count, M, num_pages, page_size):
    """(page table, free count, slots, flags)"""
    BAD_PAGE, BAD_LENGTH, NO_PAGES = 1, 2, 128
    table, slots, flags = page_table.copy(), np.full(M, -1, np.int32), 0
    B, width = table.shape
    have = min(max(int(free_count), 0), len(free_list))
    asks, total = [], 0
    for i in range(B):
        c, r0, n = int(seq_lens[i]), int(qo[i]), int(qo[i + 1]) - int(qo[i])
        hi = -(-(c + n) // page_size) if n > 0 else c // page_size
        asks.append(None)
        if n < 0 or c < 0 or r0 < 0 or r0 + n > M or (n > 0 and hi > width):
            flags |= BAD_LENGTH
            continue
        entries = table[i, c // page_size:hi] if n > 0 else table[i, :0]
        first = next((k for k, e in enumerate(entries) if e < 0), len(entries))
        if (entries[:first] >= num_pages).any() or (entries[first:] >= 0).any() or (n > 0 and c % page_size and first == 0):
            flags |= BAD_PAGE
            continue
        need = len(entries) - first
        total += need
        if need and total > have:
            flags |= NO_PAGES
            continue
        asks[i] = (c // page_size + first, need)
    taken = sum(a[1] for a in asks if a)
    at = have - taken
    for i in range(B):
        if asks[i] is None:
            continue
        first, need = asks[i]
        for g in range(first, first + need):
            page = int(free_list[at])
            at += 1
            if 0 <= page < num_pages:
                table[i, g] = page
            else:
                flags |= BAD_PAGE
        for j in range(int(qo[i + 1]) - int(qo[i])):
            pos = int(seq_lens[i]) + j
            page = table[i, pos // page_size]
            if page >= 0:
                slots[int(qo[i]) + j] = page * page_size + pos % page_size
    return table, have - taken if taken else int(free_count), slots, flags


def quantize(x, slots, cache, scale, type_):
    """One of K and V: x [M, Hkv, D] fp64; cache [pages, Hkv, P, D] uint8 and scale [pages, Hkv] fp32 are changed in place.  Returns flags."""
    BAD_PAGE, BAD_KV = 1, 256
    flags, total, r = 0, cache.shape[0] * P, 0
    while r < len(slots):
        s0 = int(slots[r])
        if not 0 <= s0 < total:
            flags |= BAD_PAGE if s0 != -1 else 0
            r += 1
            continue
        end = r + 1
        while end < len(slots) and slots[end] == slots[end - 1] + 1 and slots[end] % P:
            end += 1
        page, o = s0 // P, s0 % P
        for h in range(cache.shape[1]):
            rows = x[r:end, h]
            if not np.isfinite(rows).all():
                flags |= BAD_KV
                rows = np.where(np.isfinite(rows), rows, 0.0)
            stored = float(scale[page, h])
            old = stored if o > 0 and stored > 0 and np.isfinite(stored) else 0.0
            new = max(old, power_scale(np.abs(rows).max(), MOST[type_]))
            f32 = np.float32
            if new > old and o > 0:
                with np.errstate(invalid="ignore"):
                    cache[page, h, :o] = to_bytes((values(cache[page, h, :o], type_).astype(f32) * f32(old / new)).astype(np.float64), type_)
            q = (rows.astype(f32) / f32(new)).astype(np.float64) if new > 0 else rows * 0.0
            cache[page, h, o:o + end - r] = to_bytes(q, type_)
            scale[page, h] = new
        r = end
    return flags


def attend(q, k, v, ks, vs, page_table, seq_lens, qo, scale, type_, requests=None):
    """(out [M, Hq, D], lse [M, Hq], the mean of |V| under the probabilities [M, Hq, D], the largest sum of |scale * q * k| [M, Hq]), all fp64."""
    M, Hq, _ = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, size, lse, span = np.zeros((M, Hq, D)), np.zeros((M, Hq, D)), np.zeros((M, Hq)), np.zeros((M, Hq))
    for i in range(len(seq_lens)) if requests is None else requests:
        c, n = int(seq_lens[i]), int(qo[i + 1] - qo[i])
        pages = page_table[i, :-(-(c + n) // P)]
        for h in range(Hkv):
            K = (values(k[pages, h], type_) * ks[pages, h].astype(np.float64)[:, None, None]).reshape(-1, D)[:c + n]
            V = (values(v[pages, h], type_) * vs[pages, h].astype(np.float64)[:, None, None]).reshape(-1, D)[:c + n]
            for j in range(n):
                r, t = int(qo[i]) + j, c + j + 1
                rows = q[r, h * G:(h + 1) * G]
                z = scale * rows @ K[:t].T
                top = z.max(1, keepdims=True)
                e = np.exp(z - top)
                w = e / e.sum(1, keepdims=True)
                hs = slice(h * G, (h + 1) * G)
                out[r, hs], size[r, hs] = w @ V[:t], w @ np.abs(V[:t])
                lse[r, hs] = top[:, 0] + np.log(e.sum(1))
                span[r, hs] = (abs(scale) * np.abs(rows) @ np.abs(K[:t]).T).max(1)
    return out, lse, size, span


def tolerance(out, lse, size, span, keys):
    """How far a kernel may be off that rounds V's scaled probabilities and its output to bf16 (2^-8 each, relative) and holds the rest in fp32.

    A score is a sum of D products and two factors: off by at most (D + 4) 2^-24 span; so are the exponents, and exp2's own error is below 2^-22: a probability and
    the sum of all of them are off by twice that, relatively.  Sums over the keys add keys * 2^-24 each, the merge of split requests another few 2^-24."""
    score = (D + 4) * 2.0 ** -24 * span + 2.0 ** -22
    sums = (keys + 64) * 2.0 ** -24
    tol_out = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 * (1 + 2.0 ** -8) + 4 * score + 2 * sums)[..., None] * size + 1e-30
    tol_lse = 2 * score + sums + 2.0 ** -22 * (1 + np.abs(lse)) + 2.0 ** -22
    return tol_out, tol_lse
