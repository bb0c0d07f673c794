// spec_kv_quantize / spec_kv_dequantize: K/V rows into and out of a paged cache that holds 8 bits per element and an fp32 scale for every page and kv head.
//
// A cached element b of page p and kv head h stands for b * scale[p][h].  The scale that is written is a power of two, the smallest 2^e (e >= -126) with
// max|x| <= B 2^e (B = 448 for e4m3, 127 for int8) over the rows written to the page, and never smaller than the scale of the tokens that the page holds already, which are
// rounded again where it grows.  With powers of two every division by a scale is exact: an element is rounded once (to nearest even) by the 8-bit conversion alone,
// and rounding again costs e4m3 nothing above its subnormals.  (A scale of max|x| / 127 would use up to one more bit of int8, but each growth would shift
// every element of the page by up to half a step again.)
//
// Writing: a run is what consecutive rows put into consecutive slots of one page.  A wave owns one run of one kv head, of K or of V: its at most 16 rows are in registers at once
// (16 lanes x 16 bytes a row, 4 rows per load), so the maximum, the scale and the conversion need no second read and no workspace.  HBM-bound for prompts (2 bytes
// read, 1 written per element), a chain of dependent reads (slot, row, scale) for the rows of a decode batch.
// Reading: 16 lanes per row and kv head, 8 elements each.
#include "common.h"

namespace specv {

constexpr int kQD = 128;                     // head dimension
constexpr int kQP = 16;                      // tokens per page

// 8 consecutive cached elements as fp32
template <int TYPE>
__device__ inline void unpack8(u32x2 raw, float (&x)[8])
{
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const uint32_t b = w ? raw.y : raw.x;
        if constexpr (TYPE == SPEC_KV_E4M3) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)b, false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)b, true);
            x[4 * w] = lo[0]; x[4 * w + 1] = lo[1]; x[4 * w + 2] = hi[0]; x[4 * w + 3] = hi[1];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * w + e] = (float)(int8_t)(b >> (8 * e));
        }
    }
}

// ... and back: |x| is at most the type's largest value, rounded to nearest even
template <int TYPE>
__device__ inline u32x2 pack8(const float (&x)[8])
{
    u32x2 r;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t b;
        if constexpr (TYPE == SPEC_KV_E4M3) {
            int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w], x[4 * w + 1], 0, false);
            b = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2], x[4 * w + 3], v, true);
        } else {
            b = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) b |= ((uint32_t)(int)rintf(x[4 * w + e]) & 0xFFu) << (8 * e);
        }
        if (w) r.y = b; else r.x = b;
    }
    return r;
}

// The smallest 2^e, e >= -126, with amax <= B 2^e; 0 for 0.  B = m 2^k: the exponent of amax less k, one more where its fraction is above m's.
template <int TYPE>
__device__ inline float power_scale(float amax)
{
    constexpr int k = TYPE == SPEC_KV_E4M3 ? 8 : 6;
    constexpr uint32_t fraction = TYPE == SPEC_KV_E4M3 ? 0x600000u : 0x7E0000u;          // 448 = 1.75 x 2^8, 127 = 1.984375 x 2^6
    const uint32_t bits = __builtin_bit_cast(uint32_t, amax);
    int e = (int)(bits >> 23) - k + ((bits & 0x7FFFFFu) > fraction);                   // biased
    e = e < 1 ? 1 : e;
    return bits == 0 ? 0.0f : __builtin_bit_cast(float, (uint32_t)e << 23);
}

// Loads and stores of operands that are touched once, nontemporal where a call is too large for the memory-side cache.
template <bool STREAM, typename T>
__device__ inline T load_once(const void* at)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const T*>(at));
    else return *reinterpret_cast<const T*>(at);
}

template <bool STREAM, typename T>
__device__ inline void store_once(void* at, T x)
{
    if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<T*>(at));
    else *reinterpret_cast<T*>(at) = x;
}

struct QuantParams {
    const uint16_t* x[2];    // K, V rows
    uint8_t* cache[2];
    float* scale[2];
    const int32_t* slot_map;
    int32_t* status_flags;
    long row_stride;         // elements
    int M, Hkv, slots;       // slots = num_pages * 16
};

// WINDOW: rows whose runs a wave looks for.
template <int TYPE, int WINDOW, bool STREAM>
__global__ __launch_bounds__(256) void kv_quantize_kernel(QuantParams p)
{
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    // heads first, then K and V, then windows: waves that start together read neighbouring pieces of the same rows
    const uint32_t task = __builtin_amdgcn_readfirstlane(blockIdx.x * 4u + (threadIdx.x >> 6));
    const uint32_t unit = task / (uint32_t)p.Hkv, window = unit >> 1;
    const int h = (int)(task - unit * (uint32_t)p.Hkv), which = (int)(unit & 1u);
    const long row0 = (long)window * WINDOW;
    if (row0 >= p.M) return;
    // the window's slots, the one before (lane 0) and the 15 behind
    int slot = -1;
    const long mine = row0 - 1 + lane;
    if (lane <= WINDOW + 15 && mine >= 0 && mine < p.M) slot = p.slot_map[mine];
    const bool bad = slot < -1 || slot >= p.slots;
    if (bad) slot = -1;
    const int before = __shfl_up(slot, 1, 64);
    const bool follows = lane > 0 && slot >= 0 && before == slot - 1 && slot % kQP != 0 && before >= 0;
    const uint64_t chain = __ballot(follows);
    uint64_t starts = __ballot(lane >= 1 && lane <= WINDOW && slot >= 0 && !follows);
    int flags = __any(bad && lane >= 1 && lane <= WINDOW) ? SPEC_FLAG_BAD_PAGE : 0;

    const uint16_t* x = p.x[which];
    while (starts) {
        const int a = __ffsll((long long)starts) - 1;
        starts &= starts - 1;
        const int s0 = __builtin_amdgcn_readlane(slot, a), page = s0 / kQP, o = s0 % kQP;
        const int len = __ffsll((long long)~(chain >> (a + 1)));                       // (at most 16: a page ends the chain)
        const long r0 = row0 - 1 + a;
        uint8_t* to = p.cache[which] + ((size_t)page * p.Hkv + h) * (kQP * kQD) + l16 * 8;
        float* sp = p.scale[which] + (size_t)page * p.Hkv + h;
        // rows g, g + 4, g + 8, g + 12 of the run
        u32x4 v[4];
        const float stored = *sp;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = u32x4{0, 0, 0, 0};
            if (q * 4 + g < len) v[q] = load_once<STREAM, u32x4>(x + (r0 + q * 4 + g) * p.row_stride + (long)h * kQD + l16 * 8);
        }
        uint32_t top = 0;
        bool odd = false;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t lo = v[q][w] & 0xFFFFu, hi = v[q][w] >> 16;
                if ((lo & 0x7F80u) == 0x7F80u) { lo = 0; odd = true; }                 // infinities and NaN are stored as 0
                if ((hi & 0x7F80u) == 0x7F80u) { hi = 0; odd = true; }
                v[q][w] = lo | (hi << 16);
                top = max(top, max(lo & 0x7FFFu, hi & 0x7FFFu));                       // (magnitudes are ordered like their bits)
            }
        if (__any(odd)) flags |= SPEC_FLAG_BAD_KV;
        const float amax = four_rows_max(row16_max(__builtin_bit_cast(float, top << 16)));
        const float old = o > 0 && stored > 0.0f && stored < INFINITY ? stored : 0.0f;
        const float now = fmaxf(old, power_scale<TYPE>(amax));
        // a scale that the caller set need not be a power of two (2^127 has no reciprocal here)
        const bool power = (__builtin_bit_cast(uint32_t, now) & 0x7FFFFFu) == 0 && now < 0x1p127f;
        const float inverse = now > 0.0f ? __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, now)) : 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q * 4 + g < len) {
                float f[8];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    f[2 * w] = __builtin_bit_cast(float, v[q][w] << 16);
                    f[2 * w + 1] = __builtin_bit_cast(float, v[q][w] & 0xFFFF0000u);
                }
                if (power) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= inverse;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] /= now;
                }
                store_once<STREAM>(to + (o + q * 4 + g) * kQD, pack8<TYPE>(f));
            }
        if (now > old && o > 0) {                         // (seldom: the tokens before the run are read only here, 16384 single rows x heads 20.2 -> 18.9 us)
            const float ratio = old * inverse;            // now is a power of two here
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (q * 4 + g < o) {
                    float f[8];
                    unpack8<TYPE>(*reinterpret_cast<const u32x2*>(to + (q * 4 + g) * kQD), f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= ratio;
                    *reinterpret_cast<u32x2*>(to + (q * 4 + g) * kQD) = pack8<TYPE>(f);
                }
        }
        if (lane == 0 && !(stored == now)) *sp = now;
    }
    if (flags && lane == 0 && p.status_flags) atomicOr(p.status_flags, flags);
}

struct DequantParams {
    const uint8_t* cache[2];
    const float* scale[2];
    uint16_t* out[2];
    const int32_t* slot_map;
    int32_t* status_flags;
    long row_stride;
    int M, Hkv, slots;
};

template <int TYPE, bool STREAM>
__global__ __launch_bounds__(256) void kv_dequantize_kernel(DequantParams p)
{
    const int l16 = threadIdx.x & 15, which = blockIdx.y;
    const uint32_t pair = blockIdx.x * 16u + (threadIdx.x >> 4);
    const uint32_t row = pair / (uint32_t)p.Hkv;
    const int h = (int)(pair - row * (uint32_t)p.Hkv);
    if (row >= (uint32_t)p.M) return;
    const int slot = p.slot_map[row];
    if (slot < 0 || slot >= p.slots) {
        if (slot != -1 && l16 == 0 && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_PAGE);
        return;
    }
    const size_t unit = (size_t)(slot / kQP) * p.Hkv + h;
    const u32x2 raw = load_once<STREAM, u32x2>(p.cache[which] + (unit * kQP + slot % kQP) * kQD + l16 * 8);
    const float scale = p.scale[which][unit];
    float f[8];
    unpack8<TYPE>(raw, f);
    const u32x4 out = {pack_bf16x2(f[0] * scale, f[1] * scale), pack_bf16x2(f[2] * scale, f[3] * scale),
                       pack_bf16x2(f[4] * scale, f[5] * scale), pack_bf16x2(f[6] * scale, f[7] * scale)};
    store_once<STREAM>(p.out[which] + (long)row * p.row_stride + (long)h * kQD + l16 * 8, out);
}

static int check_rows(const char* who, const void* k, const void* v, int64_t row_stride, const int32_t* slot_map, const void* k_cache, const void* v_cache,
                      const float* k_scale, const float* v_scale, int num_pages, int M, int Hkv, int D, int page_size, int kv_type)
{
    if (M < 0 || Hkv <= 0 || num_pages < 0) return fail(SPEC_EINVAL, "%s: negative size (M=%d Hkv=%d num_pages=%d)", who, M, Hkv, num_pages);
    if (kv_type != SPEC_KV_E4M3 && kv_type != SPEC_KV_INT8) return fail(SPEC_EINVAL, "%s: unknown cache type %d", who, kv_type);
    if (D != kQD || page_size != kQP) return fail(SPEC_ESHAPE, "%s: built for D=128, page_size=16 (got D=%d page_size=%d)", who, D, page_size);
    if ((long)num_pages * page_size > 2147483647L) return fail(SPEC_ESHAPE, "%s: slots of %d pages do not fit 32 bits", who, num_pages);
    if ((long)M * Hkv > 2147483647L / 16) return fail(SPEC_ESHAPE, "%s: %d rows x %d heads beyond the launch grid", who, M, Hkv);
    if (M == 0) return SPEC_OK;
    if (!k || !v || !slot_map || !k_cache || !v_cache || !k_scale || !v_scale) return fail(SPEC_EINVAL, "%s: NULL pointer argument", who);
    if (row_stride < (int64_t)Hkv * D || row_stride % 8 != 0)
        return fail(SPEC_EINVAL, "%s: row_stride=%lld must be a multiple of 8 and at least Hkv * D", who, (long long)row_stride);
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16))
        return fail(SPEC_EINVAL, "%s: rows and caches must be 16-byte aligned", who);
    return SPEC_OK;
}

// 6 bytes are read and written per element of K and V.  Calls on three batches in turn, ordinary -> nontemporal, us: writing whole pages 49 MB 11.7 -> 12.6, 98 MB 20.5 -> 21.0, 197 MB
// 42.4 -> 38.0, 393 MB 79.2 -> 74.6; reading rows 49 MB 10.0 -> 12.4, 98 MB 24.0 -> 21.9, 197 MB 45.1 -> 40.8, 393 MB 86.9 -> 79.2 (5 TB/s; a copy of 4 GiB reaches 4.7).
static bool streams(int M, int Hkv) { return (size_t)M * Hkv * (6 * kQD) > kMemorySideCache * 5 / 16; }

template <int TYPE, int WINDOW>
static void launch_quantize_as(const QuantParams& p, hipStream_t s)
{
    const dim3 grid(((uint32_t)(p.M + WINDOW - 1) / WINDOW * (2u * (uint32_t)p.Hkv) + 3) / 4);
    if (streams(p.M, p.Hkv)) hipLaunchKernelGGL((kv_quantize_kernel<TYPE, WINDOW, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((kv_quantize_kernel<TYPE, WINDOW, false>), grid, dim3(256), 0, s, p);
}

// A wave takes the runs that start in its window one by one: with windows of 16 rows whole pages keep every wave busy, with windows of 4 single rows are not in a queue.  Windows of
// 4 / 16, us (4.5 to 5.5: what a call costs the host): pages of 8000 rows x heads 5.7 / 4.4, 16000 7.7 / 5.3, 32000 11.8 / 7.7, 128000 34 / 20; single rows, 2048 rows x heads
// 6.3 / 18.5, 16384 18.8 / 24.9, 65536 61 / 65.  (Windows of one row: 2048 5.2, 16384 19.7, 65536 70; pages of 16000 15.7.)
// The rule goes by rows x heads, which is all that the host knows of them, and is drawn for pages: single rows pay for it behind the line.
template <int TYPE>
static void launch_quantize(const QuantParams& p, hipStream_t s)
{
    if ((long)p.M * p.Hkv >= 24576) launch_quantize_as<TYPE, 16>(p, s);
    else launch_quantize_as<TYPE, 4>(p, s);
}

template <int TYPE>
static void launch_dequantize(const DequantParams& p, hipStream_t s)
{
    const dim3 grid((uint32_t)(((long)p.M * p.Hkv + 15) / 16), 2);
    if (streams(p.M, p.Hkv)) hipLaunchKernelGGL((kv_dequantize_kernel<TYPE, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((kv_dequantize_kernel<TYPE, false>), grid, dim3(256), 0, s, p);
}

}  // namespace specv

extern "C" int spec_kv_quantize(const void* k, const void* v, int64_t row_stride, const int32_t* slot_map,
                                void* k_cache, void* v_cache, float* k_scale, float* v_scale, int num_pages,
                                int M, int Hkv, int D, int page_size, int kv_type, int32_t* status_flags, void* stream)
{
    using namespace specv;
    if (int rc = check_rows("spec_kv_quantize", k, v, row_stride, slot_map, k_cache, v_cache, k_scale, v_scale, num_pages, M, Hkv, D, page_size, kv_type)) return rc;
    if (M == 0) return SPEC_OK;
    const QuantParams p{{(const uint16_t*)k, (const uint16_t*)v}, {(uint8_t*)k_cache, (uint8_t*)v_cache}, {k_scale, v_scale}, slot_map, status_flags,
                        (long)row_stride, M, Hkv, num_pages * kQP};
    if (kv_type == SPEC_KV_E4M3) launch_quantize<SPEC_KV_E4M3>(p, (hipStream_t)stream);
    else launch_quantize<SPEC_KV_INT8>(p, (hipStream_t)stream);
    return check_launch("spec_kv_quantize");
}

extern "C" int spec_kv_dequantize(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, int num_pages,
                                  const int32_t* slot_map, void* k, void* v, int64_t row_stride,
                                  int M, int Hkv, int D, int page_size, int kv_type, int32_t* status_flags, void* stream)
{
    using namespace specv;
    if (int rc = check_rows("spec_kv_dequantize", k, v, row_stride, slot_map, k_cache, v_cache, k_scale, v_scale, num_pages, M, Hkv, D, page_size, kv_type)) return rc;
    if (M == 0) return SPEC_OK;
    const DequantParams p{{(const uint8_t*)k_cache, (const uint8_t*)v_cache}, {k_scale, v_scale}, {(uint16_t*)k, (uint16_t*)v}, slot_map, status_flags,
                          (long)row_stride, M, Hkv, num_pages * kQP};
    if (kv_type == SPEC_KV_E4M3) launch_dequantize<SPEC_KV_E4M3>(p, (hipStream_t)stream);
    else launch_dequantize<SPEC_KV_INT8>(p, (hipStream_t)stream);
    return check_launch("spec_kv_dequantize");
}
