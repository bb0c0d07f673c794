// spec_verify_attn_quantized: the attention of spec_verify_attn over pages that hold K and V in 8 bits with a scale per page and kv head.
//
//   S[t] = scale * ks[page(t)] * <q, K8_t>,  out = sum_t softmax(S)[t] * vs[page(t)] * V8_t
//
// The products run on the bf16 matrix cores: every e4m3 and int8 value is a bf16 value, so the conversion loses nothing, and the scales stay in fp32: K's is part of the
// softmax scale of a page's scores, V's is a factor of the page's probabilities.  Those enter the products as the sum of two bf16 numbers, the second being what the rounding to the first
// left: 2^-16 of a probability is lost, and the output's own rounding is what remains of the error (32 x 2048 keys, 5 rows against 64 bits: 0.0022 with one bf16 number, 0.0017 with two, as an
// fp32 form has; 28.6 -> 30.2 us, 256 mixed requests 115 -> 125, 8 x 32-64k 41.4 -> 43.6).  Scores, maxima, sums and O are fp32.
//
// HBM-bound: 256 bytes of K + V per key and kv head.
//   Work, one of two ways (quant_plan says when):
//   - ranges: the batch is cut into equal ranges of work, one per workgroup and kv head, wherever the requests' borders lie, so that all workgroups are resident at once and end
//     together; a workgroup finds its range itself from the lengths (no list, no launch before it).  A request that lies in one range is finished there; pieces of others leave
//     fp32 partials, at most two per range, which a second kernel merges.
//   - whole requests: a workgroup per request and kv head (and row group, while those are fewer than the compute units), the longest first; nothing to merge.
//   Calls, us (bytes of K and V at the rate over the call): 128 x 2.6k keys x 8 heads, 1 row 118 (5.7 TB/s); 32 x 2048 x 8, 5 rows 30.6 (4.5); 256 requests of 1 to 9 rows x 8
//   125 (4.3 with the second pass over the keys of those with more than 48 rows); 8 x 32-64k in int8, 5 rows x 8 44 (2.3); 1 x 777 keys 10.1.  Without the arithmetic of the
//   steps an earlier form that took 119, 32, 118, 45 took 113, 26, 107, 33: what is left is the stream, the chain lengths -> page ids -> pages, and the merges.
//   A step: a wave owns 32 keys (two pages) of every 128; its pages go straight to its own LDS (direct loads, two steps in flight: half the bytes of bf16 pages would otherwise
//   leave HBM idle) and from there to registers.  The waves share nothing but Q until their parts are merged.
//   Operands: scores are computed transposed (S^T = K Q^T), so that exp(S^T) is the B operand of O^T += V^T P^T.  The order of d in a score is free:
//   K: lane (l16, g) holds key l16, d = 32 g .. + 31: MFMA s contracts d = 32 g + 8 s .. + 7, and Q is laid out alike;
//   V: lane (l16, g) holds d = 8 l16 .. + 7 of keys 4 g .. 4 g + 3: byte t of the four rows, paired by v_perm, converts to the A operand of output tile t, whose rows are
//      d = 8 m + t.  A lane then ends with d = 32 g .. 32 g + 31 of its query row.
#include "attn_request.h"
#include "common.h"
#include "kv_stream.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace specv {

extern Tunable g_attn_chunk_override;
extern Tunable g_attn_plan;
extern Tunable g_attn_plan_waves;

constexpr int kD = 128;                      // head dimension
constexpr int kP = 16;                       // tokens per page
constexpr int kQuantWaves = 4;               // waves per workgroup
constexpr int kQuantThreads = kQuantWaves * 64;
constexpr int kQuantStep = kQuantWaves * 32; // keys per workgroup step
constexpr int kQuantTiles = 3;               // row tiles (16 query rows) at once; a request with more takes its keys again for the next ones
constexpr int kQuantStages = 2;              // steps of a wave that are in flight
constexpr int kQuantWgsPerCu = 2;            // 64 KB of pages each
constexpr int kQuantListed = 1024;           // requests whose ranges a workgroup finds (four per thread)
constexpr int kQuantOrdered = kQuantThreads;             // whole requests are taken longest first up to so many
constexpr int kQuantPageBytes = kP * kD;
constexpr int kQuantStageBytes = 4 * kQuantPageBytes;    // two pages of K, two of V
constexpr int kQuantWaveBytes = kQuantStages * kQuantStageBytes;
constexpr float kNegBig = -3.4028235e38f;    // "nothing seen yet" running maximum (log2 domain): below every score
constexpr float kMasked = -INFINITY;         // a masked score: 0 in the exponential below every maximum
constexpr float kMaxSlack = 6.0f;            // how far a score may exceed the reference before a rescale

typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));    // (rows of the output may start at any element)

struct QuantAttnParams {
    const uint16_t* q;
    const uint8_t* k;
    const uint8_t* v;
    const float* k_scale;    // [num_pages, Hkv]
    const float* v_scale;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* qo_indptr;
    uint16_t* out;           // [M, Hq, 128] bf16
    float* lse;              // [M, Hq] or null
    int32_t* status_flags;
    // ranges > 0: pieces of range r (its first request's, and its last one's where that goes on) are slots 2 r, 2 r + 1 of [max_q_len, Hq] rows;
    // req[i] = {range of request i's first piece, pieces}
    float* part_o;           // [2 ranges, max_q_len, Hq, 128]
    float* part_m;           // running maximum, log2 domain
    float* part_l;
    u32x2* req;
    int max_pages, num_pages, Hq, Hkv, G, M, B, max_kv_len, max_q_len;
    int ranges;              // 0: a workgroup takes a whole request
    int min_work;            // of a range, and at least the work of one step of any request
    uint32_t g_magic;        // r / G = r * g_magic >> 16 for r < 256
    int by_length;           // whole requests: the longest first
    int groups;              // whole requests: row groups are workgroups of their own (1: the workgroup takes them all)
    float scale_log2e;       // >= 0
    float stream_keys;       // committed keys of the batch above which its pages are too large for the memory-side cache
    uint32_t q_sign;         // flips the sign of two query elements: a negative softmax scale
};

// two cached elements (bytes 2 HI, 2 HI + 1 of a word) as bf16
// (e4m3: times a power of two)
template <int TYPE, bool HI>
__device__ inline uint32_t bf16_pair(uint32_t raw, float power = 1.0f)
{
    if constexpr (TYPE == SPEC_KV_E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw, power, HI));
    else return pack_bf16x2((float)(int8_t)(raw >> (HI ? 16 : 0)), (float)(int8_t)(raw >> (HI ? 24 : 8)));
}

// (The empty statement keeps the words whole up to here: the compiler otherwise takes them apart where they are loaded, into a register per byte.)
template <int TYPE>
__device__ inline bf16x8 bf16_oct(uint32_t a, uint32_t b)
{
    asm("" : "+v"(a), "+v"(b));
    const u32x4 w = {bf16_pair<TYPE, false>(a), bf16_pair<TYPE, true>(a), bf16_pair<TYPE, false>(b), bf16_pair<TYPE, true>(b)};
    return __builtin_bit_cast(bf16x8, w);
}

__device__ inline bool quant_request_ok(int r0, int n, int c, const QuantAttnParams& p)
{
    return attn_request_fits(r0, n, c, p.M, p.max_q_len, p.max_kv_len);
}

// Work of one step of a request with `rows` query rows per kv head: a pass over the keys per kQuantTiles row tiles, and the tiles' products (128 keys in a full CU
// take 1.31, 1.32, 1.48, 2.92, 4.70 us with 1, 2, 3, 4, 8 tiles: up to 3 the stream bounds an even batch; in one where it does not they take 0.95, 1.36, 1.65).
__host__ __device__ constexpr int quant_step_work(int rows)
{
    const int tiles = (rows + 15) / 16;
    return (tiles + kQuantTiles - 1) / kQuantTiles * 4 + tiles;
}

// ... and of a piece besides its steps: its first pages' round trip, the merge of its waves (0 / 20 / 40: 256 mixed requests 139 / 125 / 123 us, 8 x 32-64k 48 / 45 / 44,
// 128 decode rows x 8 heads as ranges 129 / 132 / 134)
__host__ __device__ constexpr int quant_piece_work(int rows) { return ((rows + 15) / 16 + kQuantTiles - 1) / kQuantTiles * 20; }

// One piece: keys kbeg .. kend (kbeg a multiple of 128) of request i for one kv head.
struct QuantPiece { int i, r0, n, c, kbeg, kend; bool whole; size_t slot; };

// A request's first row, rows and committed tokens, the same in every lane by construction: control flow and addresses that depend on them stay scalar.
struct QuantRequest { int r0, n, c; };

// (read through the scalar cache: a vector load would be waited for together with the pages in flight behind it)
__device__ inline int scalar_load(const int32_t* x, int i)
{
    return ((const __attribute__((address_space(4))) int32_t*)reinterpret_cast<uint64_t>(x))[i];
}

__device__ inline QuantRequest quant_request(const QuantAttnParams& p, int i)
{
    const int r0 = scalar_load(p.qo_indptr, i);
    return {r0, attn_request_rows(r0, scalar_load(p.qo_indptr, i + 1)), scalar_load(p.seq_lens, i)};
}

// An address that is the same in every lane, in scalar registers whatever the compiler makes of what it is computed from.  The s_nop is the distance that a load written
// in assembly needs from a vector instruction that writes its scalar base.
__device__ inline const uint8_t* scalar_address(const uint8_t* x)
{
    const uint64_t bits = reinterpret_cast<uint64_t>(x);
    uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(bits >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)bits);
    asm volatile("s_nop 4" : "+s"(at));
    return reinterpret_cast<const uint8_t*>(at);
}

// NR: row tiles at once.
template <int NR, int TYPE>
struct QuantKernel {
    static constexpr int NW = kQuantWaves;
    static constexpr int kTileBytes = 16 * kD * 4;        // a row tile of O
    static_assert(kQuantStages == 2 && kTileBytes <= kQuantStageBytes, "the waits count the loads of one younger step; the merge has the place of the second");
    // LDS: the waves' pages, Q, the waves' maxima and sums
    static constexpr size_t kQAt = NW * kQuantWaveBytes, kMlAt = kQAt + (NR == 1 ? 0 : NR * 4 * 64 * 16), kBytes = kMlAt + 2 * NW * NR * 16 * 4;

    // Pieces one behind the other, `first` and then what next(piece, group) makes of the last one.  While a piece is computed the page ids of the next one are fetched; its
    // scales, queries and first pages fly while the waves' parts of this one are merged.
    template <typename Next>
    static __device__ __forceinline__ void run(const QuantAttnParams& p, unsigned char* smem, int kvh, QuantPiece u, int group, Next next)
    {
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int l16 = lane & 15, g = lane >> 4;
        u32x4* sQ = reinterpret_cast<u32x4*>(smem + kQAt);                             // [NR * 4][64], not with one row tile
        float* s_m = reinterpret_cast<float*>(smem + kMlAt);                           // [NW][NR * 16]
        float* s_l = s_m + NW * NR * 16;
        unsigned char* ring = smem + wave * kQuantWaveBytes;
        int bad_page = 0;

        // ---- page ids and scales of this wave's steps, 32 steps at a time: lane l holds page l % 2 of step l / 2 (page 0 stands in for a bad id, which is flagged,
        // and with scales 0 for what lies behind the piece).  K's scale is that of a score; V's is a power of two, which the conversion of e4m3 applies, and the rest, a
        // factor of the probabilities that is 1 for the scales that spec_kv_quantize sets ----
        struct Pages { int id; float ks, vm; uint32_t ve; };
        auto page_at = [&](int step) { return (step + (lane >> 1)) * (kQuantStep / kP) + 2 * wave + (lane & 1); };
        auto load_ids = [&](const QuantPiece& x, int step) {
            const int pg = page_at(step);
            int id = 0;
            if (pg * kP < x.kend - x.kbeg) {
                id = p.page_table[(size_t)x.i * p.max_pages + x.kbeg / kP + pg];
                if (id < 0 || id >= p.num_pages) { id = 0; bad_page = 1; }
            }
            return id;
        };
        auto load_scales = [&](const QuantPiece& x, int step, int id) {
            Pages r{id, 0.0f, 0.0f, 0x3F800000u};
            if (page_at(step) * kP < x.kend - x.kbeg) {
                r.ks = p.k_scale[(size_t)id * p.Hkv + kvh] * p.scale_log2e;
                r.vm = p.v_scale[(size_t)id * p.Hkv + kvh];
                if constexpr (TYPE == SPEC_KV_E4M3) {
                    const uint32_t bits = __builtin_bit_cast(uint32_t, r.vm), power = bits & 0x7F800000u;
                    r.ve = max(power, 0x00800000u);       // (0 and subnormal numbers: 2^-126)
                    r.vm = power ? __builtin_bit_cast(float, (bits & 0x807FFFFFu) | 0x3F800000u) : r.vm * 0x1p126f;
                }
            }
            return r;
        };
        // Whether the pages of a piece are read by nontemporal loads (kv_stream.h): every wave looks at a quarter of the up to 64 requests around its own.  A request with more
        // than kQuantTiles row tiles takes its keys again: ordinary loads but for the last time (256 mixed requests 133 -> 120 us).
        struct Look { float keys; bool shared; };
        auto look = [&](const QuantPiece& x) {
            if (lane >= kKvScanRequests / 4) return Look{0.0f, false};
            const KvScan s = kv_scan_lane(p.seq_lens, p.page_table, p.max_pages, p.B, p.max_kv_len, x.i, x.kbeg / kP, 4 * lane);
            return Look{s.keys, s.shared};
        };
        auto streams = [&](const QuantPiece& x, int grp, Look l) {
            const int large = __builtin_amdgcn_readfirstlane(row16_sum(l.keys) > p.stream_keys);           // (lanes 0 .. 15)
            return (grp + 1) * kQuantTiles * 16 >= p.G * x.n && large && !__any(l.shared);
        };
        // Q: one row tile stays in registers, of more tiles wave w takes fragment w of each to LDS
        constexpr int kQ = NR == 1 ? 4 : NR;
        struct Query { u32x4 x[kQ]; };
        auto load_q = [&](const QuantPiece& x, int grp) {
            Query r;
#pragma unroll
            for (int k = 0; k < kQ; ++k) {
                const int row = grp * kQuantTiles * 16 + (NR == 1 ? 0 : k) * 16 + l16, s = NR == 1 ? k : wave, j = (int)((uint32_t)row * p.g_magic >> 16);
                r.x[k] = u32x4{0, 0, 0, 0};
                if (row < p.G * x.n) r.x[k] = *reinterpret_cast<const u32x4*>(p.q + ((size_t)(x.r0 + j) * p.Hq + kvh * p.G + row - j * p.G) * kD + g * 32 + s * 8);
                r.x[k] ^= p.q_sign;
            }
            return r;
        };

        // ---- a step's two pages, HBM -> LDS: 2 direct loads of 1 KB per page.  16-byte chunk ch of K's row (key) r is stored at position ch ^ (r & 7), so that
        // 8 lanes that read the same chunk of 8 rows meet no bank twice; V stays as it is ----
        const uint32_t koff = (uint32_t)((lane >> 3) * kD + (((lane & 7) ^ (lane >> 3)) << 4)), voff = (uint32_t)lane * 16;
        auto issue_as = [&](auto nontemporal, int ids, int step) {
            constexpr bool STREAM = decltype(nontemporal)::value;
            const int a = __builtin_amdgcn_readlane(ids, 2 * (step & 31)), b = __builtin_amdgcn_readlane(ids, 2 * (step & 31) + 1);
            unsigned char* to = ring + (step & 1) * kQuantStageBytes;
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
                const size_t at = ((size_t)(pg ? b : a) * p.Hkv + kvh) * kQuantPageBytes;
                const uint8_t *from_k = scalar_address(p.k + at), *from_v = scalar_address(p.v + at);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    lds_dma16_off<STREAM>(koff, from_k + h * 1024, to + pg * kQuantPageBytes + h * 1024);
                    lds_dma16_off<STREAM>(voff, from_v + h * 1024, to + (2 + pg) * kQuantPageBytes + h * 1024);
                }
            }
        };
        auto issue = [&](bool stream, int ids, int step) {
            if (stream) issue_as(std::true_type{}, ids, step);
            else issue_as(std::false_type{}, ids, step);
        };
        constexpr int kLoads = 8;                         // of a step
        auto steps_of = [&](const QuantPiece& x) {
            const int keys = x.kend - x.kbeg - wave * 32;
            return keys <= 0 ? 0 : (keys + kQuantStep - 1) / kQuantStep;
        };
        // scales of one step: of both its pages
        struct Scales { float ks[2], vm[2], ve[2]; };
        auto scales_of = [&](const Pages& x, int step) {
            Scales r;
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
                const int l = 2 * (step & 31) + pg;
                r.ks[pg] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x.ks), l));
                r.vm[pg] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x.vm), l));
                r.ve[pg] = TYPE == SPEC_KV_E4M3 ? __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)x.ve, l)) : 1.0f;
            }
            return r;
        };

        Pages pages;
        pages.id = load_ids(u, 0);
        bool stream = streams(u, group, look(u));
        if (steps_of(u) > 0) issue(stream, pages.id, 0);
        pages = load_scales(u, 0, pages.id);
        Query query = load_q(u, group);
        if (steps_of(u) > 1) issue(stream, pages.id, 1);
        bool first = true;

        while (true) {
            const int first_row = group * kQuantTiles * 16, R = min(p.G * u.n - first_row, NR * 16), c = u.c, kend = u.kend, steps = steps_of(u);
            if constexpr (NR > 1) {
#pragma unroll
                for (int rt = 0; rt < NR; ++rt) sQ[(rt * 4 + wave) * 64 + lane] = query.x[rt];
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // the first step's pages, with the scales and queries that were requested beside them
            Scales now = scales_of(pages, 0), nxt = scales_of(pages, 1);
            if (steps > 1 && !first) issue(stream, pages.id, 1);           // (the first piece's is on its way, since nothing is merged in its place: 8 x 32-64k 43.9 -> 42.5 us)
            first = false;
            if constexpr (NR > 1) __syncthreads();
            // what comes next, and its page ids
            QuantPiece v = u;
            int v_group = group;
            const bool more = next(v, v_group);
            int v_ids = 0;
            Look v_look{0.0f, false};
            if (more) {
                v_ids = load_ids(v, 0);
                v_look = look(v);
            }

            int limit[NR];                // row sees key positions t < limit
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
                const int r = rt * 16 + l16;
                limit[rt] = r < R ? min(c + (int)((uint32_t)(first_row + r) * p.g_magic >> 16) + 1, kend) : 0;
            }
            f32x4 o[NR][8];
            float m_run[NR], l_run[NR];
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
                m_run[rt] = kNegBig;
                l_run[rt] = 0.0f;
#pragma unroll
                for (int t = 0; t < 8; ++t) o[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            }

            auto keys = [&](auto active) {
                constexpr int A = decltype(active)::value;
                for (int step = 0; step < steps; ++step) {
                    const int wbase = u.kbeg + step * kQuantStep + wave * 32;
                    // this step's pages have landed (the first one's before the loop), the next one's may fly on; once they are in registers, their place is for the
                    // step behind that
                    if (step == 0) asm volatile("" ::: "memory");
                    else if (step + 1 < steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
                    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    u32x4 kraw[2][2];
                    u32x2 vraw[2][4];
                    const unsigned char* sK = ring + (step & 1) * kQuantStageBytes;
#pragma unroll
                    for (int pg = 0; pg < 2; ++pg) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) kraw[pg][h] = *reinterpret_cast<const u32x4*>(sK + pg * kQuantPageBytes + l16 * kD + (((2 * g + h) ^ (l16 & 7)) << 4));
#pragma unroll
                        for (int r = 0; r < 4; ++r) vraw[pg][r] = *reinterpret_cast<const u32x2*>(sK + (2 + pg) * kQuantPageBytes + (4 * g + r) * kD + l16 * 8);
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    const float ks[2] = {now.ks[0], now.ks[1]}, vm[2] = {now.vm[0], now.vm[1]}, ve[2] = {now.ve[0], now.ve[1]};
                    now = nxt;
                    if (step + 2 < steps) {
                        if (((step + 2) & 31) == 0) pages = load_scales(u, step + 2, load_ids(u, step + 2));     // the next 32 steps
                        issue(stream, pages.id, step + 2);
                        nxt = scales_of(pages, step + 2);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    // (two row tiles and more: Q is read again in every step; the compiler would rather keep all of it in registers)
                    int q_lane = lane;
                    if constexpr (NR > 1) asm volatile("" : "+v"(q_lane));
                    // ---- S^T = K Q^T; scores in the log2 domain ----
                    float sc[A][8];
                    {
                        // (a score is rounded before the maximum is taken and before it is subtracted: a product fused with the subtraction would exceed its own maximum by what the
                        // rounding lost, 2^8 where scores are 2^32)
#pragma clang fp contract(off)
                        // (a fragment of Q serves both pages, and the next one is read under its products: with a read in front of every product 32 x 2048 x 8 heads took 3 us more)
                        auto q_part = [&](int rt, int s) { return __builtin_bit_cast(bf16x8, NR == 1 ? query.x[NR == 1 ? s : 0] : sQ[(rt * 4 + s) * 64 + q_lane]); };
                        f32x4 acc[2][A];
                        bf16x8 qx[A];
#pragma unroll
                        for (int rt = 0; rt < A; ++rt) {
                            acc[0][rt] = acc[1][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
                            qx[rt] = q_part(rt, 0);
                        }
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            bf16x8 qn[A];
#pragma unroll
                            for (int rt = 0; rt < A; ++rt) qn[rt] = s < 3 ? q_part(rt, s + 1) : qx[rt];
#pragma unroll
                            for (int pg = 0; pg < 2; ++pg) {
                                const u32x4 raw = kraw[pg][s >> 1];
                                const bf16x8 kf = (s & 1) ? bf16_oct<TYPE>(raw.z, raw.w) : bf16_oct<TYPE>(raw.x, raw.y);
#pragma unroll
                                for (int rt = 0; rt < A; ++rt) acc[pg][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qx[rt], acc[pg][rt], 0, 0, 0);
                            }
#pragma unroll
                            for (int rt = 0; rt < A; ++rt) qx[rt] = qn[rt];
                        }
#pragma unroll
                        for (int rt = 0; rt < A; ++rt)
#pragma unroll
                            for (int e = 0; e < 8; ++e) sc[rt][e] = acc[e >> 2][rt][e & 3] * ks[e >> 2];
                    }
                    if (wbase + 32 > min(c + 1, kend)) {
#pragma unroll
                        for (int rt = 0; rt < A; ++rt)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                sc[rt][e] = wbase + (e >> 2) * 16 + g * 4 + (e & 3) < limit[rt] ? sc[rt][e] : kMasked;
                    }
                    // The reference maximum moves only when a score exceeds it by more than kMaxSlack, so exp2(s - m_run) <= 2^kMaxSlack stays well inside fp32 and bf16 and O
                    // is rescaled a handful of times (the result is the same softmax: O and l carry the same factor).  A lane looks at its own 8 scores, and the four
                    // lanes of a query row agree on a new maximum where one of them asks for it.
                    float tmax[A];
                    bool grow = false;
#pragma unroll
                    for (int rt = 0; rt < A; ++rt) {
                        tmax[rt] = fmaxf(fmaxf(fmaxf(sc[rt][0], sc[rt][1]), fmaxf(sc[rt][2], sc[rt][3])), fmaxf(fmaxf(sc[rt][4], sc[rt][5]), fmaxf(sc[rt][6], sc[rt][7])));
                        grow |= tmax[rt] > m_run[rt] + kMaxSlack;
                    }
                    if (__any(grow)) {
#pragma unroll
                        for (int rt = 0; rt < A; ++rt)
                            if (__any(tmax[rt] > m_run[rt] + kMaxSlack)) {
                                const float m_new = fmaxf(m_run[rt], four_rows_max(tmax[rt]));
                                const float alpha = __builtin_amdgcn_exp2f(m_run[rt] - m_new);
                                m_run[rt] = m_new;
                                l_run[rt] *= alpha;
#pragma unroll
                                for (int t = 0; t < 8; ++t) o[rt][t] *= alpha;
                            }
                    }
                    const bool factors = TYPE != SPEC_KV_E4M3 || vm[0] != 1.0f || vm[1] != 1.0f;
                    bf16x8 pf[A], rest[A];
#pragma unroll
                    for (int rt = 0; rt < A; ++rt) {
                        float pr[8], psum = 0.0f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            // (masked: 0, also in a row that has seen nothing, whose m_run is kNegBig)
                            pr[e] = __builtin_amdgcn_exp2f(sc[rt][e] - m_run[rt]);
                            psum += pr[e];
                        }
                        l_run[rt] += psum;
                        if (factors) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) pr[e] *= vm[e >> 2];
                        }
                        const u32x4 pw = {pack_bf16x2(pr[0], pr[1]), pack_bf16x2(pr[2], pr[3]), pack_bf16x2(pr[4], pr[5]), pack_bf16x2(pr[6], pr[7])};
                        pf[rt] = __builtin_bit_cast(bf16x8, pw);
                        // What the rounding left is rounded in turn and has products of its own: 2^-16 of a probability is lost.
                        u32x4 left;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            left[k] = pack_bf16x2(pr[2 * k] - __builtin_bit_cast(float, pw[k] << 16), pr[2 * k + 1] - __builtin_bit_cast(float, pw[k] & 0xFFFF0000u));
                        rest[rt] = __builtin_bit_cast(bf16x8, left);
                    }
                    // ---- O^T += V^T P^T ----
                    if (wbase + 32 > kend) {
                        // slots past the range may hold anything (even NaN patterns): P is 0 there, so V must be too
#pragma unroll
                        for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (wbase + pg * 16 + g * 4 + r >= kend) vraw[pg][r] = u32x2{0, 0};
                    }
                    uint32_t pair[2][2][4];               // [page][keys 4g, 4g+1 | 4g+2, 4g+3][t / 2]: bytes {key a, key b} of t, then of t + 1
#pragma unroll
                    for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                        for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
                            for (int w = 0; w < 2; ++w) {
                                uint32_t a = w ? vraw[pg][2 * k2].y : vraw[pg][2 * k2].x, b = w ? vraw[pg][2 * k2 + 1].y : vraw[pg][2 * k2 + 1].x;
                                asm("" : "+v"(a), "+v"(b));
                                pair[pg][k2][2 * w] = __builtin_amdgcn_perm(b, a, 0x05010400u);
                                pair[pg][k2][2 * w + 1] = __builtin_amdgcn_perm(b, a, 0x07030602u);
                            }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        u32x4 w;
                        if (t & 1) w = u32x4{bf16_pair<TYPE, true>(pair[0][0][t >> 1], ve[0]), bf16_pair<TYPE, true>(pair[0][1][t >> 1], ve[0]),
                                             bf16_pair<TYPE, true>(pair[1][0][t >> 1], ve[1]), bf16_pair<TYPE, true>(pair[1][1][t >> 1], ve[1])};
                        else w = u32x4{bf16_pair<TYPE, false>(pair[0][0][t >> 1], ve[0]), bf16_pair<TYPE, false>(pair[0][1][t >> 1], ve[0]),
                                       bf16_pair<TYPE, false>(pair[1][0][t >> 1], ve[1]), bf16_pair<TYPE, false>(pair[1][1][t >> 1], ve[1])};
                        const bf16x8 vf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                        for (int rt = 0; rt < A; ++rt) o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt], o[rt][t], 0, 0, 0);
#pragma unroll
                        for (int rt = 0; rt < A; ++rt) o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, rest[rt], o[rt][t], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            if (NR >= 3 && R > 32) keys(std::integral_constant<int, NR >= 3 ? 3 : 1>{});
            else if (NR >= 2 && R > 16) keys(std::integral_constant<int, NR >= 2 ? 2 : 1>{});
            else keys(std::integral_constant<int, 1>{});

            // ---- the next piece's scales, queries and first step ----
            if (more) {
                pages = load_scales(v, 0, v_ids);
                query = load_q(v, v_group);
                stream = streams(v, v_group, v_look);
                if (steps_of(v) > 0) issue(stream, v_ids, 0);
            }
            // ---- merge the waves, a row tile at a time: each leaves its O where the pages of its second step were (16-byte chunk c of a row at position
            // c ^ (row & 7)), maxima and sums beside; a thread then takes 4 consecutive d of a row from all waves ----
            float* own = reinterpret_cast<float*>(ring + kQuantStageBytes);
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
                const float l = four_rows_sum(l_run[rt]);
                if (g == 0) {
                    s_m[wave * NR * 16 + rt * 16 + l16] = m_run[rt];
                    s_l[wave * NR * 16 + rt * 16 + l16] = l;
                }
            }
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
                if (rt * 16 >= R) break;
                if (rt > 0) __syncthreads();              // everybody has read the previous tile
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        // d = 32 g + 8 e + 4 w .. + 3
                        const int ch = 8 * g + 2 * e + w;
                        *reinterpret_cast<f32x4*>(own + l16 * kD + ((ch ^ (l16 & 7)) << 2)) =
                            f32x4{o[rt][4 * w][e], o[rt][4 * w + 1][e], o[rt][4 * w + 2][e], o[rt][4 * w + 3][e]};
                    }
                __syncthreads();
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int at = half * 8 + (tid >> 5), r = rt * 16 + at, ch = tid & 31;
                    if (r < R) {
                        float m[NW], mx = kNegBig;
#pragma unroll
                        for (int w = 0; w < NW; ++w) {
                            m[w] = s_m[w * NR * 16 + r];
                            mx = fmaxf(mx, m[w]);
                        }
                        f32x4 num = f32x4{0.f, 0.f, 0.f, 0.f};
                        float l = 0.0f;
#pragma unroll
                        for (int w = 0; w < NW; ++w) {
                            const float f = __builtin_amdgcn_exp2f(m[w] - mx);
                            num += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem + w * kQuantWaveBytes + kQuantStageBytes) + at * kD + ((ch ^ (at & 7)) << 2));
                            l += f * s_l[w * NR * 16 + r];
                        }
                        const int j = (int)((uint32_t)(first_row + r) * p.g_magic >> 16), hq = kvh * p.G + first_row + r - j * p.G;
                        if (u.whole) {
                            const size_t rowhead = (size_t)(u.r0 + j) * p.Hq + hq;
                            const float inv = 1.0f / l;
                            u32x2_any packed;
                            packed.x = pack_bf16x2(num.x * inv, num.y * inv);
                            packed.y = pack_bf16x2(num.z * inv, num.w * inv);
                            *reinterpret_cast<u32x2_any*>(p.out + rowhead * kD + ch * 4) = packed;
                            if (p.lse && ch == 0) p.lse[rowhead] = (mx + log2f(l)) * 0.6931471805599453f;
                        } else {
                            const size_t slot = (u.slot * p.max_q_len + j) * p.Hq + hq;
                            *reinterpret_cast<f32x4*>(p.part_o + slot * kD + ch * 4) = num;
                            if (ch == 0) { p.part_m[slot] = mx; p.part_l[slot] = l; }
                        }
                    }
                }
            }
            if (!more) break;
            u = v;
            group = v_group;
            pages.id = v_ids;
            __syncthreads();                              // Q and the place of the second step are free again
        }
        if (bad_page && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_PAGE);
    }
};

// RANGES: workgroup (kv head, range); else (kv head and row group, request)
template <int NR, int TYPE, bool RANGES>
__global__ __launch_bounds__(kQuantThreads, kQuantWgsPerCu) void verify_attn_quant_kernel(QuantAttnParams p)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    typedef QuantKernel<NR, TYPE> Kernel;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if constexpr (!RANGES) {
        const int group = blockIdx.x / p.Hkv, kvh = blockIdx.x - group * p.Hkv;
        int i = blockIdx.y;
        if (p.by_length) {
            // workgroups start in grid order: the longest requests first (ties: request order), so that short ones fill the end
            uint32_t* s_key = reinterpret_cast<uint32_t*>(smem);      // [kQuantOrdered], then the request
            const uint32_t key = tid < p.B ? (uint32_t)min(max(p.seq_lens[tid], 0), (1 << 23) - 1) << 8 | (uint32_t)(kQuantOrdered - 1 - tid) : 0;
            s_key[tid] = key;
            __syncthreads();
            int above = 0;
#pragma unroll 4
            for (int k = 0; k < kQuantOrdered; k += 4) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(s_key + k);
                above += (x.x > key) + (x.y > key) + (x.z > key) + (x.w > key);
            }
            if (tid < p.B && above == i) s_key[kQuantOrdered] = (uint32_t)tid;
            __syncthreads();
            i = __builtin_amdgcn_readfirstlane((int)s_key[kQuantOrdered]);
            __syncthreads();                              // (pages land there next)
        }
        const auto [r0, n, c] = quant_request(p, i);
        if (!quant_request_ok(r0, n, c, p)) {
            if (blockIdx.x == 0 && tid == 0 && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_LENGTH);
            return;
        }
        if (group * kQuantTiles * 16 >= p.G * n) return;
        Kernel::run(p, smem, kvh, QuantPiece{i, r0, n, c, 0, c + n, true, 0}, group, [&](QuantPiece& u, int& at) {
            at += p.groups;
            return at * kQuantTiles * 16 < p.G * u.n;
        });
    } else {
        const int kvh = blockIdx.x, range = blockIdx.y;
        // Every request's work and what comes before it, four requests per thread; the total gives the size of a range, and the request in which this one starts leaves its
        // number and place in LDS.
        constexpr int kPer = kQuantListed / kQuantThreads;
        int* s_scan = reinterpret_cast<int*>(smem);       // [4], then {request, work before it, its first row, rows, committed tokens}
        int work[kPer], mine = 0;
        QuantRequest request[kPer];
        bool bad = false;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = tid * kPer + k;
            work[k] = 0;
            if (i < p.B) {
                const int r0 = p.qo_indptr[i], n = attn_request_rows(r0, p.qo_indptr[i + 1]), c = p.seq_lens[i];
                request[k] = QuantRequest{r0, n, c};
                if (quant_request_ok(r0, n, c, p)) work[k] = quant_piece_work(p.G * n) + (c + n + kQuantStep - 1) / kQuantStep * quant_step_work(p.G * n);
                else bad = true;
            }
            mine += work[k];
        }
        if (bad && kvh == 0 && range == 0 && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_LENGTH);
        int incl = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(incl, d, 64);
            if (lane >= d) incl += up;
        }
        if (lane == 63) s_scan[wave] = incl;
        __syncthreads();
        int before = incl - mine, total = 0;
#pragma unroll
        for (int w = 0; w < kQuantWaves; ++w) {
            const int t = s_scan[w];
            if (w < wave) before += t;
            total += t;
        }
        total = __builtin_amdgcn_readfirstlane(total);
        const int quantum = max(p.min_work, (total + p.ranges - 1) / p.ranges);
        const int first = range * quantum, last = min(total, first + quantum);        // (32 bits hold them: see quant_plan)
        if (first >= total) return;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if (first >= before && first < before + work[k]) {
                s_scan[4] = tid * kPer + k;
                s_scan[5] = before;
                s_scan[6] = request[k].r0;
                s_scan[7] = request[k].n;
                s_scan[8] = request[k].c;
            }
            before += work[k];
        }
        __syncthreads();
        int i = __builtin_amdgcn_readfirstlane(s_scan[4]), at = __builtin_amdgcn_readfirstlane(s_scan[5]);      // request, and the work before it
        QuantRequest known{__builtin_amdgcn_readfirstlane(s_scan[6]), __builtin_amdgcn_readfirstlane(s_scan[7]), __builtin_amdgcn_readfirstlane(s_scan[8])};
        bool start = true;                                // (the first request's fields are here: a round trip less, 256 mixed requests 117.4 -> 114.8 us)
        __syncthreads();                                  // (pages land there next)
        // the next request with steps in this range, whole or in part
        auto piece_from = [&](QuantPiece& u) {
            while (at < last) {
                if (!start) known = quant_request(p, i);
                start = false;
                const auto [r0, n, c] = known;
                if (quant_request_ok(r0, n, c, p)) {
                    const int len = c + n, steps = (len + kQuantStep - 1) / kQuantStep, w = quant_step_work(p.G * n);
                    // the steps whose place lies in this range
                    const int begin = at + quant_piece_work(p.G * n);        // the place of its first step
                    const int from = begin >= first ? 0 : (first - begin + w - 1) / w, to = min(steps, max(0, first + quantum - begin + w - 1) / w);
                    const int head = begin / quantum, pieces = (begin + (steps - 1) * w) / quantum - head + 1;
                    if (from == 0 && kvh == 0 && tid == 0) p.req[i] = u32x2{(uint32_t)head, (uint32_t)pieces};
                    at = begin + steps * w;
                    if (from < to) {
                        u = QuantPiece{i++, r0, n, c, from * kQuantStep, min(len, to * kQuantStep), pieces == 1, 2 * (size_t)range + (from == 0)};
                        return true;
                    }
                }
                ++i;
            }
            return false;
        };
        QuantPiece u;
        if (!piece_from(u)) return;
        Kernel::run(p, smem, kvh, u, 0, [&](QuantPiece& v, int& group) {
            if (++group * kQuantTiles * 16 < p.G * v.n) return true;
            group = 0;
            return piece_from(v);
        });
    }
}

// Merges the pieces of requests that lie in several ranges, and writes bf16 (and lse).  A workgroup per candidate row and HEADS query heads (8, or 1 where requests have many
// pieces): a group of 32 threads, 4 consecutive d each, walks the pieces of a head, or every eighth of them; the groups are then summed in order, so that nothing depends on
// timing.
template <int HEADS>
__global__ __launch_bounds__(256) void verify_attn_quant_merge_kernel(QuantAttnParams p)
{
    constexpr int kGroups = 8 / HEADS;
    __shared__ f32x4 s_num[kGroups][32];
    __shared__ float s_den[kGroups], s_max[kGroups];
    const int row = blockIdx.x, tid = threadIdx.x, grp = tid >> 5, d4 = (tid & 31) * 4;
    const int hq = HEADS == 1 ? blockIdx.y : blockIdx.y * 8 + grp;
    // The row's request: every request's fields are read at once, with where its pieces are (not written for one that is skipped), so that the partials are one more round trip
    // away and not two (13 ragged requests 20.7 -> 20.3 us, 8 x 32-64k 42.7 -> 42.2).
    __shared__ int s_last, s_req[3];
    if (tid == 0) s_last = -1;
    __syncthreads();
    int mine = -1, r0 = 0;
    u32x2 where = {0, 0};
    for (int i = tid; i < p.B; i += 256) {
        const int at = p.qo_indptr[i], n = attn_request_rows(at, p.qo_indptr[i + 1]), c = p.seq_lens[i];
        const u32x2 q = p.req[i];
        if (quant_request_ok(at, n, c, p) && row >= at && row < at + n) { mine = i; r0 = at; where = q; }
    }
    if (mine >= 0) atomicMax(&s_last, mine);              // (one thread, unless the row ranges overlap)
    __syncthreads();
    if (mine >= 0 && mine == s_last) { s_req[0] = r0; s_req[1] = (int)where.x; s_req[2] = (int)where.y; }
    __syncthreads();
    if (s_last < 0) return;
    const int head = __builtin_amdgcn_readfirstlane(s_req[1]), pieces = __builtin_amdgcn_readfirstlane(s_req[2]);
    r0 = __builtin_amdgcn_readfirstlane(s_req[0]);
    if (pieces == 1 || hq >= p.Hq) return;                // (all of a workgroup, or it has no barrier ahead)
    const auto slot = [&](int k) { return ((2 * (size_t)(head + k) + (k == 0)) * p.max_q_len + (row - r0)) * p.Hq + hq; };
    float mx = kNegBig, den = 0.0f;
    f32x4 num = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = HEADS == 1 ? grp : 0; k0 < pieces; k0 += 4 * kGroups) {
        float m[4], l[4], mx2 = mx;
        f32x4 o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const size_t s = slot(min(k0 + k * kGroups, pieces - 1));
            m[k] = p.part_m[s];
            l[k] = p.part_l[s];
            o[k] = *reinterpret_cast<const f32x4*>(p.part_o + s * kD + d4);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) mx2 = fmaxf(mx2, m[k]);
        const float f = __builtin_amdgcn_exp2f(mx - mx2);
        num *= f;
        den *= f;
        mx = mx2;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k0 + k * kGroups < pieces) {
                const float w = __builtin_amdgcn_exp2f(m[k] - mx);
                num += w * o[k];
                den += w * l[k];
            }
    }
    if constexpr (kGroups > 1) {
        s_num[grp][tid & 31] = num;
        if ((tid & 31) == 0) { s_den[grp] = den; s_max[grp] = mx; }
        __syncthreads();
        if (tid >= 32) return;
#pragma unroll
        for (int k = 0; k < kGroups; ++k) mx = fmaxf(mx, s_max[k]);
        num = f32x4{0.f, 0.f, 0.f, 0.f};
        den = 0.0f;
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            const float w = __builtin_amdgcn_exp2f(s_max[k] - mx);
            num += w * s_num[k][tid];
            den += w * s_den[k];
        }
    }
    const float inv = 1.0f / den;
    u32x2_any packed;
    packed.x = pack_bf16x2(num.x * inv, num.y * inv);
    packed.y = pack_bf16x2(num.z * inv, num.w * inv);
    *reinterpret_cast<u32x2_any*>(p.out + ((size_t)row * p.Hq + hq) * kD + d4) = packed;
    if (p.lse && (tid & 31) == 0) p.lse[(size_t)row * p.Hq + hq] = (mx + log2f(den)) * 0.6931471805599453f;
}

// How a call is cut up.
struct QuantPlan {
    int tiles, groups;                       // row tiles at once, workgroups per request and kv head (whole requests)
    int ranges, min_work;                    // 0 ranges: whole requests
    bool by_length;                          // whole requests: the longest first
    bool many;                               // pieces per request: a workgroup per head merges them
    size_t slots, req_bytes;
};

constexpr int kQuantMinSteps = 2;            // of a range

// Ranges of a call at most, whatever its lengths: by the compute units (or the keys per range that are asked for), and by the work at its bounds, for which a request's piece
// work counts as four steps (it is 20 / 5 of one with one row tile, less with more).  Grows with B and max_kv_len alone.
static long quant_most_ranges(int B, int Hkv, int max_kv_len)
{
    const int chunk = g_attn_chunk_override, waves = g_attn_plan_waves;
    const long steps = ((long)max_kv_len + kQuantStep - 1) / kQuantStep, least = chunk > 0 ? 1 : kQuantMinSteps;
    const long ranges = chunk > 0 ? (long)B * max_kv_len / chunk + 1 : std::max<long>(1, (long)device_cu_count() * (waves > 0 ? waves : kQuantWgsPerCu) / Hkv);
    return std::min(std::min(ranges, (B * (steps + 4) + least - 1) / least), 8192L);
}

static QuantPlan quant_plan(int B, int Hq, int Hkv, int max_kv_len, int max_q_len)
{
    QuantPlan c{};
    const int G = Hq / Hkv, NR = (G * max_q_len + 15) / 16;
    c.tiles = std::min(NR, kQuantTiles);
    const int row_groups = (NR + kQuantTiles - 1) / kQuantTiles;
    const long cus = device_cu_count(), units = (long)B * Hkv;
    c.groups = units >= cus ? 1 : row_groups;
    c.by_length = B > 1 && B <= kQuantOrdered && units > cus;
    const int mode = g_attn_plan, chunk = g_attn_chunk_override;
    const long steps = ((long)max_kv_len + kQuantStep - 1) / kQuantStep, work = quant_step_work(G * max_q_len);
    const long most = B * (steps * work + quant_piece_work(G * max_q_len));            // work of the batch at its bounds
    if (mode == 2 || B > kQuantListed || most > (1L << 30)) return c;
    // Whole requests need no merge and leave no bubbles between pieces, but the longest one is as long as the call.  In us: what it takes (0.8, 1.3, 1.6 a step with 1, 2, 3 row
    // tiles) against what the ranges' second launch and partials cost (8, with more than one row tile 18 once the chip is busy) and half of what the batch takes at its bounds and
    // 6.5 TB/s (lengths are usually below them).  Ranges / whole, us, all requests at the bound | lengths from an eighth of it on, 1 row tile: 1 x 1024 keys 11.3 / 11.3, 2048 12.3 / 18.5;
    // 128 requests x heads of 2048 21.6 / 20.5 | 19.0 / 20.2, 4096 31.9 / 35.4 | 23.9 / 34.7; 256 of 4096 55.6 / 46.5 | 36.8 / 36.8, 8192 98.5 / 87.1 | 62.2 / 68.8; 3 row tiles: 1 x 512
    // 15.1 / 13.4, 1024 15.4 / 19.9; 128 of 2048 37.7 / 36.0 | 30.9 / 35.7; 256 of 2048 51.7 / 38.5 | 43.5 / 37.6, 4096 77 / 66 | 58 / 63.
    // The bounds are all that the host knows.  Where they say little the rule is off: 32 requests of 2048 keys x 8 heads, 5 rows take 32 us whole under a bound of 2053 and 40 as
    // ranges under one of 4096 or more; one request of 65000 keys among 127 of 1024, 1 row x 8 heads, bound 65536, takes 496 whole, which the rule chooses, and 84 as ranges.
    const double all_us = (double)units * max_kv_len * (2 * kD) / 6.5e6;
    const double one_us = steps * (NR == 1 ? 0.8 : NR == 2 ? 1.3 : 1.6 * row_groups);
    const double saved_us = 8.0 + (NR == 1 ? 0.0 : 10.0 * std::min(1.0, all_us / 15.0));
    if (mode != 1 && chunk <= 0 && one_us <= saved_us + 0.5 * all_us) return c;
    c.min_work = (int)((chunk > 0 ? 1 : kQuantMinSteps) * work);
    const long ranges = std::min(quant_most_ranges(B, Hkv, max_kv_len), (most + c.min_work - 1) / c.min_work);
    c.ranges = (int)ranges;
    c.many = ranges > 16L * B;
    c.slots = 2 * (size_t)ranges * max_q_len * Hq;
    c.req_bytes = round_up((size_t)B * 8, 256);
    return c;
}

static size_t quant_workspace(const QuantPlan& c)
{
    return c.ranges == 0 ? 0 : c.req_bytes + round_up(c.slots * kD * 4, 256) + 2 * round_up(c.slots * 4, 256);
}

template <int NR, int TYPE, bool RANGES>
static int launch_quant_one(const QuantAttnParams& p, dim3 grid, hipStream_t s)
{
    constexpr size_t smem = QuantKernel<NR, TYPE>::kBytes;
    static LdsGrantTable granted = {};
    if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(&verify_attn_quant_kernel<NR, TYPE, RANGES>), smem, granted, "spec_verify_attn_quantized")) return rc;
    hipLaunchKernelGGL((verify_attn_quant_kernel<NR, TYPE, RANGES>), grid, dim3(kQuantThreads), smem, s, p);
    return SPEC_OK;
}

template <int NR, int TYPE>
static int launch_quant_as(const QuantAttnParams& p, dim3 grid, hipStream_t s)
{
    return p.ranges > 0 ? launch_quant_one<NR, TYPE, true>(p, grid, s) : launch_quant_one<NR, TYPE, false>(p, grid, s);
}

template <int NR>
static int launch_quant(const QuantAttnParams& p, int kv_type, dim3 grid, hipStream_t s)
{
    return kv_type == SPEC_KV_E4M3 ? launch_quant_as<NR, SPEC_KV_E4M3>(p, grid, s) : launch_quant_as<NR, SPEC_KV_INT8>(p, grid, s);
}

}  // namespace specv

extern "C" size_t spec_verify_attn_quantized_workspace_bytes(int B, int M, int Hq, int Hkv, int D, int max_kv_len, int max_q_len)
{
    using namespace specv;
    (void)D;
    if (B <= 0 || M <= 0 || Hq <= 0 || Hkv <= 0 || max_kv_len <= 0 || Hq % Hkv != 0 || g_attn_plan == 2) return 0;
    // Also where this batch is taken as whole requests: a smaller one may be cut.
    QuantPlan c{};
    B = std::min(B, kQuantListed);
    c.ranges = (int)quant_most_ranges(B, Hkv, max_kv_len);
    c.slots = 2 * (size_t)c.ranges * (max_q_len > 0 ? max_q_len : 1) * Hq;
    c.req_bytes = round_up((size_t)B * 8, 256);
    return quant_workspace(c);
}

extern "C" int spec_verify_attn_quantized(const void* q, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                                          const int32_t* page_table, int max_pages_per_seq, int num_pages,
                                          const int32_t* seq_lens, const int32_t* qo_indptr, void* out, float* lse,
                                          int B, int M, int Hq, int Hkv, int D, int page_size, int kv_type,
                                          int max_kv_len, int max_q_len, float scale, int32_t* status_flags,
                                          void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace specv;
    if (B == 0 || M == 0) return SPEC_OK;
    if (!q || !k_cache || !v_cache || !k_scale || !v_scale || !page_table || !seq_lens || !qo_indptr || !out)
        return fail(SPEC_EINVAL, "spec_verify_attn_quantized: NULL pointer argument");
    if (B < 0 || M < 0 || Hq <= 0 || Hkv <= 0 || max_pages_per_seq <= 0 || num_pages <= 0 || max_kv_len <= 0 || max_q_len <= 0)
        return fail(SPEC_EINVAL, "spec_verify_attn_quantized: non-positive size");
    if (kv_type != SPEC_KV_E4M3 && kv_type != SPEC_KV_INT8) return fail(SPEC_EINVAL, "spec_verify_attn_quantized: unknown cache type %d", kv_type);
    if (D != kD || page_size != kP)
        return fail(SPEC_ESHAPE, "spec_verify_attn_quantized: built for D=128, page_size=16 (got D=%d page_size=%d)", D, page_size);
    if (Hq % Hkv != 0) return fail(SPEC_ESHAPE, "spec_verify_attn_quantized: Hq=%d is not a multiple of Hkv=%d", Hq, Hkv);
    const int G = Hq / Hkv;
    if ((long)G * max_q_len > 128)
        return fail(SPEC_ESHAPE, "spec_verify_attn_quantized: (Hq/Hkv)*max_q_len = %ld rows per kv head, at most 128", (long)G * max_q_len);
    if ((long)max_pages_per_seq * kP < max_kv_len)
        return fail(SPEC_EINVAL, "spec_verify_attn_quantized: page table of %d pages cannot hold max_kv_len=%d", max_pages_per_seq, max_kv_len);
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16))
        return fail(SPEC_EINVAL, "spec_verify_attn_quantized: q and the caches must be 16-byte aligned");
    if (B > 65535 || Hkv > 65535 || M > 2147483647 / Hq) return fail(SPEC_ESHAPE, "spec_verify_attn_quantized: B, Hkv or M beyond the launch grid");
    const QuantPlan c = quant_plan(B, Hq, Hkv, max_kv_len, max_q_len);
    const size_t need = quant_workspace(c);
    if (!workspace || !aligned(workspace, 256))
        return fail(SPEC_EINVAL, "spec_verify_attn_quantized: workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need)
        return fail(SPEC_EWORKSPACE, "spec_verify_attn_quantized: workspace %zu bytes, need %zu", workspace_bytes, need);

    QuantAttnParams p{};
    p.q = (const uint16_t*)q; p.k = (const uint8_t*)k_cache; p.v = (const uint8_t*)v_cache; p.k_scale = k_scale; p.v_scale = v_scale;
    p.page_table = page_table; p.seq_lens = seq_lens; p.qo_indptr = qo_indptr;
    p.out = (uint16_t*)out; p.lse = lse; p.status_flags = status_flags;
    p.max_pages = max_pages_per_seq; p.num_pages = num_pages; p.Hq = Hq; p.Hkv = Hkv; p.G = G;
    p.M = M; p.B = B; p.max_kv_len = max_kv_len; p.max_q_len = max_q_len;
    p.ranges = c.ranges; p.min_work = c.min_work; p.groups = c.groups; p.by_length = c.by_length;
    // 3/8 of the cache.  Calls on three batches in turn, ordinary -> nontemporal: 21 MB 43.7 -> 47 us, 101 MB 50 -> 47, 134 MB 34 -> 30, 680 MB 143 -> 128
    const int near = std::min(B, kKvScanRequests);
    p.stream_keys = (float)(kMemorySideCache / (2 * kD) * 3 / 8) / (float)Hkv * (float)((near + 3) / 4) / (float)near;       // (what the looked-at quarter adds up to)
    p.g_magic = 65536u / (uint32_t)G + 1;
    p.scale_log2e = fabsf(scale) * 1.4426950408889634f;
    p.q_sign = scale < 0.0f ? 0x80008000u : 0u;
    hipStream_t s = (hipStream_t)stream;
    dim3 grid(Hkv * c.groups, B);
    if (c.ranges > 0) {
        char* at = (char*)workspace;
        p.req = (u32x2*)at;
        p.part_o = (float*)(at + c.req_bytes);
        p.part_m = (float*)(at + c.req_bytes + round_up(c.slots * kD * 4, 256));
        p.part_l = (float*)((char*)p.part_m + round_up(c.slots * 4, 256));
        grid = dim3(Hkv, c.ranges);
    }
    int rc = SPEC_OK;
    switch (c.tiles) {
        case 1: rc = launch_quant<1>(p, kv_type, grid, s); break;
        case 2: rc = launch_quant<2>(p, kv_type, grid, s); break;
        default: rc = launch_quant<3>(p, kv_type, grid, s); break;
    }
    if (rc != SPEC_OK) return rc;
    rc = check_launch("spec_verify_attn_quantized");
    if (rc != SPEC_OK || c.ranges <= 1) return rc;        // (one range holds every request whole)
    if (c.many) hipLaunchKernelGGL(verify_attn_quant_merge_kernel<1>, dim3(M, Hq), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(verify_attn_quant_merge_kernel<8>, dim3(M, (Hq + 7) / 8), dim3(256), 0, s, p);
    return check_launch("spec_verify_attn_quantized (merge)");
}
