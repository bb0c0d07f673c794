// spec_verify_attn_quantized: the attention of spec_verify_attn over pages that hold K and V in 8 bits with a scale per page and kv head.
//
//   S[t] = scale * ks[page(t)] * <q, K8_t>,  out = sum_t softmax(S)[t] * vs[page(t)] * V8_t
//
// The products run on the bf16 matrix cores: every e4m3 and int8 value is a bf16 value, so the conversion loses nothing, and the scales stay in fp32: K's is part of the
// softmax scale of a page's scores, V's is a factor of the page's probabilities before they are rounded to bf16 (2^-9 each, as in spec_verify_attn).  Scores, maxima, sums and O are fp32.
//
// HBM-bound: 256 bytes of K + V per key and kv head.
//   Work: the batch is cut into equal ranges of work, one per workgroup and kv head, wherever the requests' borders lie, so that all workgroups are resident at once and end
//   together; a workgroup finds its range itself from the lengths (no list, no launch before it).  A request that lies in one range is finished there; pieces of others leave fp32
//   partials, at most two per range, which a second kernel merges.
//   A step: a wave owns 32 keys (two pages) of every 128; its pages go straight to its own LDS (direct loads, two steps in flight: half the bytes of bf16 pages would otherwise
//   leave HBM idle) and from there to registers.  The waves share nothing but Q until their parts are merged.
//   Operands: scores are computed transposed (S^T = K Q^T), so that exp(S^T) is the B operand of O^T += V^T P^T.  The order of d in a score is free:
//   K: lane (l16, g) holds key l16, d = 32 g .. + 31: MFMA s contracts d = 32 g + 8 s .. + 7, and Q is laid out alike;
//   V: lane (l16, g) holds d = 8 l16 .. + 7 of keys 4 g .. 4 g + 3: byte t of the four rows, paired by v_perm, converts to the A operand of output tile t, whose rows are
//      d = 8 m + t.  A lane then ends with d = 32 g .. 32 g + 31 of its query row.
#include "common.h"

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
constexpr int kQuantPageBytes = kP * kD;
constexpr int kQuantStageBytes = 4 * kQuantPageBytes;    // two pages of K, two of V
constexpr int kQuantWaveBytes = kQuantStages * kQuantStageBytes;
constexpr float kNegBig = -1.0e30f;          // "nothing seen yet" running maximum (log2 domain)
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
    int groups;              // whole requests: row groups are workgroups of their own (1: the workgroup takes them all)
    float scale_log2e;       // >= 0
    uint32_t q_sign;         // flips the sign of two query elements: a negative softmax scale
};

// two cached elements (bytes 2 HI, 2 HI + 1 of a word) as bf16
template <int TYPE, bool HI>
__device__ inline uint32_t bf16_pair(uint32_t raw)
{
    if constexpr (TYPE == SPEC_KV_E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw, 1.0f, HI));
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
    return n >= 1 && n <= p.max_q_len && r0 >= 0 && r0 + n <= p.M && c >= 0 && c + n <= p.max_kv_len;
}

// Work of one step of a request with `rows` query rows per kv head: a pass over the keys per kQuantTiles row tiles, and the tiles' products (128 keys in a full CU
// took 1.44, 1.60, 1.95 us with 1, 2, 3 tiles).
__host__ __device__ constexpr int quant_step_work(int rows)
{
    const int tiles = (rows + 15) / 16;
    return (tiles + kQuantTiles - 1) / kQuantTiles * 4 + tiles;
}

// One piece: keys kbeg .. kend (kbeg a multiple of 128) of request i for one kv head.
struct QuantPiece { int i, r0, n, c, kbeg, kend; bool whole; size_t slot; };

// A request's first row, rows and committed tokens, the same in every lane by construction: control flow and addresses that depend on them stay scalar.
struct QuantRequest { int r0, n, c; };

__device__ inline QuantRequest quant_request(const QuantAttnParams& p, int i)
{
    const int r0 = __builtin_amdgcn_readfirstlane(p.qo_indptr[i]), end = __builtin_amdgcn_readfirstlane(p.qo_indptr[i + 1]);
    return {r0, end - r0, __builtin_amdgcn_readfirstlane(p.seq_lens[i])};
}

// NR: row tiles at once.
template <int NR, int TYPE>
struct QuantKernel {
    static constexpr int NW = kQuantWaves;
    static constexpr int kSlices = (NR * 16 * kD * 4 + kQuantWaveBytes - 1) / kQuantWaveBytes, kSliceD = kD / kSlices, kChunks = kSliceD / 4;
    static_assert(kD % kSlices == 0 && kSliceD % 32 == 0 && NR * 16 * kSliceD * 4 <= kQuantWaveBytes, "a wave's slice of O fits its buffers");
    static_assert(kQuantStages == 2, "the waits count the loads of one younger step");
    // LDS: the waves' pages, Q, the waves' maxima and sums
    static constexpr size_t kQAt = NW * kQuantWaveBytes, kMlAt = kQAt + (NR == 1 ? 0 : NR * 4 * 64 * 16), kBytes = kMlAt + 2 * NW * NR * 16 * 4;

    static __device__ __forceinline__ void piece(const QuantAttnParams& p, unsigned char* smem, const QuantPiece& u, int kvh, int group)
    {
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int l16 = lane & 15, g = lane >> 4;
        u32x4* sQ = reinterpret_cast<u32x4*>(smem + kQAt);                             // [NR * 4][64], not with one row tile
        float* s_m = reinterpret_cast<float*>(smem + kMlAt);                           // [NW][NR * 16]
        float* s_l = s_m + NW * NR * 16;
        const int G = p.G, first_row = group * kQuantTiles * 16, R = min(G * u.n - first_row, NR * 16);
        const int c = u.c, kend = u.kend;

        // ---- page ids and scales of this wave's steps, 32 steps at a time: lane l holds page l % 2 of step l / 2 (page 0 stands in for a bad id, which is flagged,
        // and with scales 0 for what lies behind the piece) ----
        const int32_t* pt = p.page_table + (size_t)u.i * p.max_pages + (u.kbeg / kP);
        const int npages = (kend - u.kbeg + kP - 1) / kP;
        int ids = 0, bad_page = 0;
        float ksc = 0.0f, vsc = 0.0f;
        auto load_ids = [&](int step) {
            const int pg = (step + (lane >> 1)) * (kQuantStep / kP) + 2 * wave + (lane & 1);
            ids = 0;
            if (pg < npages) {
                ids = pt[pg];
                if (ids < 0 || ids >= p.num_pages) { ids = 0; bad_page = 1; }
            }
        };
        auto load_scales = [&](int step) {
            const int pg = (step + (lane >> 1)) * (kQuantStep / kP) + 2 * wave + (lane & 1);
            ksc = vsc = 0.0f;
            if (pg < npages) {
                ksc = p.k_scale[(size_t)ids * p.Hkv + kvh];
                vsc = p.v_scale[(size_t)ids * p.Hkv + kvh];
            }
        };
        load_ids(0);
        // Q fragments: one row tile stays in registers, more are read again from LDS, where wave w leaves fragment w of every tile
        bf16x8 qf[4];
        auto load_q = [&](int rt, int s) {
            const int r = rt * 16 + l16, j = (first_row + r) / G, gq = first_row + r - j * G;
            u32x4 x = {0, 0, 0, 0};
            if (r < R) x = *reinterpret_cast<const u32x4*>(p.q + ((size_t)(u.r0 + j) * p.Hq + kvh * G + gq) * kD + g * 32 + s * 8);
            return x ^ p.q_sign;
        };
        if constexpr (NR == 1) {
#pragma unroll
            for (int s = 0; s < 4; ++s) qf[s] = __builtin_bit_cast(bf16x8, load_q(0, s));
        } else {
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) sQ[(rt * 4 + wave) * 64 + lane] = load_q(rt, wave);
        }
        int limit[NR];                // row sees key positions t < limit
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            const int r = rt * 16 + l16;
            limit[rt] = r < R ? min(c + (first_row + r) / G + 1, kend) : 0;
        }

        // ---- a step's two pages, HBM -> LDS: 2 direct loads of 1 KB per page.  16-byte chunk ch of K's row (key) r is stored at position ch ^ (r & 7), so that
        // 8 lanes that read the same chunk of 8 rows meet no bank twice; V stays as it is ----
        unsigned char* ring = smem + wave * kQuantWaveBytes;
        const uint32_t koff = (uint32_t)((lane >> 3) * kD + (((lane & 7) ^ (lane >> 3)) << 4)), voff = (uint32_t)lane * 16;
        auto issue = [&](int step) {
            const int a = __builtin_amdgcn_readlane(ids, 2 * (step & 31)), b = __builtin_amdgcn_readlane(ids, 2 * (step & 31) + 1);
            unsigned char* to = ring + (step & 1) * kQuantStageBytes;
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
                const size_t at = ((size_t)(pg ? b : a) * p.Hkv + kvh) * kQuantPageBytes;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    lds_dma16_off(koff, p.k + at + h * 1024, to + pg * kQuantPageBytes + h * 1024);
                    lds_dma16_off(voff, p.v + at + h * 1024, to + (2 + pg) * kQuantPageBytes + h * 1024);
                }
            }
        };
        constexpr int kLoads = 8;                         // of a step
        const int wkeys = kend - u.kbeg - wave * 32, steps = wkeys <= 0 ? 0 : (wkeys + kQuantStep - 1) / kQuantStep;
        if (steps > 0) issue(0);
        if (steps > 1) issue(1);
        load_scales(0);                                   // (a second round trip that flies with the first pages)
        if constexpr (NR > 1) __syncthreads();
        // scales of the two steps in flight: K's of both pages, V's of both pages
        struct Scales { float k[2], v[2]; };
        auto scales_of = [&](int step) {
            Scales x;
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
                x.k[pg] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ksc), 2 * (step & 31) + pg));
                x.v[pg] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, vsc), 2 * (step & 31) + pg));
            }
            return x;
        };
        Scales now = scales_of(0), next = scales_of(1);

        f32x4 o[NR][8];
        float m_run[NR], l_run[NR];
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            m_run[rt] = kNegBig;
            l_run[rt] = 0.0f;
#pragma unroll
            for (int t = 0; t < 8; ++t) o[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        auto run = [&](auto active) {
            constexpr int A = decltype(active)::value;
            for (int step = 0; step < steps; ++step) {
                const int wbase = u.kbeg + step * kQuantStep + wave * 32;
                // this step's pages have landed, the next one's may fly on; once they are in registers, their place is for the step behind that
                if (step + 1 < steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
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
                float ks[2] = {now.k[0] * p.scale_log2e, now.k[1] * p.scale_log2e};
                const float vs[2] = {now.v[0], now.v[1]};
                now = next;
                if (step + 2 < steps) {
                    if (((step + 2) & 31) == 0) {         // the next 32 steps
                        load_ids(step + 2);
                        load_scales(step + 2);
                    }
                    issue(step + 2);
                    next = scales_of(step + 2);
                }
                __builtin_amdgcn_sched_barrier(0);
                // (two row tiles and more: Q is read again in every step; the compiler would rather keep all of it in registers)
                int q_lane = lane;
                if constexpr (NR > 1) asm volatile("" : "+v"(q_lane));
                // ---- S^T = K Q^T; sc * ks is a score in the log2 domain ----
                float sc[A][8];
#pragma unroll
                for (int pg = 0; pg < 2; ++pg) {
                    f32x4 acc[A];
#pragma unroll
                    for (int rt = 0; rt < A; ++rt) acc[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const u32x4 raw = kraw[pg][s >> 1];
                        const bf16x8 kf = (s & 1) ? bf16_oct<TYPE>(raw.z, raw.w) : bf16_oct<TYPE>(raw.x, raw.y);
#pragma unroll
                        for (int rt = 0; rt < A; ++rt) {
                            const bf16x8 qx = NR == 1 ? qf[s] : __builtin_bit_cast(bf16x8, sQ[(rt * 4 + s) * 64 + q_lane]);
                            acc[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qx, acc[rt], 0, 0, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int rt = 0; rt < A; ++rt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[rt][pg * 4 + e] = acc[rt][e];
                }
                const bool need_mask = wbase + 32 > min(c + 1, kend);
                if (need_mask) {                          // (a scale may be 0: masked scores are scaled ones)
#pragma unroll
                    for (int rt = 0; rt < A; ++rt)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            sc[rt][e] = wbase + (e >> 2) * 16 + g * 4 + (e & 3) < limit[rt] ? sc[rt][e] * ks[e >> 2] : kNegBig;
                    ks[0] = ks[1] = 1.0f;
                }
                // The reference maximum moves only when a score exceeds it by more than kMaxSlack, so exp2(s - m_run) <= 2^kMaxSlack stays well inside fp32 and bf16 and O
                // is rescaled a handful of times (the result is the same softmax: O and l carry the same factor).  A lane looks at its own 8 scores, and the four lanes
                // of a query row agree on a new maximum where one of them asks for it.
                float tmax[A];
                bool grow = false;
#pragma unroll
                for (int rt = 0; rt < A; ++rt) {
                    const float a = fmaxf(fmaxf(sc[rt][0], sc[rt][1]), fmaxf(sc[rt][2], sc[rt][3])), b = fmaxf(fmaxf(sc[rt][4], sc[rt][5]), fmaxf(sc[rt][6], sc[rt][7]));
                    tmax[rt] = fmaxf(a * ks[0], b * ks[1]);
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
                bf16x8 pf[A];
#pragma unroll
                for (int rt = 0; rt < A; ++rt) {
                    float pr[8], psum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        pr[e] = __builtin_amdgcn_exp2f(fmaf(sc[rt][e], ks[e >> 2], -m_run[rt]));
                        // (a row that has seen nothing at all has m_run == kNegBig)
                        if (need_mask) pr[e] = sc[rt][e] > 0.5f * kNegBig ? pr[e] : 0.0f;
                        psum += pr[e];
                    }
                    l_run[rt] += psum;
                    const u32x4 pw = {pack_bf16x2(pr[0] * vs[0], pr[1] * vs[0]), pack_bf16x2(pr[2] * vs[0], pr[3] * vs[0]),
                                      pack_bf16x2(pr[4] * vs[1], pr[5] * vs[1]), pack_bf16x2(pr[6] * vs[1], pr[7] * vs[1])};
                    pf[rt] = __builtin_bit_cast(bf16x8, pw);
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
                uint32_t pair[2][2][4];                   // [page][keys 4g, 4g+1 | 4g+2, 4g+3][t / 2]: bytes {key a, key b} of t, then of t + 1
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
                    if (t & 1) w = u32x4{bf16_pair<TYPE, true>(pair[0][0][t >> 1]), bf16_pair<TYPE, true>(pair[0][1][t >> 1]),
                                         bf16_pair<TYPE, true>(pair[1][0][t >> 1]), bf16_pair<TYPE, true>(pair[1][1][t >> 1])};
                    else w = u32x4{bf16_pair<TYPE, false>(pair[0][0][t >> 1]), bf16_pair<TYPE, false>(pair[0][1][t >> 1]),
                                   bf16_pair<TYPE, false>(pair[1][0][t >> 1]), bf16_pair<TYPE, false>(pair[1][1][t >> 1])};
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                    for (int rt = 0; rt < A; ++rt) o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt], o[rt][t], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        if (NR >= 3 && R > 32) run(std::integral_constant<int, NR >= 3 ? 3 : 1>{});
        else if (NR >= 2 && R > 16) run(std::integral_constant<int, NR >= 2 ? 2 : 1>{});
        else run(std::integral_constant<int, 1>{});
        if (bad_page && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_PAGE);

        // ---- merge the waves, in slices of d: each leaves its O where its pages were (16-byte chunk c of a row at position c ^ (row & 7)), maxima and sums beside; a thread then
        // takes 4 consecutive d of a row from all waves ----
        float* own = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            const float l = four_rows_sum(l_run[rt]);
            if (g == 0) {
                s_m[wave * NR * 16 + rt * 16 + l16] = m_run[rt];
                s_l[wave * NR * 16 + rt * 16 + l16] = l;
            }
        }
#pragma unroll
        for (int sl = 0; sl < kSlices; ++sl) {
            if (sl > 0) __syncthreads();                  // everybody has read the previous slice
            if (32 * g / kSliceD == sl) {
#pragma unroll
                for (int rt = 0; rt < NR; ++rt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            // d = 32 g + 8 e + 4 w .. + 3
                            const int ch = (32 * g % kSliceD) / 4 + 2 * e + w;
                            *reinterpret_cast<f32x4*>(own + (rt * 16 + l16) * kSliceD + ((ch ^ (l16 & 7)) << 2)) =
                                f32x4{o[rt][4 * w][e], o[rt][4 * w + 1][e], o[rt][4 * w + 2][e], o[rt][4 * w + 3][e]};
                        }
            }
            __syncthreads();
            for (int e = tid; e < R * kChunks; e += kQuantThreads) {
                const int r = e / kChunks, ch = e % kChunks;
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
                    num += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem + w * kQuantWaveBytes) + r * kSliceD + ((ch ^ (r & 7)) << 2));
                    l += f * s_l[w * NR * 16 + r];
                }
                const int j = (first_row + r) / G, gq = first_row + r - j * G;
                if (u.whole) {
                    const size_t rowhead = (size_t)(u.r0 + j) * p.Hq + kvh * G + gq;
                    u32x2_any packed;
                    packed.x = pack_bf16x2(num.x / l, num.y / l);
                    packed.y = pack_bf16x2(num.z / l, num.w / l);
                    *reinterpret_cast<u32x2_any*>(p.out + rowhead * kD + sl * kSliceD + ch * 4) = packed;
                    if (p.lse && sl == 0 && ch == 0) p.lse[rowhead] = (mx + log2f(l)) * 0.6931471805599453f;
                } else {
                    const size_t at = (u.slot * p.max_q_len + j) * p.Hq + kvh * G + gq;
                    *reinterpret_cast<f32x4*>(p.part_o + at * kD + sl * kSliceD + ch * 4) = num;
                    if (sl == 0 && ch == 0) { p.part_m[at] = mx; p.part_l[at] = l; }
                }
            }
        }
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
        const int group = blockIdx.x / p.Hkv, kvh = blockIdx.x - group * p.Hkv, i = blockIdx.y;
        const auto [r0, n, c] = quant_request(p, i);
        if (!quant_request_ok(r0, n, c, p)) {
            if (blockIdx.x == 0 && tid == 0 && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_LENGTH);
            return;
        }
        const QuantPiece u{i, r0, n, c, 0, c + n, true, 0};
        for (int at = group; at * kQuantTiles * 16 < p.G * n; at += p.groups) {
            if (at > group) __syncthreads();              // the buffers are free again
            Kernel::piece(p, smem, u, kvh, at);
        }
    } else {
        const int kvh = blockIdx.x, range = blockIdx.y;
        // Every request's work and what comes before it, four requests per thread; the total gives the size of a range, and the request in which this one starts leaves its
        // number and place in LDS.
        constexpr int kPer = kQuantListed / kQuantThreads;
        int* s_scan = reinterpret_cast<int*>(smem);       // [8], then {request, work before it}
        int work[kPer], mine = 0;
        bool bad = false;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = tid * kPer + k;
            work[k] = 0;
            if (i < p.B) {
                const int r0 = p.qo_indptr[i], n = p.qo_indptr[i + 1] - r0, c = p.seq_lens[i];
                if (quant_request_ok(r0, n, c, p)) work[k] = (c + n + kQuantStep - 1) / kQuantStep * quant_step_work(p.G * n);
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
        const int first = range * quantum, last = min(total, first + quantum);        // (at most total + ranges * min_work: the host sees to 32 bits)
        if (first >= total) return;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if (first >= before && first < before + work[k]) { s_scan[4] = tid * kPer + k; s_scan[5] = before; }
            before += work[k];
        }
        __syncthreads();
        int i = __builtin_amdgcn_readfirstlane(s_scan[4]), at = __builtin_amdgcn_readfirstlane(s_scan[5]);      // `at`: the work before request i
        while (at < last) {
            __syncthreads();                              // the buffers are free again
            const auto [r0, n, c] = quant_request(p, i);
            if (quant_request_ok(r0, n, c, p)) {
                const int len = c + n, steps = (len + kQuantStep - 1) / kQuantStep, w = quant_step_work(p.G * n);
                // the steps whose place lies in this range
                const int from = at >= first ? 0 : (first - at + w - 1) / w, to = min(steps, (first + quantum - at + w - 1) / w);
                const int head = at / quantum, pieces = (at + (steps - 1) * w) / quantum - head + 1;
                if (from == 0 && kvh == 0 && tid == 0) p.req[i] = u32x2{(uint32_t)head, (uint32_t)pieces};
                if (from < to) {
                    const QuantPiece u{i, r0, n, c, from * kQuantStep, min(len, to * kQuantStep), pieces == 1, 2 * (size_t)range + (from == 0)};
                    for (int group = 0; group * kQuantTiles * 16 < p.G * n; ++group) {
                        if (group > 0) __syncthreads();
                        Kernel::piece(p, smem, u, kvh, group);
                    }
                }
                at += steps * w;
            }
            ++i;
        }
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
    int count = 0;
    for (int k = 0; k < p.B; k += 256) count += __syncthreads_count(k + tid < p.B && p.qo_indptr[k + tid] <= row);
    const int i = __builtin_amdgcn_readfirstlane(count) - 1;          // the last request that starts at or before the row
    if (i < 0) return;
    const int r0 = p.qo_indptr[i], n = p.qo_indptr[i + 1] - r0, c = p.seq_lens[i];
    if (!quant_request_ok(r0, n, c, p) || row < r0 || row >= r0 + n) return;
    const u32x2 q = p.req[i];
    const int head = (int)q.x, pieces = (int)q.y;
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
    bool many;                               // pieces per request: a workgroup per head merges them
    size_t slots, req_bytes;
};

constexpr int kQuantMinSteps = 2;            // of a range

static QuantPlan quant_plan(int B, int Hq, int Hkv, int max_kv_len, int max_q_len)
{
    QuantPlan c{};
    const int G = Hq / Hkv, NR = (G * max_q_len + 15) / 16;
    c.tiles = std::min(NR, kQuantTiles);
    const int row_groups = (NR + kQuantTiles - 1) / kQuantTiles;
    const long cus = device_cu_count(), units = (long)B * Hkv;
    c.groups = units >= cus ? 1 : row_groups;
    const int mode = g_attn_plan, chunk = g_attn_chunk_override, waves = g_attn_plan_waves;
    const long steps = ((long)max_kv_len + kQuantStep - 1) / kQuantStep, work = quant_step_work(G * max_q_len);
    const long most = B * steps * work;      // work of the batch at its bounds
    if (mode == 2 || B > kQuantListed || steps < 2 * kQuantMinSteps || most > (1L << 30)) return c;
    c.min_work = (int)(kQuantMinSteps * work);
    long ranges = std::max<long>(1, cus * (waves > 0 ? waves : kQuantWgsPerCu) / Hkv);
    if (chunk > 0) { ranges = (long)B * max_kv_len / chunk + 1; c.min_work = (int)work; }
    ranges = std::min(std::min<long>(ranges, (most + c.min_work - 1) / c.min_work), 8192L);
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
    if (B <= 0 || M <= 0 || Hq <= 0 || Hkv <= 0 || max_kv_len <= 0 || Hq % Hkv != 0) return 0;
    return quant_workspace(quant_plan(B, Hq, Hkv, max_kv_len, max_q_len > 0 ? max_q_len : 1));
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
    if (need > 0 && (!workspace || !aligned(workspace, 256)))
        return fail(SPEC_EINVAL, "spec_verify_attn_quantized: workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need)
        return fail(SPEC_EWORKSPACE, "spec_verify_attn_quantized: workspace %zu bytes, need %zu", workspace_bytes, need);

    QuantAttnParams p{};
    p.q = (const uint16_t*)q; p.k = (const uint8_t*)k_cache; p.v = (const uint8_t*)v_cache; p.k_scale = k_scale; p.v_scale = v_scale;
    p.page_table = page_table; p.seq_lens = seq_lens; p.qo_indptr = qo_indptr;
    p.out = (uint16_t*)out; p.lse = lse; p.status_flags = status_flags;
    p.max_pages = max_pages_per_seq; p.num_pages = num_pages; p.Hq = Hq; p.Hkv = Hkv; p.G = G;
    p.M = M; p.B = B; p.max_kv_len = max_kv_len; p.max_q_len = max_q_len;
    p.ranges = c.ranges; p.min_work = c.min_work; p.groups = c.groups;
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
