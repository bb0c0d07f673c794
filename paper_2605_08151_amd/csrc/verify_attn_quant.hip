// spec_verify_attn_quantized: the attention of spec_verify_attn over pages that hold K and V in 8 bits with a scale per page and kv head.
//
//   S[t] = scale * ks[page(t)] * <q, K8_t>,  out = sum_t softmax(S)[t] * vs[page(t)] * V8_t
//
// The products run on the bf16 matrix cores: every e4m3 and int8 value is a bf16 value, so the conversion loses nothing, and the scales stay in fp32: K's is part of the
// softmax scale of a page's scores, V's is a factor of the page's probabilities before they are rounded to bf16 (2^-9 each, as in spec_verify_attn).  Scores, maxima, sums and O are fp32.
//
// HBM-bound: 256 bytes of K + V per key and kv head.  As in verify_attn.hip a workgroup streams one chunk of one request's keys for one kv head, a wave owns 32 keys
// (two pages) of every step, scores are computed transposed (S^T = K Q^T, so that exp(S^T) is the B operand of O^T += V^T P^T), chunks leave fp32 partials and a second kernel
// merges them.  Unlike there nothing of K and V goes through LDS: the order of d in a score is free, and with half the bytes a lane's operands are what it loads itself:
//   K: lane (l16, g) holds key l16, d = 32 g .. + 31: MFMA s contracts d = 32 g + 8 s .. + 7, and Q is laid out alike;
//   V: lane (l16, g) holds d = 8 l16 .. + 7 of keys 4 g .. 4 g + 3: byte t of the four rows, paired by v_perm, converts to the A operand of output tile t, whose rows are
//      d = 8 m + t.  A lane then ends with d = 32 g .. 32 g + 31 of its query row.
// The next step's K is requested as soon as this one's is converted, its V likewise.
#include "attn_params.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace specv {

extern Tunable g_attn_chunk_override;
extern Tunable g_attn_plan;
extern Tunable g_attn_plan_waves;

constexpr int kQuantWaves = 4;               // waves per workgroup
constexpr int kQuantStep = kQuantWaves * 32; // keys per workgroup step
constexpr int kQuantTiles = 3;               // row tiles (16 query rows) a workgroup takes at most
constexpr int kQuantStages = 2;              // steps of a wave that are in flight
constexpr int kQuantPageBytes = kP * kD;
constexpr int kQuantStageBytes = 4 * kQuantPageBytes;    // two pages of K, two of V

struct QuantAttnParams {
    AttnParams a;                            // (k_cache, v_cache: not used)
    const uint8_t* k;
    const uint8_t* v;
    const float* k_scale;                    // [num_pages, Hkv]
    const float* v_scale;
    int page_slots;                          // 4-byte slots of a chunk's page ids in LDS
    uint32_t q_sign;                         // flips the sign of two query elements: a negative softmax scale (a.scale_log2e is its magnitude)
};

constexpr int kQuantWgsPerCu = 2;            // 64 KB of pages in flight each

// two cached elements (bytes 2 HI, 2 HI + 1 of a word) as bf16
template <int TYPE, bool HI>
__device__ inline uint32_t bf16_pair(uint32_t raw)
{
    if constexpr (TYPE == SPEC_KV_E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw, 1.0f, HI));
    else return pack_bf16x2((float)(int8_t)(raw >> (HI ? 16 : 0)), (float)(int8_t)(raw >> (HI ? 24 : 8)));
}

// (The empty statement keeps the words whole up to here: the compiler otherwise takes them apart where they are loaded, a step earlier, into a register per byte.)
template <int TYPE>
__device__ inline bf16x8 bf16_oct(uint32_t a, uint32_t b)
{
    asm("" : "+v"(a), "+v"(b));
    const u32x4 w = {bf16_pair<TYPE, false>(a), bf16_pair<TYPE, true>(a), bf16_pair<TYPE, false>(b), bf16_pair<TYPE, true>(b)};
    return __builtin_bit_cast(bf16x8, w);
}

// NR: row tiles per workgroup; FINAL: no request is split, the workgroup normalises and writes bf16 itself.
template <int NR, int TYPE, bool FINAL>
__global__ __launch_bounds__(kQuantWaves * 64, kQuantWgsPerCu) void verify_attn_quant_kernel(QuantAttnParams qp)
{
    constexpr int NW = kQuantWaves, kThreads = NW * 64;
    constexpr int kWaveBytes = kQuantStages * kQuantStageBytes;
    constexpr int kSlices = (NR * 16 * kD * 4 + kWaveBytes - 1) / kWaveBytes, kSliceD = kD / kSlices, kChunks = kSliceD / 4;
    static_assert(kD % kSlices == 0 && kSliceD % 32 == 0 && NR * 16 * kSliceD * 4 <= kWaveBytes, "a wave's slice of O fits its buffers");
    const AttnParams& p = qp.a;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    u32x4* sQ = reinterpret_cast<u32x4*>(smem + NW * kWaveBytes);                        // [NR * 4][64], not with one row tile
    float* sScale = reinterpret_cast<float*>(sQ + (NR == 1 ? 0 : NR * 4 * 64));          // scales of the chunk's pages: K's, then V's
    int32_t* sPT = reinterpret_cast<int32_t*>(sScale + 2 * qp.page_slots);               // ... and their ids

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    // the first dimension of the grid: kv heads, and the row groups of each
    const int groups = (p.G * p.max_q_len + NR * 16 - 1) / (NR * 16);
    const int hx = p.head_first ? blockIdx.x : blockIdx.y, piece = p.head_first ? blockIdx.y : blockIdx.x;
    const int kvh = hx / groups, group = hx - kvh * groups;
    int split, i, ns_plan = 0, pb_plan = 0;
    if (p.plan_items) {
        if (piece >= p.plan_hdr[0]) return;
        const int* it = p.plan_items + 4 * (size_t)piece;
        i = __builtin_amdgcn_readfirstlane(it[0]);
        split = __builtin_amdgcn_readfirstlane(it[1]);
        ns_plan = __builtin_amdgcn_readfirstlane(it[2]);
        pb_plan = __builtin_amdgcn_readfirstlane(it[3]);
    } else {
        i = blockIdx.z;
        split = FINAL ? piece : piece_of_place(p.turn, p.splits, piece, i);
    }
    const int r0 = p.qo_indptr[i], n = p.qo_indptr[i + 1] - r0, c = p.seq_lens[i];
    if (!request_ok(r0, n, c, p)) {
        if (!p.plan_items && split == 0 && hx == 0 && tid == 0 && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_LENGTH);
        return;
    }
    const int len = c + n;
    const int ns = p.plan_items ? ns_plan : (len + p.chunk_target - 1) / p.chunk_target;
    if (split >= ns) return;
    const int G = p.G, first_row = group * NR * 16, R = min(G * n - first_row, NR * 16);    // rows first_row .. first_row + R of the request and kv head
    if (R <= 0) return;
    const int chunk = (((len + ns - 1) / ns) + kP - 1) & ~(kP - 1);
    const int kbeg = split * chunk;
    const int kend = min(len, kbeg + chunk);
    const size_t part_base = p.plan_items ? (size_t)pb_plan : (size_t)r0 * p.Hq * p.splits;
    const size_t part_ns = p.plan_items ? (size_t)ns : (size_t)p.splits;
    const int nrt = (R + 15) >> 4;

    // page ids of the chunk, validated once (page 0 stands in for a bad id, which is flagged)
    const int32_t* pt = p.page_table + (size_t)i * p.max_pages;
    int bad_page = 0;
    const int npages = (kend - kbeg + kP - 1) / kP;
    for (int pg = tid; pg < npages; pg += kThreads) {
        int page = pt[kbeg / kP + pg];
        if (page < 0 || page >= p.num_pages) { page = 0; bad_page = 1; }
        sPT[pg] = page;
    }
    // Q fragments: one row tile stays in registers, more are read again from LDS, where wave w leaves fragment w of every tile
    bf16x8 qf[4];
    auto load_q = [&](int rt, int s) {
        const int r = rt * 16 + l16, j = (first_row + r) / G, gq = first_row + r - j * G;
        u32x4 x = {0, 0, 0, 0};
        if (r < R) x = *reinterpret_cast<const u32x4*>(p.q + ((size_t)(r0 + j) * p.Hq + kvh * G + gq) * kD + g * 32 + s * 8);
        return x ^ qp.q_sign;
    };
    if constexpr (NR == 1) {
#pragma unroll
        for (int s = 0; s < 4; ++s) qf[s] = __builtin_bit_cast(bf16x8, load_q(0, s));
    } else {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) sQ[(rt * 4 + wave) * 64 + lane] = load_q(rt, wave);
    }
    int limit[NR];                    // row sees key positions t < limit
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        const int r = rt * 16 + l16;
        limit[rt] = r < R ? min(c + (first_row + r) / G + 1, kend) : 0;
    }
    __syncthreads();

    // This wave's two pages of a step, HBM -> LDS: 2 direct loads of 1 KB per page; places past the range are read from page 0 and masked.  16-byte chunk ch of K's row
    // (key) r is stored at position ch ^ (r & 7), so that 8 lanes that read the same chunk of 8 rows meet no bank twice; V stays as it is.
    unsigned char* ring = smem + wave * kWaveBytes;
    const uint32_t koff = (uint32_t)((lane >> 3) * kD + (((lane & 7) ^ (lane >> 3)) << 4)), voff = (uint32_t)lane * 16;
    auto issue = [&](int wbase, int stage) {
        const int a = __builtin_amdgcn_readfirstlane(sPT[(wbase - kbeg) / kP]);
        const int b = wbase + kP < kend ? __builtin_amdgcn_readfirstlane(sPT[(wbase - kbeg) / kP + 1]) : 0;
        unsigned char* to = ring + stage * kQuantStageBytes;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
            const size_t at = ((size_t)(pg ? b : a) * p.Hkv + kvh) * kQuantPageBytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                lds_dma16_off(koff, qp.k + at + h * 1024, to + pg * kQuantPageBytes + h * 1024);
                lds_dma16_off(voff, qp.v + at + h * 1024, to + (2 + pg) * kQuantPageBytes + h * 1024);
            }
        }
    };
    constexpr int kLoads = 8;                             // of a stage
    const int wfirst = kbeg + wave * 32;
#pragma unroll
    for (int st = 0; st < kQuantStages; ++st)
        if (wfirst + st * kQuantStep < kend) issue(wfirst + st * kQuantStep, st);
    // (behind the first pages' requests: a second round trip that flies with them)
    for (int pg = tid; pg < 2 * qp.page_slots; pg += kThreads) {
        const int at = pg < qp.page_slots ? pg : pg - qp.page_slots;
        sScale[pg] = at < npages ? (pg < qp.page_slots ? qp.k_scale : qp.v_scale)[(size_t)sPT[at] * p.Hkv + kvh] : 0.0f;
    }
    __syncthreads();

    f32x4 o[NR][8];
    float m_run[NR], l_run[NR];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        m_run[rt] = kNegBig;
        l_run[rt] = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) o[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    auto run_chunk = [&](auto active) {
    constexpr int A = decltype(active)::value;
    int stage = 0;
    for (int wbase = wfirst; wbase < kend; wbase += kQuantStep) {
        // this step's pages have landed, the next one's may fly on; once they are in registers, their place is for the step behind that
        if (wbase + kQuantStep < kend) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads * (kQuantStages - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        u32x4 kraw[2][2];
        u32x2 vraw[2][4];
        const unsigned char* sK = ring + stage * kQuantStageBytes;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
#pragma unroll
            for (int h = 0; h < 2; ++h) kraw[pg][h] = *reinterpret_cast<const u32x4*>(sK + pg * kQuantPageBytes + l16 * kD + (((2 * g + h) ^ (l16 & 7)) << 4));
#pragma unroll
            for (int r = 0; r < 4; ++r) vraw[pg][r] = *reinterpret_cast<const u32x2*>(sK + (2 + pg) * kQuantPageBytes + (4 * g + r) * kD + l16 * 8);
        }
        float ks[2], vs[2];
        const int at = (wbase - kbeg) / kP;               // (a page that is not there has scales 0)
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) { ks[pg] = sScale[at + pg] * p.scale_log2e; vs[pg] = sScale[qp.page_slots + at + pg]; }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (wbase + kQuantStages * kQuantStep < kend) issue(wbase + kQuantStages * kQuantStep, stage);
        stage = stage + 1 == kQuantStages ? 0 : stage + 1;
        // (two row tiles: Q is read again in every step, 32 registers less; three have room for 48)
        int q_lane = lane;
        if constexpr (NR == 2) asm volatile("" : "+v"(q_lane));
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
        if (need_mask) {                                  // (a scale may be 0: masked scores are scaled ones)
#pragma unroll
            for (int rt = 0; rt < A; ++rt)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sc[rt][e] = wbase + (e >> 2) * 16 + g * 4 + (e & 3) < limit[rt] ? sc[rt][e] * ks[e >> 2] : kNegBig;
            ks[0] = ks[1] = 1.0f;
        }
        // The reference maximum moves only when a score exceeds it by more than kMaxSlack (see verify_attn.hip): a lane looks at its own 8 scores, and the four
        // lanes of a query row agree on a new maximum where one of them asks for it.
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
        uint32_t pair[2][2][4];       // [page][keys 4g, 4g+1 | 4g+2, 4g+3][t / 2]: bytes {key a, key b} of t, then of t + 1
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
            if (t & 1) w = u32x4{bf16_pair<TYPE, true>(pair[0][0][t >> 1]), bf16_pair<TYPE, true>(pair[0][1][t >> 1]), bf16_pair<TYPE, true>(pair[1][0][t >> 1]), bf16_pair<TYPE, true>(pair[1][1][t >> 1])};
            else w = u32x4{bf16_pair<TYPE, false>(pair[0][0][t >> 1]), bf16_pair<TYPE, false>(pair[0][1][t >> 1]), bf16_pair<TYPE, false>(pair[1][0][t >> 1]), bf16_pair<TYPE, false>(pair[1][1][t >> 1])};
            const bf16x8 vf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
            for (int rt = 0; rt < A; ++rt) o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt], o[rt][t], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    };
    switch (nrt) {
        case 1: run_chunk(std::integral_constant<int, 1>{}); break;
        case 2: if constexpr (NR >= 2) run_chunk(std::integral_constant<int, 2>{}); break;
        default: if constexpr (NR >= 3) run_chunk(std::integral_constant<int, 3>{}); break;
    }
    if (bad_page && p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_PAGE);

    // ---- merge the waves, in slices of d: each leaves its O (16-byte chunk c of a row at position c ^ (row & 7)), maxima and sums; a thread then takes 4
    // consecutive d of a row from all waves ----
    float* s_m = sScale;                                  // [NW][NR * 16] (every wave has read its scales, see the barrier)
    float* s_l = s_m + NW * NR * 16;
    float* own = reinterpret_cast<float*>(ring);
    __syncthreads();
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
        if (sl > 0) __syncthreads();                      // everybody has read the previous slice
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
        for (int e = tid; e < R * kChunks; e += kThreads) {
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
                num += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem + w * kWaveBytes) + r * kSliceD + ((ch ^ (r & 7)) << 2));
                l += f * s_l[w * NR * 16 + r];
            }
            const int j = (first_row + r) / G, gq = first_row + r - j * G;
            if (FINAL) {
                const size_t rowhead = (size_t)(r0 + j) * p.Hq + kvh * G + gq;
                u32x2_any packed;
                packed.x = pack_bf16x2(num.x / l, num.y / l);
                packed.y = pack_bf16x2(num.z / l, num.w / l);
                *reinterpret_cast<u32x2_any*>(p.out + rowhead * kD + sl * kSliceD + ch * 4) = packed;
                if (p.lse && sl == 0 && ch == 0) p.lse[rowhead] = (mx + log2f(l)) * 0.6931471805599453f;
            } else {
                const size_t slot = part_base + ((size_t)j * p.Hq + kvh * G + gq) * part_ns + split;
                *reinterpret_cast<f32x4*>(p.part_o + slot * kD + sl * kSliceD + ch * 4) = num;
                if (sl == 0 && ch == 0) { p.part_m[slot] = mx; p.part_l[slot] = l; }
            }
        }
    }
}

// How a call is cut up: keys per split of the fixed chunks, or the work list.
struct QuantPlan {
    int tiles, groups;                       // row tiles per workgroup, workgroups per (chunk, kv head)
    int chunk, splits;
    bool list;
    int target_items, max_items;
    size_t hdr_bytes, req_bytes, items_bytes, slots;
};

constexpr int kQuantMinChunk = 256, kQuantMaxChunk = 4096;

static QuantPlan quant_plan(int B, int M, int Hq, int Hkv, int max_kv_len, int max_q_len)
{
    QuantPlan c{};
    const int NR = (Hq / Hkv * max_q_len + 15) / 16;
    c.groups = (NR + kQuantTiles - 1) / kQuantTiles;
    c.tiles = (NR + c.groups - 1) / c.groups;
    const long cus = device_cu_count(), per_cu = kQuantWgsPerCu;
    const int forced = g_attn_chunk_override;
    long target = forced > 0 ? forced : (long)B * Hkv * max_kv_len / (cus * per_cu);
    if (forced <= 0) target = std::min<long>(std::max<long>(target, kQuantMinChunk), 4096);
    target = std::min<long>(std::min<long>(target, kQuantMaxChunk), max_kv_len);
    c.chunk = (int)((target + kQuantStep - 1) / kQuantStep * kQuantStep);
    c.splits = (max_kv_len + c.chunk - 1) / c.chunk;
    c.list = B <= 1024 && g_attn_plan != 2 && (g_attn_plan == 1 || (c.splits > 1 && max_kv_len >= 4096 && B > 1));
    const int plan_waves = g_attn_plan_waves;
    const long t = std::max<long>(1, cus * (plan_waves > 0 ? plan_waves : per_cu) / Hkv);
    c.target_items = (int)t;
    c.max_items = (int)std::min<long>(std::max<long>(t + B, (long)B * ((max_kv_len + kQuantMaxChunk - 1) / kQuantMaxChunk)), 2147483647L);
    c.hdr_bytes = 256;
    c.req_bytes = round_up((size_t)B * 8, 256);
    c.items_bytes = round_up((size_t)c.max_items * 16, 256);
    c.slots = c.list ? (size_t)c.max_items * max_q_len * Hq : (c.splits > 1 ? (size_t)M * Hq * c.splits : 0);
    return c;
}

static size_t quant_workspace(const QuantPlan& c)
{
    return (c.list ? c.hdr_bytes + c.req_bytes + c.items_bytes : 0) + round_up(c.slots * kD * 4, 256) + 2 * round_up(c.slots * 4, 256);
}

// LDS: the waves' pages, Q, and the scales and ids of a chunk's pages (where the waves' maxima and sums stand at the end)
static size_t quant_smem(int NR, int page_slots)
{
    return (size_t)kQuantWaves * kQuantStages * kQuantStageBytes + (NR == 1 ? 0 : (size_t)NR * 16 * kD * 2) + std::max<size_t>((size_t)page_slots * 12, (size_t)kQuantWaves * NR * 16 * 8);
}

template <int NR, int TYPE, bool FINAL>
static int launch_quant_one(const QuantAttnParams& p, dim3 grid, hipStream_t s)
{
    const size_t smem = quant_smem(NR, p.page_slots);
    static LdsGrantTable granted = {};
    if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(&verify_attn_quant_kernel<NR, TYPE, FINAL>), smem, granted, "spec_verify_attn_quantized")) return rc;
    hipLaunchKernelGGL((verify_attn_quant_kernel<NR, TYPE, FINAL>), grid, dim3(kQuantWaves * 64), smem, s, p);
    return SPEC_OK;
}

template <int NR, int TYPE>
static int launch_quant_as(const QuantAttnParams& p, dim3 grid, hipStream_t s)
{
    return p.a.splits == 1 ? launch_quant_one<NR, TYPE, true>(p, grid, s) : launch_quant_one<NR, TYPE, false>(p, grid, s);
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
    return quant_workspace(quant_plan(B, M, Hq, Hkv, max_kv_len, max_q_len > 0 ? max_q_len : 1));
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
    if (B > 65535 || Hkv > 8191 || M > 2147483647 / Hq) return fail(SPEC_ESHAPE, "spec_verify_attn_quantized: B, Hkv or M beyond the launch grid");
    const QuantPlan c = quant_plan(B, M, Hq, Hkv, max_kv_len, max_q_len);
    const size_t need = quant_workspace(c);
    if (need > 0 && (!workspace || !aligned(workspace, 256)))
        return fail(SPEC_EINVAL, "spec_verify_attn_quantized: workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need)
        return fail(SPEC_EWORKSPACE, "spec_verify_attn_quantized: workspace %zu bytes, need %zu", workspace_bytes, need);

    QuantAttnParams p{};
    AttnParams& a = p.a;
    a.q = (const uint16_t*)q;
    a.page_table = page_table; a.seq_lens = seq_lens; a.qo_indptr = qo_indptr;
    a.out = (uint16_t*)out; a.lse = lse; a.status_flags = status_flags;
    a.max_pages = max_pages_per_seq; a.num_pages = num_pages; a.Hq = Hq; a.Hkv = Hkv; a.G = G;
    a.M = M; a.max_kv_len = max_kv_len; a.max_q_len = max_q_len; a.B = B;
    a.chunk_target = c.chunk; a.splits = c.splits;
    a.scale_log2e = fabsf(scale) * 1.4426950408889634f;
    p.q_sign = scale < 0.0f ? 0x80008000u : 0u;
    p.k = (const uint8_t*)k_cache; p.v = (const uint8_t*)v_cache; p.k_scale = k_scale; p.v_scale = v_scale;
    hipStream_t s = (hipStream_t)stream;
    char* parts = (char*)workspace;
    dim3 grid(c.splits, Hkv * c.groups, B);               // (pieces, kv heads and their row groups, requests)
    if (c.list) {
        if (c.slots * kD > 2147483647u) return fail(SPEC_ESHAPE, "spec_verify_attn_quantized: work list beyond 32-bit slots");
        int32_t* hdr = (int32_t*)parts;
        int32_t* req = (int32_t*)(parts + c.hdr_bytes);
        int32_t* items = (int32_t*)(parts + c.hdr_bytes + c.req_bytes);
        parts += c.hdr_bytes + c.req_bytes + c.items_bytes;
        if (int rc = launch_attn_plan(a, B, c.target_items, kQuantStep, kQuantMinChunk, kQuantMaxChunk, c.max_items, hdr, req, items, s)) return rc;
        a.plan_hdr = hdr; a.plan_req = req; a.plan_items = items;
        a.chunk_target = kQuantMaxChunk;
        a.splits = 2;                                     // "somebody is split": partials and the merge
        grid = dim3(c.max_items, Hkv * c.groups, 1);
    }
    a.part_o = (float*)parts;
    a.part_m = (float*)(parts + round_up(c.slots * kD * 4, 256));
    a.part_l = (float*)(parts + round_up(c.slots * kD * 4, 256) + round_up(c.slots * 4, 256));
    p.page_slots = (std::min(a.chunk_target, max_kv_len) / kP + 3) & ~1;     // a step's second page may lie one behind the chunk's last
    a.turn = piece_turn(Hkv, a.splits);
    a.head_first = grid.x <= 65535;                       // (the second dimension's limit)
    if (a.head_first) grid = dim3(grid.y, grid.x, grid.z);
    int rc = SPEC_OK;
    switch (c.tiles) {
        case 1: rc = launch_quant<1>(p, kv_type, grid, s); break;
        case 2: rc = launch_quant<2>(p, kv_type, grid, s); break;
        default: rc = launch_quant<3>(p, kv_type, grid, s); break;
    }
    if (rc != SPEC_OK) return rc;
    rc = check_launch("spec_verify_attn_quantized");
    if (rc != SPEC_OK) return rc;
    if (a.splits == 1) return SPEC_OK;
    return launch_attn_merge(a, B, c.list ? (c.target_items + B) / B <= 8 : a.splits <= 16, s);
}
