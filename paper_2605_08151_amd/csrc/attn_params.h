// What the attention kernels on bf16 pages (verify_attn.hip) and on 8-bit pages (verify_attn_quant.hip) share: their parameters, a request's checks and order, and the launches
// of the work list's and the merge's kernels, which know nothing of the cache.
#pragma once

#include "batch_rules.h"
#include "common.h"

namespace specv {

constexpr int kD = 128;                      // head dimension
constexpr int kP = 16;                       // tokens per page
constexpr float kNegBig = -1.0e30f;          // "nothing seen yet" running maximum (log2 domain)
constexpr float kMaxSlack = 6.0f;            // how far a step's maximum may exceed the reference before a rescale

typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));    // (rows of the output may start at any element)

struct AttnParams {
    const uint16_t* q;
    const uint16_t* k_cache;
    const uint16_t* v_cache;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* qo_indptr;
    uint16_t* out;      // [M, Hq, 128] bf16
    float* lse;         // [M, Hq] or null
    float* part_o;      // [M*Hq, splits, 128]
    float* part_m;      // [M*Hq, splits]   running max, log2 domain
    float* part_l;      // [M*Hq, splits]
    int32_t* status_flags;
    // balanced work list written by verify_attn_plan_kernel (all null when requests are split by the fixed
    // chunk_target instead): hdr = {items, keys per chunk, K/V too large for the memory-side cache}; req[i] = {splits of request i, first partial slot};
    // items[k] = {request, split, splits of the request, first partial slot}
    const int32_t* parent;     // tree verification: row-local parent of every candidate row ([M], -1 for a root), or null = chains
    const int32_t* plan_hdr;
    const int32_t* plan_req;
    const int32_t* plan_items;
    int max_pages, num_pages, Hq, Hkv, G, M, max_kv_len, max_q_len, chunk_target, splits;
    float scale_log2e;
    int B;
    // Workgroups that start together take the heads of one piece: their pages are neighbours in HBM (a page of all heads is one stretch of Hkv * 4 KB), and are
    // read at about the same time.  Pieces first -> heads first: 128 requests x 8 heads x 2.6k keys 266.7 -> 220.7 us (5.2 -> 6.3 TB/s)
    int head_first;
    PieceTurn turn;            // fixed chunks: which piece of its request a place in the grid stands for
    // Fixed chunks, at most 64 requests, more workgroups than CUs: the requests with the longest contexts go first (see longest_first)
    int by_length;
    int page_slots;            // see attn_page_slots
    float stream_keys;         // committed keys of the batch above which its K/V is too large for the memory-side cache (0: it never is)
};

__device__ inline bool request_ok(int r0, int n, int c, const AttnParams& p)
{
    return n >= 1 && n <= p.max_q_len && r0 >= 0 && r0 + n <= p.M && c >= 0 && c + n <= p.max_kv_len;
}

// Request number `rank` in the order of committed keys, longest first (ties: request order), and its metadata.  A lane per request (at most 64); one memory round trip,
// like reading the request of the grid's own order.  Workgroups start in grid order, one per CU, so that the last ones decide when the call ends: 64 requests of
// 1-4k keys x 8 heads, 5 rows 114.0 -> 105.7 us; 16 trees of 0.5-4k keys x 8 heads 40.0 -> 38.3.
struct RequestRef { int i, r0, n, c; };

__device__ inline RequestRef longest_first(const AttnParams& p, int rank)
{
    const int lane = threadIdx.x & 63;
    int c = 0, q0 = 0, q1 = 0;
    if (lane < p.B) { c = p.seq_lens[lane]; q0 = p.qo_indptr[lane]; q1 = p.qo_indptr[lane + 1]; }
    // lanes past the batch: below all others
    const uint32_t key = (uint32_t)min(max(c, 0), (1 << 25) - 1) * 64u + (uint32_t)(63 - lane);
    int above = 0;
#pragma unroll
    for (int k = 0; k < 64; ++k) above += (uint32_t)__builtin_amdgcn_readlane((int)key, k) > key;
    const int i = __ffsll((long long)__ballot(above == rank)) - 1;
    const int r0 = __builtin_amdgcn_readlane(q0, i);
    return {i, r0, __builtin_amdgcn_readlane(q1, i) - r0, __builtin_amdgcn_readlane(c, i)};
}

// The launches of the work list's kernel and of the merge of split requests (verify_attn.hip).
int launch_attn_plan(const AttnParams& p, int B, int target_items, int step_keys, int min_chunk, int max_chunk, int max_items, int32_t* hdr, int32_t* req,
                     int32_t* items, hipStream_t s);
int launch_attn_merge(const AttnParams& p, int B, bool few, hipStream_t s);

}  // namespace specv
