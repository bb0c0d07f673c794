// spec_kv_reserve: pages for the rows that are about to be written, and the slot of every row (the counterpart of spec_kv_commit, which returns the pages of
// rejected rows; paper, Appendix "Target side": the candidates' K/V enter the cache before they are verified).
//
//   hi_i = ceil((c_i + n_i) / P), first_i = the first unmapped logical page from c_i / P on, need_i = hi_i - first_i;
//   with the needs' running sums e_i (before request i) and the total T of those served, logical page g of request i becomes free_list[F - T + e_i + g - first_i],
//   F = *free_count, and row j of request i is slot page(c_i + j) * P + (c_i + j) mod P.
// The running sums order the requests; everything else is independent.  One workgroup does it all for the rounds of a decode batch (a launch and a few dependent reads:
// latency); with more rows the same workgroup leaves two words per request and a grid over the rows follows.
#include "common.h"

namespace specv {

constexpr int kReserveThreads = 1024;
constexpr int kReserveDeep = 16;             // entries of a long range that a lane has in flight
constexpr int kReserveShort = 4;             // so many table entries are looked at by the request's own thread, longer ranges by a wave

struct ReserveParams {
    int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* qo_indptr;
    const int32_t* free_list;
    int32_t* free_count;
    int32_t* slot_map;
    int32_t* status_flags;
    int32_t* hdr;            // {first place of the pages taken in the free list}
    u32x2* req;              // [B] {first logical page to map, its place among the pages taken}; a request without slots has first = INT32_MAX
    int max_pages, num_pages, free_capacity, B, M, P;
};

constexpr int kUnserved = 0x7FFFFFFF;

// What a request asks for; ok: its lengths fit the table and the row range.
struct ReserveRange { int lo, hi, c, r0, n; bool ok, descends; };

__device__ inline ReserveRange reserve_range(const ReserveParams& p, int i)
{
    ReserveRange q;
    q.r0 = p.qo_indptr[i];
    const long end = p.qo_indptr[i + 1], n = end - q.r0;
    q.c = p.seq_lens[i];
    q.n = (int)n;
    q.descends = n < 0;
    const long len = q.c + n, hi = (len + p.P - 1) / p.P;
    q.ok = n >= 0 && q.c >= 0 && q.r0 >= 0 && end <= p.M && len <= 0x7FFFFFFFL && (n == 0 || hi <= p.max_pages);
    q.lo = q.ok ? q.c / p.P : 0;
    q.hi = q.ok && n > 0 ? (int)hi : q.lo;                // (no rows: nothing is looked at)
    return q;
}

// Slot of row `row` of request i, whose rows r0 .. end - 1 are positions c on; enters the id of a page that the row is the first of.
__device__ inline void reserve_row(const ReserveParams& p, int row, int i, int r0, int end, int c, int start, int first, int place)
{
    int slot = -1;
    if (i >= 0 && first != kUnserved && row >= r0 && row < end) {
        const int pos = c + (row - r0), g = pos / p.P, at = pos - g * p.P;
        int32_t* entry = p.page_table + (size_t)i * p.max_pages + g;
        int page;
        if (g < first) {
            page = *entry;                                // (mapped before the call, and looked at when the requests were counted)
        } else {
            page = p.free_list[start + place + (g - first)];
            if (page < 0 || page >= p.num_pages) {
                page = -1;
                if (p.status_flags) atomicOr(p.status_flags, SPEC_FLAG_BAD_PAGE);
            } else if (at == 0) {                         // a page that is mapped here begins with a row of this call
                *entry = page;
            }
        }
        if (page >= 0) slot = page * p.P + at;
    }
    p.slot_map[row] = slot;
}

// The request of a row: the last one that starts at or before it.
__device__ inline int reserve_request_of(const int32_t* qo, int B, int row)
{
    int lo = -1, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (qo[mid] <= row) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// ROWS: at most 1024 requests (one block), whose rows this workgroup does as well.
template <bool ROWS>
__global__ __launch_bounds__(kReserveThreads) void kv_reserve_kernel(ReserveParams p)
{
    __shared__ long wave_total[kReserveThreads / 64];
    __shared__ long block_total;
    __shared__ int s_first[kReserveThreads], s_place[kReserveThreads], s_long[kReserveThreads];
    __shared__ int32_t s_qo[kReserveThreads], s_end[kReserveThreads], s_c[kReserveThreads];
    __shared__ int s_longs, s_taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int count = *p.free_count;
    const int have = count < 0 ? 0 : (count < p.free_capacity ? count : p.free_capacity);
    if (tid == 0) s_taken = 0;
    long base = 0;
    int flags = 0;
    // Offsets that descend can give a row to two requests, of which the search finds one: the other's pages would be taken and not entered.  So nobody is served then.  (Up to
    // 1024 requests are looked at below, in their only block.)
    int descends = 0;
    if constexpr (!ROWS) {
        for (int i = tid; i < p.B; i += kReserveThreads) descends |= p.qo_indptr[i + 1] < p.qo_indptr[i];
        descends = __syncthreads_or(descends);
    }
    for (int block = 0; block < p.B; block += kReserveThreads) {
        if (tid == 0) s_longs = 0;
        __syncthreads();                                  // (also: the arrays of the block before have been read)
        const int i = block + tid;
        ReserveRange q{0, 0, 0, 0, 0, false, false};
        bool ok = false;
        int first = 0;
        if (i < p.B) {
            q = reserve_range(p, i);
            ok = q.ok;
            if (!ok) flags |= SPEC_FLAG_BAD_LENGTH;
            first = q.hi;
            const int32_t* e = p.page_table + (size_t)i * p.max_pages;
            if (q.hi - q.lo > kReserveShort) {
                s_long[atomicAdd(&s_longs, 1)] = i;       // (any order: each is looked at by itself)
            } else {
                for (int g = q.lo; g < q.hi; ++g) {
                    const int page = e[g];
                    if (page < 0) first = min(first, g);
                    else if (page >= p.num_pages || first < g) ok = false;
                }
            }
            s_first[tid] = first;
            s_qo[tid] = q.r0;
            s_end[tid] = q.r0 + q.n;
            s_c[tid] = q.c;
        }
        if constexpr (ROWS) descends = __syncthreads_or(q.descends);
        else __syncthreads();
        for (int k = wave; k < s_longs; k += kReserveThreads / 64) {
            const int j = __builtin_amdgcn_readfirstlane(s_long[k]);
            struct { int lo, hi; } w{s_c[j - block] / p.P, 0};
            w.hi = (int)(((long)s_c[j - block] + (s_end[j - block] - s_qo[j - block]) + p.P - 1) / p.P);
            const int32_t* e = p.page_table + (size_t)j * p.max_pages;
            int f = w.hi, last = -1;                      // first unmapped, last mapped
            bool bad = false;
            for (int g0 = w.lo; g0 < w.hi; g0 += 64 * kReserveDeep) {
                int page[kReserveDeep];
#pragma unroll
                for (int u = 0; u < kReserveDeep; ++u) page[u] = e[min(g0 + u * 64 + lane, w.hi - 1)];
#pragma unroll
                for (int u = 0; u < kReserveDeep; ++u) {
                    const int g = min(g0 + u * 64 + lane, w.hi - 1);
                    if (page[u] < 0) f = min(f, g);
                    else { last = max(last, g); bad |= page[u] >= p.num_pages; }
                }
            }
            for (int d = 32; d >= 1; d >>= 1) { f = min(f, __shfl_xor(f, d, 64)); last = max(last, __shfl_xor(last, d, 64)); }
            if (__any(bad) || last > f) f = -1;
            if (lane == 0) s_first[j - block] = f;
        }
        __syncthreads();
        if (i < p.B) {
            first = s_first[tid];
            if (first < 0) ok = false;
            if (ok && q.n > 0 && q.c % p.P != 0 && first == q.lo) ok = false;     // the page of its last tokens is not there
            if (!ok && q.ok) flags |= SPEC_FLAG_BAD_PAGE;
            if (descends) { ok = false; flags |= SPEC_FLAG_BAD_LENGTH; }
        }
        const long need = i < p.B && ok ? q.hi - first : 0;
        long incl = need;
        for (int d = 1; d < 64; d <<= 1) {
            const long up = __shfl_up(incl, d, 64);
            if (lane >= d) incl += up;
        }
        if (lane == 63) wave_total[wave] = incl;
        __syncthreads();
        if (wave == 0) {
            const long t = lane < kReserveThreads / 64 ? wave_total[lane] : 0;
            long ti = t;
            for (int d = 1; d < 16; d <<= 1) {
                const long up = __shfl_up(ti, d, 64);
                if (lane >= d) ti += up;
            }
            if (lane < kReserveThreads / 64) wave_total[lane] = ti - t;
            if (lane == kReserveThreads / 64 - 1) block_total = ti;
        }
        __syncthreads();
        incl += base + wave_total[wave];
        if (i < p.B) {
            // in the requests' order, as far as the free list goes; who needs no page is always served
            if (ok && need > 0) {
                if (incl <= have) atomicMax(&s_taken, (int)incl);
                else { ok = false; flags |= SPEC_FLAG_NO_PAGES; }
            }
            const int place = ok ? (int)(incl - need) : 0;
            first = ok ? first : kUnserved;
            if (ROWS) { s_first[tid] = first; s_place[tid] = need > 0 ? place : 0; }
            else p.req[i] = u32x2{(uint32_t)first, (uint32_t)(need > 0 ? place : 0)};
        }
        base += block_total;
        __syncthreads();
    }
    const int taken = s_taken, start = have - taken;
    if (tid == 0) {
        if (taken > 0) *p.free_count = start;
        if (!ROWS) p.hdr[0] = start;
    }
    if (flags && p.status_flags) atomicOr(p.status_flags, flags);
    if (ROWS)
        for (int row = tid; row < p.M; row += kReserveThreads) {
            const int i = reserve_request_of(s_qo, p.B, row);
            if (i >= 0) reserve_row(p, row, i, s_qo[i], s_end[i], s_c[i], start, s_first[i], s_place[i]);
            else p.slot_map[row] = -1;
        }
}

__global__ __launch_bounds__(256) void kv_reserve_rows_kernel(ReserveParams p)
{
    const int row = blockIdx.x * 256 + threadIdx.x;
    if (row >= p.M) return;
    const int i = reserve_request_of(p.qo_indptr, p.B, row);
    if (i < 0) { p.slot_map[row] = -1; return; }
    const u32x2 q = p.req[i];
    reserve_row(p, row, i, p.qo_indptr[i], p.qo_indptr[i + 1], p.seq_lens[i], p.hdr[0], (int)q.x, (int)q.y);
}

}  // namespace specv

extern "C" size_t spec_kv_reserve_workspace_bytes(int B)
{
    return B <= 0 ? 0 : 256 + specv::round_up((size_t)B * 8, 256);
}

extern "C" int spec_kv_reserve(int32_t* page_table, int max_pages_per_seq, int num_pages, const int32_t* seq_lens, const int32_t* qo_indptr,
                               const int32_t* free_list, int32_t free_capacity, int32_t* free_count, int32_t* slot_map,
                               int B, int M, int page_size, int32_t* status_flags, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace specv;
    if (B < 0 || M < 0 || page_size <= 0 || max_pages_per_seq < 0 || num_pages < 0 || free_capacity < 0)
        return fail(SPEC_EINVAL, "spec_kv_reserve: negative size (B=%d M=%d page_size=%d max_pages=%d num_pages=%d cap=%d)", B, M, page_size,
                    max_pages_per_seq, num_pages, free_capacity);
    if (B == 0 && M == 0) return SPEC_OK;
    // (without requests there are only rows to mark)
    if ((B > 0 && (!page_table || !seq_lens || !qo_indptr || !free_list)) || !free_count || (M > 0 && !slot_map))
        return fail(SPEC_EINVAL, "spec_kv_reserve: NULL pointer argument");
    if ((long)num_pages * page_size > 2147483647L)
        return fail(SPEC_ESHAPE, "spec_kv_reserve: slots of %d pages x %d tokens do not fit 32 bits", num_pages, page_size);
    const size_t need = spec_kv_reserve_workspace_bytes(B);
    if (need > 0 && (!workspace || !aligned(workspace, 256))) return fail(SPEC_EINVAL, "spec_kv_reserve: workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need) return fail(SPEC_EWORKSPACE, "spec_kv_reserve: workspace %zu bytes, need %zu", workspace_bytes, need);
    ReserveParams p{page_table, seq_lens, qo_indptr, free_list, free_count, slot_map, status_flags, (int32_t*)workspace,
                    (u32x2*)((char*)workspace + 256), max_pages_per_seq, num_pages, free_capacity, B, M, page_size};
    const bool one = B == 0 || (B <= kReserveThreads && M <= 8192);
    if (one) {
        hipLaunchKernelGGL(kv_reserve_kernel<true>, dim3(1), dim3(kReserveThreads), 0, (hipStream_t)stream, p);
        return check_launch("spec_kv_reserve");
    }
    hipLaunchKernelGGL(kv_reserve_kernel<false>, dim3(1), dim3(kReserveThreads), 0, (hipStream_t)stream, p);
    if (int rc = check_launch("spec_kv_reserve")) return rc;
    if (M == 0) return SPEC_OK;
    hipLaunchKernelGGL(kv_reserve_rows_kernel, dim3((M + 255) / 256), dim3(256), 0, (hipStream_t)stream, p);
    return check_launch("spec_kv_reserve (rows)");
}
