// Which requests of a batch the attention kernels compute.  Plain arithmetic without device types: the kernels and a CPU test share it.  Offsets and lengths come from device
// memory and may hold anything: no sum or difference here leaves 32 bits.
#pragma once

namespace specv {

// Query rows of a request whose offsets are r0 and end; 0 where the offsets are not ascending or negative.
constexpr int attn_request_rows(int r0, int end) { return r0 >= 0 && end > r0 ? end - r0 : 0; }

// n rows from r0 on (n from attn_request_rows) behind c committed tokens lie within the call's bounds (all of them positive).
constexpr bool attn_request_fits(int r0, int n, int c, int M, int max_q_len, int max_kv_len)
{
    return n >= 1 && n <= max_q_len && r0 <= M - n && c >= 0 && c <= max_kv_len - n;
}

}  // namespace specv
