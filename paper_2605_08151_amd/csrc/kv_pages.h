// Tokens and pages of a paged cache.  Plain arithmetic without device types: the kernels and a CPU test share it.
#pragma once

namespace specv {

// Pages of P tokens each that hold `tokens` >= 0; tokens + P - 1 need not fit 32 bits.
constexpr int pages_of(int tokens, int P)
{
    const int whole = tokens / P;
    return whole + (whole * P != tokens);
}

// n rows behind c tokens: a length that 32 bits hold.  (Offsets and lengths come from device memory and may hold anything.)
constexpr bool kv_length_fits(int n, int c) { return n >= 1 && c >= 0 && c <= 0x7FFFFFFF - n; }

// Rows between two offsets, 0 where they do not ascend; the difference of any two 32-bit numbers is one of at most 2^32 - 1, of which those beyond 2^31 - 1 are no rows either.
constexpr int kv_rows(int from, int to)
{
    const long n = (long)to - from;
    return n >= 1 && n <= 0x7FFFFFFF ? (int)n : 0;
}

}  // namespace specv
