// Layout of a paged key-value cache and what the kernels that read or write it
// share.
//
// A plane (the keys, or the values, of one layer) is n_pages pages of
// page_bytes bytes.  A binary16 page is [kv heads][page][D] binary16; an int4
// page is codes [kv heads][page][D/2] (two signed codes a byte, low nibble =
// even d) followed by binary16 scales [kv heads][page], one for a token's D
// values of a head (SymQuant with G = D).  Token t of sequence b is in page
// table[b * width + t / page], at t % page.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apex4_internal.h"

namespace apex4 {

inline int64_t kv_page_bytes(bool i4, int64_t kv_heads, int64_t D, int64_t page) {
    return kv_heads * page * (i4 ? D / 2 + 2 : 2 * D);
}

namespace {   // internal linkage in every translation unit that includes it

// The page that holds token t (t >= 0), or -1 where the table has none that
// lies in the plane.
__device__ __forceinline__ int page_of(const KvView& c, int b, int64_t t) {
    const int64_t i = t >> c.page_shift;
    if (i >= c.width) return -1;
    const int id = c.table[static_cast<int64_t>(b) * c.width + i];
    return static_cast<uint32_t>(id) < static_cast<uint32_t>(c.n_pages) ? id : -1;
}

// Sequence b's cached tokens, the new ones included, as far as the table and
// the caller's bound reach.
__device__ __forceinline__ int cached_tokens(const KvView& c, int b) {
    const int64_t most = static_cast<int64_t>(c.width) << c.page_shift;
    int64_t n = c.kv_len[b];
    n = n < 0 ? 0 : n;
    n = n < most ? n : most;
    return static_cast<int>(n < c.max_len ? n : c.max_len);
}

// The sequence that token i of the packed new tokens belongs to: the last b
// with q_start[b] <= i (q_start ascending, q_start[0] = 0).  nullptr: one token
// a sequence.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int B, int i) {
    if (!q_start) return i;
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (q_start[mid] <= i) lo = mid; else hi = mid - 1;
    }
    return lo;
}

}  // namespace
}  // namespace apex4
