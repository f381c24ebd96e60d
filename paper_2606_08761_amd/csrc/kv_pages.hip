// The pages of a paged cache: reserving, sharing, freeing and compacting them on
// the device, without the host knowing their numbers.
//
// The state is a table of page ids for every sequence slot, the slots' lengths
// and one reference count a page; a page is free where its count is zero, and
// free pages are handed out lowest first, so that every result is a function of
// the state alone.  The bookkeeping of reserve, fork and compact is one
// workgroup: it reads the counts 16384 at a time, ahead of what else it looks up,
// and ranks the pages it looks for by one scan (a cache of 288 GB has some ten
// thousand pages); a chain of a few latencies.  The data then moves in one launch over
// all planes, bound by HBM: 2 page_bytes a moved page and plane.
//
// Measured: the bookkeeping 8 to 10 us a call (32 forks of 63 pages, or 24 sequences
// of up to 128, in pools of some thousand pages), freeing 3 to 5 us, and moving the
// pages that such a batch leaves behind, 0.59 GB read and as much written in 8
// planes of 32 KB pages, 227 us: 5.2 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apex4_internal.h"

namespace apex4 {
namespace {

constexpr int kThreads = 1024;
constexpr int kWavesPerGroup = kThreads / 64;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Exclusive prefix sum over the workgroup's threads, and the total.
__device__ __forceinline__ int scan(int v, int* total) {
    __shared__ int wave_sum[kWavesPerGroup];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
        const int t = __shfl_up(s, i, 64);
        if (lane >= i) s += t;
    }
    __syncthreads();  // the sums of the call before are read
    if (lane == 63) wave_sum[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kWavesPerGroup; ++i) {
        before += i < wave ? wave_sum[i] : 0;
        all += wave_sum[i];
    }
    *total = all;
    return before + s - v;
}

// A chunk of kSpan pages: a thread has every 1024th, bit i of its word for page
// 1024 i + thread of the chunk, so that the loads lie side by side and do not wait
// for one another.
constexpr int kPer = 16, kSpan = kPer * kThreads;
// Numbers i that hold a page at all: a small pool's chunk has few.
__device__ __forceinline__ int numbers_of(int n_pages, int chunk) {
    const int64_t n = (n_pages - static_cast<int64_t>(chunk) * kSpan + kThreads - 1) / kThreads;
    return n < kPer ? static_cast<int>(n) : kPer;
}
__device__ __forceinline__ uint32_t live_bits(const int32_t* refs, int n_pages, int chunk) {
    const int64_t p0 = static_cast<int64_t>(chunk) * kSpan + threadIdx.x;
    const int numbers = numbers_of(n_pages, chunk);
    int32_t r[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        r[i] = 0;
        if (i < numbers && p0 + i * kThreads < n_pages) r[i] = refs[p0 + i * kThreads];
    }
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) bits |= r[i] > 0 ? 1u << i : 0u;
    return bits;
}
__device__ __forceinline__ uint32_t pages_here(int n_pages, int chunk) {  // which of the bits are pages at all
    const int64_t left = n_pages - static_cast<int64_t>(chunk) * kSpan - threadIdx.x;
    return left <= 0 ? 0u : left > kSpan - kThreads ? 0xFFFFu : (1u << ((left + kThreads - 1) / kThreads)) - 1u;
}
__device__ __forceinline__ int chunks_of(int n_pages) { return (n_pages + kSpan - 1) / kSpan; }

// Ranks the set bits of a chunk in page order: before[16 i + wave] is the number
// of those before a wave's pages of number i.  Returns how many there are.
__device__ __forceinline__ int rank_bits(uint32_t bits, int numbers, int32_t* before) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // what is there is read
    for (int i = 0; i < numbers; ++i) {
        const int n = __popcll(__ballot(bits >> i & 1u));
        if ((threadIdx.x & 63) == 0) before[i * kWavesPerGroup + wave] = n;
    }
    __syncthreads();
    const bool mine = static_cast<int>(threadIdx.x) < numbers * kWavesPerGroup;
    int all;
    const int at = scan(mine ? before[threadIdx.x] : 0, &all);
    if (mine) before[threadIdx.x] = at;
    __syncthreads();
    return all;
}
// The rank of the thread's page i among the set bits (or, of one that is not set,
// how many come before it).
__device__ __forceinline__ int rank_of(uint32_t bits, int i, const int32_t* before) {
    const uint64_t mask = __ballot(bits >> i & 1u);
    return before[i * kWavesPerGroup + (threadIdx.x >> 6)] + __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1ull));
}

// Writes the free pages to list[0 .. most), in ascending order; returns how many
// there are, or some number >= most once that many are found.  live0: live_bits of
// the first chunk, loaded before.
__device__ __forceinline__ int list_free(const int32_t* refs, int n_pages, uint32_t live0, int32_t* before, int32_t* list,
                                         int most) {
    int found = 0;
    for (int c = 0; c < chunks_of(n_pages) && found < most; ++c) {
        const uint32_t free = ~(c ? live_bits(refs, n_pages, c) : live0) & pages_here(n_pages, c);
        const int numbers = numbers_of(n_pages, c), all = rank_bits(free, numbers, before);
        for (int i = 0; i < numbers; ++i) {
            const int at = found + rank_of(free, i, before);
            if ((free >> i & 1u) && at < most) list[at] = c * kSpan + i * kThreads + threadIdx.x;
        }
        found += all;
    }
    return found;
}

__device__ __forceinline__ int pages_for(int64_t tokens, int shift) {
    return static_cast<int>((tokens + (int64_t{1} << shift) - 1) >> shift);
}

// Gives every listed sequence the pages for new_len tokens.  All or nothing:
// *status = pages missing, -1 where a length does not fit the table.
__global__ __launch_bounds__(kThreads) void reserve_kernel(int32_t* __restrict__ table, int slots, int width,
                                                           int32_t* __restrict__ kv_len, int32_t* __restrict__ refs,
                                                           int n_pages, const int32_t* __restrict__ seqs,
                                                           const int32_t* __restrict__ new_len, int n, int shift,
                                                           int32_t* __restrict__ status, int32_t* free_list,
                                                           int32_t* first) {
    __shared__ int too_long;
    __shared__ int32_t before_of[kPer * kWavesPerGroup];
    const uint32_t live0 = live_bits(refs, n_pages, 0);
    if (threadIdx.x == 0) too_long = 0;
    __syncthreads();
    int need_all = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        int need = 0;
        if (i < n) {
            const int s = seqs[i];
            if (static_cast<uint32_t>(s) < static_cast<uint32_t>(slots)) {
                const int have = pages_for(max(kv_len[s], 0), shift), want = pages_for(max(new_len[i], 0), shift);
                if (want > width) too_long = 1;
                need = max(want - have, 0);
                if (want > width) need = 0;
            }
        }
        int all;
        const int before = scan(need, &all);
        if (i < n) first[i] = need_all + before;
        if (need_all > n_pages - all) need_all = n_pages + 1;  // more than there are: the sum must not wrap
        else need_all += all;
    }
    __syncthreads();
    if (too_long) {
        if (threadIdx.x == 0) *status = -1;
        return;
    }
    const int found = need_all > n_pages ? 0 : list_free(refs, n_pages, live0, before_of, free_list, need_all);
    if (need_all > found) {
        if (threadIdx.x == 0) *status = need_all - found;
        return;
    }
    __syncthreads();  // the lists are written
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < n; i += kWavesPerGroup) {
        const int s = seqs[i];
        if (static_cast<uint32_t>(s) >= static_cast<uint32_t>(slots)) continue;
        const int len = max(kv_len[s], 0), want_len = max(new_len[i], 0);
        const int have = pages_for(len, shift), more = pages_for(want_len, shift) - have;
        for (int k = lane; k < more; k += 64) {
            const int p = free_list[first[i] + k];
            table[static_cast<int64_t>(s) * width + have + k] = p;
            refs[p] = 1;
        }
        if (lane == 0 && want_len > len) kv_len[s] = want_len;
    }
    if (threadIdx.x == 0) *status = 0;
}

// Children share their parents' full pages and get a page of their own for what
// is left; its data is copied by the launch after (src, dst; src = -1: none).
__global__ __launch_bounds__(kThreads) void fork_kernel(int32_t* __restrict__ table, int slots, int width,
                                                        int32_t* __restrict__ kv_len, int32_t* __restrict__ refs,
                                                        int n_pages, const int32_t* __restrict__ parents,
                                                        const int32_t* __restrict__ children, int n, int shift,
                                                        int32_t* __restrict__ status, int32_t* free_list,
                                                        int32_t* src, int32_t* dst) {
    auto valid = [&](int s) { return static_cast<uint32_t>(s) < static_cast<uint32_t>(slots); };
    // a page of its own: where the parent's length ends inside a page of its table
    auto parts = [&](int s) {
        const int len = max(kv_len[s], 0);
        return (len & ((1 << shift) - 1)) != 0 && (len >> shift) < width;
    };
    __shared__ int32_t before_of[kPer * kWavesPerGroup];
    const uint32_t live0 = live_bits(refs, n_pages, 0);
    int need = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        const int one = i < n && valid(parents[i]) && valid(children[i]) && parts(parents[i]);
        int all;
        const int before = scan(one, &all);
        if (i < n) dst[i] = one ? need + before : -1;
        need += all;
    }
    // (the list has room for as many as there are pages; all free ones are counted then)
    const int found = list_free(refs, n_pages, live0, before_of, free_list, min(need, n_pages));
    const bool enough = found >= need;
    if (threadIdx.x == 0) *status = enough ? 0 : need - found;
    __syncthreads();  // the lists are written, and no count changes before they are
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < n; i += kWavesPerGroup) {
        const int p = parents[i], ch = children[i];
        if (!enough || !valid(p) || !valid(ch)) {
            if (lane == 0) src[i] = -1;
            continue;
        }
        const int len = max(kv_len[p], 0), full = min(len >> shift, width);
        const int32_t* from = table + static_cast<int64_t>(p) * width;
        int32_t* to = table + static_cast<int64_t>(ch) * width;
        const int rank = dst[i];
        for (int k = lane; k < width; k += 64) {
            int id = -1;
            if (k < full) {
                id = from[k];
                if (static_cast<uint32_t>(id) < static_cast<uint32_t>(n_pages)) atomicAdd(&refs[id], 1);
            } else if (k == full && rank >= 0) {
                id = free_list[rank];
                refs[id] = 1;  // free: no other child adds to it
                const int last = from[k];
                src[i] = static_cast<uint32_t>(last) < static_cast<uint32_t>(n_pages) ? last : -1;
                dst[i] = id;
            }
            to[k] = id;
        }
        if (lane == 0) {
            kv_len[ch] = len;
            if (rank < 0) src[i] = -1;
        }
    }
}

__global__ __launch_bounds__(256) void free_kernel(int32_t* __restrict__ table, int slots, int width,
                                                   int32_t* __restrict__ kv_len, int32_t* __restrict__ refs, int n_pages,
                                                   const int32_t* __restrict__ seqs, int n) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= n) return;
    const int s = seqs[i];
    if (static_cast<uint32_t>(s) >= static_cast<uint32_t>(slots)) return;
    int32_t* row = table + static_cast<int64_t>(s) * width;
    for (int k = lane; k < width; k += 64) {
        const int id = row[k];
        if (static_cast<uint32_t>(id) < static_cast<uint32_t>(n_pages)) {
            if (atomicSub(&refs[id], 1) <= 0) atomicAdd(&refs[id], 1);  // was free: stays so
        }
        row[k] = -1;
    }
    if (lane == 0) kv_len[s] = 0;
}

// Live pages past the number of live pages move to the free ones below it:
// src[i] -> dst[i] (both ascending) for i < *count; to[p] is page p's new id.
// held[i]: the references of src[i].
__global__ __launch_bounds__(kThreads) void compact_plan_kernel(int32_t* __restrict__ refs, int n_pages,
                                                                int32_t* __restrict__ status, int32_t* to, int32_t* src,
                                                                int32_t* dst, int32_t* held, int32_t* __restrict__ count) {
    __shared__ int below_of;
    __shared__ int32_t before_of[kPer * kWavesPerGroup];
    const uint32_t live0 = live_bits(refs, n_pages, 0);
    const int chunks = chunks_of(n_pages);
    int live = 0;
    for (int c = 0; c < chunks; ++c) live += rank_bits(c ? live_bits(refs, n_pages, c) : live0, numbers_of(n_pages, c), before_of);
    // live pages below page `live`: the others, and as many free pages, change places
    if (threadIdx.x == 0) below_of = live;
    __syncthreads();
    int found = 0;
    for (int c = 0; c < chunks; ++c) {
        const uint32_t bits = c ? live_bits(refs, n_pages, c) : live0;
        const int all = chunks == 1 ? 0 : rank_bits(bits, numbers_of(n_pages, c), before_of);
        if (live / kSpan == c && live < n_pages) {
            const int at = found + rank_of(bits, live % kSpan / kThreads, before_of);
            if (live % kThreads == static_cast<int>(threadIdx.x)) below_of = at;
        }
        found += all;
    }
    __syncthreads();
    const int below = below_of, moves = live - below;
    found = 0;
    for (int c = 0; c < chunks; ++c) {
        const uint32_t bits = c ? live_bits(refs, n_pages, c) : live0;
        const int all = chunks == 1 ? 0 : rank_bits(bits, numbers_of(n_pages, c), before_of);
        for (int i = 0; i < numbers_of(n_pages, c); ++i) {
            const int at = found + rank_of(bits, i, before_of);  // live pages before page p
            const int64_t p = static_cast<int64_t>(c) * kSpan + i * kThreads + threadIdx.x;
            const bool is_live = bits >> i & 1u;
            if (p < n_pages) {
                if (is_live && p >= live) {
                    src[at - below] = static_cast<int>(p);
                    held[at - below] = refs[p];
                } else {
                    to[p] = static_cast<int>(p);
                    if (!is_live && p < live) dst[p - at] = static_cast<int>(p);
                }
            }
        }
        found += all;
    }
    __syncthreads();  // the lists are written, and the counts read
    for (int i = threadIdx.x; i < moves; i += kThreads) {
        const int s = src[i], d = dst[i];
        to[s] = d;
        refs[d] = held[i];
        refs[s] = 0;
    }
    if (threadIdx.x == 0) {
        *count = moves;
        *status = live;
    }
}

// Copies page src[i] to dst[i] in every plane, i < n (*count where that is
// given); pairs outside the pool are left out, and no destination is another
// pair's source.  A workgroup moves 16 KB pieces.  table: every entry p becomes
// to[p].
constexpr int kPiece = 16 << 10;
__global__ __launch_bounds__(256) void copy_pages_kernel(uint8_t* __restrict__ pool, int planes, int64_t page_bytes,
                                                         int n_pages, const int32_t* __restrict__ src,
                                                         const int32_t* __restrict__ dst, int n,
                                                         const int32_t* __restrict__ count, int32_t* __restrict__ table,
                                                         int64_t entries, const int32_t* __restrict__ to) {
    if (table) {
        const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < entries; i += stride) {
            const int id = table[i];
            if (static_cast<uint32_t>(id) < static_cast<uint32_t>(n_pages)) table[i] = to[id];
        }
    }
    if (count) n = *count;
    const int pieces = static_cast<int>((page_bytes + kPiece - 1) / kPiece);
    const int64_t items = static_cast<int64_t>(n) * planes * pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int piece = static_cast<int>(item % pieces);
        const int64_t r = item / pieces;
        const int i = static_cast<int>(r / planes), plane = static_cast<int>(r % planes);
        const int s = src[i], d = dst[i];
        if (static_cast<uint32_t>(s) >= static_cast<uint32_t>(n_pages) || static_cast<uint32_t>(d) >= static_cast<uint32_t>(n_pages))
            continue;
        const int64_t at = static_cast<int64_t>(piece) * kPiece;
        const uint8_t* a = pool + (static_cast<int64_t>(plane) * n_pages + s) * page_bytes + at;
        uint8_t* b = pool + (static_cast<int64_t>(plane) * n_pages + d) * page_bytes + at;
        const int bytes = static_cast<int>(page_bytes - at < kPiece ? page_bytes - at : kPiece);  // a multiple of 16
        u32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int o = (j * 256 + threadIdx.x) * 16;
            if (o < bytes) v[j] = *reinterpret_cast<const u32x4*>(a + o);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int o = (j * 256 + threadIdx.x) * 16;
            if (o < bytes) *reinterpret_cast<u32x4*>(b + o) = v[j];
        }
    }
}

// One workgroup a piece, up to some rounds of the compute units.
unsigned copy_blocks(int64_t items) {
    const int64_t most = static_cast<int64_t>(device_cu_count()) * 32;
    return static_cast<unsigned>(items < 1 ? 1 : items < most ? items : most);
}

}  // namespace

hipError_t launch_pages_reserve(const PageTable& p, const int32_t* seqs, const int32_t* new_len, int n, int32_t* status,
                                int32_t* work, hipStream_t stream) {
    reserve_kernel<<<1, kThreads, 0, stream>>>(p.table, p.slots, p.width, p.kv_len, p.refs, p.n_pages, seqs, new_len, n,
                                               p.page_shift, status, work, work + p.n_pages);
    return hipGetLastError();
}

hipError_t launch_pages_copy(uint8_t* pool, int planes, int64_t page_bytes, int n_pages, const int32_t* src,
                             const int32_t* dst, int n, hipStream_t stream) {
    const int64_t pieces = (page_bytes + kPiece - 1) / kPiece;
    copy_pages_kernel<<<copy_blocks(pieces * planes * n), 256, 0, stream>>>(pool, planes, page_bytes, n_pages, src, dst, n,
                                                                            nullptr, nullptr, 0, nullptr);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PageTable& p, uint8_t* pool, int planes, int64_t page_bytes, const int32_t* parents,
                             const int32_t* children, int n, int32_t* status, int32_t* work, hipStream_t stream) {
    int32_t* src = work + p.n_pages;
    int32_t* dst = src + n;
    fork_kernel<<<1, kThreads, 0, stream>>>(p.table, p.slots, p.width, p.kv_len, p.refs, p.n_pages, parents, children, n,
                                            p.page_shift, status, work, src, dst);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_pages_copy(pool, planes, page_bytes, p.n_pages, src, dst, n, stream);
}

hipError_t launch_pages_free(const PageTable& p, const int32_t* seqs, int n, hipStream_t stream) {
    free_kernel<<<(n + 3) / 4, 256, 0, stream>>>(p.table, p.slots, p.width, p.kv_len, p.refs, p.n_pages, seqs, n);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const PageTable& p, uint8_t* pool, int planes, int64_t page_bytes, int32_t* status,
                                int32_t* work, hipStream_t stream) {
    // a page moves to another: no more than half of them
    int32_t *to = work, *src = to + p.n_pages, *held = src + (p.n_pages + 1) / 2, *dst = src + p.n_pages + 1, *count = dst + p.n_pages;
    compact_plan_kernel<<<1, kThreads, 0, stream>>>(p.refs, p.n_pages, status, to, src, dst, held, count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t pieces = (page_bytes + kPiece - 1) / kPiece;
    copy_pages_kernel<<<copy_blocks(pieces * planes * (p.n_pages / 2)), 256, 0, stream>>>(
        pool, planes, page_bytes, p.n_pages, src, dst, 0, count, p.table, static_cast<int64_t>(p.slots) * p.width, to);
    return hipGetLastError();
}

}  // namespace apex4
