// The pages of a paged cache: reserving, sharing, freeing and compacting them on
// the device, without the host knowing their numbers.
//
// The state is a table of page ids for every sequence slot, the slots' lengths
// and one reference count a page; a page is free where its count is zero, and
// free pages are handed out lowest first, so that every result is a function of
// the state alone.  The bookkeeping of reserve, fork and compact is one
// workgroup: it reads the counts 4096 at a time and ranks the pages it looks for
// by a scan (a cache of 288 GB has some ten thousand pages, a few steps; a pass
// costs about 2 us, and the launch).  The data then moves in one launch over
// all planes, bound by HBM: 2 page_bytes a moved page and plane.
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

// Writes the pages p in [from, to) with pick(refs[p]) to list[0 .. most), in
// ascending order; returns how many there are, or some number >= most once that
// many are found.
template <class Pick>
__device__ __forceinline__ int list_pages(const int32_t* refs, int from, int to, Pick pick, int32_t* list, int most) {
    int found = 0;
    for (int p0 = from; p0 < to && found < most; p0 += 4 * kThreads) {
        const int p = p0 + 4 * threadIdx.x;
        int n = 0, take[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            take[i] = p + i < to && pick(refs[p + i]);
            n += take[i];
        }
        int all;
        int at = found + scan(n, &all);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (take[i]) {
                if (at < most) list[at] = p + i;
                ++at;
            }
        found += all;
    }
    return found;
}

struct IsFree {
    __device__ bool operator()(int32_t r) const { return r <= 0; }
};
struct IsLive {
    __device__ bool operator()(int32_t r) const { return r > 0; }
};

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
    const int found = need_all > n_pages ? 0 : list_pages(refs, 0, n_pages, IsFree(), free_list, need_all);
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
    int need = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        const int one = i < n && valid(parents[i]) && valid(children[i]) && parts(parents[i]);
        int all;
        const int before = scan(one, &all);
        if (i < n) dst[i] = one ? need + before : -1;
        need += all;
    }
    const int found = need > n_pages ? 0 : list_pages(refs, 0, n_pages, IsFree(), free_list, need);
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
__global__ __launch_bounds__(kThreads) void compact_plan_kernel(int32_t* __restrict__ refs, int n_pages,
                                                                int32_t* __restrict__ status, int32_t* to, int32_t* src,
                                                                int32_t* dst, int32_t* __restrict__ count) {
    int live = 0;
    for (int p0 = 0; p0 < n_pages; p0 += 4 * kThreads) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = p0 + 4 * threadIdx.x + i;
            if (p < n_pages) {
                n += refs[p] > 0;
                to[p] = p;
            }
        }
        int all;
        scan(n, &all);
        live += all;
    }
    const int holes = list_pages(refs, 0, live, IsFree(), dst, n_pages);
    list_pages(refs, live, n_pages, IsLive(), src, n_pages);
    __syncthreads();  // the lists are written
    for (int i = threadIdx.x; i < holes; i += kThreads) {
        to[src[i]] = dst[i];
        refs[dst[i]] = refs[src[i]];
        refs[src[i]] = 0;
    }
    if (threadIdx.x == 0) {
        *count = holes;
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
    int32_t *to = work, *src = to + p.n_pages, *dst = src + p.n_pages, *count = dst + p.n_pages;
    compact_plan_kernel<<<1, kThreads, 0, stream>>>(p.refs, p.n_pages, status, to, src, dst, count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t pieces = (page_bytes + kPiece - 1) / kPiece;
    copy_pages_kernel<<<copy_blocks(pieces * planes * (p.n_pages / 2)), 256, 0, stream>>>(
        pool, planes, page_bytes, p.n_pages, src, dst, 0, count, p.table, static_cast<int64_t>(p.slots) * p.width, to);
    return hipGetLastError();
}

}  // namespace apex4
