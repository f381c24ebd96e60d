// Sampling: a token for every row of logits from one given random number.
//
// In the order of falling logits (equal ones by index, lowest first) w = 2^((x - max) c),
// c = log2(e) / temperature; top-k keeps the first k; top-p of those the shortest
// beginning that holds p of their sum; min-p those with w >= min_p.  All three keep a
// beginning of that order, so one border does: a logit, and an index among those equal to
// it.  The token is the first, by index, whose running sum of kept weights passes u times
// their sum.
//
// Weights are computed in binary64 and held as whole numbers of 2^-45 of the largest
// one: their sums are exact in any order, so that no result depends on which thread was
// first.  A weight is rounded by half such a unit, so running sums, and with them a border and the
// token's share, are off by n 2^-46 of the largest weight at most for n logits.  (In binary32 one row in some
// hundred of a flat distribution over 10^5 tokens would get another token.)  A logit 46
// octaves below the largest weighs nothing.
//
// A workgroup takes a row; rows of up to 126 KB stay in LDS, longer ones are read again,
// through a ring in LDS that keeps four loads a wave in flight and no registers.  Passes
// over the row:
//   1  the largest logit;
//   2  only for top-k or top-p: counts and sums by buckets of 1/16 octave below it, the sums
//      by quarters of the row (of a small top-k's top-p later, over the list); a scan
//      gives the bucket of the border;
//   3  the logits down to that bucket into a list, if it holds them; then all that follows
//      goes over the list.  If not, the bucket's own go there, and the weights before it
//      are known by quarters, or are summed by the waves' parts of the row.  The range of
//      the bucket's logits is split into 1024 until one value is left, and for equal ones
//      their indexes, 256 and then 1 at a time (where the list does not even hold the bucket,
//      over the row);
//   4  the token: by indexes in the list, or by the quarter that holds it and that one's
//      sixteenths, or by the waves' parts, then the logits of the part.
//
// Bound by the arithmetic of a row's one compute unit and by the steps that follow each
// other.  48 rows of 32000 binary16 logits with top-p take 31 to 34 us, of which the load
// and pass 1 are 2.7, pass 2 8.5 (3.3 without weights), pass 3 6.3, each search through
// the bins 1.2, the token 2.4 from the list or 5 from the row; with top-k 50 19 us, with
// both 25, with neither 14.  256 rows of 131072 binary32 logits with top-p: 112 us; pass 1 comes from
// memory in 20 us, the others as fast from the cache behind it, and weights add 20 to pass 2.
// Tried: weights one after the other, each in its own branch (+4 to 8 %), pass 3 that weighs
// all that is before the bucket (+18 us there), sixteen waves for a scan of the bins (+0.6
// us), places in the list by a scan of the wave instead of ballots (+2 %).
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "apex4_internal.h"

namespace apex4 {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBuckets = 736;          // 1/16 octave each
constexpr int kStageBytes = 126 << 10; // of a row in LDS
constexpr int kSharedLogits = 48 << 10;  // rows from here on are shared where they are few
constexpr int kLdsBytes = 160 << 10, kMostList = 8704;
constexpr uint32_t kShortList = 4096;  // logits
// top-p of up to so many that top-k keeps weighs them alone (256 rows of 131072 binary32 logits,
// top-k 50, top-p 0.9: 78 us, all of them weighed 97; 48 of 32000: 25 and 29).
constexpr int kFewKept = 1024;
constexpr int kDepth = 4, kRingBytes = kWaves * kDepth * 1024;
constexpr int kSteps = 512, kStepBits = 9;  // table of 2^(i / 512)
constexpr double kMagic = 0x1.8p52;    // added to a number below 2^51: its nearest whole one in the low bits
constexpr float kNothing = -__builtin_inff();

struct Shared {
    alignas(16) u64 bucket_w[kBuckets];
    alignas(16) u64 bin_w[1024];
    uint32_t bin_n[1024];
    double table[kSteps];
    alignas(16) uint32_t bucket_n[kBuckets];
    u64 wave_w[kWaves];
    u64 part_w[kWaves];   // of the waves' parts of the row, or at 4 q of its quarter q
    uint32_t wave_n[kWaves];
    float wave_max[kWaves];
    // the border's bin: what lies before it and in it
    u64 before_w, in_w, goal, total;
    uint32_t before_n, in_n;
    int bin;
    uint32_t listed, low, high, first;
};

// In pass 2 of a row that is one workgroup's the buckets' sums are held by quarters of the
// row: the first in bucket_w, two where the bins are later, the last in the list's place.
constexpr int kQuarters = 4, kQuarterWaves = kWaves / kQuarters;
static_assert(offsetof(Shared, bin_n) == offsetof(Shared, bin_w) + 1024 * 8 && 2 * kBuckets * 8 <= 1024 * 12, "two of them where the bins are");
__device__ __forceinline__ u64* quarter(Shared& sm, u64* list, int q) {
    return q == 0 ? sm.bucket_w : q == kQuarters - 1 ? list : sm.bin_w + (q - 1) * kBuckets;
}

// What the workgroups that share a row leave for the next launch.
struct Work {
    u64 part_w[kWaves];
    u64 bucket_w[kBuckets];
    u64 list[kMostList];
    uint32_t bucket_n[kBuckets];
    float max[kWaves];
    uint32_t listed, first;
    uint32_t unused[2];
};
static_assert(sizeof(Work) % 16 == 0, "aligned");

__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// The next number below that of k; below 0 it is not -0, which is not less.
__device__ __forceinline__ float under(uint32_t k) { return unordered(k == 0x80000000u ? k - 2u : k - 1u); }

typedef __attribute__((address_space(3))) uint8_t lds_u8;
__device__ __forceinline__ u32x4 read_lds(uint32_t at) {
    return *(const __attribute__((address_space(3))) u32x4*)static_cast<uintptr_t>(at);
}
// 16 bytes a lane from base + off straight into LDS at `to` + 16 lane.  The compiler does
// not see these loads: landed_but() waits for all but the last N of the wave's (and for its
// reads of LDS).  The wait states let M0, and a base that came out of a vector
// instruction, settle.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(uint32_t to, uint32_t off, const uint8_t* base) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(off),
                 "s"(static_cast<uint64_t>(hi) << 32 | lo)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void landed_but() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

// What the passes need to know of a row.
template <bool F16, bool STAGED>
struct Row {
    static constexpr int kVec = F16 ? 8 : 4;  // logits of 16 bytes, a piece
    const uint8_t* base;   // 16-byte aligned, at or before the first logit
    u32x4* staged;
    uint32_t ring;         // the ring's place in LDS
    const double* table;
    int skip, V, pieces;   // logits between base and the first; pieces that hold the row
    int from, to;          // the pieces that the passes go over
    bool infinite;         // the largest logit is infinite: its like count as 0, the others as nothing
    float scale, scaled, c32;  // below() is the scaled difference times c32
    double max, c64;       // 512 c

    static constexpr uint32_t kNone = F16 ? 0xFC00FC00u : 0xFF800000u;  // -infinity
    // A piece as it was read, with -infinity for what is not of the row.
    __device__ __forceinline__ u32x4 trimmed(u32x4 v, int piece) const {
        if ((piece == 0 && skip) || piece == pieces - 1) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                const int i = piece * kVec + j - skip;
                if (i >= 0 && i < V) continue;
                if constexpr (F16) v[j >> 1] = j & 1 ? (v[j >> 1] & 0xFFFFu) | (kNone & 0xFFFF0000u) : (v[j >> 1] & 0xFFFF0000u) | (kNone & 0xFFFFu);
                else v[j] = kNone;
            }
        }
        return v;
    }
    __device__ __forceinline__ static float raw(const u32x4& v, int j) {
        if constexpr (F16) return __half2float(__ushort_as_half(static_cast<unsigned short>(j & 1 ? v[j >> 1] >> 16 : v[j >> 1] & 0xFFFFu)));
        else return __uint_as_float(v[j]);
    }
    __device__ __forceinline__ float finite(float x) const {
        if (infinite) {
            asm volatile("");  // a branch of the whole wave, not three instructions for every logit
            x = x == -kNothing ? 0.f : kNothing;
        }
        return x;
    }
    // Logit i of the row.
    __device__ __forceinline__ float at(int i) const {
        const void* p = STAGED ? static_cast<const void*>(staged) : base;
        if constexpr (F16) return finite(__half2float(__ushort_as_half(static_cast<const uint16_t*>(p)[i + skip])));
        else return finite(static_cast<const float*>(p)[i + skip]);
    }
    // f(logits, index of the first) for the thread's pieces; wave w has the w-th sixteenth of
    // them, all its lanes together (a lane without a piece has -infinity).
    template <class F>
    __device__ __forceinline__ void each_piece(F f) const {
        const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = threadIdx.x & 63;
        const int part = (to - from + kWaves - 1) / kWaves, begin = from + wave * part, end = min(to, begin + part), n = (end - begin + 63) / 64;
        const uint32_t slots = ring + wave * (kDepth * 1024);
        auto fetch = [&](int it) {
            const int i = min(begin + 64 * it + lane, pieces - 1);
            copy_to_lds(slots + it % kDepth * 1024, static_cast<uint32_t>(i) * 16u, base);
        };
        if constexpr (!STAGED)
            for (int it = 0; it < kDepth && it < n; ++it) fetch(it);
        for (int it = 0; it < n; ++it) {
            const int i = begin + 64 * it + lane;
            u32x4 v;
            if constexpr (STAGED) {
                v = staged[min(i, pieces - 1)];
            } else {
                if (it + kDepth <= n) landed_but<kDepth - 1>();
                else landed_but<0>();
                v = trimmed(read_lds(slots + it % kDepth * 1024 + lane * 16), min(i, pieces - 1));
                landed_but<kDepth - 1>();  // it is read before its place is loaded again
                if (it + kDepth < n) fetch(it + kDepth);
            }
            if (i >= end) v = u32x4{kNone, kNone, kNone, kNone};
            float x[kVec];
#pragma unroll
            for (int j = 0; j < kVec; ++j) x[j] = finite(raw(v, j));
            f(x, i * kVec - skip);
        }
    }
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        each_piece([&](const float(&x)[kVec], int i) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) f(x[j], i + j);
        });
    }
    __device__ __forceinline__ int part() const { return (pieces + kWaves - 1) / kWaves; }  // pieces of a part of the row

    // 1/16 octaves below the largest: rises as x falls.  NaN and -infinity are not below
    // kBuckets: they are not live.
    __device__ __forceinline__ float below(float x) const { return fmaf(-scale, x, scaled) * c32; }
    __device__ __forceinline__ static bool live(float y) { return y < static_cast<float>(kBuckets); }
    // 2^45 2^((x - max) c), the power not below -60, in binary64: 512 (x - max) c = k + f, |f| <=
    // 1/2, the table's 2^(k % 512 / 512), a power of two (which only adds to its exponent), and
    // e^r - 1, r = f ln 2 / 512, by its series to r^3 (what follows is below 2^-46).  Each fma
    // is written out: a row's sums of different passes are compared, so all have the same bits.
    __device__ __forceinline__ double weight(float x) const {
        const double d = static_cast<double>(x) - max, t = fma(d, c64, kMagic), f = fma(d, c64, -(t - kMagic));
        const int k = static_cast<int>(__double_as_longlong(t));
        constexpr double l = 0.69314718055994530942 / kSteps;
        const double p = f * fma(f, fma(f, l * l * l / 6, l * l / 2), l);
        const u64 two = static_cast<u64>(__double_as_longlong(table[k & (kSteps - 1)])) + (static_cast<u64>(static_cast<uint32_t>(k & -kSteps) << (20 - kStepBits)) << 32);
        const double a = __longlong_as_double(static_cast<long long>(two));
        return fma(a, p, a);
    }
    // f(j, weight) for a piece's logits; four of them are worked out side by side (one after the
    // other they would wait for the table, and eight do not fit the registers), those that
    // are not asked for as any number.
    template <class F>
    __device__ __forceinline__ void weights(const float (&x)[kVec], F f) const {
#pragma unroll
        for (int g = 0; g < kVec; g += 4) {
            double w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = weight(x[g + q]);
            asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));  // not put off into f's branches
#pragma unroll
            for (int q = 0; q < 4; ++q) f(g + q, w[q]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    static constexpr u64 kZero = 0x4330000000000000ull;  // the bits of 2^52
    // The bits of 2^52 + w: w rounded to a whole number, 0 .. 2^45, above kZero.
    __device__ __forceinline__ static u64 above(double w) { return static_cast<u64>(__double_as_longlong(w + 0x1p52)); }
    __device__ __forceinline__ static u64 whole(double w) { return above(w) - kZero; }
    // The same, or kZero if not `in`: what is left of w without its high half is nothing beside 2^52.
    __device__ __forceinline__ static u64 above_if(bool in, double w) {
        const u64 bits = static_cast<u64>(__double_as_longlong(w));
        return above(__longlong_as_double(static_cast<long long>(in ? bits : bits & 0xFFFFFFFFull)));
    }
};

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_before(uint32_t v) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xF, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ void add_before(uint32_t& n, u64& w) {
    const uint32_t lo = from_before<CTRL, ROWS>(static_cast<uint32_t>(w)), hi = from_before<CTRL, ROWS>(static_cast<uint32_t>(w >> 32));
    n += from_before<CTRL, ROWS>(n);
    w += static_cast<u64>(hi) << 32 | lo;
}
// Running sums over the wave's lanes, the lane's own included: by 1, 2, 4 and 8 lanes
// inside rows of 16, then the rows' last lanes into the rows behind them.
__device__ __forceinline__ void wave_scan(uint32_t& n, u64& w) {
    add_before<0x111, 0xF>(n, w);
    add_before<0x112, 0xF>(n, w);
    add_before<0x114, 0xF>(n, w);
    add_before<0x118, 0xF>(n, w);
    add_before<0x142, 0xA>(n, w);
    add_before<0x143, 0xC>(n, w);
}

// Running sums over the waves, in lanes 0 .. 15, of what the last lane of each has in (n, w).
// Has one barrier, and wants one before the next.
static_assert(kWaves == 16, "a row of lanes");
__device__ __forceinline__ void across_waves(Shared& sm, uint32_t& n, u64& w) {
    const int lane = threadIdx.x & 63;
    if (lane == 63) {
        sm.wave_n[threadIdx.x >> 6] = n;
        sm.wave_w[threadIdx.x >> 6] = w;
    }
    __syncthreads();
    n = sm.wave_n[lane & 15];
    w = sm.wave_w[lane & 15];
    add_before<0x111, 0xF>(n, w);
    add_before<0x112, 0xF>(n, w);
    add_before<0x114, 0xF>(n, w);
    add_before<0x118, 0xF>(n, w);
}
__device__ __forceinline__ u64 of_lane(u64 w, int lane) {
    return static_cast<u64>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(w >> 32), lane))) << 32 |
           static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(w), lane));
}

// The workgroup's sums, to every thread.  Begins with a barrier.
__device__ __forceinline__ void group_sum(Shared& sm, uint32_t& n, u64& w) {
    wave_scan(n, w);
    __syncthreads();
    across_waves(sm, n, w);
    n = __builtin_amdgcn_readlane(static_cast<int>(n), kWaves - 1);
    w = of_lane(w, kWaves - 1);
}

// The largest whole number that is not above u total (total >= 1), and below total.
__device__ __forceinline__ u64 share_of(float u, u64 total) {
    if (!(u > 0.f)) return 0ull;
    if (u >= 1.f) return total - 1;
    int e;
    const u64 f = static_cast<u64>(ldexpf(frexpf(u, &e), 24));  // u = f 2^(e - 24)
    const int shift = 24 - e;
    return shift < 128 ? static_cast<u64>(static_cast<unsigned __int128>(f) * total >> shift) : 0ull;
}

// The least whole number that is a share p of total, above 0.
__device__ __forceinline__ u64 least_share(float p, u64 total) {
    const double s = ceil(static_cast<double>(p) * static_cast<double>(total));
    return s > 1.0 ? static_cast<u64>(s) : 1ull;
}

// What a border is looked for by: the k-th; the first whose running sum reaches the goal; or
// that with the goal for a share `part` of all, or for passing it.
struct Target {
    enum Kind { kCount, kSum, kShare, kPass } kind;
    uint32_t k;
    u64 goal;
    float part;
};

// Of the bins with counts ns and sums ws the one in which what comes after (base_n, base_w)
// reaches the target: to sm.bin, or -1, before_*, in_*, and the goal and the sum of all.
// Four waves do it, one a SIMD and a lane with four bins: sixteen take twice the time for the
// scans that all of them repeat.  The bins are complete at a barrier before, what the last
// call left has been read at one; ends in a barrier.
template <int BINS, bool N, bool W>
__device__ __forceinline__ void find_bin(Shared& sm, const uint32_t* ns, const u64* ws, uint32_t base_n, u64 base_w, const Target& target) {
    constexpr int kFinders = 4;
    static_assert(BINS % 4 == 0 && BINS <= kFinders * 256, "four bins a lane");
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t n[4] = {0, 0, 0, 0}, sum_n = 0, end_n = 0;
    u64 w[4] = {0, 0, 0, 0}, sum_w = 0, end_w = 0;
    if (wave < kFinders) {
        if (4 * tid < BINS) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (N) n[q] = ns[4 * tid + q];
                if (W) w[q] = ws[4 * tid + q];
            }
        }
        end_n = sum_n = n[0] + n[1] + n[2] + n[3];
        end_w = sum_w = w[0] + w[1] + w[2] + w[3];
        wave_scan(end_n, end_w);
        if ((tid & 63) == 63) {
            sm.wave_n[wave] = end_n;
            sm.wave_w[wave] = end_w;
        }
        if (tid == 0) sm.bin = -1;
    }
    __syncthreads();
    if (wave < kFinders) {
        u64 total = 0;
#pragma unroll
        for (int i = 0; i < kFinders; ++i) {
            const uint32_t one_n = sm.wave_n[i];
            const u64 one_w = sm.wave_w[i];
            base_n += i < wave ? one_n : 0u;
            base_w += i < wave ? one_w : 0ull;
            total += one_w;
        }
        u64 goal = target.goal;
        if (W && target.kind == Target::kShare) goal = least_share(target.part, total);
        if (W && target.kind == Target::kPass) goal = share_of(target.part, total) + 1;
        const bool by_n = N && (!W || target.kind == Target::kCount);
        auto reached = [&](uint32_t at_n, u64 at_w) { return by_n ? at_n >= target.k : at_w >= goal; };
        end_n += base_n;
        end_w += base_w;
        uint32_t at_n = end_n - sum_n;
        u64 at_w = end_w - sum_w;
        if (reached(end_n, end_w) && !reached(at_n, at_w)) {
            int q = 0;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                if (q == i && !reached(at_n + n[i], at_w + w[i])) {
                    at_n += n[i];
                    at_w += w[i];
                    q = i + 1;
                }
            }
            sm.bin = 4 * tid + q;
            sm.before_n = at_n;
            sm.before_w = at_w;
            sm.in_n = q == 0 ? n[0] : q == 1 ? n[1] : q == 2 ? n[2] : n[3];
            sm.in_w = q == 0 ? w[0] : q == 1 ? w[1] : q == 2 ? w[2] : w[3];
        }
        if (tid == 0) {
            sm.goal = goal;
            sm.total = total;
        }
    }
    __syncthreads();
}

// Kept are logits above `key`, and those equal to it up to index `last`; their sum.
struct Border {
    uint32_t key;
    int last;
    u64 sum;
};

// What the list holds: nothing, the bucket of the border, or all down to it.
enum Held : int { kNoList, kBucket, kAll };

// What goes into a list with room for `room` logits: up to `most` all of them.  Where pass 2
// left the quarters' sums a long list costs more than a quarter (48 rows of 32000 that keep
// 7900: 37.4 us with all in the list, 33.6 with the bucket; that keep 2400: 30.2 and 32.9).
__device__ __forceinline__ int held_by(uint32_t before, uint32_t members, uint32_t room, uint32_t most) {
    return before + members <= min(room, most) ? kAll : members <= room ? kBucket : kNoList;
}

// The logits of the bucket from `top` to `end` (1/16 octaves), or all down to it, into `list`,
// *listed of them so far; returns the thread's sum of the kept weights before it (parts).
template <class R>
__device__ __forceinline__ u64 collect(const R& row, u64* list, uint32_t* listed, uint32_t room, int held, float top, float end, bool parts,
                                       double least) {
    // a piece's wanted logits into the list, one count for a wave
    auto append = [&](const bool (&wanted)[R::kVec], const float(&x)[R::kVec], int i) {
        u64 lanes[R::kVec];
        uint32_t n = 0;
#pragma unroll
        for (int j = 0; j < R::kVec; ++j) {
            lanes[j] = __ballot(wanted[j]);
            n += __builtin_popcountll(lanes[j]);
        }
        if (n == 0) return;
        uint32_t at = 0;
        if ((threadIdx.x & 63) == 0) at = atomicAdd(listed, n);
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int j = 0; j < R::kVec; ++j) {
            if (lanes[j] == 0) continue;
            const uint32_t place = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(lanes[j] >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(lanes[j]), at));
            if (wanted[j] && place < room) list[place] = static_cast<u64>(ordered(x[j])) << 32 | static_cast<uint32_t>(i + j);
            at += __builtin_popcountll(lanes[j]);
        }
    };
    u64 sum = 0;
    if (held == kAll) {
        row.each_piece([&](const float(&x)[R::kVec], int i) {
            bool wanted[R::kVec];
#pragma unroll
            for (int j = 0; j < R::kVec; ++j) wanted[j] = row.below(x[j]) < end;
            append(wanted, x, i);
        });
    } else {
        row.each_piece([&](const float(&x)[R::kVec], int i) {
            bool wanted[R::kVec], before = false;
#pragma unroll
            for (int j = 0; j < R::kVec; ++j) {
                const float y = row.below(x[j]);
                wanted[j] = (y >= top) & (y < end);
                before |= y < top;
            }
            append(wanted, x, i);
            if (!parts || !__any(before)) return;
            row.weights(x, [&](int j, double w) { sum += R::above_if((row.below(x[j]) < top) & (w >= least), w); });
            sum -= R::kVec * R::kZero;
        });
    }
    return sum;
}

// A border's search in the bucket that find_bin left in sm.  The list is filled by the first (held < 0), or was by an earlier launch
// (work: the list, and in sm.part_w the parts); the second one's border is not behind the
// first's.  parts: the sums of the kept weights before the bucket are left in sm.part_w (min-p's
// `least` included) where the list holds the bucket alone: of the quarters, if pass 2 left
// their buckets (quartered, which says afterwards if it is so) and min-p keeps all before the
// bucket's end, or of the waves' parts.  fresh: the buckets' sums are not there yet and come from
// the list, which holds all that top-k can keep.
template <class R>
__device__ __forceinline__ Border search(Shared& sm, const R& row, u64* list, uint32_t room, const Target& target, bool weigh, bool parts, bool fresh,
                                         double least, const Work* work, bool& quartered, int& held, uint32_t& listed) {
    const int tid = threadIdx.x;
    const int bucket = sm.bin;
    uint32_t before_n = sm.before_n;
    const uint32_t members = sm.in_n;
    u64 before_w = sm.before_w;
    const float top = static_cast<float>(bucket), end = static_cast<float>(bucket + 1);  // 1/16 octaves
    if (tid == 0) {
        sm.low = 0xFFFFFFFFu;
        sm.high = 0u;
    }
    uint32_t low = 0xFFFFFFFFu, high = 0u;
    auto member = [&](float x) {
        low = min(low, ordered(x));
        high = max(high, ordered(x));
    };
    if (held != kAll) {
        const bool ready = held < 0 && work != nullptr;
        held = held_by(before_n, members, room, quartered && parts ? kShortList : room);
        listed = held == kAll ? before_n + members : members;
        // (the bucket's end is at 2^-((bucket + 1) / 16) but for the roundings of below())
        quartered = quartered && parts && held == kBucket && least <= exp2(45.0 - 1e-3 - (bucket + 1) * (1.0 / 16.0));
        if (quartered) {
            const int wave = tid >> 6, lane = tid & 63;
            if (wave > 0 && wave < kQuarters) {
                const u64* q = quarter(sm, list, wave);
                u64 sum = 0;
                for (int i = lane; i < bucket; i += 64) sum += q[i];
                uint32_t none = 0;
                wave_scan(none, sum);
                if (lane == 63) sm.part_w[wave] = sum;
            }
            __syncthreads();
            if (tid == 0) {
                const u64 w1 = sm.part_w[1], w2 = sm.part_w[2], w3 = sm.part_w[3];
                for (int i = 0; i < kWaves; ++i) sm.part_w[i] = 0ull;
                sm.part_w[0] = before_w - w1 - w2 - w3;
                sm.part_w[kQuarterWaves] = w1;
                sm.part_w[2 * kQuarterWaves] = w2;
                sm.part_w[3 * kQuarterWaves] = w3;
            }
        }
        if (tid == 0) sm.listed = 0u;
        __syncthreads();
        if (held == kNoList) {
            row.each([&](float x, int) {
                const float y = row.below(x);
                if (y >= top && y < end) member(x);
            });
        } else if (ready) {
            for (uint32_t i = tid; i < listed; i += kThreads) list[i] = work->list[i];
        } else {
            u64 sum = collect(row, list, &sm.listed, room, held, top, end, parts && !quartered, least);
            uint32_t none = 0;
            wave_scan(none, sum);
            if ((tid & 63) == 63 && !quartered) sm.part_w[tid >> 6] = sum;
        }
    }
    __syncthreads();
    if (held != kNoList) {
        for (uint32_t i = tid; i < listed; i += kThreads) {
            const float x = unordered(static_cast<uint32_t>(list[i] >> 32)), y = row.below(x);
            if (y >= top && y < end) member(x);
            if (fresh) atomicAdd(&sm.bucket_w[static_cast<int>(y)], R::whole(row.weight(x)));
        }
    }
    if (high) {
        atomicMin(&sm.low, low);
        atomicMax(&sm.high, high);
    }
    __syncthreads();
    low = sm.low;
    high = sm.high;
    if (fresh) {
        find_bin<kBuckets, true, true>(sm, sm.bucket_n, sm.bucket_w, 0u, 0ull, target);
        before_w = sm.before_w;
    }
    // f(key, index): the bucket's are all the logits from low to high
    auto each = [&](auto f) {
        if (held != kNoList) {
            for (uint32_t i = tid; i < listed; i += kThreads) f(static_cast<uint32_t>(list[i] >> 32), static_cast<int>(list[i] & 0xFFFFFFFFu));
        } else {
            row.each([&](float x, int i) { f(ordered(x), i); });
        }
    };
    Border b;
    for (;;) {
        const uint32_t range = high - low;
        const int shift = range < 1024u ? 0 : 22 - __builtin_clz(range);
        sm.bin_n[tid] = 0u;
        sm.bin_w[tid] = 0ull;
        __syncthreads();
        each([&](uint32_t key, int) {
            if (key < low || key > high) return;
            const uint32_t bin = (high - key) >> shift;
            atomicAdd(&sm.bin_n[bin], 1u);
            if (weigh) atomicAdd(&sm.bin_w[bin], R::whole(row.weight(unordered(key))));
        });
        __syncthreads();
        find_bin<1024, true, true>(sm, sm.bin_n, sm.bin_w, before_n, before_w, target);
        before_n = sm.before_n;
        before_w = sm.before_w;
        const uint32_t first = high - (static_cast<uint32_t>(sm.bin) << shift);
        if (shift == 0) {
            b.key = first;
            break;
        }
        const uint32_t span = (1u << shift) - 1u;
        low = first - low > span ? first - span : low;
        high = first;
        __syncthreads();  // sm's fields are read
    }
    // of the equal ones, the first `take` by index
    const uint32_t equal = sm.in_n;
    const u64 w = weigh ? R::whole(row.weight(unordered(b.key))) : 0ull;
    uint32_t take = equal;
    if (target.kind == Target::kCount) {
        take = target.k - before_n;
    } else {
        const double t = ceil(static_cast<double>(target.goal - before_w) / static_cast<double>(w));
        take = t < 1.0 ? 1u : t > equal ? equal : static_cast<uint32_t>(t);
        while (take > 1 && before_w + (take - 1) * w >= target.goal) --take;
        while (take < equal && before_w + take * w < target.goal) ++take;
    }
    b.sum = before_w + take * w;
    b.last = row.V;
    if (take < equal) {
        int first = 0;
        uint32_t done = 0;
        const Target nth = {Target::kCount, take, 0ull, 0.f};
        for (int shift = 8; shift >= 0; shift -= 8) {  // V <= 2^18
            __syncthreads();
            sm.bin_n[tid] = 0u;
            __syncthreads();
            each([&](uint32_t key, int i) {
                const int bin = (i - first) >> shift;
                if (key == b.key && bin >= 0 && bin < 1024) atomicAdd(&sm.bin_n[bin], 1u);
            });
            __syncthreads();
            find_bin<1024, true, false>(sm, sm.bin_n, nullptr, done, 0ull, nth);
            done = sm.before_n;
            first += sm.bin << shift;
        }
        b.last = first;
    }
    __syncthreads();
    return b;
}

// A row is one workgroup's, in one launch, or sixteen workgroups share its passes, in four.
enum Phase : int {
    kWhole,
    kMax,      // pass 1, and the counts are cleared
    kCount,    // pass 2, or where no border is the parts' sums
    kCollect,  // pass 3
    kRest,     // the border inside its bucket, and the token: one workgroup
};

template <bool F16, bool STAGED, int PHASE>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a, uint32_t room, int list_at) {
    extern __shared__ __align__(16) uint8_t smem[];
    Shared& sm = *reinterpret_cast<Shared*>(smem);
    u64* list = reinterpret_cast<u64*>(smem + list_at);
    using R = Row<F16, STAGED>;
    constexpr int kSize = F16 ? 2 : 4;
    constexpr bool kShares = PHASE == kMax || PHASE == kCount || PHASE == kCollect;

    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t b = kShares ? blockIdx.x / kWaves : blockIdx.x;
    const int share = kShares ? blockIdx.x % kWaves : 0;
    Work* work = PHASE == kWhole ? nullptr : static_cast<Work*>(a.workspace) + b;
    const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits) + static_cast<uintptr_t>(b * a.stride) * kSize;
    R row;
    row.base = reinterpret_cast<const uint8_t*>(at & ~static_cast<uintptr_t>(15));
    row.staged = reinterpret_cast<u32x4*>(smem + (sizeof(Shared) + 15) / 16 * 16);
    row.ring = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_u8*)(smem + (sizeof(Shared) + 15) / 16 * 16)));
    row.table = sm.table;
    row.skip = static_cast<int>(at & 15) / kSize;
    row.V = a.V;
    row.pieces = (row.skip + a.V + R::kVec - 1) / R::kVec;
    row.from = kShares ? min(row.pieces, share * row.part()) : 0;
    row.to = kShares ? min(row.pieces, row.from + row.part()) : row.pieces;
    row.infinite = false;

    const float t = a.temperature ? a.temperature[b] : a.temperature_all, p = a.top_p ? a.top_p[b] : a.top_p_all;
    const float least = a.min_p ? a.min_p[b] : a.min_p_all, u = a.u[b];
    const int k = a.top_k ? a.top_k[b] : a.top_k_all;

    // 1: the largest logit
    float m = kNothing;
    auto larger = [&](float x) { m = x > m ? x : m; };
    if constexpr (STAGED) {
        const int part = row.part(), end = min(row.pieces, (wave + 1) * part);
        for (int i = wave * part + lane; i < end; i += 64) {
            const u32x4 v = row.trimmed(reinterpret_cast<const u32x4*>(row.base)[i], i);
            row.staged[i] = v;
#pragma unroll
            for (int j = 0; j < R::kVec; ++j) larger(R::raw(v, j));
        }
    } else if constexpr (PHASE == kWhole || PHASE == kMax) {
        row.each([&](float x, int) { larger(x); });
    }
    if constexpr (PHASE == kWhole || PHASE == kMax) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) larger(__shfl_xor(m, d, 64));
        if (lane == 0) sm.wave_max[wave] = m;
    }
    if (tid == 0) sm.first = 0xFFFFFFFFu;
    if (tid < kBuckets) {
        sm.bucket_n[tid] = 0u;
        sm.bucket_w[tid] = 0ull;
        if constexpr (PHASE == kWhole)
            for (int q = 1; q < kQuarters; ++q) quarter(sm, list, q)[tid] = 0ull;
    }
    if (tid < kSteps) sm.table[tid] = exp2(45.0 + tid * (1.0 / kSteps));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) larger(PHASE == kWhole || PHASE == kMax ? sm.wave_max[i] : work->max[i]);
    if constexpr (PHASE == kMax) {
        constexpr int kEach = (kBuckets + kWaves - 1) / kWaves;
        if (tid < kEach && share * kEach + tid < kBuckets) {
            work->bucket_n[share * kEach + tid] = 0u;
            work->bucket_w[share * kEach + tid] = 0ull;
        }
        if (tid == 0) {
            work->max[share] = m;
            work->part_w[share] = 0ull;
            if (share == 0) {
                work->listed = 0u;
                work->first = 0xFFFFFFFFu;
            }
        }
        return;
    }
    if (m == kNothing) {  // nothing can be chosen
        if (!kShares && tid == 0) {
            a.tokens[b] = -1;
            if (a.probs) a.probs[b] = 0.f;
        }
        return;
    }
    row.infinite = __builtin_amdgcn_readfirstlane(m == -kNothing);
    if (row.infinite) m = 0.f;
    // settings that leave the first alone: the largest logit, the lowest index of equal ones
    if (!(t > 0.f) || k == 1 || p <= 0.f || least > 1.f) {
        if constexpr (PHASE == kWhole || PHASE == kCount) {
            uint32_t first = 0xFFFFFFFFu;
            row.each([&](float x, int i) {
                if (x == m) first = min(first, static_cast<uint32_t>(i));
            });
            if (first != 0xFFFFFFFFu) atomicMin(PHASE == kCount ? &work->first : &sm.first, first);
            __syncthreads();
        }
        if (!kShares && tid == 0) {
            a.tokens[b] = static_cast<int>(PHASE == kRest ? work->first : sm.first);
            if (a.probs) a.probs[b] = 1.f;
        }
        return;
    }
    const double c = 1.4426950408889634074 / static_cast<double>(t);
    row.max = m;
    row.c64 = kSteps * c;
    // Halves, whose difference cannot overflow.  A temperature below some 2^-120 would take their
    // factor past binary32 and logits thousands of octaves down for live ones; there the differences
    // that count are small numbers and are made larger, unless the largest logit's next is far below it anyhow.
    row.scale = c >= 0x1p120 && fabsf(m) < 0x1p60f ? 0x1p60f : 0.5f;
    row.scaled = row.scale * m;
    row.c32 = fminf(static_cast<float>(16.0 * c / row.scale), 3.4e38f);  // 0 times it is 0

    // 2, 3: the border
    const bool by_k = k > 1 && k < a.V, by_p = p < 1.f;
    const double floor_w = least > 0.f ? 0x1p45 * static_cast<double>(least) : 0.0;
    Border border = {0u, a.V, 0ull};
    int held = -1;
    uint32_t listed = 0;
    bool found = false, quartered = PHASE == kWhole && by_p;  // a border; the quarters' buckets, then their sums, are there
    // top-p of what a small top-k keeps: only that is weighed, in the list (if it holds all of it)
    bool few = PHASE == kWhole && by_k && by_p && k <= kFewKept;
    if (by_k || by_p) {
        if constexpr (PHASE == kWhole || PHASE == kCount) {
            u64* sums = PHASE == kWhole ? quarter(sm, list, __builtin_amdgcn_readfirstlane(wave) / kQuarterWaves) : sm.bucket_w;
            for (bool first = true;; first = false) {
                row.each_piece([&](const float(&x)[R::kVec], int) {
                    float y[R::kVec];
                    bool live = false;
#pragma unroll
                    for (int j = 0; j < R::kVec; ++j) {
                        y[j] = row.below(x[j]);
                        live |= R::live(y[j]);
                    }
                    if (!__any(live)) return;
                    if (first) {
#pragma unroll
                        for (int j = 0; j < R::kVec; ++j)
                            if (R::live(y[j])) atomicAdd(&sm.bucket_n[static_cast<int>(y[j])], 1u);
                    }
                    if (by_p && !few)
                        row.weights(x, [&](int j, double w) {
                            if (R::live(y[j])) atomicAdd(&sums[static_cast<int>(y[j])], R::whole(w));
                        });
                });
                __syncthreads();
                if (!few) break;
                find_bin<kBuckets, true, false>(sm, sm.bucket_n, nullptr, 0u, 0ull, Target{Target::kCount, static_cast<uint32_t>(k), 0ull, 0.f});
                if (sm.bin >= 0 && sm.before_n + sm.in_n <= room) break;
                few = false;
                __syncthreads();
            }
            if (PHASE == kWhole && by_p && !few && tid < kBuckets)
                for (int q = 1; q < kQuarters; ++q) sm.bucket_w[tid] += quarter(sm, list, q)[tid];
        } else if (tid < kBuckets) {
            sm.bucket_n[tid] = work->bucket_n[tid];
            sm.bucket_w[tid] = work->bucket_w[tid];
        }
        __syncthreads();
        if constexpr (PHASE == kCount) {
            if (tid < kBuckets && sm.bucket_n[tid]) {
                atomicAdd(&work->bucket_n[tid], sm.bucket_n[tid]);
                if (sm.bucket_w[tid]) atomicAdd(&work->bucket_w[tid], sm.bucket_w[tid]);
            }
            return;
        }
        for (int i = 0; i < 2; ++i) {  // top-k, then top-p of what it keeps
            if (!(i ? by_p : by_k)) continue;
            Target target = {i ? found ? Target::kSum : Target::kShare : Target::kCount, static_cast<uint32_t>(k), found ? least_share(p, border.sum) : 0ull, p};
            if (i || !few) find_bin<kBuckets, true, true>(sm, sm.bucket_n, sm.bucket_w, 0u, 0ull, target);
            if (sm.bin < 0) {  // fewer than k
                __syncthreads();
                continue;
            }
            target.goal = sm.goal;
            if (i) target.kind = Target::kSum;
            if constexpr (PHASE == kCollect) {
                held = held_by(sm.before_n, sm.in_n, room, room);
                u64 sum = 0;
                if (held != kNoList)
                    sum = collect(row, work->list, &work->listed, room, held, static_cast<float>(sm.bin), static_cast<float>(sm.bin + 1), i || !by_p, floor_w);
                uint32_t none = 0;
                group_sum(sm, none, sum);
                if (tid == 0) work->part_w[share] = sum;
                return;
            } else {
                if (PHASE == kRest && !found && tid < kWaves) sm.part_w[tid] = work->part_w[tid];
                border = search(sm, row, list, room, target, by_p, i || !by_p, !i && few, floor_w, work, quartered, held, listed);
                found = true;
            }
        }
    }

    // 4: the token.  The weight of a logit if it is kept, or 0: above `low`, and not one of
    // those equal to the border's that come after its last.
    // Where no border is, what is 100 octaves below the largest stays out (46 to 1000 would do:
    // a difference of few steps of binary32 is rounded by half a step), and what is no number.
    const float dead = fminf(m - static_cast<float>(100.0 / c), under(ordered(m)));
    const float low = border.key ? under(border.key) : dead;
    const float tied = border.last < a.V ? unordered(border.key) : __builtin_nanf("");
    auto kept = [&](float x, int i) -> u64 {
        if (!(x > low) || (x == tied && i > border.last)) return 0ull;
        const double w = row.weight(x);
        return w >= floor_w ? R::whole(w) : 0ull;
    };
    // the thread's share of the kept weights
    auto kept_sum = [&]() -> u64 {
        u64 sum = 0;
        const bool ties = border.last < a.V;
        row.each_piece([&](const float(&v)[R::kVec], int i) {
            float x[R::kVec], most = kNothing;
#pragma unroll
            for (int j = 0; j < R::kVec; ++j) x[j] = v[j];
            if (ties) {
#pragma unroll
                for (int j = 0; j < R::kVec; ++j)
                    if (x[j] == tied && i + j > border.last) x[j] = kNothing;
            }
#pragma unroll
            for (int j = 0; j < R::kVec; ++j) most = fmaxf(most, x[j]);
            if (!__any(most > low)) return;
            row.weights(x, [&](int j, double w) { sum += R::above_if((x[j] > low) & (w >= floor_w), w); });
            sum -= R::kVec * R::kZero;
        });
        return sum;
    };
    if constexpr (kShares) {  // no border: the parts' sums, in the launch that finds that out
        if (PHASE == kCount || by_k) {
            u64 sum = kept_sum();
            uint32_t none = 0;
            group_sum(sm, none, sum);
            if (tid == 0) work->part_w[share] = sum;
        }
        return;
    }
    auto done = [&](int i, float x, u64 total) {
        a.tokens[b] = i;
        if (a.probs) a.probs[b] = static_cast<float>(row.weight(x) / static_cast<double>(total));
    };
    if (held == kAll) {
        // by indexes, 256 at a time, then 1
        int first = 0;
        u64 total = 0, passed = 0;
        Target target = {Target::kPass, 0u, 0ull, u};
        for (int shift = 8; shift >= 0; shift -= 8) {
            sm.bin_w[tid] = 0ull;
            __syncthreads();
            for (uint32_t e = tid; e < listed; e += kThreads) {
                const int i = static_cast<int>(list[e] & 0xFFFFFFFFu), bin = (i - first) >> shift;
                if (bin < 0 || bin >= 1024) continue;
                const u64 w = kept(unordered(static_cast<uint32_t>(list[e] >> 32)), i);
                if (w) atomicAdd(&sm.bin_w[bin], w);
            }
            __syncthreads();
            find_bin<1024, false, true>(sm, nullptr, sm.bin_w, 0u, passed, target);
            if (shift) {
                total = sm.total;
                target.kind = Target::kSum;
                target.goal = sm.goal;
            }
            passed = sm.before_w;
            first += sm.bin << shift;
            __syncthreads();
        }
        for (uint32_t e = tid; e < listed; e += kThreads)
            if (static_cast<int>(list[e] & 0xFFFFFFFFu) == first) done(first, unordered(static_cast<uint32_t>(list[e] >> 32)), total);
        return;
    }
    const int part = row.part();
    bool summed = true;
    if (held == kBucket && (quartered || !(by_k && by_p))) {  // the parts' sums, but for the bucket's, are there
        for (uint32_t e = tid; e < listed; e += kThreads) {
            const uint32_t key = static_cast<uint32_t>(list[e] >> 32);
            const int i = static_cast<int>(list[e] & 0xFFFFFFFFu), p = (i + row.skip) / R::kVec / part;
            const u64 w = kept(unordered(key), i);
            if (w) atomicAdd(&sm.part_w[quartered ? p / kQuarterWaves * kQuarterWaves : p], w);
        }
    } else if (PHASE == kRest && !found) {
        if (tid < kWaves) sm.part_w[tid] = work->part_w[tid];
    } else {
        summed = quartered = false;
    }
    // the part that holds the token; of a quarter its sixteenths are summed first
    u64 total = 0, goal = 0;
    int w;
    for (bool first = true;; first = false) {
        if (!summed) {
            u64 sum = kept_sum();
            uint32_t none = 0;
            wave_scan(none, sum);
            if (lane == 63) sm.part_w[wave] = sum;
        }
        __syncthreads();
        if (first) {
#pragma unroll
            for (int i = 0; i < kWaves; ++i) total += sm.part_w[i];
            goal = share_of(u, total);
        }
        w = 0;
        while (w < kWaves - 1 && goal >= sm.part_w[w]) goal -= sm.part_w[w++];
        if (!quartered) break;
        quartered = summed = false;
        row.from = min(row.pieces, w * part);
        row.to = min(row.pieces, (w + kQuarterWaves) * part);
        __syncthreads();
    }
    // that part's logits, a run of them a thread
    const int each = (row.to - row.from + kWaves - 1) / kWaves;
    const int begin = max(0, (row.from + w * each) * R::kVec - row.skip), end = min(a.V, min(row.to, row.from + (w + 1) * each) * R::kVec - row.skip);
    const int run = (end - begin + kThreads - 1) / kThreads, first = min(end, begin + tid * run), last = min(end, first + run);
    u64 own = 0;
    for (int i = first; i < last; ++i) own += kept(row.at(i), i);
    sm.bin_w[tid] = own;
    __syncthreads();
    find_bin<1024, false, true>(sm, nullptr, sm.bin_w, 0u, 0ull, Target{Target::kSum, 0u, goal + 1, 0.f});
    if (tid == sm.bin) {
        u64 left = goal - sm.before_w;
        for (int i = first; i < last; ++i) {
            const float x = row.at(i);
            const u64 v = kept(x, i);
            if (left < v) {
                done(i, x, total);
                break;
            }
            left -= v;
        }
    }
}

template <bool F16, bool STAGED, int PHASE>
hipError_t run(const SampleArgs& a, int64_t groups, int row_bytes, hipStream_t st) {
    static std::atomic<uint64_t> done{0};
    constexpr int fixed = (sizeof(Shared) + 15) / 16 * 16;
    static_assert(fixed + kStageBytes + 1024 * 8 <= kLdsBytes && fixed + kRingBytes + kMostList * 8 <= kLdsBytes && 1024 >= kBuckets, "fits a compute unit's LDS");
    const auto k = sample_kernel<F16, STAGED, PHASE>;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(k), kLdsBytes, done);
    if (e != hipSuccess) return e;
    const int list_at = fixed + (STAGED ? row_bytes : kRingBytes), left = (kLdsBytes - list_at) / 8, room = left < kMostList ? left : kMostList;
    const bool lists = PHASE == kWhole || PHASE == kRest;
    k<<<dim3(static_cast<unsigned>(groups)), dim3(kThreads), list_at + (lists ? room * 8 : 0), st>>>(a, static_cast<uint32_t>(room), list_at);
    return hipGetLastError();
}

template <bool F16>
hipError_t run_shared(const SampleArgs& a, int64_t B, hipStream_t st) {
    hipError_t e = run<F16, false, kMax>(a, B * kWaves, 0, st);
    if (e == hipSuccess) e = run<F16, false, kCount>(a, B * kWaves, 0, st);
    if (e == hipSuccess) e = run<F16, false, kCollect>(a, B * kWaves, 0, st);
    return e == hipSuccess ? run<F16, false, kRest>(a, B, 0, st) : e;
}

}  // namespace

// Sharing takes three more launches (some 8 us where the host keeps up, 15 where it does
// not) and a row's passes a sixteenth of their time.  top-p, us one workgroup a row and
// shared: 131072 binary32 logits 1 row 86 and 43, 32 rows 89 and 64, 64 rows 88 and 96;
// 65000 of binary16 1 row 48 and 37, 16 rows 54 and 46, 32 rows 52 and 57; 32000 1 row 23 and
// 26, 32 rows 34 and 54.
int64_t sample_workspace(int64_t B, int64_t V) {
    const bool shared = B > 0 && V >= kSharedLogits && B * kWaves * kSharedLogits <= device_cu_count() * V;
    return shared ? B * static_cast<int64_t>(sizeof(Work)) : 0;
}

hipError_t launch_sample(const SampleArgs& a, int64_t B, bool f16, hipStream_t stream) {
    if (sample_workspace(B, a.V)) return f16 ? run_shared<true>(a, B, stream) : run_shared<false>(a, B, stream);
    const int bytes = (a.V * (f16 ? 2 : 4) + 15) / 16 * 16 + 16;  // a row that begins inside a piece has one more
    if (bytes <= kStageBytes) return f16 ? run<true, true, kWhole>(a, B, bytes, stream) : run<false, true, kWhole>(a, B, bytes, stream);
    return f16 ? run<true, false, kWhole>(a, B, bytes, stream) : run<false, false, kWhole>(a, B, bytes, stream);
}

}  // namespace apex4
