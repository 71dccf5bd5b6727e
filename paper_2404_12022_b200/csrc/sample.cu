// Sampling from filtered distributions (temperature, top-k, top-p, min-p) with given uniform numbers, alone and as the
// verification of a draft tree (Section "Inference stage" with sampled instead of greedy tokens).
//
// Definition, per row of logits x with largest value m:
//     weight   w_i = exp((x_i - m) / T), zero where that is below 2^-1000
//     order    larger x first, lower index among equals
//     kept     the first top_k of the order; of those, the ones whose running weight before them is below
//              top_p * (weight of the first top_k); of those, the ones with w_i >= min_p
//     token    the first kept i in index order whose running kept weight exceeds uniform * (kept weight)
// Every filter keeps a prefix of the order, so a kept set is one pair (x, index): the first element left out.
//
// The token is a whole number, and the cut of a flat distribution moves all that follows it, so weights and sums are
// held in 64 bits (relative error about 1e-12), whatever the order of a sum.  The tokens below 2^-31 of the largest are
// added up in 32 in rows of up to 2^20 (kLongTail): all of them weigh V 2^-31 of the whole at most, their sum is off by 2e-5
// of that (weights 1e-5, as many roundings of 2^-25 as a thread has tokens), and so by 2e-5 V 2^-31 < 1e-8 of the whole: a
// sixth of the step of a uniform number or a top_p.  Longer rows add them up in 64.  Nothing is added by atomics but counts.
//
// A row is split over the blocks of a cluster (one block where the rows fill the GPU by themselves), its slices in
// shared memory; one read of the logits.  A histogram of the tokens over the logarithm of their weight (1/64 octave per
// bin) bounds the running weight at every bin, which leaves the cut in a zone of a bin or a few; the zone's tokens (or
// the whole kept set, where it is small) are sorted by the cluster's first block and the cut is found exactly.  A small
// top-k needs no weights at all: the k-th largest of the threads' maxima is a lower bound of the k-th largest token.
// bf16 rows are counted by value instead, which needs no weights per token until the cut is known.
// Bound by instructions per token (30 to 50 per pass and token, a third of them 64-bit; at 64 registers, two blocks per SM, with
// 24 to 126 bytes of spills) and, for few long rows, by the chain of a cluster's steps, not by HBM: 4 x 32000 in bf16 13 us,
// 256 x 32003 in fp16 26 us, 64 x 131072 in fp32 98 us (top-p), 4096 x 32000 in bf16 436 us (top-p).
//
// Compiled once per type of the logits (HT_SAMPLE_DTYPE, the number of the type), side by side; fp32 brings the entry.
#include <float.h>
#include <limits.h>

#include "accept.cuh"

namespace ht {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kBins = 2048;
constexpr int kBinsPerOctave = 64;
constexpr int kList = 1024;               // tokens that are sorted at most
// Kept sets up to this are sorted whole and drawn from in one step instead of cut in their zone and walked.  1024 rows of 32000 in
// fp16, top-k and top-p, at 64 / 128 / 256: k = 50 49.7 us in all three, k = 100 69.3 / 54.7 / 54.8 us, k = 200 82.5 / 82.4 / 69.2 us.
constexpr unsigned int kShort = 256;
constexpr int kMaxTeam = 8;               // blocks per row
constexpr int kLongTail = 1 << 20;        // longer rows sum the tokens below 2^-31 of the largest in 64 bits

struct SampleSmem {
    union {
        unsigned int hist[kBins];
        unsigned long long list[kList];
    };
    double pow2[kBinsPerOctave];          // 2^(i / 64)
    double wsum[kSampleWarps];            // per warp, of the block's latest sum
    double part[kSampleWarps];            // per warp: kept weight of its range of the row
    double scan[3 * kSampleWarps];
    double short_w[kShort], short_sum;
    float wmax[kSampleWarps];
    unsigned int wcount[kSampleWarps];
    struct {
        double d;
        float f;
        unsigned int u;
    } slot[2];                            // what the row's other blocks read, by turns
    long long value_at;                   // value_cut: the cut's value (its bin; -1: none) and, in the low half, how many of it are kept
    int n_list, n_above, zone_lo, zone_hi, answer, first_thread;
    unsigned int total;
    float cut_x;
    int cut_i;
};

// Ordered integer of a value: larger value, larger integer; -0 counts as 0.
__device__ __forceinline__ unsigned int order_key(float x) {
    const unsigned int u = __float_as_uint(x + 0.f);
    return u ^ ((unsigned int)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned int k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// In constant memory, where an instruction reads them as operands (as literals each would be put together in two
// registers first, for every token anew).
constexpr double kLn2By64 = 0.693147180559945309417 / 64.0;
static __constant__ double kSeries[5] = {1.0, kLn2By64, kLn2By64 *kLn2By64 / 2.0, kLn2By64 *kLn2By64 *kLn2By64 / 6.0,
                                  kLn2By64 *kLn2By64 *kLn2By64 *kLn2By64 / 24.0};
static __constant__ double kMagicC = 6755399441055744.0 + (1 << 30);      // 1.5 * 2^52 + the bias below: adding it rounds to a whole number

// Weight of a logit.  exp(d / T) = 2^(t / 64) with t = 64 log2(e) d / T.  k = t rounded is the token's bin (its distance
// to the largest in 1/64 octaves) and leaves |r| <= 1/2: k = 64 n + i, a table of 2^(i / 64), the Taylor series of
// e^(r ln2 / 64) to the fourth power (the next term is below 4e-14) and n into the exponent.  All in 64 bits.
struct Weights {
    double m, c;                          // largest logit, 64 log2(e) / T
    float m32, low, c32;                  // largest logit; logits below `low` lie in the last bin; log2(e) / T
    const double *pow2;
    static constexpr unsigned int kBias = 1u << 30;                // keeps k's 32 bits away from a change of sign
    // distance in bins of a logit that is not below `low`, and the two factors of its weight
    __device__ __forceinline__ int split(float x, double &q, double &s) const {
        const double d = (double)x - m;
        const double kd = fma(d, c, kMagicC);
        const unsigned int k = (unsigned int)__double2loint(kd);
        const double r = fma(d, c, kMagicC - kd);
        q = kSeries[4];
#pragma unroll
        for (int i = 3; i >= 0; --i) q = fma(q, r, kSeries[i]);
        s = *reinterpret_cast<const double *>(reinterpret_cast<const char *>(pow2) + ((k << 3) & 0x1f8u));
        // (the bias leaves no trace above bit 31)
        s = __hiloint2double((int)((unsigned int)__double2hiint(s) + ((k & ~63u) << 14)), __double2loint(s));
        return (int)(kBias - k);
    }
    // the distance in bins as such
    __device__ __forceinline__ double depth(float x) const { return (m - (double)x) * c; }
    // any logit: zero below 2^-1000
    __device__ __forceinline__ double operator()(float x) const {
        double q, s;
        split(x, q, s);
        return ((double)x - m) * c >= -64000.0 ? q * s : 0.0;
    }
    // the weight of a logit below `low` (under 2^-31 of the largest) to 1e-5 where it counts: the exponent, -31 to about -60, is
    // formed from three roundings of 2^-24
    __device__ __forceinline__ float small(float x) const {
        float y;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"((x - m32) * c32));
        return y;
    }
};

// A block's slice of a row: vectors [v_lo, v_hi) of 16 bytes, in shared memory at the phase they have in global memory
// with -inf around the row (kStaged), or in global memory.  NaN reads as -inf; where the largest value is +inf
// (`peak`), +inf reads as 0 and all else as -inf.
template <typename T, bool kStaged>
struct Row {
    static constexpr int VE = Vec16<T>::n;
    const T *base;                        // vector v_lo (kStaged) or vector 0; element i of the row is number phase + i from vector 0
    int phase, V, v_lo, v_hi;
    bool peak;
    __device__ __forceinline__ void load(int v, float *x) const {
        if (kStaged) {
            unpack16<T>(*reinterpret_cast<const uint4 *>(base + (v - v_lo) * VE), x);
            return;
        }
        const int i0 = v * VE - phase;
        if (i0 >= 0 && i0 + VE <= V) {
            unpack16<T>(*reinterpret_cast<const uint4 *>(base + (size_t)v * VE), x);
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e) x[e] = (i0 + e >= 0 && i0 + e < V) ? to_float<T>(base[(size_t)v * VE + e]) : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) x[e] = clean(x[e]);
    }
    __device__ __forceinline__ int index(int v, int e) const { return v * VE - phase + e; }
    // the vectors of warp w: consecutive, so that sums per warp are sums over ranges of the index
    __device__ __forceinline__ int warp_first(int w) const { return v_lo + (int)((long long)(v_hi - v_lo) * w / kSampleWarps); }
    // f(value, index) for this thread's elements.  Two at a time: the loop's code, not its loads, is what has to be short.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        const int w = threadIdx.x >> 5, end = warp_first(w + 1) * (VE / 2);
#pragma unroll 1
        for (int j = warp_first(w) * (VE / 2) + (threadIdx.x & 31); j < end; j += 32) {
            float x0, x1;
            const int i = 2 * j - phase;
            if (kStaged) {
                pair(base + 2 * j - v_lo * VE, x0, x1);
            } else {
                x0 = i >= 0 && i < V ? clean(to_float<T>(base[2 * (size_t)j])) : -INFINITY;
                x1 = i + 1 >= 0 && i + 1 < V ? clean(to_float<T>(base[2 * (size_t)j + 1])) : -INFINITY;
            }
            f(x0, i);
            f(x1, i + 1);
        }
    }
    __device__ __forceinline__ float clean(float x) const {
        if (!(x == x)) x = -INFINITY;
        return peak ? (x == INFINITY ? 0.f : -INFINITY) : x;
    }
    static __device__ __forceinline__ void pair(const float *p, float &x0, float &x1) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        x0 = v.x;
        x1 = v.y;
    }
    static __device__ __forceinline__ void pair(const __half *p, float &x0, float &x1) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(p));
        x0 = v.x;
        x1 = v.y;
    }
    static __device__ __forceinline__ void pair(const __nv_bfloat16 *p, float &x0, float &x1) {
        const unsigned int u = *reinterpret_cast<const unsigned int *>(p);
        x0 = __uint_as_float(u << 16);
        x1 = __uint_as_float(u & 0xFFFF0000u);
    }
};

// The kept set: elements ahead of (x, index) in the order; at first everything above -inf.
struct Cut {
    float x;
    int index;
    __device__ __forceinline__ bool keeps(float v, int i) const { return v > x || (v == x && i < index); }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
// Sum over the block, the same in every thread; the warps' sums stay in sm.wsum until the next call.
__device__ __forceinline__ double block_sum(SampleSmem &sm, double v) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm.wsum[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kSampleWarps; ++w) s += sm.wsum[w];
    return s;
}
__device__ __forceinline__ unsigned int block_count(SampleSmem &sm, unsigned int v) {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm.wcount[threadIdx.x >> 5] = v;
    __syncthreads();
    unsigned int s = 0;
#pragma unroll
    for (int w = 0; w < kSampleWarps; ++w) s += sm.wcount[w];
    return s;
}
// Exclusive running sum over the threads of the block; `total` receives the sum.
template <typename S>
__device__ __forceinline__ S block_scan(S v, S *warp_buf, S *total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    S incl = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const S o = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += o;
    }
    __syncthreads();
    if (lane == 31) warp_buf[w] = incl;
    __syncthreads();
    S before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kSampleWarps; ++i) {
        if (i == w) before = all;
        all += warp_buf[i];
    }
    *total = all;
    S excl = __shfl_up_sync(0xffffffffu, incl, 1);
    if (lane == 0) excl = 0;
    return before + excl;
}

// The same for two sums and a count at once.
struct Sums {
    double up, dn;
    unsigned int c;
};
__device__ __forceinline__ Sums block_scan3(const Sums v, Sums *warp_buf, Sums *total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    Sums in = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const double up = __shfl_up_sync(0xffffffffu, in.up, off), dn = __shfl_up_sync(0xffffffffu, in.dn, off);
        const unsigned int c = __shfl_up_sync(0xffffffffu, in.c, off);
        if (lane >= off) { in.up += up; in.dn += dn; in.c += c; }
    }
    __syncthreads();
    if (lane == 31) warp_buf[w] = in;
    __syncthreads();
    Sums before{0.0, 0.0, 0u}, all{0.0, 0.0, 0u};
#pragma unroll
    for (int i = 0; i < kSampleWarps; ++i) {
        if (i == w) before = all;
        all.up += warp_buf[i].up; all.dn += warp_buf[i].dn; all.c += warp_buf[i].c;
    }
    *total = all;
    Sums ex{__shfl_up_sync(0xffffffffu, in.up, 1), __shfl_up_sync(0xffffffffu, in.dn, 1), __shfl_up_sync(0xffffffffu, in.c, 1)};
    if (lane == 0) ex = Sums{0.0, 0.0, 0u};
    return Sums{before.up + ex.up, before.dn + ex.dn, before.c + ex.c};
}

// The blocks that share a row: a cluster (kTeam), or one block.  Values cross through `slot`, by turns, so that one
// barrier per exchange is enough: a block can be one exchange ahead of another, not two.
template <bool kTeam>
struct Team {
    SampleSmem &sm;
    int rank, size, turn;
    template <typename U>
    __device__ __forceinline__ U *of(U *p, int r) const {    // block r's copy of a shared variable
        if (!kTeam) return p;
        U *q;
        asm("mapa.u64 %0, %1, %2;" : "=l"(q) : "l"(p), "r"(r));
        return q;
    }
    __device__ __forceinline__ void barrier() const {
        if (kTeam) asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
    }
    __device__ __forceinline__ double sum(double block_value) {              // of the blocks' values, in their order
        if (!kTeam) return block_value;
        if (threadIdx.x == 0) sm.slot[turn].d = block_value;
        barrier();
        double s = 0.0;
        for (int r = 0; r < size; ++r) s += *of(&sm.slot[turn].d, r);
        turn ^= 1;
        return s;
    }
    // ... and what the blocks ahead of this one have
    __device__ __forceinline__ double sum(double block_value, double &before) {
        before = 0.0;
        if (!kTeam) return block_value;
        if (threadIdx.x == 0) sm.slot[turn].d = block_value;
        barrier();
        double s = 0.0;
        for (int r = 0; r < size; ++r) {
            if (r == rank) before = s;
            s += *of(&sm.slot[turn].d, r);
        }
        turn ^= 1;
        return s;
    }
    __device__ __forceinline__ unsigned int count(unsigned int block_value) {
        if (!kTeam) return block_value;
        if (threadIdx.x == 0) sm.slot[turn].u = block_value;
        barrier();
        unsigned int s = 0;
        for (int r = 0; r < size; ++r) s += *of(&sm.slot[turn].u, r);
        turn ^= 1;
        return s;
    }
    // the largest of f, and the smallest and largest of u
    __device__ __forceinline__ float max(float block_value) {
        if (!kTeam) return block_value;
        if (threadIdx.x == 0) sm.slot[turn].f = block_value;
        barrier();
        float s = -INFINITY;
        for (int r = 0; r < size; ++r) s = fmaxf(s, *of(&sm.slot[turn].f, r));
        turn ^= 1;
        return s;
    }
    __device__ __forceinline__ int min_int(int block_value) {
        if (!kTeam) return block_value;
        if (threadIdx.x == 0) sm.slot[turn].u = (unsigned int)block_value;
        barrier();
        int s = INT_MAX;
        for (int r = 0; r < size; ++r) s = ::min(s, (int)*of(&sm.slot[turn].u, r));
        turn ^= 1;
        return s;
    }
    __device__ __forceinline__ unsigned int max_key(unsigned int block_value) {
        if (!kTeam) return block_value;
        if (threadIdx.x == 0) sm.slot[turn].u = block_value;
        barrier();
        unsigned int s = 0;
        for (int r = 0; r < size; ++r) s = ::max(s, *of(&sm.slot[turn].u, r));
        turn ^= 1;
        return s;
    }
    __device__ __forceinline__ unsigned int min_key(unsigned int block_value) {
        if (!kTeam) return block_value;
        return ~max_key(~block_value);
    }
};

// Ascending sort of list[0, n), n <= kList, by the whole block: a bitonic network on the next power of two, two
// neighbouring entries per thread.  Entries up to 32 apart meet by shuffles, within a warp and without a barrier; farther
// ones through shared memory (ten of the 55 steps for 1024 entries).
__device__ __forceinline__ void sort_list(SampleSmem &sm, int n) {
    static_assert(kList == 2 * kSampleThreads, "two entries per thread");
    int size = 2;
    while (size < n) size <<= 1;
    const int i0 = 2 * threadIdx.x, lane = threadIdx.x & 31;
    __syncthreads();
    unsigned long long a = i0 < n ? sm.list[i0] : ~0ull, b = i0 + 1 < n ? sm.list[i0 + 1] : ~0ull;
    const bool active = i0 - 2 * lane < size;               // whole warps
    for (int k = 2; k <= size; k <<= 1) {
        const bool up = (i0 & k) == 0;
        for (int j = k >> 1; j >= 64; j >>= 1) {
            __syncthreads();
            if (active) { sm.list[i0] = a; sm.list[i0 + 1] = b; }
            __syncthreads();
            if (active) {
                const unsigned long long oa = sm.list[i0 ^ j], ob = sm.list[(i0 + 1) ^ j];
                const bool keep_small = ((i0 & j) == 0) == up;
                a = keep_small ? ::min(a, oa) : ::max(a, oa);
                b = keep_small ? ::min(b, ob) : ::max(b, ob);
            }
        }
        if (active) {
            for (int j = ::min(k >> 1, 32); j >= 2; j >>= 1) {
                const unsigned long long oa = __shfl_xor_sync(0xffffffffu, a, j >> 1), ob = __shfl_xor_sync(0xffffffffu, b, j >> 1);
                const bool keep_small = ((i0 & j) == 0) == up;
                a = keep_small ? ::min(a, oa) : ::max(a, oa);
                b = keep_small ? ::min(b, ob) : ::max(b, ob);
            }
            if ((a > b) == up) {
                const unsigned long long o = a;
                a = b;
                b = o;
            }
        }
    }
    __syncthreads();
    if (active) { sm.list[i0] = a; sm.list[i0 + 1] = b; }
    __syncthreads();
}
// A token as a list entry that sorts in the order: larger key first, lower index among equals.
__device__ __forceinline__ unsigned long long list_entry(float x, int i) { return ((unsigned long long)~order_key(x) << 32) | (unsigned)i; }
__device__ __forceinline__ float entry_value(unsigned long long e) { return key_value(~(unsigned int)(e >> 32)); }
__device__ __forceinline__ int entry_index(unsigned long long e) { return (int)(unsigned int)e; }

// The first entry of the sorted list[0, n) at which `above` plus the weight of the entries ahead reaches `goal`; n if none.
// `sum_all` receives the weight of the whole list.
__device__ __forceinline__ int list_cut(SampleSmem &sm, const Weights &wt, int n, double above, double goal, double *sum_all) {
    constexpr int PER = kList / kSampleThreads;
    double w[PER], mine = 0.0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = threadIdx.x * PER + u;
        w[u] = i < n ? wt(entry_value(sm.list[i])) : 0.0;
        mine += w[u];
    }
    if (threadIdx.x == 0) sm.answer = n;
    double before = above + block_scan(mine, sm.wsum, sum_all);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = threadIdx.x * PER + u;
        if (i < n && !(before < goal)) {
            atomicMin(&sm.answer, i);
            break;
        }
        before += w[u];
    }
    __syncthreads();
    const int r = sm.answer;
    __syncthreads();
    return r;
}

// Draws from list[0, n) (any order, all kept, the first of the order with weight 1 among them).
__device__ __forceinline__ int list_draw(SampleSmem &sm, const Weights &wt, int n, double u) {
    if (n == 1) return entry_index(sm.list[0]);
    constexpr int PER = kList / kSampleThreads;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int i = threadIdx.x + x * kSampleThreads;
        if (i < n) {
            const unsigned long long e = sm.list[i];
            sm.list[i] = (e << 32) | (e >> 32);             // index first
        }
    }
    sort_list(sm, n);
    double w[PER], mine = 0.0, sum;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int i = threadIdx.x * PER + x;
        w[x] = i < n ? wt(key_value(~(unsigned int)sm.list[i])) : 0.0;
        mine += w[x];
    }
    if (threadIdx.x == 0) { sm.answer = INT_MAX; sm.first_thread = -1; }
    double running = block_scan(mine, sm.wsum, &sum);
    const double goal = u * sum;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int i = threadIdx.x * PER + x;
        running += w[x];
        if (i < n && w[x] > 0.0) {
            if (running > goal) atomicMin(&sm.answer, i);
            atomicMax(&sm.first_thread, i);                  // the last one with a weight, should none exceed the goal
        }
    }
    __syncthreads();
    const int at = sm.answer != INT_MAX ? sm.answer : sm.first_thread;
    return (int)(unsigned int)(sm.list[at] >> 32);
}

// What a block answers: a token, that another block of the row has it, or that besides nothing of this block's shared memory
// is read any more.
constexpr int kElsewhere = -2, kGone = -3;

// bf16 rows in shared memory are counted by value: 13 binades of either sign, 128 values each, and the few nearer to zero
// as one bin, in the order of the values.  Behind the row's slice in shared memory: counts, and the values' weights.
constexpr int kSide = 13 * 128;
constexpr int kValues = 2 * kSide + 1;
constexpr size_t kValueBytes = ((size_t)kValues * (sizeof(unsigned int) + sizeof(double)) + 31) / 16 * 16;
template <typename T, bool kStaged> struct ByValue { static constexpr bool on = false; };
template <> struct ByValue<__nv_bfloat16, true> { static constexpr bool on = true; };

template <typename T, bool kStaged, bool kTeam>
struct Sampler {
    static constexpr int VE = Vec16<T>::n;
    static constexpr bool kByValue = ByValue<T, kStaged>::on;
    SampleSmem &sm;
    Team<kTeam> &team;
    Row<T, kStaged> row;
    Weights wt;
    float m;                              // largest logit
    double *value_weight;                 // [kValues] and behind them counts (kByValue)

    // The cut behind the last element of value x that `in` keeps: where x is the value that `in` cuts through, `in` itself.
    __device__ __forceinline__ Cut last_of(float x, const Cut &in) { return x == in.x ? in : Cut{x, INT_MAX}; }

    // The cut among the elements of value key_value(key) that `in` keeps, behind the first `ties` of them in index order.
    // By the list, or, where they are more than it holds, by halving the range of the indexes, one pass per step.
    __device__ __noinline__ Cut tie_cut(const Cut in, unsigned int key, unsigned int ties) {
        open_list();
        row.each([&](float x, int i) { if (order_key(x) == key && in.keeps(x, i)) append(x, i); });
        const int n = close_list();
        if (n <= kList) {
            Cut c = last_of(key_value(key), in);
            if (!kTeam || team.rank == 0) {
                sort_list(sm, n);
                if (ties < (unsigned int)n) c = Cut{key_value(key), entry_index(sm.list[ties])};
            }
            return share(c);
        }
        team.barrier();
        int a = 0, z = row.V;                                // the first index with `ties` equal elements ahead of it
        while (a < z) {
            const int mid = a + (z - a) / 2;
            unsigned int c = 0;
            row.each([&](float x, int i) { c += order_key(x) == key && i < mid && in.keeps(x, i); });
            if (team.count(block_count(sm, c)) >= ties) z = mid;
            else a = mid + 1;
        }
        return a < row.V ? Cut{key_value(key), a} : last_of(key_value(key), in);
    }

    // Cut behind the first `goal` elements of the order, by a radix selection on the values' keys (11, 11 and 10 bits): exact
    // for every distribution, three passes.  For a cut below 2^-32 of the largest weight, where the bins end, and where a
    // step of a zone still holds more than the list (22 rows of 22318 in bf16, k = 1789 among them: halving the range of
    // the keys took 96 us, this takes 40).
    __device__ __noinline__ Cut radix_cut(const Cut in, unsigned int goal) {
        unsigned int prefix = 0, above = 0;
#pragma unroll 1
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), width = round == 2 ? 10 : 11;
            const unsigned int mask = (1u << width) - 1u;
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += kSampleThreads) sm.hist[i] = 0u;
            __syncthreads();
            row.each([&](float x, int i) {
                const unsigned int key = order_key(x);
                if (in.keeps(x, i) && (round == 0 || key >> (shift + width) == prefix)) atomicAdd(&sm.hist[mask - ((key >> shift) & mask)], 1u);
            });
            team.barrier();
            merge_counts();
            find_count(goal - above);                        // (there are at least `goal` of them)
            prefix = (prefix << width) | (mask - (unsigned int)*team.of(&sm.zone_lo, 0));
            above += (unsigned int)*team.of(&sm.n_above, 0);
            team.barrier();                                  // (read by all before the next round's answer)
        }
        return tie_cut(in, prefix, goal - above);
    }

    // Cut behind the elements before which less than top_p of the kept weight has come, by halving the range of the keys: exact
    // for every distribution, one pass over the row per step.  For rows whose zone does not fit the list: very many equal
    // tokens, or a cut among tokens below 2^-32 of the largest.  The goal is formed from the same 64-bit sum as what it is
    // compared with (sums of the same terms in the same order, which only grow as terms are added): all of the weight
    // reaches it.  The total of the passes before has its far tail from 32 bits and may exceed that sum.
    __device__ __noinline__ Cut slow_cut(const Cut in, float top_p) {
        auto weight_from = [&](unsigned int key) {
            double w = 0.0;
            row.each([&](float x, int i) { if (in.keeps(x, i) && order_key(x) >= key) w += wt(x); });
            return team.sum(block_sum(sm, w));
        };
        const double goal = (double)top_p * weight_from(0u);
        unsigned int lo = 0, hi = order_key(m);              // the answer: the largest key whose elements at or above it reach the goal
        while (lo < hi) {
            const unsigned int mid = lo + (hi - lo) / 2 + 1;
            if (weight_from(mid) >= goal) lo = mid;
            else hi = mid - 1;
        }
        const double above = weight_from(lo + 1), each_w = wt(key_value(lo));        // (lo is the key of a finite value)
        // elements equal to it, in index order, are kept while the weight before them is below the goal
        unsigned int ties = 1, most = (unsigned int)row.V;
        while (ties < most) {
            const unsigned int mid = ties + (most - ties) / 2;
            if (above + (double)mid * each_w >= goal) most = mid;
            else ties = mid + 1;
        }
        return tie_cut(in, lo, ties);
    }

    __device__ __forceinline__ void open_list() {            // (a barrier of the row lies behind every open_list)
        __syncthreads();
        if (threadIdx.x == 0) sm.n_list = 0;
        team.barrier();
    }
    __device__ __forceinline__ void append(float x, int i) { // to the first block's list
        const int at = atomicAdd(team.of(&sm.n_list, 0), 1);
        if (at < kList) *team.of(&sm.list[at], 0) = list_entry(x, i);
    }
    __device__ __forceinline__ int close_list() {            // entries asked for; they may exceed what the list holds
        team.barrier();
        return *team.of(&sm.n_list, 0);
    }

    // A part of the order where the cut must lie: bins [lo, hi], hi < kBins - 1, and where those hold more than the list
    // takes, steps [fine_lo, fine_hi] of them: kBins even steps from bin lo to bin hi.
    struct Zone {
        int lo, hi, fine_lo, fine_hi;
        __device__ __forceinline__ double start() const { return lo - 0.5; }
        __device__ __forceinline__ double step() const { return (hi - lo + 1) * (1.0 / kBins); }
    };
    __device__ __forceinline__ int fine_step(const Zone &z, float x) const {
        const int f = (int)((wt.depth(x) - z.start()) * ((double)kBins / (z.hi - z.lo + 1)));
        return ::min(::max(f, 0), kBins - 1);
    }

    // Gathers the kept elements of the zone into the first block's list (kCount: counts them by their steps instead).
    // kAbove: *above receives the weight of the kept elements ahead of the zone; sm.part the warps' shares of it.
    template <bool kAbove, bool kFine, bool kCount>
    __device__ __forceinline__ int gather(const Cut &in, const Zone z, double *above) {
        if (kCount) {
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += kSampleThreads) sm.hist[i] = 0u;
            __syncthreads();
        } else {
            open_list();
        }
        double w = 0.0;
        const float bottom = fmaxf(wt.low, in.x);
        row.each([&](float x, int i) {
            if (x >= bottom) {
                if (x == in.x && i >= in.index) return;
                double q, s;
                const int b = wt.split(x, q, s);
                if (b > z.hi) return;
                bool ahead = b < z.lo;
                if (!ahead) {
                    if (kCount) {
                        atomicAdd(&sm.hist[fine_step(z, x)], 1u);
                        return;
                    }
                    const int f = kFine ? fine_step(z, x) : 0;
                    ahead = kFine && f < z.fine_lo;
                    if (!ahead && (!kFine || f <= z.fine_hi)) append(x, i);
                }
                if (kAbove && ahead) w = fma(q, s, w);
            }
        });
        if (kAbove) {
            *above = team.sum(block_sum(sm, w));
            if (threadIdx.x < kSampleWarps) sm.part[threadIdx.x] = sm.wsum[threadIdx.x];
        }
        if (kCount) {
            if (!kAbove) team.barrier();
            merge_counts();
            return 0;
        }
        return close_list();
    }

    // The blocks' counts summed in the first one's (a barrier of the row lies behind the counting).
    __device__ __forceinline__ void merge_counts() {
        if (kTeam && team.rank == 0) {
            for (int i = threadIdx.x; i < kBins; i += kSampleThreads) {
                unsigned int c[kMaxTeam], all = sm.hist[i];
#pragma unroll
                for (int r = 1; r < kMaxTeam; ++r) c[r] = r < team.size ? *team.of(&sm.hist[i], r) : 0u;
#pragma unroll
                for (int r = 1; r < kMaxTeam; ++r) all += c[r];
                sm.hist[i] = all;
            }
        }
    }

    // The cut of top_p by counts per value: every value's weight is formed once instead of every token's (4096 rows of
    // 32000: 536 -> 439 us).  False where the cut lies among the values next to zero or weights that count lie
    // beyond the bins (negative and larger than twice the largest logit, and 32).  sm.part: the warps' kept weights.
    __device__ __forceinline__ bool value_cut(float top_p, Cut &cut) {
        constexpr int PER = (kValues + kSampleThreads - 1) / kSampleThreads;
        unsigned int *const count = reinterpret_cast<unsigned int *>(value_weight + kValues);
        const int top = (int)((__float_as_uint(fmaxf(fabsf(m), 16.f)) >> 16) | 0x7fu), a0 = top - kSide + 1;   // of the magnitudes' bits
        auto bin = [&](unsigned int bits, int &t) {           // bits: the value's, as a float's; t: 0 .. kSide - 1 where it has a bin
            t = (int)((bits >> 16) & 0x7fffu) - a0;
            return (int)bits < 0 ? kSide + 1 + t : kSide - 1 - t;
        };
        auto value = [&](int b) {
            const unsigned int a = b < kSide ? (unsigned int)(top - b) : (b == kSide ? 0u : (unsigned int)(a0 + b - kSide - 1) | 0x8000u);
            return __uint_as_float(a << 16);
        };
        __syncthreads();
        for (int i = threadIdx.x; i < kValues; i += kSampleThreads) count[i] = 0u;
        __syncthreads();
        double w_near = 0.0;
        float w_low = 0.f;
        unsigned int beyond = 0;
        row.each([&](float x, int) {
            int t;
            const int b = bin(__float_as_uint(x), t);
            if ((unsigned int)t < (unsigned int)kSide) {
                atomicAdd(&count[b], 1u);
            } else if (t < 0) {
                w_near += wt(x);
            } else {
                beyond |= x >= wt.low;
                w_low += wt.small(x);
            }
        });
        const double near_zero = team.sum(block_sum(sm, w_near)), low = team.sum(block_sum(sm, (double)w_low));
        if (team.count((unsigned int)__syncthreads_or((int)beyond)) != 0) return false;
        // the values' weights, in every block; their counts and running weights in the first one
        double mass[PER], mine = 0.0;
        unsigned int c[PER];
#pragma unroll 1
        for (int q = 0; q < PER; ++q) {
            const int b = threadIdx.x * PER + q;
            if (b < kValues) value_weight[b] = wt(value(b));
        }
        if (!kTeam || team.rank == 0) {
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int b = threadIdx.x * PER + q;
                c[q] = b < kValues ? count[b] : 0u;
                if (kTeam && b < kValues)
                    for (int r = 1; r < team.size; ++r) c[q] += *team.of(&count[b], r);
                mass[q] = b == kSide ? near_zero : (c[q] ? c[q] * value_weight[b] : 0.0);
                mine += mass[q];
            }
            double all, before = block_scan(mine, sm.wsum, &all);
            const double goal = (double)top_p * (all + low);
            if (threadIdx.x == 0) sm.value_at = -1;
            __syncthreads();
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int b = threadIdx.x * PER + q;
                // (two threads' running sums are rounded apart: both may claim the goal at their border, so the answer is one store)
                if (b != kSide && before < goal && before + mass[q] >= goal) {
                    // of the equal tokens those before which less than the goal has come
                    const double each_w = value_weight[b], n = ceil((goal - before) / each_w);
                    unsigned int ties = n < 1.0 ? 1u : (n > (double)c[q] ? c[q] : (unsigned int)n);
                    while (ties > 1 && !(before + (double)(ties - 1) * each_w < goal)) --ties;
                    while (ties < c[q] && before + (double)ties * each_w < goal) ++ties;
                    sm.value_at = ((long long)b << 32) | ties;
                }
                before += mass[q];
            }
        }
        team.barrier();
        const long long value_at = *team.of(&sm.value_at, 0);
        if (value_at < 0) return false;
        const int at = (int)(value_at >> 32);
        const unsigned int ties = (unsigned int)value_at;
        // kept weights and equal tokens by warp
        double w = 0.0;
        unsigned int equal = 0;
        row.each([&](float x, int) {
            int t;
            const int b = bin(__float_as_uint(x), t);
            if ((unsigned int)t < (unsigned int)kSide) {
                if (b < at) w += value_weight[b];
                else equal += b == at;
            } else if (t < 0 && at > kSide) {
                w += wt(x);
            }
        });
        w = warp_sum(w);
        equal = __reduce_add_sync(0xffffffffu, equal);
        const int warp = threadIdx.x >> 5;
        __syncthreads();
        if ((threadIdx.x & 31) == 0) { sm.part[warp] = w; sm.wcount[warp] = equal; }
        __syncthreads();
        unsigned int in_block = 0;
#pragma unroll
        for (int i = 0; i < kSampleWarps; ++i) in_block += sm.wcount[i];
        double ahead;
        team.sum((double)in_block, ahead);
        // the equal tokens of the blocks and warps ahead come first; the first one left out lies in warp `edge`, if in this block
        int left = (int)ties - (int)ahead, edge = -1, edge_left = 0;
#pragma unroll
        for (int i = 0; i < kSampleWarps; ++i) {
            const int n = (int)sm.wcount[i];
            if (left >= 0 && left < n) { edge = i; edge_left = left; }
            if ((int)threadIdx.x == i) sm.part[i] += (double)::min(::max(left, 0), n) * value_weight[at];
            left -= n;
        }
        int index = INT_MAX;
        if (edge >= 0) {
            const float v = value(at);
            const int first = row.warp_first(edge), n = row.warp_first(edge + 1) - first, per = (n + kSampleThreads - 1) / kSampleThreads;
            const int v0 = first + ::min(n, (int)threadIdx.x * per), v1 = first + ::min(n, ((int)threadIdx.x + 1) * per);
            unsigned int n_mine = 0, all;
            for (int k = v0; k < v1; ++k) {
                float x[VE];
                row.load(k, x);
#pragma unroll
                for (int e = 0; e < VE; ++e) n_mine += x[e] == v;
            }
            unsigned int seen = block_scan(n_mine, sm.wcount, &all);
            if (seen <= (unsigned int)edge_left && (unsigned int)edge_left < seen + n_mine)
                for (int k = v0; k < v1; ++k) {
                    float x[VE];
                    row.load(k, x);
                    for (int e = 0; e < VE; ++e)
                        if (x[e] == v && seen++ == (unsigned int)edge_left) sm.answer = row.index(k, e);
                }
            __syncthreads();
            index = sm.answer;
        }
        cut = Cut{value(at), team.min_int(index)};
        __syncthreads();
        return true;
    }

    __device__ __forceinline__ bool long_row() const { return !kStaged && row.V > kLongTail; }     // (rows in shared memory are shorter)

    // Weight of this thread's kept elements below `low`, in 64 bits (for rows longer than kLongTail; out of line: the code of
    // the pass that all rows take is what has to be short).
    __device__ __noinline__ double deep_weight(const Cut &in) const {
        double w = 0.0;
        row.each([&](float x, int i) { if (x < wt.low && in.keeps(x, i)) w += wt(x); });
        return w;
    }

    // Counts of the kept elements by bin, summed over the row's blocks in the first one, and (kWeight) their weight.
    // The histogram shares its memory with the list: a barrier of the row lies between the uses.
    // kAll: nothing is cut off yet.
    template <bool kWeight, bool kAll>
    __device__ __forceinline__ double histogram(const Cut &in) {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kSampleThreads) sm.hist[i] = 0u;
        __syncthreads();
        double w = 0.0;
        float w_low = 0.f;
        unsigned int low = 0;                                // the last bin may hold most of the row: counted in registers
        const float top = kAll ? wt.low : fmaxf(wt.low, in.x);
        const bool deep = kAll || in.x < wt.low;             // are any elements of the last bin kept?
        row.each([&](float x, int i) {
            if (x >= top) {
                if (!kAll && x == in.x && i >= in.index) return;
                double q, s;
                const int b = wt.split(x, q, s);
                atomicAdd(&sm.hist[::min(b, kBins - 1)], 1u);
                if (kWeight) w = fma(q, s, w);
            } else if (deep && (kAll || in.keeps(x, i))) {
                low += kWeight || x > -INFINITY;             // (with weights the last bin's count only bounds: -inf may be in it)
                if (kWeight) w_low += wt.small(x);
            }
        });
        low = __reduce_add_sync(0xffffffffu, low);
        if ((threadIdx.x & 31) == 0) atomicAdd(&sm.hist[kBins - 1], low);
        double sum = 0.0;
        if (kWeight) {
            if (long_row()) {
                w_low = 0.f;
                w += deep_weight(in);
            }
            sum = team.sum(block_sum(sm, w + (double)w_low));
        } else {
            team.barrier();
        }
        merge_counts();
        return sum;
    }

    // First bin at which the running count reaches `goal` (sm.zone_lo = -1: none does), the count before it
    // (sm.n_above) and in it (sm.total).
    __device__ __forceinline__ void find_count(unsigned int goal) {
        constexpr int PER = kBins / kSampleThreads;
        __syncthreads();
        if (!kTeam || team.rank == 0) {
            unsigned int c[PER], mine = 0, all;
#pragma unroll
            for (int u = 0; u < PER; ++u) mine += c[u] = sm.hist[threadIdx.x * PER + u];
            unsigned int before = block_scan(mine, sm.wcount, &all);
            if (threadIdx.x == 0) sm.zone_lo = -1;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                if (before < goal && before + c[u] >= goal) {
                    sm.zone_lo = threadIdx.x * PER + u;
                    sm.n_above = (int)before;
                    sm.total = c[u];
                }
                before += c[u];
            }
        }
        team.barrier();
    }

    // Bins that may hold the cut of a running weight, `total` being the weight of all.  With every element of a bin taken
    // at the bin's upper or lower end, running sums `up` and `dn` enclose the running weight M_b at the end of bin b from
    // the front, and what is left behind it encloses it from the back (a cut close to the end has little behind it):
    //     max(dn_b, total - (up_all - up_b)) <= M_b <= min(up_b, total - (dn_all - dn_b)).
    // kFine: the same for the steps of a zone, from the front alone, `total` being the weight ahead of the zone.
    // sm.zone_lo: the first bin where the upper bound reaches the goal, sm.zone_hi: the first where the lower one does,
    // sm.total: elements up to zone_hi, sm.n_above: before zone_lo.  Bins' edges are formed in 32 bits: 1e-5 relative covers that; the last bin has no
    // lower end.
    template <bool kFine>
    __device__ __forceinline__ void find_weight(double goal, double total, const Zone z) {
        constexpr int PER = kBins / kSampleThreads;
        __syncthreads();
        if (!kTeam || team.rank == 0) {
            unsigned int c[PER];
            double up[PER], dn[PER];
            Sums mine{0.0, 0.0, 0u}, all;
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int b = threadIdx.x * PER + u;
                c[u] = sm.hist[b];
                if (kFine) {
                    up[u] = c[u] * (exp2(-(z.start() + b * z.step()) / kBinsPerOctave) * (1.0 + 1e-9));
                    dn[u] = c[u] * (exp2(-(z.start() + (b + 1) * z.step()) / kBinsPerOctave) * (1.0 - 1e-9));
                } else {
                    const float edge = exp2f((0.5f - (float)b) / kBinsPerOctave);
                    up[u] = c[u] * ((double)edge * 1.00001);
                    dn[u] = b == kBins - 1 ? 0.0 : c[u] * ((double)edge * (0.98922 * 0.99999));   // 2^(-1/64) = 0.989228...
                }
                mine.c += c[u];
                mine.up += up[u];
                mine.dn += dn[u];
            }
            Sums run = block_scan3(mine, reinterpret_cast<Sums *>(sm.scan), &all);
            if (threadIdx.x == 0) { sm.zone_lo = kBins - 1; sm.zone_hi = kBins - 1; sm.total = all.c; sm.n_above = 0; }
            __syncthreads();
            int lo = INT_MAX, hi = INT_MAX;                  // this thread's first bins that reach the goal
            unsigned int run_c[PER];
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int b = threadIdx.x * PER + u;
                run.up += up[u];
                run.dn += dn[u];
                run_c[u] = run.c += c[u];
                if ((kFine ? total + run.up : fmin(run.up, total - (all.dn - run.dn))) >= goal) lo = ::min(lo, b);
                if ((kFine ? total + run.dn : fmax(run.dn, total - (all.up - run.up))) >= goal) hi = ::min(hi, b);
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_min_sync(0xffffffffu, hi);
            if ((threadIdx.x & 31) == 0) {
                atomicMin(&sm.zone_lo, lo);
                atomicMin(&sm.zone_hi, hi);
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                if ((int)threadIdx.x * PER + u == sm.zone_hi) sm.total = run_c[u];
                if ((int)threadIdx.x * PER + u == sm.zone_lo) sm.n_above = (int)(run_c[u] - c[u]);
            }
        }
        team.barrier();
    }

    // Weight of an element for the draw: ahead of the cut and w >= floor.
    __device__ __forceinline__ double kept_weight(const Cut &cut, double floor, float x, int i) const {
        if (!cut.keeps(x, i)) return 0.0;
        const double w = wt(x);
        return w >= floor ? w : 0.0;
    }

    // sm.part: the warps' kept weights.
    __device__ __forceinline__ void sum_kept(const Cut &cut, double floor, bool exact) {
        double mine = 0.0;
        float low = 0.f;
        if (floor > 0.0 || exact || long_row()) {
            row.each([&](float x, int i) { mine += kept_weight(cut, floor, x, i); });
        } else {
            const float top = fmaxf(wt.low, cut.x);
            const bool deep = cut.x < wt.low;
            row.each([&](float x, int i) {
                if (x >= top) {
                    if (x == cut.x && i >= cut.index) return;
                    double q, s;
                    wt.split(x, q, s);
                    mine = fma(q, s, mine);
                } else if (deep && cut.keeps(x, i)) {
                    low += wt.small(x);
                }
            });
        }
        mine = warp_sum(mine + (double)low);
        if ((threadIdx.x & 31) == 0) sm.part[threadIdx.x >> 5] = mine;
        __syncthreads();
    }

    // The token, given the warps' kept weights in sm.part: the block that holds it walks one warp's range.
    __device__ __forceinline__ int locate(const Cut &cut, double floor, double u) {
        double block = 0.0, before;
        for (int w = 0; w < kSampleWarps; ++w) block += sm.part[w];
        const double goal = u * team.sum(block, before);
        int seg = -1;
        for (int w = 0; w < kSampleWarps; ++w) {
            const double s = sm.part[w];
            if (s > 0.0) {
                if (before + s > goal) { seg = w; break; }
                before += s;
            }
        }
        // the first block of the row with such a warp
        const int owner_block = team.min_int(seg >= 0 ? team.rank : INT_MAX);
        if (owner_block == INT_MAX) {                         // uniform = 1 (or rounding): the last one with a weight
            int last = -1;
            row.each([&](float x, int i) { if (kept_weight(cut, floor, x, i) > 0.0) last = ::max(last, i); });
            last = __reduce_max_sync(0xffffffffu, last);
            __syncthreads();
            if (threadIdx.x == 0) sm.answer = -1;
            __syncthreads();
            if ((threadIdx.x & 31) == 0) atomicMax(&sm.answer, last);
            __syncthreads();
            last = -1 - team.min_int(-1 - sm.answer);         // the largest
            return team.rank == 0 ? last : kElsewhere;
        }
        if (owner_block != team.rank) return kElsewhere;
        const int first = row.warp_first(seg), n = row.warp_first(seg + 1) - first;
        const int per = (n + kSampleThreads - 1) / kSampleThreads;
        const int v0 = first + ::min(n, (int)threadIdx.x * per), v1 = first + ::min(n, ((int)threadIdx.x + 1) * per);
        double mine = 0.0;
        for (int v = v0; v < v1; ++v) {
            float x[VE];
            row.load(v, x);
#pragma unroll
            for (int e = 0; e < VE; ++e) mine += kept_weight(cut, floor, x[e], row.index(v, e));
        }
        __syncthreads();
        if (threadIdx.x == 0) { sm.first_thread = INT_MAX; sm.answer = -1; }
        double all, running = before + block_scan(mine, sm.wsum, &all);
        // the first thread whose range passes the goal; should rounding leave none, the last with a weight
        if (mine > 0.0 && running + mine > goal) atomicMin(&sm.first_thread, (int)threadIdx.x);
        if (mine > 0.0) atomicMax(&sm.answer, (int)threadIdx.x);
        __syncthreads();
        const int owner = sm.first_thread != INT_MAX ? sm.first_thread : sm.answer;
        __syncthreads();
        if ((int)threadIdx.x == owner) {
            int best = -1;
            bool found = false;
            for (int v = v0; v < v1 && !found; ++v) {
                float x[VE];
                row.load(v, x);
                for (int e = 0; e < VE && !found; ++e) {
                    const double w = kept_weight(cut, floor, x[e], row.index(v, e));
                    if (w > 0.0) {
                        running += w;
                        best = row.index(v, e);
                        found = running > goal;
                    }
                }
            }
            sm.answer = best;
        }
        __syncthreads();
        return sm.answer;
    }

    // The k-th largest of the block's thread maxima, rounded down to the upper sixteen bits of its key: two steps of a
    // radix selection with 256 counts each.
    __device__ __forceinline__ unsigned int kth_maximum(float thread_max, int k) {
        const unsigned int mine = order_key(thread_max);
        unsigned int prefix = 0;
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const int shift = 24 - 8 * step;
            __syncthreads();
            if (threadIdx.x < 256) sm.hist[threadIdx.x] = 0u;
            __syncthreads();
            if (step == 0 || mine >> 24 == prefix) atomicAdd(&sm.hist[(mine >> shift) & 255u], 1u);
            __syncthreads();
            if (threadIdx.x < 32) {                          // lane l: counts 255 - 8 l and the seven below
                unsigned int c[8], sum = 0, before;
#pragma unroll
                for (int u = 0; u < 8; ++u) sum += c[u] = sm.hist[255 - 8 * threadIdx.x - u];
                before = sum;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const unsigned int o = __shfl_up_sync(0xffffffffu, before, off);
                    if ((int)threadIdx.x >= off) before += o;
                }
                before -= sum;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    if ((int)before < k && (int)(before + c[u]) >= k) {
                        sm.zone_lo = 255 - 8 * (int)threadIdx.x - u;
                        sm.n_above = (int)before;
                    }
                    before += c[u];
                }
            }
            __syncthreads();
            prefix = step == 0 ? (unsigned int)sm.zone_lo : (prefix << 8) | (unsigned int)sm.zone_lo;
            k -= sm.n_above;
        }
        return prefix << 16;
    }

    // The cut that the first block found, told to all.
    __device__ __forceinline__ Cut share(const Cut &cut) {
        if (threadIdx.x == 0 && team.rank == 0) { sm.cut_x = cut.x; sm.cut_i = cut.index; }
        team.barrier();
        return Cut{*team.of(&sm.cut_x, 0), *team.of(&sm.cut_i, 0)};
    }

    __device__ __forceinline__ int sample(float thread_max, int top_k, float top_p, float min_p, float uniform) {
        // (nothing exceeds all of the weight: a rounded sum must not, so 1 becomes a number that no sum reaches)
        const double u = uniform < 1.f ? (double)uniform : 2.0, floor = min_p > 0.f ? (double)min_p : 0.0;
        const bool first = !kTeam || team.rank == 0;
        Cut cut{-INFINITY, INT_MIN};                          // keeps everything above -inf (padding has indexes below 0)
        const bool p_on = top_p < 1.f;
        if (top_k > 0 && top_k < row.V) {
            if (top_k <= kSampleThreads) {
                // Lower bounds of the k-th largest token: the k-th largest of a block's thread maxima, and the smallest of
                // the blocks' ceil(k / blocks)-th largest.
                unsigned int key = team.max_key(kth_maximum(thread_max, top_k));
                // (the first admits about k tokens per block: the second is worth its time where those may not fit the list)
                if (kTeam && team.size * top_k > kList / 2) key = ::max(key, team.min_key(kth_maximum(thread_max, (top_k + team.size - 1) / team.size)));
                const float bound = key <= order_key(-INFINITY) ? -INFINITY : key_value(key);
                open_list();
                row.each([&](float x, int i) { if (x >= bound && x > -INFINITY) append(x, i); });
                int n = close_list();
                if (n <= kList) {
                    if (!first) return kGone;
                    sort_list(sm, n);
                    n = ::min(n, top_k);
                    return finish_list(n, p_on, top_p, -1.0, floor, u);
                }
                team.barrier();                               // (the first block's list is done with)
            }
            histogram<false, true>(cut);
            find_count((unsigned int)top_k);
            const int zone = *team.of(&sm.zone_lo, 0), above = *team.of(&sm.n_above, 0);
            const unsigned int inside = *team.of(&sm.total, 0);
            if (zone >= 0) {                                  // at least k tokens above -inf
                bool done = false;
                if (zone < kBins - 1) {
                    Zone z{zone, zone, 0, kBins - 1};
                    int ahead = above, n;
                    if (inside <= kList) {
                        n = gather<false, false, false>(cut, z, nullptr);
                    } else {                                  // step by step
                        gather<false, false, true>(cut, z, nullptr);
                        find_count((unsigned int)(top_k - above));
                        z.fine_lo = z.fine_hi = ::max(*team.of(&sm.zone_lo, 0), 0);
                        ahead += *team.of(&sm.n_above, 0);
                        n = gather<false, true, false>(cut, z, nullptr);
                    }
                    if (n >= 1 && n <= kList) {
                        Cut c = cut;
                        if (first) {
                            sort_list(sm, n);
                            const bool within = top_k - ahead < n;
                            const unsigned long long e = sm.list[within ? top_k - ahead : n - 1];
                            c = Cut{entry_value(e), within ? entry_index(e) : INT_MAX};
                        }
                        cut = share(c);
                        done = true;
                    }
                }
                if (!done) cut = radix_cut(cut, (unsigned int)top_k);
            }
            team.barrier();
        }
        bool cut_by_value = false;
        if constexpr (kByValue) {
            if (p_on && cut.x == -INFINITY) {
                cut_by_value = value_cut(top_p, cut);
                if (cut_by_value && floor == 0.0 && u > 0.0) return locate(cut, 0.0, u);
            }
        }
        if (p_on && !cut_by_value) {
            const double Z = cut.x == -INFINITY ? histogram<true, true>(cut) : histogram<true, false>(cut);
            const double goal = (double)top_p * Z;
            Zone z{0, 0, 0, kBins - 1};
            find_weight<false>(goal, Z, z);
            z.hi = *team.of(&sm.zone_hi, 0);
            z.lo = ::min(*team.of(&sm.zone_lo, 0), z.hi);
            const unsigned int upto = *team.of(&sm.total, 0), before = (unsigned int)*team.of(&sm.n_above, 0);
            bool done = false;
            if (z.hi < kBins - 1 && upto <= kShort) {         // a short kept set: all of it in the list
                z.lo = 0;
                const int n = gather<false, false, false>(cut, z, nullptr);
                if (!first) return kGone;
                sort_list(sm, n);
                return finish_list(n, true, top_p, Z, floor, u);
            }
            if (z.hi < kBins - 1) {
                double above;
                int n;
                if (upto - before <= kList) {
                    n = gather<true, false, false>(cut, z, &above);
                } else {                                      // step by step
                    gather<true, false, true>(cut, z, &above);
                    find_weight<true>(goal, above, z);
                    z.fine_hi = *team.of(&sm.zone_hi, 0);
                    z.fine_lo = ::min(*team.of(&sm.zone_lo, 0), z.fine_hi);
                    n = gather<true, true, false>(cut, z, &above);
                }
                if (n >= 1 && n <= kList) {
                    Cut c = cut;
                    if (first) {
                        sort_list(sm, n);
                        double sum;
                        const int at = list_cut(sm, wt, n, above, goal, &sum);
                        c = at < n ? Cut{entry_value(sm.list[at]), entry_index(sm.list[at])} : last_of(entry_value(sm.list[n - 1]), cut);
                    }
                    const Cut p_cut = share(c);
                    if (floor == 0.0 && u > 0.0) {
                        // the warps' kept weights: what lies ahead of the zone, and their tokens of the list
                        add_list(n, p_cut);
                        return locate(p_cut, 0.0, u);
                    }
                    cut = p_cut;
                    done = true;
                }
            }
            if (!done) cut = slow_cut(cut, top_p);
        }
        sum_kept(cut, floor, u == 0.0);
        return locate(cut, floor, u);
    }

    // Adds the kept tokens of the first block's list[0, n) to the warps' weights in sm.part, in the list's order.
    __device__ __forceinline__ void add_list(int n, const Cut &cut) {
        if (kTeam && team.rank != 0) {
            for (int i = threadIdx.x; i < n; i += kSampleThreads) sm.list[i] = *team.of(&sm.list[i], 0);
        }
        team.barrier();
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const int i0 = row.index(row.warp_first(w), 0), i1 = row.index(row.warp_first(w + 1), 0);
        double mine = 0.0;
        for (int i = lane; i < n; i += 32) {
            const unsigned long long e = sm.list[i];
            const int at = entry_index(e);
            if (at >= i0 && at < i1 && cut.keeps(entry_value(e), at)) mine += wt(entry_value(e));
        }
        mine = warp_sum(mine);
        __syncwarp();
        if (lane == 0) sm.part[w] += mine;
        __syncthreads();
    }

    // finish_list for the usual few tokens, one per thread: one running sum settles top_p and min_p, and each kept token adds
    // up the weights of the kept ones at or below its index itself.
    __device__ __forceinline__ int finish_short(int n, bool p_on, float top_p, double total, double floor, double u) {
        const int i = threadIdx.x;
        const bool mine = i < n;
        const unsigned long long e = mine ? sm.list[i] : 0ull;
        const double w = mine ? wt(entry_value(e)) : 0.0;
        double sum;
        const double before = block_scan(w, sm.wsum, &sum);
        if (total < 0.0) total = sum;
        // (a prefix: both conditions fall with the order)
        const bool keep = mine && (i == 0 || ((!p_on || before < (double)top_p * total) && w >= floor));
        n = __syncthreads_count(keep);
        if (i < kShort) sm.short_w[i] = keep ? w : 0.0;
        if (i == n - 1) sm.short_sum = before + w;
        if (i == 0) { sm.answer = INT_MAX; sm.first_thread = -1; }
        __syncthreads();
        if (keep && w > 0.0) {
            const int at = entry_index(e);
            double upto = 0.0;
            for (int j = 0; j < n; ++j) upto += entry_index(sm.list[j]) <= at ? sm.short_w[j] : 0.0;
            if (upto > u * sm.short_sum) atomicMin(&sm.answer, at);
            atomicMax(&sm.first_thread, at);                 // the last one with a weight, should none exceed the goal
        }
        __syncthreads();
        return sm.answer != INT_MAX ? sm.answer : sm.first_thread;
    }

    // list[0, n): the first n of the order.  total < 0: the weight that top_p refers to is the list's own.
    __device__ __forceinline__ int finish_list(int n, bool p_on, float top_p, double total, double floor, double u) {
        if (n <= (int)kShort) return finish_short(n, p_on, top_p, total, floor, u);
        if (n > 1 && p_on) {
            double sum;
            if (total < 0.0) {
                list_cut(sm, wt, n, 0.0, INFINITY, &sum);
                total = sum;
            }
            n = ::max(1, list_cut(sm, wt, n, 0.0, (double)top_p * total, &sum));
        }
        if (n > 1 && floor > 0.0) {
            int c = 0;
            for (int i = threadIdx.x; i < n; i += kSampleThreads) c += wt(entry_value(sm.list[i])) >= floor;
            n = ::max(1, (int)block_count(sm, (unsigned int)c));
        }
        return list_draw(sm, wt, n, u);
    }
};

// Copies vectors [v_lo, v_hi) of the row into shared memory at their own 16-byte phase (nothing outside the row is read),
// -inf around the row.
template <typename T>
__device__ __forceinline__ void stage_row(T *dst, const T *src, int V, int phase, int v_lo, int v_hi) {
    constexpr int VE = Vec16<T>::n;
    const T *base = src - phase;
    for (int v = v_lo + threadIdx.x; v < v_hi; v += kSampleThreads) {
        const int i0 = v * VE - phase;
        T *d = dst + (v - v_lo) * VE;
        if (i0 >= 0 && i0 + VE <= V) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(d)), "l"(base + (size_t)v * VE) : "memory");
        } else {
            for (int e = 0; e < VE; ++e) d[e] = (i0 + e >= 0 && i0 + e < V) ? src[i0 + e] : from_float<T>(-INFINITY);
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}

// Is a parameter of sequence b out of range, or one of the uniform numbers that this thread looks at?
template <int kThreads>
__device__ __forceinline__ bool bad_sequence(const SampleArgs &a, int b, float Tm, float top_p, float min_p) {
    bool bad = !(Tm >= 0.f) || Tm == INFINITY || !(top_p == top_p) || !(min_p <= 1.f);
    for (int i = threadIdx.x; i < a.R; i += kThreads) {
        const float x = a.uniform[(size_t)b * a.N + i];
        bad |= !(x >= 0.f && x <= 1.f);
    }
    return bad;
}

template <typename T, bool kStaged, bool kTeam, bool kVerify>
__global__ void __launch_bounds__(kSampleThreads, 2)
sample_kernel(const SampleArgs a) {
    constexpr int VE = Vec16<T>::n;
    extern __shared__ uint4 s_dyn[];
    __shared__ SampleSmem sm;
    __shared__ int s_last;
    Team<kTeam> team{sm, 0, 1, 0};
    if (kTeam) {
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(team.rank));
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(team.size));
    }
    const int unit = kTeam ? (int)blockIdx.x / team.size : (int)blockIdx.x;
    const int b = unit / a.R, r = unit - b * a.R;
    if (threadIdx.x < kBinsPerOctave) sm.pow2[threadIdx.x] = exp2((double)threadIdx.x / kBinsPerOctave);
    // The launch is serialized programmatically behind the kernel ahead of it in the stream: from here on everything
    // that kernel wrote may be read.  A kernel serialized behind this one may set itself up meanwhile.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const T *src = static_cast<const T *>(a.logits) + ((size_t)b * a.N + r) * a.V;
    Row<T, kStaged> row;
    row.phase = (int)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
    row.V = a.V;
    const int vecs = (row.phase + a.V + VE - 1) / VE, share = (vecs + team.size - 1) / team.size;
    row.v_lo = min(vecs, team.rank * share);
    row.v_hi = min(vecs, row.v_lo + share);
    row.peak = false;
    if (kStaged) stage_row<T>(reinterpret_cast<T *>(s_dyn), src, a.V, row.phase, row.v_lo, row.v_hi);
    row.base = kStaged ? reinterpret_cast<const T *>(s_dyn) : src - row.phase;
    // parameters of the sequence; every block of it comes to the same decision
    const float Tm = a.temperature ? a.temperature[b] : 1.f;
    const int top_k = a.top_k ? a.top_k[b] : 0;
    const float top_p = a.top_p ? a.top_p[b] : 1.f;
    const float min_p = a.min_p ? a.min_p[b] : 0.f;
    bool bad = a.checked ? a.status[b] != HT_STATUS_OK : bad_sequence<kSampleThreads>(a, b, Tm, top_p, min_p);
    if (kStaged) asm volatile("cp.async.wait_group 0;" ::: "memory");
    bad = __syncthreads_or(bad);
    int token = -1;
    if (!bad) {
        // largest value (NaN aside); staged rows are rewritten without NaN
        float mx = -INFINITY;
        {
            const int w = threadIdx.x >> 5, end = row.warp_first(w + 1);
            for (int v = row.warp_first(w) + (threadIdx.x & 31); v < end; v += 32) {
                float x[VE];
                row.load(v, x);
                bool nan = false;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    nan |= !(x[e] == x[e]);
                    mx = fmaxf(mx, x[e]);                    // (the other operand where one is NaN)
                }
                if (kStaged && nan) {
                    T *d = reinterpret_cast<T *>(s_dyn) + (v - row.v_lo) * VE;
                    for (int e = 0; e < VE; ++e)
                        if (!(x[e] == x[e])) d[e] = from_float<T>(-INFINITY);
                }
            }
        }
        float m = mx;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
        if ((threadIdx.x & 31) == 0) sm.wmax[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSampleWarps; ++w) m = fmaxf(m, sm.wmax[w]);
        m = team.max(m);
        if (m == -INFINITY) {
            // nothing above -inf: the first -inf, or 0 in a row of NaNs, as the greedy verification has it
            if (team.rank == 0) {
                if (threadIdx.x == 0) sm.answer = INT_MAX;
                __syncthreads();
                for (int i = threadIdx.x; i < a.V; i += kSampleThreads)
                    if (to_float<T>(src[i]) == -INFINITY) { atomicMin(&sm.answer, i); break; }
                __syncthreads();
                token = sm.answer == INT_MAX ? 0 : sm.answer;
            } else {
                token = kElsewhere;
            }
        } else if (Tm == 0.f || top_k == 1 || top_p <= 0.f) {
            if (threadIdx.x == 0) sm.answer = INT_MAX;
            __syncthreads();
            int first = INT_MAX;
            row.each([&](float x, int i) { if (x == m) first = min(first, i); });
            first = __reduce_min_sync(0xffffffffu, first);
            if ((threadIdx.x & 31) == 0) atomicMin(&sm.answer, first);
            __syncthreads();
            token = team.min_int(sm.answer);
            if (team.rank != 0) token = kElsewhere;
        } else {
            if (m == INFINITY) {                             // the +inf tokens share the weight, the others have none
                if (kStaged) {
                    T *d = reinterpret_cast<T *>(s_dyn);
                    for (int i = threadIdx.x; i < (row.v_hi - row.v_lo) * VE; i += kSampleThreads)
                        d[i] = from_float<T>(to_float<T>(d[i]) == INFINITY ? 0.f : -INFINITY);
                }
                row.peak = true;
                m = 0.f;
                mx = mx == INFINITY ? 0.f : -INFINITY;
                __syncthreads();
            }
            const double log2e = 1.4426950408889634074;
            // (`low` may lie a little inside the last bin or the one before: what is not below it is told by its bin)
            const float low = (float)((double)m - (double)(kBins - 1) / kBinsPerOctave / log2e * (double)Tm);
            Sampler<T, kStaged, kTeam> s{sm, team, row,
                                         Weights{(double)m, kBinsPerOctave * log2e / (double)Tm, m, fmaxf(low, -FLT_MAX),
                                                 (float)fmin(log2e / (double)Tm, 1e30), sm.pow2}, m,
                                         reinterpret_cast<double *>(s_dyn + share)};     // (the same place in every block)
            token = s.sample(mx, top_k, top_p, min_p, a.uniform[(size_t)b * a.N + r]);
        }
    }
    // A block leaves only when no other block of the row may still read its shared memory (the barrier does not wait for
    // blocks that have left).
    if (kTeam && token != kGone) team.barrier();
    if (bad ? team.rank != 0 : token <= kElsewhere) return;
    if (!kVerify) {
        if (threadIdx.x == 0) {
            a.token[(size_t)b * a.N + r] = token;
            if (r == 0 && !a.checked) a.status[b] = bad ? HT_STATUS_BAD_PARAM : HT_STATUS_OK;
        }
        return;
    }
    // Verification: the block that stores a sequence's last token searches its tree (the count protocol of the greedy
    // verification).  Rows that are not sampled read -1.
    if (r == 0)
        for (int i = a.R + threadIdx.x; i < a.N; i += kSampleThreads) a.token[(size_t)b * a.N + i] = -1;
    __syncthreads();
    if (threadIdx.x == 0) {
        a.token[(size_t)b * a.N + r] = token;
        unsigned before;
        __threadfence();
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], %2;" : "=r"(before) : "l"(a.accept_len + b), "r"(kTicket) : "memory");
        s_last = before / kTicket == (unsigned)(a.R - 1);
    }
    __syncthreads();
    if (!s_last) return;
    if (bad) {
        for (int j = threadIdx.x; j < a.max_path; j += kSampleThreads) a.accept_path[(size_t)b * a.max_path + j] = -1;
        if (threadIdx.x == 0) {
            a.status[b] = HT_STATUS_BAD_PARAM;
            a.next_token[b] = -1;
            a.accept_len[b] = 0;
        }
        return;
    }
    TreeSmem &ts = *reinterpret_cast<TreeSmem *>(s_dyn);      // the row is done with
    if (threadIdx.x == 0) ts.staged_b = -1;
    __syncthreads();
    stage_tree(ts, b, a.tokens, a.parent, a.root_pred, a.N, a.T);
    accept_sequence(ts, b, a.tokens, a.parent, a.root_pred, a.token, a.N, a.T, a.max_path, a.accept_len, a.accept_path, a.next_token,
                    a.status, 0);
}

// Shared memory a block may take beyond its static part (227 KB per SM in all).
constexpr size_t kSampleDynMax = 227 * 1024 - sizeof(SampleSmem) - 1024;
static_assert(kSampleDynMax / sizeof(__nv_bfloat16) * kMaxTeam <= kLongTail, "rows in shared memory sum the far tail in 32 bits");

template <typename T, bool kStaged, bool kTeam, bool kVerify>
static cudaError_t launch_shape(const SampleArgs &a, int team, size_t smem, cudaStream_t s) {
    static bool raised[64];                                  // per device: the kernel's shared memory limit
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    auto kernel = sample_kernel<T, kStaged, kTeam, kVerify>;
    if (dev < 0 || dev >= 64 || !raised[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSampleDynMax);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) raised[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((long long)a.B * a.R * team));
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)team;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kTeam ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T>
cudaError_t launch_sample_t(const SampleArgs &a, const char *what, cudaStream_t s) {
    // Blocks per row: as many as it takes for the slices to fit shared memory two to an SM, and, where the rows are too few to
    // fill the GPU, slices of 8 KB -- but a row of up to 32 KB stays whole, since a cluster's steps cost more than they share.
    // Whole / shared out, 16 rows: 16000 in bf16, top-p 17.1 / 29.3 us, top-k 9.1 / 12.2 us, no filter 11.5 / 11.7 us; 8000 in
    // fp32 15.8 / 21.4, 8.4 / 11.7, 8.7 / 10.1 us; beyond, one row of 32000 in fp16 by two blocks / eight: no filter
    // 14.4 / 11.1 us, top-p 27.5 / 23.0 us.
    const long long rows = (long long)a.B * a.R;
    const size_t by_value = ByValue<T, true>::on ? kValueBytes : 0;
    auto slice = [&](int team) { return (((size_t)a.V * sizeof(T) + 15 + 15) / 16 + team - 1) / team * 16 + by_value; };
    const bool divisible = (size_t)a.V * sizeof(T) > 32768;
    int team = 1;
    while (team < kMaxTeam && (slice(team) > kSampleDynMax / 2 || (divisible && rows * team <= sm_count() && slice(team) - by_value > 8192))) team *= 2;
    const bool staged = slice(team) <= kSampleDynMax;
    const size_t tree = a.tokens ? sizeof(TreeSmem) : 0;
    const size_t smem = staged && slice(team) > tree ? slice(team) : tree;
    trace("%s -> %d block(s) per row, %s", what, team, staged ? "staged" : "from global memory");
    if (a.tokens) {
        if (!staged) return launch_shape<T, false, true, true>(a, team, smem, s);
        return team > 1 ? launch_shape<T, true, true, true>(a, team, smem, s) : launch_shape<T, true, false, true>(a, team, smem, s);
    }
    if (!staged) return launch_shape<T, false, true, false>(a, team, smem, s);
    return team > 1 ? launch_shape<T, true, true, false>(a, team, smem, s) : launch_shape<T, true, false, false>(a, team, smem, s);
}

#ifndef HT_SAMPLE_DTYPE
#define HT_SAMPLE_DTYPE 0
#endif
#if HT_SAMPLE_DTYPE == 1
template cudaError_t launch_sample_t<__half>(const SampleArgs &, const char *, cudaStream_t);
#elif HT_SAMPLE_DTYPE == 2
template cudaError_t launch_sample_t<__nv_bfloat16>(const SampleArgs &, const char *, cudaStream_t);
#else
static_assert(HT_F32 == 0 && HT_F16 == 1 && HT_BF16 == 2, "the numbers of the types");
extern template cudaError_t launch_sample_t<__half>(const SampleArgs &, const char *, cudaStream_t);
extern template cudaError_t launch_sample_t<__nv_bfloat16>(const SampleArgs &, const char *, cudaStream_t);

// The status words ahead of a call with more than kManyRows rows per sequence, where every block's own look at all of its
// sequence's uniform numbers would add up to the square of the rows.  One sequence of 1000 tokens in bf16, top-p, by the
// blocks' own looks / with this kernel: 256 rows 17.3 / 19.2 us, 2048 rows 99.9 / 99.7 us, 32768 rows 1731 / 1484 us.
constexpr int kManyRows = 2048, kCheckThreads = 1024;
__global__ void __launch_bounds__(kCheckThreads)
check_sequences_kernel(const SampleArgs a) {
    const int b = blockIdx.x;
    const bool bad = __syncthreads_or(bad_sequence<kCheckThreads>(a, b, a.temperature ? a.temperature[b] : 1.f, a.top_p ? a.top_p[b] : 1.f,
                                                                  a.min_p ? a.min_p[b] : 0.f));
    if (threadIdx.x == 0) a.status[blockIdx.x] = bad ? HT_STATUS_BAD_PARAM : HT_STATUS_OK;
}

int launch_sample(const SampleArgs &args, int dtype, const char *what, cudaStream_t s) {
    SampleArgs a = args;
    a.checked = a.R > kManyRows;
    if (a.checked) {
        check_sequences_kernel<<<a.B, kCheckThreads, 0, s>>>(a);
        const int rc = check_launch(what);
        if (rc != HT_OK) return rc;
    }
    cudaError_t e;
    switch (dtype) {
        case HT_F32: e = launch_sample_t<float>(a, what, s); break;
        case HT_F16: e = launch_sample_t<__half>(a, what, s); break;
        default: e = launch_sample_t<__nv_bfloat16>(a, what, s); break;
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(HT_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    return HT_OK;
}
#endif  // HT_SAMPLE_DTYPE

}  // namespace ht
