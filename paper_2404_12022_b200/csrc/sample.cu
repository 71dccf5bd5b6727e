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
// held in 64 bits (relative error about 1e-13): a row's answer does not depend on how its sum was split.  Nothing is
// added by atomics but counts.
//
// One block per row, the row in shared memory.  A histogram of the tokens over the logarithm of their weight (1/64
// octave per bin) bounds the running weight at every bin, which leaves the cut in a zone of a bin or a few; the zone's
// tokens (or the whole kept set, where it is small) are sorted and the cut is found exactly.  A small top-k needs no
// weights at all: the k-th largest of the threads' maxima is a lower bound of the k-th largest token.
#include <limits.h>

#include "accept.cuh"

namespace ht {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kBins = 2048;
constexpr int kBinsPerOctave = 64;
constexpr int kList = 1024;               // tokens that are sorted at most
constexpr float kLog2eF = 1.4426950408889634f;

struct SampleSmem {
    union {
        unsigned int hist[kBins];
        unsigned long long list[kList];
    };
    double pow2[16];                      // 2^(i / 16)
    double wsum[kSampleWarps];
    float wmax[kSampleWarps];
    unsigned int wcount[kSampleWarps];
    int n_list, n_above, zone_lo, zone_hi, answer, first_thread;
    unsigned int total;
};

// Ordered integer of a value: larger value, larger integer; -0 counts as 0.
__device__ __forceinline__ unsigned int order_key(float x) {
    const unsigned int u = __float_as_uint(x + 0.f);
    return u ^ ((unsigned int)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned int k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Weight of a logit.  exp(d / T) = 2^(t / 16) with t = 16 log2(e) d / T = 16 n + i + r, |r| <= 1/2: a table of
// 2^(i / 16) (16 doubles: a gather without bank conflicts), the Taylor series of e^(r ln2 / 16) to the fifth power (the
// next term is below 2e-13) and n into the exponent.  All in 64 bits.
struct Weights {
    double m, c;                          // largest logit, 16 log2(e) / T
    const double *pow2;
    __device__ __forceinline__ double operator()(float x) const {
        const double t = ((double)x - m) * c;
        if (!(t >= -16000.0)) return 0.0;
        constexpr double kMagic = 6755399441055744.0;          // 1.5 * 2^52: adding it rounds to a whole number
        const double kd = t + kMagic;
        const int k = __double2loint(kd);
        const double r = t - (kd - kMagic);
        constexpr double a = 0.693147180559945309417 / 16.0;   // ln 2 / 16
        double q = a * a * a * a * a / 120.0;
        q = fma(q, r, a * a * a * a / 24.0);
        q = fma(q, r, a * a * a / 6.0);
        q = fma(q, r, a * a / 2.0);
        q = fma(q, r, a);
        q = fma(q, r, 1.0);
        const double w = q * pow2[k & 15];
        return __hiloint2double(__double2hiint(w) + ((k >> 4) << 20), __double2loint(w));
    }
};

// A row: in shared memory at the 16-byte phase it has in global memory, with -inf around it (kStaged), or in global
// memory.  NaN reads as -inf; where the largest value is +inf (`peak`), +inf reads as 0 and all else as -inf.
template <typename T, bool kStaged>
struct Row {
    static constexpr int VE = Vec16<T>::n;
    const T *base;                        // vector 0 (16-byte aligned); element i of the row is base[phase + i]
    int phase, V, vecs;
    bool peak;
    __device__ __forceinline__ void load(int v, float *x) const {
        if (kStaged) {
            unpack16<T>(*reinterpret_cast<const uint4 *>(base + v * VE), x);
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
        for (int e = 0; e < VE; ++e) {
            if (!(x[e] == x[e])) x[e] = -INFINITY;
            if (peak) x[e] = x[e] == INFINITY ? 0.f : -INFINITY;
        }
    }
    __device__ __forceinline__ int index(int v, int e) const { return v * VE - phase + e; }
    // the vectors of warp w: consecutive, so that sums per warp are sums over ranges of the index
    __device__ __forceinline__ int warp_first(int w) const { return (int)((long long)vecs * w / kSampleWarps); }
    // f(value, index) for this thread's elements
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        const int w = threadIdx.x >> 5, end = warp_first(w + 1);
        for (int v = warp_first(w) + (threadIdx.x & 31); v < end; v += 32) {
            float x[VE];
            load(v, x);
#pragma unroll
            for (int e = 0; e < VE; ++e) f(x[e], index(v, e));
        }
    }
};

// The kept set: elements ahead of (key, index) in the order.
struct Cut {
    unsigned int key;
    int index;
    __device__ __forceinline__ bool keeps(float x, int i) const {
        const unsigned int k = order_key(x);
        return k > key || (k == key && i < index);
    }
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

// Ascending sort of list[0, n), n <= kList, by the whole block (bitonic network on the next power of two).
__device__ __forceinline__ void sort_list(SampleSmem &sm, int n) {
    int size = 2;
    while (size < n) size <<= 1;
    __syncthreads();
    for (int i = n + threadIdx.x; i < size; i += kSampleThreads) sm.list[i] = ~0ull;
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int t = threadIdx.x; t < size / 2; t += kSampleThreads) {
                const int i = 2 * t - (t & (j - 1)), o = i + j;
                const unsigned long long a = sm.list[i], b = sm.list[o];
                if ((a > b) == ((i & k) == 0)) {
                    sm.list[i] = b;
                    sm.list[o] = a;
                }
            }
        }
    __syncthreads();
}
// A token as a list entry that sorts in the order: larger key first, lower index among equals.
__device__ __forceinline__ unsigned long long list_entry(float x, int i) { return ((unsigned long long)~order_key(x) << 32) | (unsigned)i; }
__device__ __forceinline__ unsigned int entry_key(unsigned long long e) { return ~(unsigned int)(e >> 32); }
__device__ __forceinline__ int entry_index(unsigned long long e) { return (int)(unsigned int)e; }

__device__ __forceinline__ void append(SampleSmem &sm, float x, int i) {
    const int at = atomicAdd(&sm.n_list, 1);
    if (at < kList) sm.list[at] = list_entry(x, i);
}

// The first entry of the sorted list[0, n) at which `above` plus the weight of the entries ahead reaches `goal`; n if none.
// `sum_all` receives the weight of the whole list.
__device__ __forceinline__ int list_cut(SampleSmem &sm, const Weights &wt, int n, double above, double goal, double *sum_all) {
    constexpr int PER = kList / kSampleThreads;
    double w[PER], mine = 0.0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = threadIdx.x * PER + u;
        w[u] = i < n ? wt(key_value(entry_key(sm.list[i]))) : 0.0;
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
    unsigned long long e[PER];
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int i = threadIdx.x + x * kSampleThreads;
        if (i < n) {
            e[x] = sm.list[i];
            sm.list[i] = (e[x] << 32) | (e[x] >> 32);       // index first
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

template <typename T, bool kStaged>
struct Sampler {
    SampleSmem &sm;
    Row<T, kStaged> row;
    Weights wt;
    float m, cf;                          // largest logit; bins per unit of logit

    __device__ __forceinline__ int bin(float x) const {
        const float y = (m - x) * cf;
        return y < (float)(kBins - 1) ? (int)y : kBins - 1;
    }

    // Elements ahead of the cut of a running count (top_k > 0) or weight (goal), by halving the range of the keys and
    // then of the indexes: exact for every distribution, one pass over the row per step.  For rows whose zone does not
    // fit the list: very many equal tokens, or a cut among tokens below 2^-32 of the largest.
    __device__ __forceinline__ Cut slow_cut(const Cut &in, unsigned int count_goal, double goal) {
        auto reaches = [&](unsigned int key, double *weight, unsigned int *count) {
            double w = 0.0;
            unsigned int c = 0;
            row.each([&](float x, int i) {
                if (x > -INFINITY && order_key(x) >= key && in.keeps(x, i)) {
                    ++c;
                    if (!count_goal) w += wt(x);
                }
            });
            *count = block_count(sm, c);
            *weight = count_goal ? 0.0 : block_sum(sm, w);
            return count_goal ? *count >= count_goal : *weight >= goal;
        };
        unsigned int lo = 0, hi = order_key(m);              // the answer: the largest key whose elements at or above it reach the goal
        double w;
        unsigned int c;
        while (lo < hi) {
            const unsigned int mid = lo + (hi - lo) / 2 + 1;
            if (reaches(mid, &w, &c)) lo = mid;
            else hi = mid - 1;
        }
        double w_above;
        unsigned int c_above;
        if (lo == 0xFFFFFFFFu) { w_above = 0.0; c_above = 0; }
        else reaches(lo + 1, &w_above, &c_above);
        // elements equal to it, in index order, are kept while the running count or weight before them is below the goal
        unsigned int ties;
        if (count_goal) {
            ties = count_goal - c_above;
        } else {
            const double each_w = wt(key_value(lo));
            const double n = each_w > 0.0 ? ceil((goal - w_above) / each_w) : 1.0;
            ties = n < 1.0 ? 1u : (n > 2.0e9 ? 2000000000u : (unsigned int)n);
            while (ties > 1 && !(w_above + (double)(ties - 1) * each_w < goal)) --ties;
            while (w_above + (double)ties * each_w < goal && ties < 2000000000u) ++ties;
        }
        int a = 0, z = row.V;                                // the first index with `ties` equal elements ahead of it
        while (a < z) {
            const int mid = a + (z - a) / 2;
            unsigned int n = 0;
            row.each([&](float x, int i) { n += order_key(x) == lo && i < mid && in.keeps(x, i); });
            if (block_count(sm, n) >= ties) z = mid;
            else a = mid + 1;
        }
        return Cut{lo, a};
    }

    // Gathers the kept elements of bins [lo, hi] into the list; returns their number, which may exceed what the list holds.
    // `above`: weight of the kept elements of lower bins (where asked for).
    __device__ __forceinline__ int gather(const Cut &in, int lo, int hi, double *above) {
        __syncthreads();
        if (threadIdx.x == 0) sm.n_list = 0;
        __syncthreads();
        double w = 0.0;
        row.each([&](float x, int i) {
            const int b = bin(x);
            if (b <= hi && x > -INFINITY && in.keeps(x, i)) {
                if (b >= lo) append(sm, x, i);
                else if (above) w += wt(x);
            }
        });
        if (above) *above = block_sum(sm, w);
        __syncthreads();
        return sm.n_list;
    }

    // Counts of the kept elements by bin, and their weight.
    template <bool kWeight>
    __device__ __forceinline__ double histogram(const Cut &in) {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kSampleThreads) sm.hist[i] = 0u;
        __syncthreads();
        double w = 0.0;
        unsigned int low = 0;                                // the last bin may hold most of the row: counted in registers
        row.each([&](float x, int i) {
            if (x > -INFINITY && in.keeps(x, i)) {
                const int b = bin(x);
                if (b < kBins - 1) atomicAdd(&sm.hist[b], 1u);
                else ++low;
                if (kWeight) w += wt(x);
            }
        });
        low = block_count(sm, low);
        if (threadIdx.x == 0) sm.hist[kBins - 1] = low;
        return kWeight ? block_sum(sm, w) : 0.0;
    }

    // First bin at which the running count reaches `goal` (sm.zone_lo = sm.zone_hi), counts before it (sm.n_above) and in all (sm.total).
    __device__ __forceinline__ void find_count(unsigned int goal) {
        constexpr int PER = kBins / kSampleThreads;
        __syncthreads();
        unsigned int c[PER], mine = 0, all;
#pragma unroll
        for (int u = 0; u < PER; ++u) mine += c[u] = sm.hist[threadIdx.x * PER + u];
        unsigned int before = block_scan(mine, sm.wcount, &all);
        if (threadIdx.x == 0) { sm.total = all; sm.zone_lo = -1; }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            if (before < goal && before + c[u] >= goal) {
                sm.zone_lo = threadIdx.x * PER + u;
                sm.n_above = (int)before;
            }
            before += c[u];
        }
        __syncthreads();
    }

    // Bins that may hold the cut of a running weight, `total` being the weight of all.  With every element of a bin taken
    // at the bin's upper or lower end, running sums `up` and `dn` enclose the running weight M_b at the end of bin b from
    // the front, and what is left behind it encloses it from the back (a cut close to the end has little behind it):
    //     max(dn_b, total - (up_all - up_b)) <= M_b <= min(up_b, total - (dn_all - dn_b)).
    // sm.zone_lo: the first bin where the upper bound reaches the goal, sm.zone_hi: the first where the lower one does,
    // sm.total: elements up to zone_hi.  Bins are formed in 32 bits: 1e-5 relative covers what their edges move by; the
    // last bin has no lower end.
    __device__ __forceinline__ void find_weight(double goal, double total) {
        constexpr int PER = kBins / kSampleThreads;
        __syncthreads();
        unsigned int c[PER], mine_c = 0, all_c;
        double up[PER], dn[PER], mine_up = 0.0, mine_dn = 0.0, all_up, all_dn;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int b = threadIdx.x * PER + u;
            c[u] = sm.hist[b];
            const float edge = exp2f(-(float)b / kBinsPerOctave);
            up[u] = c[u] * ((double)edge * 1.00001);
            dn[u] = b == kBins - 1 ? 0.0 : c[u] * ((double)edge * (0.98922 * 0.99999));   // 2^(-1/64) = 0.989228...
            mine_c += c[u];
            mine_up += up[u];
            mine_dn += dn[u];
        }
        unsigned int before_c = block_scan(mine_c, sm.wcount, &all_c);
        double sum_up = block_scan(mine_up, sm.wsum, &all_up);
        double sum_dn = block_scan(mine_dn, sm.wsum, &all_dn);
        if (threadIdx.x == 0) { sm.zone_lo = kBins - 1; sm.zone_hi = kBins - 1; sm.total = all_c; }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int b = threadIdx.x * PER + u;
            sum_up += up[u];
            sum_dn += dn[u];
            if (fmin(sum_up, total - (all_dn - sum_dn)) >= goal) atomicMin(&sm.zone_lo, b);
            if (fmax(sum_dn, total - (all_up - sum_up)) >= goal) atomicMin(&sm.zone_hi, b);
        }
        __syncthreads();
        const int hi = sm.zone_hi;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            before_c += c[u];
            if (threadIdx.x * PER + u == hi) sm.total = before_c;
        }
        __syncthreads();
    }

    // The token by one pass of sums and the walk of one warp's range: kept = ahead of the cut and w >= floor.
    __device__ __forceinline__ int draw(const Cut &cut, double floor, double u) {
        auto weight = [&](float x, int i) {
            if (!(x > -INFINITY) || !cut.keeps(x, i)) return 0.0;
            const double w = wt(x);
            return w >= floor ? w : 0.0;
        };
        double mine = 0.0;
        row.each([&](float x, int i) { mine += weight(x, i); });
        const double goal = u * block_sum(sm, mine);
        double before = 0.0;
        int seg = -1;
        for (int w = 0; w < kSampleWarps; ++w) {
            const double s = sm.wsum[w];
            if (s > 0.0) {
                if (before + s > goal) { seg = w; break; }
                before += s;
            }
        }
        __syncthreads();
        if (seg < 0) {                                        // uniform = 1: the last one with a weight
            if (threadIdx.x == 0) sm.answer = -1;
            __syncthreads();
            int last = -1;
            row.each([&](float x, int i) { if (weight(x, i) > 0.0) last = max(last, i); });
            atomicMax(&sm.answer, last);
            __syncthreads();
            return sm.answer;
        }
        const int first = row.warp_first(seg), n = row.warp_first(seg + 1) - first;
        const int per = (n + kSampleThreads - 1) / kSampleThreads;
        const int v0 = first + min(n, (int)threadIdx.x * per), v1 = first + min(n, ((int)threadIdx.x + 1) * per);
        mine = 0.0;
        for (int v = v0; v < v1; ++v) {
            float x[Row<T, kStaged>::VE];
            row.load(v, x);
#pragma unroll
            for (int e = 0; e < Row<T, kStaged>::VE; ++e) mine += weight(x[e], row.index(v, e));
        }
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
                float x[Row<T, kStaged>::VE];
                row.load(v, x);
#pragma unroll
                for (int e = 0; e < Row<T, kStaged>::VE; ++e) {
                    const double w = weight(x[e], row.index(v, e));
                    if (!found && w > 0.0) {
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

    __device__ int sample(float thread_max, float Tm, int top_k, float top_p, float min_p, float uniform) {
        const double u = (double)uniform, floor = min_p > 0.f ? (double)min_p : 0.0;
        Cut cut{0u, INT_MAX};                                 // keeps everything above -inf
        bool p_on = top_p < 1.f;
        if (top_k > 0 && top_k < row.V) {
            if (top_k <= kSampleThreads) {
                // the k-th largest of the threads' maxima bounds the k-th largest token from below
                const unsigned int mine = order_key(thread_max);
                unsigned int key = 0;
                for (int bit = 31; bit >= (sizeof(T) == 2 ? 13 : 0); --bit) {     // (a 16-bit value has no lower bits: fp16 reaches bit 13)
                    const unsigned int cand = key | (1u << bit);
                    if (__syncthreads_count(mine >= cand) >= top_k) key = cand;
                }
                if (threadIdx.x == 0) sm.n_list = 0;
                __syncthreads();
                row.each([&](float x, int i) { if (x > -INFINITY && order_key(x) >= key) append(sm, x, i); });
                __syncthreads();
                int n = sm.n_list;
                if (n <= kList) {
                    sort_list(sm, n);
                    n = min(n, top_k);
                    return finish_list(n, p_on, top_p, -1.0, floor, u);
                }
            }
            histogram<false>(cut);
            find_count((unsigned int)top_k);
            if (sm.zone_lo >= 0) {                            // more than k tokens above -inf
                const int zone = sm.zone_lo, above = sm.n_above;
                bool done = false;
                if (zone < kBins - 1) {
                    const int n = gather(cut, zone, zone, nullptr);
                    if (n <= kList) {
                        sort_list(sm, n);
                        if (top_k - above < n) cut = Cut{entry_key(sm.list[top_k - above]), entry_index(sm.list[top_k - above])};
                        else cut = Cut{entry_key(sm.list[n - 1]), INT_MAX};
                        done = true;
                    }
                }
                if (!done) cut = slow_cut(cut, (unsigned int)top_k, 0.0);
            }
        }
        if (p_on) {
            const double Z = histogram<true>(cut);
            const double goal = (double)top_p * Z;
            find_weight(goal, Z);
            const int lo = sm.zone_lo, hi = sm.zone_hi;
            const unsigned int upto = sm.total;
            if (hi < kBins - 1 && upto <= kList) {            // the whole kept set fits the list
                const int n = gather(cut, 0, hi, nullptr);
                sort_list(sm, n);
                return finish_list(n, true, top_p, Z, floor, u);
            }
            bool done = false;
            if (hi < kBins - 1) {
                double above;
                const int n = gather(cut, lo, hi, &above);
                if (n <= kList) {
                    sort_list(sm, n);
                    double sum;
                    const int at = list_cut(sm, wt, n, above, goal, &sum);
                    cut = at < n ? Cut{entry_key(sm.list[at]), entry_index(sm.list[at])} : Cut{entry_key(sm.list[n - 1]), INT_MAX};
                    done = true;
                }
            }
            if (!done) cut = slow_cut(cut, 0u, goal);
        }
        return draw(cut, floor, u);
    }

    // list[0, n): the first n of the order.  total < 0: the weight that top_p refers to is the list's own.
    __device__ __forceinline__ int finish_list(int n, bool p_on, float top_p, double total, double floor, double u) {
        if (n > 1 && p_on) {
            double sum;
            if (total < 0.0) {
                list_cut(sm, wt, n, 0.0, INFINITY, &sum);
                total = sum;
            }
            n = max(1, list_cut(sm, wt, n, 0.0, (double)top_p * total, &sum));
        }
        if (n > 1 && floor > 0.0) {
            int c = 0;
            for (int i = threadIdx.x; i < n; i += kSampleThreads) c += wt(key_value(entry_key(sm.list[i]))) >= floor;
            n = max(1, (int)block_count(sm, (unsigned int)c));
        }
        return list_draw(sm, wt, n, u);
    }
};

// Copies the row into shared memory at its own 16-byte phase (nothing outside the row is read), -inf around it.
template <typename T>
__device__ __forceinline__ void stage_row(T *dst, const T *src, int V, int phase, int vecs) {
    constexpr int VE = Vec16<T>::n;
    const T *base = src - phase;
    for (int v = threadIdx.x; v < vecs; v += kSampleThreads) {
        const int i0 = v * VE - phase;
        if (i0 >= 0 && i0 + VE <= V) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + v * VE)), "l"(base + (size_t)v * VE) : "memory");
        } else {
            for (int e = 0; e < VE; ++e) dst[v * VE + e] = (i0 + e >= 0 && i0 + e < V) ? src[i0 + e] : from_float<T>(-INFINITY);
        }
    }
    asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
    __syncthreads();
}

template <typename T, bool kStaged, bool kVerify>
__global__ void __launch_bounds__(kSampleThreads, 2)
sample_kernel(const SampleArgs a) {
    constexpr int VE = Vec16<T>::n;
    extern __shared__ uint4 s_dyn[];
    __shared__ SampleSmem sm;
    __shared__ int s_last;
    const int b = blockIdx.x / a.R, r = blockIdx.x - b * a.R;
    const T *src = static_cast<const T *>(a.logits) + ((size_t)b * a.N + r) * a.V;
    Row<T, kStaged> row;
    row.phase = (int)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
    row.V = a.V;
    row.vecs = (row.phase + a.V + VE - 1) / VE;
    row.peak = false;
    if (threadIdx.x < 16) sm.pow2[threadIdx.x] = exp2((double)threadIdx.x / 16.0);
    // parameters of the sequence; every block of it comes to the same decision
    const float Tm = a.temperature ? a.temperature[b] : 1.f;
    const int top_k = a.top_k ? a.top_k[b] : 0;
    const float top_p = a.top_p ? a.top_p[b] : 1.f;
    const float min_p = a.min_p ? a.min_p[b] : 0.f;
    bool bad = !(Tm >= 0.f) || Tm == INFINITY || !(top_p == top_p) || !(min_p <= 1.f);
    for (int i = threadIdx.x; i < a.R; i += kSampleThreads) {
        const float x = a.uniform[(size_t)b * a.N + i];
        bad |= !(x >= 0.f && x <= 1.f);
    }
    bad = __syncthreads_or(bad);
    int token = -1;
    if (!bad) {
        if (kStaged) {
            T *dst = reinterpret_cast<T *>(s_dyn);
            stage_row<T>(dst, src, a.V, row.phase, row.vecs);
            row.base = dst;
        } else {
            row.base = src - row.phase;
        }
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
                    T *d = reinterpret_cast<T *>(s_dyn) + v * VE;
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
        if (m == -INFINITY) {
            // nothing above -inf: the first -inf, or 0 in a row of NaNs, as the greedy verification has it
            if (threadIdx.x == 0) sm.answer = INT_MAX;
            __syncthreads();
            for (int i = threadIdx.x; i < a.V; i += kSampleThreads)
                if (to_float<T>(src[i]) == -INFINITY) { atomicMin(&sm.answer, i); break; }
            __syncthreads();
            token = sm.answer == INT_MAX ? 0 : sm.answer;
        } else if (Tm == 0.f || top_k == 1 || top_p <= 0.f) {
            if (threadIdx.x == 0) sm.answer = INT_MAX;
            __syncthreads();
            int first = INT_MAX;
            row.each([&](float x, int i) { if (x == m) first = min(first, i); });
            first = __reduce_min_sync(0xffffffffu, first);
            if ((threadIdx.x & 31) == 0) atomicMin(&sm.answer, first);
            __syncthreads();
            token = sm.answer;
        } else {
            if (m == INFINITY) {                             // the +inf tokens share the weight, the others have none
                if (kStaged) {
                    T *d = reinterpret_cast<T *>(s_dyn);
                    for (int i = threadIdx.x; i < row.vecs * VE; i += kSampleThreads)
                        d[i] = from_float<T>(to_float<T>(d[i]) == INFINITY ? 0.f : -INFINITY);
                }
                row.peak = true;
                m = 0.f;
                mx = mx == INFINITY ? 0.f : -INFINITY;
                __syncthreads();
            }
            const float cf = fminf(kBinsPerOctave * kLog2eF / Tm, 1e30f);
            Sampler<T, kStaged> s{sm, row, Weights{(double)m, 16.0 * 1.4426950408889634074 / (double)Tm, sm.pow2}, m, cf};
            token = s.sample(mx, Tm, top_k, top_p, min_p, a.uniform[(size_t)b * a.N + r]);
        }
    }
    if (!kVerify) {
        if (threadIdx.x == 0) {
            a.token[(size_t)b * a.N + r] = token;
            if (r == 0) a.status[b] = bad ? HT_STATUS_BAD_PARAM : HT_STATUS_OK;
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

template <typename T, bool kStaged, bool kVerify>
static cudaError_t launch_shape(const SampleArgs &a, size_t smem, cudaStream_t s) {
    static bool raised[64];                                  // per device: the kernel's shared memory limit
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !raised[dev]) {
        e = cudaFuncSetAttribute(sample_kernel<T, kStaged, kVerify>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSampleDynMax);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) raised[dev] = true;
    }
    sample_kernel<T, kStaged, kVerify><<<(unsigned)((long long)a.B * a.R), kSampleThreads, smem, s>>>(a);
    return cudaPeekAtLastError();
}

template <typename T>
static cudaError_t launch_t(const SampleArgs &a, cudaStream_t s) {
    const size_t staged = ((size_t)a.V * sizeof(T) + 15 + 15) / 16 * 16;
    const size_t tree = a.tokens ? sizeof(TreeSmem) : 0;
    if (staged <= kSampleDynMax) {
        const size_t smem = staged > tree ? staged : tree;
        return a.tokens ? launch_shape<T, true, true>(a, smem, s) : launch_shape<T, true, false>(a, smem, s);
    }
    return a.tokens ? launch_shape<T, false, true>(a, tree, s) : launch_shape<T, false, false>(a, tree, s);
}

int launch_sample(const SampleArgs &a, int dtype, const char *what, cudaStream_t s) {
    cudaError_t e;
    switch (dtype) {
        case HT_F32: e = launch_t<float>(a, s); break;
        case HT_F16: e = launch_t<__half>(a, s); break;
        default: e = launch_t<__nv_bfloat16>(a, s); break;
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(HT_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    return HT_OK;
}

}  // namespace ht
