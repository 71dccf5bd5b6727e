// Norm of each query and key head, rotary embedding and placement of the new K / V rows behind the context, in one pass
// (the step ahead of tree attention for models that normalise their heads or rotate them otherwise than the plain
// half-split embedding does; ht_rope_kv_append is the plain form).  Per head of D features x:
//     y = x * rsqrt(mean(x^2) + eps) * (w + weight_offset)
//     the first rot_dim features of y in pairs (a, b): (a cos - b sin, b cos + a sin) of the angle pos * f_i
// with pair i = (i, i + rot_dim / 2) or (2 i, 2 i + 1), and the frequencies f_i formed on the host in 64 bits.
//
// Every value is read once and written once: bound by HBM for prompts, by the launch and one round trip to memory for a
// tree's rows.  A block takes rows of the batch by turns.  A head is D / 2 features by lanes that hold two 16-byte
// vectors each, chosen so that both features of every pair meet in one lane: the rotation needs no exchange, the mean a
// shuffle over 4 to 16 lanes.  A lane keeps its place within the head for all heads of a row, so the cosines and sines
// are loaded into registers once per row; up to three heads per lane are in flight, and as soon as one has been used the
// next row's vectors are asked for in its place.  Angles: the position times the frequency in turns, in 64 bits, its
// fraction to 32 (a position of a hundred thousand leaves a 32-bit product no low bits); products and sums in 32 bits,
// one rounding to the type.
//
// 8 x 2048 rows of 80 heads in bf16 (671 MB): 142 us = 4.7 TB/s, 0.72 of the measured copy rate; the instructions of 16
// values per lane and head (about 250 per warp and head group) are what is left.  One row per block took 203 us (the
// chain position -> angle -> table -> heads once per row), one barrier per row 157 us.  1 x 91 rows of 96 heads: 4.3 us.
#include <math.h>

#include "ht_common.cuh"

namespace ht {

struct RopeTurns {
    double f[64];                 // turns per position of pair i
};

struct PlaceArgs {
    const void *q_in, *k_in, *v_in, *q_weight, *k_weight;
    void *q_out, *k_cache, *v_cache;
    const int32_t *pos, *kv_len;
    int32_t *status;
    int N, Hq, Hkv, cap, rot, norm;
    int chunks;                   // of kPlaceAhead * (heads per block pass) heads
    long long rows;
    float eps, offset, magnitude;
    long long q_stride, k_stride, v_stride, stride_b, stride_h;
};

// 16 bytes of rounded values, a pair per conversion.
__device__ __forceinline__ uint4 pack16(const float *x, float) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack16(const float *x, __half) {
    __half2 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
    return *reinterpret_cast<const uint4 *>(h);
}
__device__ __forceinline__ uint4 pack16(const float *x, __nv_bfloat16) {
    __nv_bfloat162 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    return *reinterpret_cast<const uint4 *>(h);
}

constexpr int kPlaceThreads = 256;
constexpr int kPlaceAhead = 3;    // heads per lane whose vectors are asked for before the angles are formed

template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kPlaceThreads, 2)
norm_rope_kernel(const PlaceArgs p, const PageMap pm, const __grid_constant__ RopeTurns turns) {
    // lets a kernel that is serialized programmatically behind this one (the attention call) set itself up meanwhile
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int VE = Vec16<T>::n, LPH = D / (2 * VE), HPB = kPlaceThreads / LPH;     // lanes per head, heads per block pass
    constexpr int kBatch = kPlaceThreads / 64;           // rows whose tables are formed at once: a thread per pair
    __shared__ float s_cos[2][kBatch][D / 2], s_sin[2][kBatch][D / 2];
    const int half_rot = p.rot >> 1;
    const int group = threadIdx.x / LPH, j = threadIdx.x - group * LPH;
    // this lane's two vectors within a head
    int v0, v1;
    bool rotates;
    if (kInterleaved) {
        v0 = j;
        v1 = j + LPH;
        rotates = true;                                  // (decided pair by pair)
    } else {
        const int R = half_rot / VE;                     // lanes that hold rotated pairs
        rotates = j < R;
        v0 = rotates ? j : 2 * j;
        v1 = rotates ? j + R : 2 * j + 1;
    }
    // A block keeps one chunk of kPlaceAhead * HPB heads for all its rows: what a lane's heads are is settled here.
    enum { kQ = 0, kK = 1, kV = 2, kNone = 3 };
    const int chunk = (int)(blockIdx.x % (unsigned)p.chunks), step = (int)(gridDim.x / (unsigned)p.chunks);
    int kind[kPlaceAhead], head[kPlaceAhead];
    const uint4 *src[kPlaceAhead];
    unsigned int ahead[kPlaceAhead];                     // vectors from a row of the block to its next (checked on the host)
    long long row = blockIdx.x / (unsigned)p.chunks;
#pragma unroll
    for (int u = 0; u < kPlaceAhead; ++u) {
        const int h = chunk * kPlaceAhead * HPB + group + u * HPB;
        kind[u] = h < p.Hq ? kQ : (h < p.Hq + p.Hkv ? kK : (h < p.Hq + 2 * p.Hkv ? kV : kNone));
        head[u] = kind[u] == kQ ? h : (kind[u] == kK ? h - p.Hq : h - p.Hq - p.Hkv);
        const T *base = static_cast<const T *>(kind[u] == kQ ? p.q_in : (kind[u] == kK ? p.k_in : p.v_in));
        const long long stride = kind[u] == kQ ? p.q_stride : (kind[u] == kK ? p.k_stride : p.v_stride);
        src[u] = reinterpret_cast<const uint4 *>(base + row * stride + (long long)head[u] * D) + v0;
        ahead[u] = (unsigned int)(stride / VE * step);
    }
    const int apart = v1 - v0;
    uint4 in0[kPlaceAhead], in1[kPlaceAhead];
    auto ask = [&](int u) {                              // the vectors of this lane's head u, and on to the block's next row
        if (kind[u] != kNone) {
            in0[u] = src[u][0];
            in1[u] = src[u][apart];
        }
        src[u] += ahead[u];
    };
#pragma unroll
    for (int u = 0; u < kPlaceAhead; ++u) ask(u);
    // the query weights stay in registers (ones without weights); the few key heads read theirs where they need them
    float wq[2 * VE];
    {
        const uint4 *w = static_cast<const uint4 *>(p.q_weight);
        if (w) {
            unpack16<T>(__ldg(w + v0), wq);
            unpack16<T>(__ldg(w + v1), wq + VE);
        }
#pragma unroll
        for (int e = 0; e < 2 * VE; ++e) wq[e] = w ? wq[e] + p.offset : 1.f;
    }
    // Cosines and sines of the positions of the block's next four rows, one pair per thread, into one of two sets of tables
    // while the other one is in use; the positions have been asked for a batch earlier.
    const int me_row = threadIdx.x >> 6, me_pair = threadIdx.x & 63;
    auto position = [&](long long first) {
        const long long at = first + (long long)me_row * step;
        return me_pair < half_rot && at < p.rows ? p.pos[at] : 0;
    };
    auto form_tables = [&](int at, int turn) {
        if (me_pair >= half_rot) return;
        const double t = (double)at * turns.f[me_pair];
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        s_cos[turn][me_row][me_pair] = c * p.magnitude;
        s_sin[turn][me_row][me_pair] = s * p.magnitude;
    };
    form_tables(position(row), 0);
    int pos_next = position(row + kBatch * step);
    for (int i = 0; row < p.rows; row += step, ++i) {
        const long long next = row + step;
        const int k = i % kBatch, turn = (i / kBatch) & 1;
        const int b = (int)((unsigned)row / (unsigned)p.N), r = (int)row - b * p.N;
        const int L = p.kv_len[b];
        const bool bad = L < 0 || (long long)L + p.N > p.cap;
        // where cache row L + r of this sequence starts, short of the head's offset
        long long row_off = (long long)b * p.stride_b + (long long)(L + r) * D;
        bool no_page = false;
        if (pm.table && !bad) {
            const int page = pm.table[(size_t)b * pm.max_pages + ((L + r) >> pm.shift)];
            no_page = (unsigned)page >= (unsigned)pm.n_pages;     // the row's K and V are not stored; its q is written
            row_off = (long long)page * pm.page_stride + (long long)((L + r) & ((1 << pm.shift) - 1)) * D;
        }
        if (r == 0 && chunk == 0) {                      // the sequence's word, by one block: its length, its pages
            int bad_page = 0;
            if (!bad && pm.table)
                for (int i = (L >> pm.shift) + threadIdx.x; i <= (L + p.N - 1) >> pm.shift; i += kPlaceThreads)
                    bad_page |= (unsigned)pm.table[(size_t)b * pm.max_pages + i] >= (unsigned)pm.n_pages;
            bad_page = __syncthreads_or(bad_page);
            if (threadIdx.x == 0) p.status[b] = bad ? HT_STATUS_BAD_LEN : (bad_page ? HT_STATUS_BAD_PAGE : HT_STATUS_OK);
        }
        if (k == 0) {
            __syncthreads();                             // the batch's tables are complete, the other ones' readers are done
            if (row + kBatch * step < p.rows) {
                form_tables(pos_next, turn ^ 1);
                pos_next = position(row + 2 * kBatch * step);
            }
        }
        // The lane's pairs, for all heads of the row.  Half-split: the VE pairs of vector v0; interleaved: VE / 2 pairs of
        // v0, then VE / 2 of v1.
        float cs[VE], sn[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const int pair = kInterleaved ? (e < VE / 2 ? v0 * (VE / 2) + e : v1 * (VE / 2) + e - VE / 2) : j * VE + e;
            cs[e] = pair < half_rot ? s_cos[turn][k][pair] : 1.f;
            sn[e] = pair < half_rot ? s_sin[turn][k][pair] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kPlaceAhead; ++u) {
            uint4 out0 = in0[u], out1 = in1[u];
            if (next < p.rows) ask(u);                   // the place is free for the next row's vectors
            float x[2 * VE];
            unpack16<T>(out0, x);
            unpack16<T>(out1, x + VE);
            float ss = 0.f, ss1 = 0.f;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                ss = fmaf(x[e], x[e], ss);
                ss1 = fmaf(x[VE + e], x[VE + e], ss1);
            }
            ss += ss1;
#pragma unroll
            for (int off = LPH / 2; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
            if (bad || kind[u] == kNone || (kind[u] != kQ && no_page)) continue;
            if (kind[u] != kV) {
                if (p.norm & (kind[u] == kQ ? HT_HEAD_NORM_Q : HT_HEAD_NORM_K)) {
                    const float inv = rsqrtf(fmaf(ss, 1.f / D, p.eps));
                    if (kind[u] == kQ) {
#pragma unroll
                        for (int e = 0; e < 2 * VE; ++e) x[e] *= inv * wq[e];
                    } else {
                        const uint4 *w = static_cast<const uint4 *>(p.k_weight);
                        float wk[2 * VE];
                        if (w) {
                            unpack16<T>(__ldg(w + v0), wk);
                            unpack16<T>(__ldg(w + v1), wk + VE);
                        }
#pragma unroll
                        for (int e = 0; e < 2 * VE; ++e) x[e] *= w ? inv * (wk[e] + p.offset) : inv;
                    }
                }
                if (rotates) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        const int a = kInterleaved ? 2 * e : e, c = kInterleaved ? 2 * e + 1 : e + VE;
                        // an unrotated pair stays as it is, infinities included (interleaved: within a rotating lane)
                        if (!kInterleaved || (e < VE / 2 ? v0 * (VE / 2) + e : v1 * (VE / 2) + e - VE / 2) < half_rot) {
                            const float xa = x[a], xc = x[c];
                            x[a] = xa * cs[e] - xc * sn[e];
                            x[c] = xc * cs[e] + xa * sn[e];
                        }
                    }
                }
                out0 = pack16(x, T());
                out1 = pack16(x + VE, T());
            }
            T *dst = kind[u] == kQ ? static_cast<T *>(p.q_out) + (row * p.Hq + head[u]) * D
                                   : static_cast<T *>(kind[u] == kK ? p.k_cache : p.v_cache) + row_off + head[u] * p.stride_h;
            uint4 *to = reinterpret_cast<uint4 *>(dst) + v0;
            to[0] = out0;
            to[apart] = out1;
        }
    }
}

// Turns per position of each pair.  By parts (Peng et al., "YaRN", arXiv 2309.00071, Section 3.2): a pair that turns
// more than `high` times over the original context keeps its frequency, one that turns less than `low` times has it
// divided by the factor, with a linear ramp in between.
static RopeTurns make_turns(const ht_head_desc &h) {
    RopeTurns t{};
    const double two_pi = 6.283185307179586476925;
    const double ratio = h.rot_dim > 0 ? pow((double)h.rope_base, -2.0 / h.rot_dim) : 1.0;
    double plain = 1.0 / two_pi;                         // base^(-2i / rot_dim) / 2 pi, by products: 63 roundings of 2^-53 at most
    for (int i = 0; i < h.rot_dim / 2; ++i, plain *= ratio) {
        double f = plain;
        if (h.scaling == HT_ROPE_LINEAR) {
            f /= h.factor;
        } else if (h.scaling == HT_ROPE_BY_PARTS) {
            double keep = ((double)h.orig_len * f - h.low) / ((double)h.high - h.low);
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
            f *= keep + (1.0 - keep) / h.factor;
        }
        t.f[i] = f;
    }
    return t;
}

// Blocks of a kernel that the device holds at once.
template <typename Kernel>
static int resident_blocks(Kernel kernel) {
    int dev = 0, sms = 0, per_sm = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kPlaceThreads, 0) != cudaSuccess || sms <= 0 || per_sm <= 0) {
        cudaGetLastError();
        return 148;
    }
    return sms * per_sm;
}

template <typename T, int D, bool kInterleaved>
static int launch_form(const PlaceArgs &a, const PageMap &pm, const RopeTurns &turns, cudaStream_t s) {
    static int resident[64];                             // per device
    int dev = 0;
    cudaGetDevice(&dev);
    int *slot = (dev >= 0 && dev < 64) ? &resident[dev] : nullptr;
    int blocks = slot ? *slot : 0;
    if (blocks == 0) {
        blocks = resident_blocks(norm_rope_kernel<T, D, kInterleaved>);
        if (slot) *slot = blocks;
    }
    constexpr int kChunk = kPlaceAhead * kPlaceThreads * 2 * Vec16<T>::n / D;       // heads a block takes of a row
    PlaceArgs args = a;
    args.chunks = (a.Hq + 2 * a.Hkv + kChunk - 1) / kChunk;
    long long turns_at_once = blocks / args.chunks;      // rows
    turns_at_once = turns_at_once < 1 ? 1 : (turns_at_once > a.rows ? a.rows : turns_at_once);
    const long long widest = a.q_stride > a.k_stride ? (a.q_stride > a.v_stride ? a.q_stride : a.v_stride) : (a.k_stride > a.v_stride ? a.k_stride : a.v_stride);
    while (turns_at_once > 1 && widest / Vec16<T>::n * turns_at_once > 0xffffffffLL) turns_at_once /= 2;     // (a block's step between rows is a 32-bit count of vectors)
    if (widest / Vec16<T>::n > 0xffffffffLL) return fail(HT_ERR_UNSUPPORTED, "row stride too large");
    norm_rope_kernel<T, D, kInterleaved><<<(unsigned)(turns_at_once * args.chunks), kPlaceThreads, 0, s>>>(args, pm, turns);
    return check_launch("ht_norm_rope_kv_append");
}

template <typename T>
static int launch_t(const PlaceArgs &a, const PageMap &pm, const RopeTurns &turns, int D, bool interleaved, cudaStream_t s) {
    if (D == 64) return interleaved ? launch_form<T, 64, true>(a, pm, turns, s) : launch_form<T, 64, false>(a, pm, turns, s);
    return interleaved ? launch_form<T, 128, true>(a, pm, turns, s) : launch_form<T, 128, false>(a, pm, turns, s);
}

int launch_norm_rope(const ht_attn_desc &d, const ht_head_desc &h, const void *q_in, const void *k_in, const void *v_in,
                     const void *q_weight, const void *k_weight, const int32_t *pos, const int32_t *kv_len, void *q_out,
                     void *kc, void *vc, int32_t *status, cudaStream_t s, const PageMap &pm) {
    PlaceArgs a{};
    a.q_in = q_in; a.k_in = k_in; a.v_in = v_in; a.q_weight = q_weight; a.k_weight = k_weight;
    a.q_out = q_out; a.k_cache = kc; a.v_cache = vc; a.pos = pos; a.kv_len = kv_len; a.status = status;
    a.N = d.N; a.Hq = d.Hq; a.Hkv = d.Hkv; a.cap = d.cap; a.rot = h.rot_dim; a.norm = h.norm;
    a.eps = h.eps; a.offset = h.weight_offset; a.magnitude = h.magnitude == 0.f ? 1.f : h.magnitude;
    a.q_stride = h.q_stride ? h.q_stride : (long long)d.Hq * d.D;
    a.k_stride = h.k_stride ? h.k_stride : (long long)d.Hkv * d.D;
    a.v_stride = h.v_stride ? h.v_stride : (long long)d.Hkv * d.D;
    a.stride_h = pm.table ? pm.head_stride : (d.kv_stride_h ? d.kv_stride_h : (long long)d.cap * d.D);
    a.stride_b = d.kv_stride_b ? d.kv_stride_b : (long long)d.Hkv * d.cap * d.D;
    const RopeTurns turns = make_turns(h);
    a.rows = (long long)d.B * d.N;
    const bool il = h.interleaved != 0;
    switch (d.dtype) {
        case HT_F32: return launch_t<float>(a, pm, turns, d.D, il, s);
        case HT_F16: return launch_t<__half>(a, pm, turns, d.D, il, s);
        default: return launch_t<__nv_bfloat16>(a, pm, turns, d.D, il, s);
    }
}

}  // namespace ht
