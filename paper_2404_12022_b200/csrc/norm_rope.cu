// Norm of each query and key head, rotary embedding and placement of the new K / V rows behind the context, in one pass
// (the step ahead of tree attention for models that normalise their heads or rotate them otherwise than the plain
// half-split embedding does; ht_rope_kv_append is the plain form).  Per head of D features x:
//     y = x * rsqrt(mean(x^2) + eps) * (w + weight_offset)
//     the first rot_dim features of y in pairs (a, b): (a cos - b sin, b cos + a sin) of the angle pos * f_i
// with pair i = (i, i + rot_dim / 2) or (2 i, 2 i + 1), and the frequencies f_i formed on the host in 64 bits.
//
// Every value is read once and written once: bound by HBM for prompts (8 x 2048 rows of 80 heads: see the launcher), by
// the launch and one round trip to memory for a tree's rows.  One block per (sequence, row).  A head is D / 2 features
// by lanes that hold two 16-byte vectors each, chosen so that both features of every pair meet in one lane: the rotation
// needs no exchange, the mean a shuffle over 4 to 16 lanes.  A lane keeps its place within the head for all heads of
// the row, so the cosines and sines are loaded into registers once; the first heads' vectors are on their way while the
// angles are formed.  Angles: the position times the frequency in turns, in 64 bits, its fraction to 32 (a position of
// a hundred thousand leaves a 32-bit product no low bits); products and sums in 32 bits, one rounding to the type.
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
    float eps, offset, magnitude;
    long long q_stride, k_stride, v_stride, stride_b, stride_h;
};

constexpr int kPlaceThreads = 256;
constexpr int kPlaceAhead = 3;    // heads per lane whose vectors are asked for before the angles are formed

template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kPlaceThreads)
norm_rope_kernel(const PlaceArgs p, const PageMap pm, const __grid_constant__ RopeTurns turns) {
    // lets a kernel that is serialized programmatically behind this one (the attention call) set itself up meanwhile
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int VE = Vec16<T>::n, LPH = D / (2 * VE), HPB = kPlaceThreads / LPH;     // lanes per head, heads per block pass
    __shared__ float s_cos[D / 2], s_sin[D / 2];
    const int b = blockIdx.x / p.N, r = blockIdx.x - b * p.N;
    const int L = p.kv_len[b];
    const bool bad = L < 0 || (long long)L + p.N > p.cap;
    if (r == 0) {                                        // the sequence's word, by one block: its length, its pages
        int bad_page = 0;
        if (!bad && pm.table)
            for (int i = (L >> pm.shift) + threadIdx.x; i <= (L + p.N - 1) >> pm.shift; i += kPlaceThreads)
                bad_page |= (unsigned)pm.table[(size_t)b * pm.max_pages + i] >= (unsigned)pm.n_pages;
        bad_page = __syncthreads_or(bad_page);
        if (threadIdx.x == 0) p.status[b] = bad ? HT_STATUS_BAD_LEN : (bad_page ? HT_STATUS_BAD_PAGE : HT_STATUS_OK);
    }
    if (bad) return;
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
    // where cache row L + r of this sequence starts, short of the head's offset
    long long row_off = (long long)b * p.stride_b + (long long)(L + r) * D;
    bool no_page = false;
    if (pm.table) {
        const int page = pm.table[(size_t)b * pm.max_pages + ((L + r) >> pm.shift)];
        no_page = (unsigned)page >= (unsigned)pm.n_pages;     // the row's K and V are not stored; its q is written
        row_off = (long long)page * pm.page_stride + (long long)((L + r) & ((1 << pm.shift) - 1)) * D;
    }
    const size_t row = (size_t)b * p.N + r;
    const int heads = p.Hq + 2 * p.Hkv;
    auto source = [&](int h) -> const uint4 * {
        const T *src = h < p.Hq            ? static_cast<const T *>(p.q_in) + row * p.q_stride + (size_t)h * D
                       : h < p.Hq + p.Hkv ? static_cast<const T *>(p.k_in) + row * p.k_stride + (size_t)(h - p.Hq) * D
                                          : static_cast<const T *>(p.v_in) + row * p.v_stride + (size_t)(h - p.Hq - p.Hkv) * D;
        return reinterpret_cast<const uint4 *>(src);
    };
    uint4 in0[kPlaceAhead], in1[kPlaceAhead];
    auto ask = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kPlaceAhead; ++u) {
            const int h = h0 + u * HPB;
            if (h < heads) {
                const uint4 *src = source(h);
                in0[u] = src[v0];
                in1[u] = src[v1];
            }
        }
    };
    ask(group);
    for (int i = threadIdx.x; i < half_rot; i += kPlaceThreads) {
        const double t = (double)p.pos[row] * turns.f[i];
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        s_cos[i] = c * p.magnitude;
        s_sin[i] = s * p.magnitude;
    }
    __syncthreads();
    // The lane's pairs, for all heads of the row.  Half-split: the VE pairs of vector v0; interleaved: VE / 2 pairs of
    // v0, then VE / 2 of v1.
    float cs[VE], sn[VE];
    bool turned[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        const int pair = kInterleaved ? (e < VE / 2 ? v0 * (VE / 2) + e : v1 * (VE / 2) + e - VE / 2) : j * VE + e;
        turned[e] = pair < half_rot;
        cs[e] = turned[e] ? s_cos[pair] : 1.f;
        sn[e] = turned[e] ? s_sin[pair] : 0.f;
    }
    for (int h0 = group; h0 - group < heads; h0 += kPlaceAhead * HPB) {      // (uniform over the block: the shuffles below need whole warps)
        if (h0 != group) ask(h0);
#pragma unroll
        for (int u = 0; u < kPlaceAhead; ++u) {
            const int h = h0 + u * HPB;
            if (h - group >= heads) break;
            const bool is_q = h < p.Hq, is_k = !is_q && h < p.Hq + p.Hkv;
            float x[2 * VE];
            unpack16<T>(in0[u], x);
            unpack16<T>(in1[u], x + VE);
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 2 * VE; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
            for (int off = LPH / 2; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
            if (h >= heads || (!is_q && no_page)) continue;
            uint4 out0 = in0[u], out1 = in1[u];
            if (is_q || is_k) {
                if (p.norm & (is_q ? HT_HEAD_NORM_Q : HT_HEAD_NORM_K)) {
                    const float inv = 1.f / sqrtf(ss * (1.f / D) + p.eps);
                    const uint4 *w = static_cast<const uint4 *>(is_q ? p.q_weight : p.k_weight);
                    if (w) {
                        float wf[2 * VE];
                        unpack16<T>(__ldg(w + v0), wf);
                        unpack16<T>(__ldg(w + v1), wf + VE);
#pragma unroll
                        for (int e = 0; e < 2 * VE; ++e) x[e] *= inv * (wf[e] + p.offset);
                    } else {
#pragma unroll
                        for (int e = 0; e < 2 * VE; ++e) x[e] *= inv;
                    }
                }
                if (rotates) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        const int a = kInterleaved ? 2 * e : e, c = kInterleaved ? 2 * e + 1 : e + VE;
                        if (turned[e]) {
                            const float xa = x[a], xc = x[c];
                            x[a] = xa * cs[e] - xc * sn[e];
                            x[c] = xc * cs[e] + xa * sn[e];
                        }
                    }
                }
                T o[2 * VE];
#pragma unroll
                for (int e = 0; e < 2 * VE; ++e) o[e] = from_float<T>(x[e]);
                out0 = *reinterpret_cast<const uint4 *>(o);
                out1 = *reinterpret_cast<const uint4 *>(o + VE);
            }
            T *dst = is_q   ? static_cast<T *>(p.q_out) + (row * p.Hq + h) * D
                     : is_k ? static_cast<T *>(p.k_cache) + row_off + (size_t)(h - p.Hq) * p.stride_h
                            : static_cast<T *>(p.v_cache) + row_off + (size_t)(h - p.Hq - p.Hkv) * p.stride_h;
            reinterpret_cast<uint4 *>(dst)[v0] = out0;
            reinterpret_cast<uint4 *>(dst)[v1] = out1;
        }
    }
}

// Turns per position of each pair.  By parts (Peng et al., "YaRN", arXiv 2309.00071, Section 3.2): a pair that turns
// more than `high` times over the original context keeps its frequency, one that turns less than `low` times has it
// divided by the factor, with a linear ramp in between.
static RopeTurns make_turns(const ht_head_desc &h) {
    RopeTurns t{};
    const double two_pi = 6.283185307179586476925;
    for (int i = 0; i < h.rot_dim / 2; ++i) {
        double f = pow((double)h.rope_base, -2.0 * i / h.rot_dim) / two_pi;
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

template <typename T>
static int launch_t(const PlaceArgs &a, const PageMap &pm, const RopeTurns &turns, int D, bool interleaved, unsigned blocks, cudaStream_t s) {
    if (D == 64) {
        if (interleaved) norm_rope_kernel<T, 64, true><<<blocks, kPlaceThreads, 0, s>>>(a, pm, turns);
        else norm_rope_kernel<T, 64, false><<<blocks, kPlaceThreads, 0, s>>>(a, pm, turns);
    } else {
        if (interleaved) norm_rope_kernel<T, 128, true><<<blocks, kPlaceThreads, 0, s>>>(a, pm, turns);
        else norm_rope_kernel<T, 128, false><<<blocks, kPlaceThreads, 0, s>>>(a, pm, turns);
    }
    return check_launch("ht_norm_rope_kv_append");
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
    const unsigned blocks = (unsigned)((long long)d.B * d.N);
    const bool il = h.interleaved != 0;
    switch (d.dtype) {
        case HT_F32: return launch_t<float>(a, pm, turns, d.D, il, blocks, s);
        case HT_F16: return launch_t<__half>(a, pm, turns, d.D, il, blocks, s);
        default: return launch_t<__nv_bfloat16>(a, pm, turns, d.D, il, blocks, s);
    }
}

}  // namespace ht
