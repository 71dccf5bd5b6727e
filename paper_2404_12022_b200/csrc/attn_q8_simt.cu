// Tree attention over an 8-bit cache on the fp32 ALUs: fp32 queries, heads of 64, groups that are no power of two -- what the
// tensor-core kernel (attn_q8.cu) does not take -- contiguous or paged.  The split-KV design of attn_simt.cu:
//   block = 8 warps, a query row of one head each; 32 keys at a time are staged as fp32 values (code * 2^e), lane j scores
//   key j, running maximum and sum by shuffles, each lane owns D / 32 output features; with several splits (m, l, O) parts
//   go to the workspace and a second kernel merges them.
// Bound by the ALUs: 2 x 32 x D products per row and step against 64 D bytes.  Steps of context rows that no row of the block sees
// (outside the window and behind the first tokens) are jumped over.  1 x 91 rows of 32 heads of 128 on 1024 keys in fp32: 295 us = 5.4 TFLOP/s;
// heads of 64 in bf16 161 us.
#include "q8.cuh"

namespace ht {
namespace q8simt {

constexpr int kRows = 8;          // query rows (warps) per block
constexpr int kKeys = 32;         // keys per staged tile
constexpr int kMaxWords = 32;     // ancestor words per row -> N <= 1024
constexpr float kLog2e = 1.4426950408889634f;

struct Params {
    const void *q;
    const unsigned char *kc, *vc, *k_scale, *v_scale;
    void *out;
    float *part;                  // [B, N, Hq, splits, 2 + D] when splits > 1
    const int32_t *kv_len, *parent;
    int32_t *status;
    int B, N, Hq, Hkv, cap, splits, window, sinks;
    long long stride_b, stride_h, scale_b, scale_h;      // bytes; between pages where paged
    float scale_log2;
    PageMap pm;
};

// The number a code stands for times the row's power of two (the two codes that e4m3 keeps for NaN: +-480, as in attn_q8.cu).
__device__ __forceinline__ float decode(uint32_t byte, float factor) {
    return __uint_as_float((byte & 0x80u) << 24 | (byte & 0x7Fu) << 20) * 0x1p120f * factor;
}

template <typename T, int D>
__global__ void __launch_bounds__(kRows * 32)
attn_q8_simt_kernel(const Params p) {
    constexpr int DPL = D / 32;
    __shared__ float Ks[kKeys][D + 1];
    __shared__ float Vs[kKeys][D];
    __shared__ float Qs[kRows][D];
    __shared__ uint32_t anc[kRows][kMaxWords];
    __shared__ int s_bad, s_lo;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = blockIdx.y;
    const int b = blockIdx.z / p.splits, split = blockIdx.z - b * p.splits;
    const int r = blockIdx.x * kRows + warp;
    const int N = p.N, L = p.kv_len[b];
    const int32_t *par = p.parent + (size_t)b * N;

    // Legality of this sequence's inputs; every block of the sequence comes to the same decision.
    if (threadIdx.x == 0) { s_bad = 0; s_lo = 0x7fffffff; }
    __syncthreads();
    for (int c = threadIdx.x; c < N; c += blockDim.x)
        if (par[c] < -1 || par[c] >= c) s_bad = HT_STATUS_BAD_TREE;
    __syncthreads();
    int code = s_bad;
    if (L < 0 || (long long)L + N > p.cap) code = HT_STATUS_BAD_LEN;
    const long long first_seen = p.window > 0 ? max(0ll, (long long)L - p.window + 1) : 0ll;
    if (p.pm.table && code == HT_STATUS_OK) {
        __syncthreads();
        for (int i = threadIdx.x; i <= (L + N - 1) >> p.pm.shift; i += blockDim.x) {
            const long long row0 = (long long)i << p.pm.shift;        // pages that no row sees need no entry
            const bool seen = row0 + (1 << p.pm.shift) > first_seen || row0 < p.sinks;
            if (seen && (unsigned)p.pm.table[(size_t)b * p.pm.max_pages + i] >= (unsigned)p.pm.n_pages) s_bad = HT_STATUS_BAD_PAGE;
        }
        __syncthreads();
        code = s_bad;
    }
    if (blockIdx.x == 0 && h == 0 && split == 0 && threadIdx.x == 0) p.status[b] = code;
    if (code != HT_STATUS_OK) return;

    const int words = (N + 31) >> 5;
    const bool row_ok = r < N;
    for (int w = lane; w < words; w += 32) anc[warp][w] = 0;
    __syncwarp();
    int row_lo = 0;
    if (row_ok) {
        if (lane == 0) {
            int depth = 0, back = 0;
            if (p.window > 0) {
                for (int c = par[r]; c >= 0; c = par[c]) ++depth;
                row_lo = (int)max(0ll, (long long)L + depth - p.window + 1);
            }
            for (int c = r; c >= 0; c = par[c], ++back)
                if (p.window == 0 || back < p.window || (long long)L + depth - back < p.sinks) anc[warp][c >> 5] |= 1u << (c & 31);
            atomicMin(&s_lo, row_lo);
        }
        row_lo = __shfl_sync(0xffffffffu, row_lo, 0);
    }
    const T *qrow = static_cast<const T *>(p.q) + (((size_t)b * N + (row_ok ? r : 0)) * p.Hq + h) * D;
    for (int x = lane; x < D; x += 32) Qs[warp][x] = to_float<T>(qrow[x]);
    __syncthreads();
    const int block_lo = min(s_lo, L);                 // (tree rows stand where their depth puts them: never jumped over)

    const int total = L + N;
    int chunk = (total + p.splits - 1) / p.splits;
    chunk = (chunk + kKeys - 1) / kKeys * kKeys;
    const long long k_begin = (long long)split * chunk;
    const int k_end = (int)min((long long)total, k_begin + chunk);
    const int hk = h / (p.Hq / p.Hkv);

    float m = -INFINITY, l = 0.f, o[DPL];
#pragma unroll
    for (int i = 0; i < DPL; ++i) o[i] = 0.f;

    for (long long k0l = k_begin; k0l < k_end; k0l += kKeys) {
        int k0 = (int)k0l;
        if (k0 >= p.sinks && k0 + kKeys <= block_lo) {     // nobody of the block sees these: on to the step with the first key seen
            k0 += (block_lo - k0) / kKeys * kKeys;
            k0l = k0;
            if (k0 >= k_end) break;
        }
        __syncthreads();                               // previous tile fully consumed
        constexpr int VPR = D / 16;                    // 16-byte pieces per row
        for (int t = threadIdx.x; t < kKeys * VPR; t += blockDim.x) {
            const int j = t / VPR, v = t - j * VPR, key = k0 + j;
            if (key < k_end && (key >= first_seen || key < p.sinks)) {        // what no row sees is no data, whatever lies there
                long long row = (long long)b * p.stride_b + (long long)hk * p.stride_h + (long long)key * D;
                long long at = (long long)b * p.scale_b + (long long)hk * p.scale_h + key;
                if (p.pm.table) {
                    const int page = p.pm.table[(size_t)b * p.pm.max_pages + (key >> p.pm.shift)];       // inside the pool: looked at above
                    const int in = key & ((1 << p.pm.shift) - 1);
                    row = (long long)page * p.stride_b + (long long)hk * p.stride_h + (long long)in * D;
                    at = (long long)page * p.scale_b + (long long)hk * p.scale_h + in;
                }
                const int ek = p.k_scale[at], ev = p.v_scale[at];
                // a row that is not a number in K or V makes its score so, and counts for nobody who does not see it
                const bool nan = ek == 255 || ev == 255;
                const float fk = nan ? __uint_as_float(0x7FC00000u) : (ek == 0 ? 0x1p-127f : __uint_as_float((uint32_t)ek << 23));
                const float fv = nan ? 0.f : (ev == 0 ? 0x1p-127f : __uint_as_float((uint32_t)ev << 23));
                const uint4 kw = ld_nc16(p.kc + row + v * 16), vw = ld_nc16(p.vc + row + v * 16);
                const uint32_t kk[4] = {kw.x, kw.y, kw.z, kw.w}, vv[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    Ks[j][v * 16 + e] = decode(kk[e / 4] >> (8 * (e % 4)) & 255u, fk);
                    Vs[j][v * 16 + e] = decode(vv[e / 4] >> (8 * (e % 4)) & 255u, fv);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) Ks[j][v * 16 + e] = Vs[j][v * 16 + e] = 0.f;
            }
        }
        __syncthreads();
        if (!row_ok) continue;

        const int key = k0 + lane;
        float s = 0.f;
#pragma unroll 8
        for (int x = 0; x < D; ++x) s = fmaf(Qs[warp][x], Ks[lane][x], s);
        s *= p.scale_log2;
        bool visible = key < k_end;
        if (visible && key >= L) {
            const int c = key - L;
            visible = (anc[warp][c >> 5] >> (c & 31)) & 1u;
        } else {
            visible = visible && (key >= row_lo || key < p.sinks);
        }
        if (!__any_sync(0xffffffffu, visible)) continue;   // nothing of this step is visible to the row
        s = visible ? s : -INFINITY;
        float tile_max = s;                                // (a score that is no number is passed over here, and met in the sum)
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) tile_max = fmaxf(tile_max, __shfl_xor_sync(0xffffffffu, tile_max, off));
        const float m_new = fmaxf(m, tile_max);
        const float base = m_new == -INFINITY ? 0.f : m_new;
        const float corr = m == -INFINITY ? 0.f : exp2f(m - base);
        const float pj = visible ? exp2f(s - base) : 0.f;
        float psum = pj;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) psum += __shfl_xor_sync(0xffffffffu, psum, off);
        l = l * corr + psum;
        m = m_new;
#pragma unroll
        for (int i = 0; i < DPL; ++i) o[i] *= corr;
#pragma unroll 4
        for (int j = 0; j < kKeys; ++j) {
            const float pb = __shfl_sync(0xffffffffu, pj, j);
#pragma unroll
            for (int i = 0; i < DPL; ++i) o[i] = fmaf(pb, Vs[j][lane + 32 * i], o[i]);
        }
    }
    if (!row_ok) return;
    if (p.splits == 1) {
        T *orow = static_cast<T *>(p.out) + (((size_t)b * N + r) * p.Hq + h) * D;
        const float inv = 1.f / l;
#pragma unroll
        for (int i = 0; i < DPL; ++i) orow[lane + 32 * i] = from_float<T>(o[i] * inv);
    } else {
        float *pp = p.part + ((((size_t)b * N + r) * p.Hq + h) * p.splits + split) * (2 + D);
        if (lane == 0) { pp[0] = m; pp[1] = l; }
#pragma unroll
        for (int i = 0; i < DPL; ++i) pp[2 + lane + 32 * i] = o[i];
    }
}

// One warp per (b, r, h): out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.
template <typename T, int D>
__global__ void __launch_bounds__(128)
attn_q8_combine_kernel(const Params p) {
    constexpr int DPL = D / 32;
    const long long item = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (item >= (long long)p.B * p.N * p.Hq) return;
    const int b = (int)(item / ((long long)p.N * p.Hq));
    if (p.status[b] != HT_STATUS_OK) return;           // written by the main kernel on this stream
    const float *pp = p.part + (size_t)item * p.splits * (2 + D);
    float M = -INFINITY;
    for (int s = 0; s < p.splits; ++s) M = fmaxf(M, pp[(size_t)s * (2 + D)]);
    float l = 0.f, o[DPL];
#pragma unroll
    for (int i = 0; i < DPL; ++i) o[i] = 0.f;
    for (int s = 0; s < p.splits; ++s) {
        const float *ps = pp + (size_t)s * (2 + D);
        if (ps[0] == -INFINITY) {                      // nothing visible, or nothing that is a number
            l += ps[1];
            continue;
        }
        const float w = exp2f(ps[0] - M);
        l += w * ps[1];
#pragma unroll
        for (int i = 0; i < DPL; ++i) o[i] = fmaf(w, ps[2 + lane + 32 * i], o[i]);
    }
    T *orow = static_cast<T *>(p.out) + (size_t)item * D;
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < DPL; ++i) orow[lane + 32 * i] = from_float<T>(o[i] * inv);
}

}  // namespace q8simt

// Blocks for eight per SM, with 256 keys at least per split (1 x 91 rows of 32 heads on 1024 keys in fp32: four splits 295 us, two 324,
// none 323, eight 292; heads of 64 in bf16: 161, 176, 170 and 163).
static int choose_splits_q8(const ht_attn_desc &d) {
    if (d.num_splits > 0) return d.num_splits;
    const long long blocks = (long long)((d.N + q8simt::kRows - 1) / q8simt::kRows) * d.Hq * d.B, target = 8ll * sm_count();
    long long s = (target + blocks - 1) / blocks;
    const long long by_len = ((long long)d.cap + 255) / 256;
    if (s > by_len) s = by_len;
    return (int)(s > 64 ? 64 : (s < 1 ? 1 : s));
}

size_t attn_q8_simt_workspace(const ht_attn_desc &d, int *splits_out) {
    const int splits = choose_splits_q8(d);
    if (splits_out) *splits_out = splits;
    return splits == 1 ? 0 : (size_t)d.B * d.N * d.Hq * splits * (2 + d.D) * sizeof(float);
}

template <typename T, int D>
static int launch_simt_form(const q8simt::Params &p, cudaStream_t s) {
    const dim3 grid((p.N + q8simt::kRows - 1) / q8simt::kRows, p.Hq, p.B * p.splits);
    q8simt::attn_q8_simt_kernel<T, D><<<grid, q8simt::kRows * 32, 0, s>>>(p);
    const int rc = check_launch("ht_tree_attention_q8 (simt)");
    if (rc != HT_OK || p.splits == 1) return rc;
    const long long items = (long long)p.B * p.N * p.Hq;
    q8simt::attn_q8_combine_kernel<T, D><<<(unsigned)((items + 3) / 4), 128, 0, s>>>(p);
    return check_launch("ht_tree_attention_q8 (simt combine)");
}

int launch_attn_q8_simt(const ht_attn_desc &d, const ht_window_desc &w, const void *q, const void *kc, const void *vc, const Q8Scales &scales,
                        const int32_t *kv_len, const int32_t *parent, void *out, void *ws, size_t ws_bytes, int32_t *status, cudaStream_t s,
                        const PageMap &pm) {
    q8simt::Params p{};
    const size_t need = attn_q8_simt_workspace(d, &p.splits);
    if (need > ws_bytes) return fail(HT_ERR_WORKSPACE, "workspace holds %zu bytes, %zu needed", ws_bytes, need);
    if (d.N > q8simt::kMaxWords * 32) return fail(HT_ERR_UNSUPPORTED, "N = %d exceeds %d query rows", d.N, q8simt::kMaxWords * 32);
    if (d.Hq > 65535 || (long long)d.B * p.splits > 65535) return fail(HT_ERR_UNSUPPORTED, "Hq or B * splits exceeds 65535");
    p.q = q; p.kc = static_cast<const unsigned char *>(kc); p.vc = static_cast<const unsigned char *>(vc);
    p.k_scale = scales.k; p.v_scale = scales.v; p.out = out; p.part = static_cast<float *>(ws);
    p.kv_len = kv_len; p.parent = parent; p.status = status;
    p.B = d.B; p.N = d.N; p.Hq = d.Hq; p.Hkv = d.Hkv; p.cap = d.cap;
    p.window = w.window; p.sinks = w.window > 0 ? w.sinks : 0;
    p.stride_h = pm.table ? pm.head_stride : (d.kv_stride_h ? d.kv_stride_h : (long long)d.cap * d.D);
    p.stride_b = pm.table ? pm.page_stride : (d.kv_stride_b ? d.kv_stride_b : (long long)d.Hkv * d.cap * d.D);
    p.scale_b = scales.stride_b; p.scale_h = scales.stride_h;
    p.scale_log2 = (d.scale > 0.f ? d.scale : 1.f / sqrtf((float)d.D)) * q8simt::kLog2e;
    p.pm = pm;
#define HT_FORM(T) (d.D == 64 ? launch_simt_form<T, 64>(p, s) : launch_simt_form<T, 128>(p, s))
    switch (d.dtype) {
        case HT_F32: return HT_FORM(float);
        case HT_F16: return HT_FORM(__half);
        default: return HT_FORM(__nv_bfloat16);
    }
#undef HT_FORM
}

}  // namespace ht
