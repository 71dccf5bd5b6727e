// Tree attention over an 8-bit cache on the 5th-generation tensor cores (Section "Tree attention": the same rows see the
// same keys; only what the cache holds differs).  A cache row of a KV head is D = 128 codes in e4m3 and one power of two.
//
// The kernel is the one of attn_tc.cu (two operands on the 5th-generation tensor cores, the softmax in registers, units cut into
// parts) fed with half the bytes, and what matters is who turns codes into numbers, at what cost:
//   S = Q K^T   takes K's codes as they are (kind::f8f6f4).  Q goes as a sum of parts in e4m3 -- bf16: two, which hold its eight
//               bits exactly, fp16: three -- each row relative to a power of two of its own; a key's power of two multiplies its
//               column of scores in the softmax, one packed multiplication per two scores.
//   O += P V    takes V in fp16, widened tile by tile in shared memory by four warps of their own: the weights need more than
//               e4m3's bits, and the type of both operands is one.  A code in fp16 is exact; a tile's rows are taken relative to the
//               largest of their powers of two, which the softmax adds to its exponents, so that a weight is held as what multiplies V's
//               fp16 values.
// Widening K as well kept the converting warps busy longer than the softmax where keys are shared: 16 x 67 rows of 64 on 8 heads
// on 8192 keys 763 us, and 580 as it stands (4 x 91 rows of 32 heads on 4096 keys 68 and 73.5 us, 1 x 91 on 1024 16 and 21: with
// few tiles per CTA it is the chain ahead of the first product that counts).  No unit is saturated (4 x 91 on 4096: issue slots
// 40 %, tensor pipe 20 %, shared memory 28 %): a tile's chain of waits is what bounds it, widening V and the maxima a tenth of the
// time each.
//
// The roles of a CTA (768 threads, one CTA per SM):
//   warp 20         copies: code tiles (16 KiB, 128-byte swizzle), and with K's the 256 scale bytes of K's and V's rows
//   warps 16-19     Q rows from global memory into parts, once per segment (the first one's: the softmax warps, idle till then);
//                   K's powers of two as floats; thread i widens row i of each V tile: eight 16-byte reads, sixteen 16-byte
//                   writes, both free of bank conflicts
//   warp 21         issues the products
//   warps 0-15      softmax: two streams of eight warps on alternate tiles, so that one's loads, maxima and waits lie under the
//                   other's exponentials; a row's 128 keys are shared by two threads of a stream
//
// A window keeps, of the context, the rows within `window` positions of the query row and the first `sinks`; tiles
// between the two that no row of the sequence sees are not in the list of tiles at all.  More than 128 query rows per KV
// head are several row tiles: the CTAs of a group take the same range of keys side by side, one row tile each, so that a
// key tile crosses DRAM once and comes to the others from L2.
//
// Every wait is bounded.  A warp whose wait has run out (or that sees that another's has) touches nothing more: the copying,
// converting and issuing warps leave their loops, without arriving anywhere; the softmax warps go on through their barriers alone.
// What is in flight is waited for before the CTA leaves, and the sequences' status words say HT_STATUS_TIMEOUT.
#include <stddef.h>

#include "attn_tc.cuh"
#include "q8.cuh"

namespace ht {
namespace q8 {

using namespace tc;

constexpr int kQ8Threads = 768;
constexpr int kConvThreads = 128, kConvWarp = 16, kCopyWarp = 20, kMmaWarp = 21;
constexpr int kWide = 2;                    // ring of V tiles in fp16
constexpr int kRawK = 3, kRawV = 2;         // rings of code tiles
constexpr int kParts = 3;                   // parts of Q at most
constexpr int kRawBytes = kTile * kD;
constexpr float kWeightLift = 7.f;          // weights are held as 2^7 of what they are: up to 2^15 where the reference lags, and 2^-31 before fp16 loses them

// What the kernel needs besides Params and PagedParams.
struct Q8Params {
    const void *q;
    const unsigned char *k_scale, *v_scale;    // bytes: 2^(byte - 127); 255 marks a row that is not a number
    long long scale_b, scale_h;                // bytes between sequences (pages, if paged) / heads
    int window, sinks;                         // window 0: none
    int near_keys;                             // tiles reaching past context row kv_len - near_keys send P as a hi + lo pair
    int group;                                 // CTAs that take the row tiles of one range of keys side by side (1: row tiles are in the list)
};

struct __align__(1024) SmemQ8 {
    unsigned char q[kParts][kRawBytes];
    unsigned char wide[kWide][kEntryBytes];
    unsigned char raw_k[kRawK][kRawBytes], raw_v[kRawV][kRawBytes];
    unsigned char scale[kRawK][2][kTile];      // of the rows of the K tile in the slot, and of V's
    float factor[4][kTile];                    // powers of two of K's rows, four tiles at a time
    int32_t ref[4][2];                         // what factor, and V's fp16 values, are relative to (tile_exponent)
    int32_t q_exp[4][kRows];                   // exponents of a segment's Q rows, four segments at a time
    float mx[2][2][kRows], sum[2][2][kRows];   // by stream and half of a row's keys
    float ref_row[2][kRows];                   // the streams' references
    int32_t len[kMaxB], nkt[kMaxB], pre[kMaxB + 1];
    int32_t len_listed[kMaxB];                 // context rows less those of tiles that are not in the list
    int32_t seen[kMaxB];                       // where the farthest window begins (0: no window)
    int32_t gap_at[kMaxB], gap[kMaxB];         // tiles [gap_at, gap_at + gap) of the sequence are not in the list
    int32_t plan[kPlanWords];
    int32_t row_lo[kRows];                     // first context row that the window shows the row
    unsigned long long k_full[kRawK], k_empty[kRawK], v_full[kRawV], v_empty[kRawV], w_full[kWide], w_empty[kWide];
    unsigned long long q_empty, s_full[2], p_ready[2], o_done[2], ref_full[4], q_ready[4], mma_drain;
    int abort, wait_kcycles;                   // as in Smem
    uint32_t tmem_base;
    int merge_here[2];
    int direct;
    int32_t pg[kPgTiles][kPgSub];
    uint32_t anc[kMaxWords][kRows];            // last member: only ceil(N / 32) words are allocated
};
static_assert(sizeof(SmemQ8) + 1024 <= 232448, "shared memory of a CTA");
static_assert(kXchgBytes <= kWide * kEntryBytes + (kParts + kRawK + kRawV) * kRawBytes, "the exchange area is the Q buffer and the rings");

// Tile of the sequence that is the kt-th of its list.
__device__ __forceinline__ int tile_of(const SmemQ8 &sm, int b, int kt) { return kt < sm.gap_at[b] ? kt : kt + sm.gap[b]; }

__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, void *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// 16 consecutive TMEM columns of this thread's lane.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float *v) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// ---------------------------------------------------------------------------------------
// Codes to fp16 values
// ---------------------------------------------------------------------------------------
// Two codes in the lower / upper half of w -> two fp16 values, exactly.
__device__ __forceinline__ uint32_t widen_lo(uint32_t w) {
    uint32_t d;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(d) : "r"(w));
    return d;
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t w) {
    uint32_t d;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(d) : "r"(w));
    return d;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// 2^e, e in [-126, 127].
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Rows of a tile that hold data: below `valid`, and not in [hide_lo, hide_hi), behind the first tokens and ahead of the farthest
// window: no row of the sequence sees those, and whatever a spare page holds may lie there.
struct TileRows {
    int valid, hide_lo, hide_hi;
    __device__ __forceinline__ bool all() const { return valid >= kTile && (hide_hi <= 0 || hide_lo >= kTile); }
    __device__ __forceinline__ bool data(int row) const { return row < valid && !(row >= hide_lo && row < hide_hi); }
};
// The bytes of the lane's four rows, 4 * lane and on, that are data.
__device__ __forceinline__ uint32_t data_bytes(const TileRows &rows, int lane) {
    uint32_t keep = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) keep |= rows.data(4 * lane + i) ? 255u << (8 * i) : 0u;
    return keep;
}
// The exponent that a tile's values are taken relative to, from the scale bytes of its rows (of this lane's, those in `keep`;
// rows marked as no numbers do not count): `below` less than the largest.  Alike in all lanes of the warp.
__device__ __forceinline__ int tile_exponent(const unsigned char *scale, int lane, uint32_t keep, int below) {
    const uint32_t w = *reinterpret_cast<const uint32_t *>(scale + 4 * lane) & keep;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t byte = w >> (8 * i) & 255u;
        top = max(top, byte != 255u ? byte : 0u);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    return max((int)top - 127 - below, -100);
}

// One row of a V tile: raw tile and fp16 tile both in rows of 128 bytes with 16-byte pieces exchanged by the row's number
// (128-byte swizzle); the fp16 tile as two slabs of 64 features.  factor: the row's power of two, twice; zero: nothing of the row
// is data.
__device__ __forceinline__ void widen_row(const unsigned char *raw, unsigned char *wide, int row, bool zero, uint32_t factor) {
    const int sw = row & 7;
    const uint4 *src = reinterpret_cast<const uint4 *>(raw + row * 128);
    unsigned char *dst = wide + row * 128;
    if (zero) factor = 0u;
    const uint32_t keep = zero ? 0u : 0xFFFFFFFFu;          // (whatever the bytes are, NaN included)
#pragma unroll 1
    for (int c0 = 0; c0 < 8; c0 += 4) {
        uint4 in[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) in[c] = src[(c0 + c) ^ sw];
        uint4 *slab = reinterpret_cast<uint4 *>(dst + (c0 >> 2) * kSlabBytes);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t w4[4] = {in[c].x & keep, in[c].y & keep, in[c].z & keep, in[c].w & keep};
            uint32_t out[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                out[2 * i] = mul_f16x2(widen_lo(w4[i]), factor);
                out[2 * i + 1] = mul_f16x2(widen_hi(w4[i]), factor);
            }
            slab[(2 * c) ^ sw] = make_uint4(out[0], out[1], out[2], out[3]);
            slab[(2 * c + 1) ^ sw] = make_uint4(out[4], out[5], out[6], out[7]);
        }
    }
}

__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    unsigned short w;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(w) : "f"(hi), "f"(lo));
    return w;
}
// A row of Q (128 values in global memory, or none) times 2^-e, which brings its largest value to 128 .. 256, as a sum of parts
// in e4m3: each part takes four bits and leaves the rest, exactly, to the next, down to 2^-9.  bf16's eight bits are two
// parts' wherever a value is not 2^9 times smaller than the row's largest, fp16's eleven three parts' down to 2^6 times
// smaller; below, what is left over is at most 2^-10, 2^-17 of the largest value.  e is 0 for a row of zeros.  A row with an
// infinity or a NaN has no result that is a number (its scores are infinite or none, whatever the keys): all of it becomes NaN, as
// the conversion would make 448 of an infinity.  Four lanes next to one another take a row; `quarter` is this one's, and all lanes of the warp are here.
template <bool kBf16>
struct QuarterRow {
    uint4 in[4];
    __device__ __forceinline__ void load(const uint4 *src, int quarter) {
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i] = src ? __ldg(src + 2 * (quarter + (i >> 1) * 4) + (i & 1)) : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ int split(unsigned char (*q)[kRawBytes], int row, int quarter) const {
        constexpr int kOwnParts = kBf16 ? 2 : 3;
        uint32_t top = 0;                                   // the bits of the largest magnitude, in the type's 16
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t w4[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, max(w4[i] >> 16 & 0x7FFFu, w4[i] & 0x7FFFu));
        }
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const float largest = kBf16 ? __uint_as_float(top << 16) : __half2float(__ushort_as_half((unsigned short)top));
        const uint32_t bits = __float_as_uint(largest);
        const int e = bits == 0u || bits >= 0x7F800000u ? 0 : max((int)(bits >> 23) - 134, -100);
        const float factor = bits >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : pow2(-e);
#pragma unroll
        for (int k = 0; k < 2; ++k) {                       // 16 values: 16 bytes of each part
            const int c = quarter + 4 * k;
            float x[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint4 v = in[2 * k + (i >> 2)];
                const uint32_t w = (i & 3) == 0 ? v.x : ((i & 3) == 1 ? v.y : ((i & 3) == 2 ? v.z : v.w));
                float a, b;
                if (kBf16) {
                    a = __uint_as_float(w << 16);
                    b = __uint_as_float(w & 0xFFFF0000u);
                } else {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
                    a = f.x;
                    b = f.y;
                }
                x[2 * i] = a * factor;
                x[2 * i + 1] = b * factor;
            }
#pragma unroll
            for (int part = 0; part < kOwnParts; ++part) {
                uint32_t out[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo = to_e4m3x2(x[4 * i], x[4 * i + 1]), hi = to_e4m3x2(x[4 * i + 2], x[4 * i + 3]);
                    out[i] = lo | hi << 16;
                    if (part + 1 < kOwnParts) {
                        const uint32_t l = widen_lo(lo), h = widen_lo(hi);
                        const float2 fl = __half22float2(*reinterpret_cast<const __half2 *>(&l)), fh = __half22float2(*reinterpret_cast<const __half2 *>(&h));
                        x[4 * i] -= fl.x;
                        x[4 * i + 1] -= fl.y;
                        x[4 * i + 2] -= fh.x;
                        x[4 * i + 3] -= fh.y;
                    }
                }
                *reinterpret_cast<uint4 *>(q[part] + row * 128 + ((c ^ (row & 7)) << 4)) = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
        return e;
    }
};
// The row of Q that is row `row` of row tile rt of a segment; nullptr: padding.
__device__ __forceinline__ const uint4 *q_row(const Params &p, const Q8Params &qp, const Segment &at, int rt, int row) {
    const int node = rt * p.rows_per_tile_nodes + row / p.g, head = at.hk * p.g + row % p.g;
    return node < p.N ? static_cast<const uint4 *>(qp.q) + (((long long)at.b * p.N + node) * p.Hq + head) * (kD * 2 / 16) : nullptr;
}

// The products, issued by one lane of a warp whose lanes all walk the same code: descriptors, slots and phases are then uniform
// values, which the instructions take as they are (computed by one lane alone they are moved to uniform registers one by one).
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t e;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(e));
    return e;
}
// D[tmem] (+)= A[smem] B[smem]^T, e4m3
__device__ __forceinline__ void mma_codes(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t elected) {
    asm volatile(
        "{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 e, %5, 0;\n@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
        ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
// D[tmem] (+)= A[tmem] B[smem], fp16
__device__ __forceinline__ void mma_pv(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t elected) {
    asm volatile(
        "{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 e, %5, 0;\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t bar_addr, uint32_t elected) {
    asm volatile("{\n.reg .pred e;\nsetp.ne.b32 e, %1, 0;\n@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}"
                 ::"r"(bar_addr), "r"(elected) : "memory");
}

// ---------------------------------------------------------------------------------------
// Plan
// ---------------------------------------------------------------------------------------
// Validates every sequence and fills len / nkt / pre and the gaps, as plan_sequences does for a list without gaps.  Called
// by all threads of a block; ends with a barrier.
__device__ __forceinline__ void plan_q8(const Params &p, const Q8Params &qp, SmemQ8 &sm, bool write_status, bool errors_only, int units_per_head,
                                        const RangeAsk &ask) {
    const int my_b = threadIdx.x;
    const int my_L = my_b < p.B ? p.kv_len[my_b] : 0;
    const int entries = p.B * p.N;
    bool saw_bad = false;
    for (int i = threadIdx.x; i < entries; i += kQ8Threads) {
        const int b = fast_div(i, p.N), par = p.parent[i];
        saw_bad = saw_bad || par < -1 || par >= i - b * p.N;
    }
    if (__syncthreads_or(saw_bad)) {
        for (int b = threadIdx.x; b < p.B; b += kQ8Threads) sm.nkt[b] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < entries; i += kQ8Threads) {
            const int b = i / p.N, par = p.parent[i];
            if (par < -1 || par >= i - b * p.N) sm.nkt[b] = -1;      // benign race: all writers store -1
        }
        __syncthreads();
        saw_bad = my_b < p.B && sm.nkt[my_b] < 0;
        __syncthreads();
    } else {
        saw_bad = false;
    }
    if (my_b < p.B) {
        const int L = my_L;
        int code = HT_STATUS_OK;
        if (saw_bad) code = HT_STATUS_BAD_TREE;
        if (L < 0 || (long long)L + p.N > p.cap) code = HT_STATUS_BAD_LEN;
        int n = 0, gap_at = 0, gap = 0, seen = 0;
        if (code == HT_STATUS_OK) {
            n = (L + p.N + kTile - 1) / kTile;
            gap_at = n;
            if (qp.window > 0) {
                seen = max(L - qp.window + 1, 0);            // rows that hang off the context see the farthest
                const int first = seen / kTile, kept = (int)(((long long)min(qp.sinks, L) + kTile - 1) / kTile);
                if (first > kept) {
                    gap_at = kept;
                    gap = first - kept;
                }
            }
            n -= gap;
        }
        sm.len[my_b] = L;
        sm.seen[my_b] = seen;
        sm.len_listed[my_b] = L - gap * kTile;
        sm.nkt[my_b] = n;
        sm.gap_at[my_b] = gap_at;
        sm.gap[my_b] = gap;
        if (write_status && (code != HT_STATUS_OK || !errors_only)) p.status[my_b] = code;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        // prefix sums of the units' tiles, 32 sequences at a time
        int before = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int b = b0 + (int)threadIdx.x;
            const int mine = b < p.B ? sm.nkt[b] * p.Hkv * units_per_head : 0;
            int inc = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xFFFFFFFFu, inc, off);
                if ((int)threadIdx.x >= off) inc += o;
            }
            if (b < p.B) sm.pre[b] = before + inc - mine;
            before += __shfl_sync(0xFFFFFFFFu, inc, 31);
        }
        if (threadIdx.x == 0) sm.pre[p.B] = before;
        __syncwarp();
        if (threadIdx.x == 0) plan_range(sm.len_listed, sm.nkt, sm.pre, p.B, p.Hkv, units_per_head, ask, sm.plan);
    }
    __syncthreads();
}

__device__ __forceinline__ void softmax_sync() {            // the 512 softmax threads
    asm volatile("bar.sync 1, 512;" ::: "memory");
}
// Barrier of the two warps that share 32 rows of a tile (ids from 2 on); the second form tells whether any thread brought `mine`.
__device__ __forceinline__ void pair_sync(int id) {
    asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
}
__device__ __forceinline__ bool pair_any(int id, bool mine) {
    uint32_t any;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %2, 0;\nbarrier.cta.red.or.pred q, %1, 64, p;\nselp.u32 %0, 1, 0, q;\n}"
                 : "=r"(any) : "r"(id), "r"((uint32_t)mine) : "memory");
    return any != 0;
}

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xFFFFFFFFu : (n <= 0 ? 0u : (1u << n) - 1u); }

// 16 scores of this thread's row from TMEM, each times its key's power of two (a NaN for a key that is no number); kMasked: the
// keys whose bit in `vis` is clear -inf, whatever they were.
template <bool kMasked>
__device__ __forceinline__ void load_scores(float (&x)[16], uint32_t addr, const float *factor, uint32_t vis) {
    tmem_ld16(addr, x);
    float4 f[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) f[c] = reinterpret_cast<const float4 *>(factor)[c];
    tmem_ld_wait();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        x[4 * c] *= f[c].x;
        x[4 * c + 1] *= f[c].y;
        x[4 * c + 2] *= f[c].z;
        x[4 * c + 3] *= f[c].w;
    }
    if (kMasked) {
#pragma unroll
        for (int c = 0; c < 16; ++c) x[c] = ((vis >> c) & 1u) ? x[c] : -INFINITY;
    }
}
// What a tile costs here is decided by how much code its scores run through, more than by its arithmetic: the loops below hold 16
// keys each and are not unrolled (unrolled over a thread's 64 keys: 4 x 91 rows on 4096 keys 95 us, in two runs of 32 78 us).
// The largest of this thread's 64 scores.
template <bool kMasked>
__device__ __forceinline__ float scores_max(uint32_t addr, const float *factor, unsigned long long vis) {
    float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll 1
    for (int q = 0; q < 64; q += 16) {
        float x[16];
        load_scores<kMasked>(x, addr + q, factor + q, (uint32_t)(vis >> q));
#pragma unroll
        for (int c = 0; c < 16; c += 4) {
            mx0 = max3(mx0, x[c], x[c + 1]);
            mx1 = max3(mx1, x[c + 2], x[c + 3]);
        }
    }
    return fmaxf(mx0, mx1);
}
// Their weights 2^(scale x + lift), the sum returned, P to TMEM over scores already consumed: packed 16-bit pairs in the half's
// columns [0, 32), or (kHiLo) as pairs hi + lo, chunk by chunk of 32 keys, hi in the chunk's columns [0, 16) and lo in [16, 32).
template <bool kMasked, bool kHiLo>
__device__ __forceinline__ float scores_weights(uint32_t addr, const float *factor, unsigned long long vis, float scale, float lift) {
    float sum0 = 0.f, sum1 = 0.f;
    uint32_t held[8];                                        // kHiLo: a chunk's first eight pairs of lo, until its scores are consumed
#pragma unroll 1
    for (int q = 0; q < 64; q += 16) {
        float x[16];
        load_scores<kMasked>(x, addr + q, factor + q, (uint32_t)(vis >> q));
        uint32_t r[8], r_lo[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float p0 = ex2(fmaf(x[2 * c], scale, lift)), p1 = ex2(fmaf(x[2 * c + 1], scale, lift));
            sum0 += p0;
            sum1 += p1;
            r[c] = pack2<false>(p0, p1);
            if (kHiLo) r_lo[c] = pack2_rest<false>(p0, p1, r[c]);
        }
        if (!kHiLo) {
            tmem_st8(addr + q / 2, r);
        } else if (q & 16) {
            tmem_st8(addr + q - 8, r);
            tmem_st8(addr + q, held);
            tmem_st8(addr + q + 8, r_lo);
        } else {
            tmem_st8(addr + q, r);
#pragma unroll
            for (int c = 0; c < 8; ++c) held[c] = r_lo[c];
        }
    }
    return sum0 + sum1;
}

// Merge of the parts of a cut unit by the 512 softmax threads of the CTA that delivered the last part: four threads to a row, 32
// features each, 16 at a time, so that the loads of several parts are on their way together within the kernel's 80 registers.
// Which CTA comes last, and whether the last of two finishes the unit from its accumulators instead, is a matter of timing: the
// arithmetic is the same, product by product, so that the result is not.
template <bool kBf16>
__device__ __noinline__ void merge_parts_q8(const Params &p, const CutUnit &cu, int per, int tid) {
    const int row = tid & 127, quarter = tid >> 7;
    const int node = cu.rt * p.rows_per_tile_nodes + row / p.g;
    if (node >= p.N) return;
    auto part = [&](int c) {
        const int slot = 2 * (c * cu.cta_mul + cu.cta_add) + ((max(cu.t0, c * per) == c * per) ? 0 : 1);
        return p.part + (size_t)slot * kSlotFloats;
    };
    float M = -INFINITY, l = 0.f;
#pragma unroll 4
    for (int c = cu.c_lo; c <= cu.c_hi; ++c) {
        const float *at = part(c) + kRows * kD + row;
        const float m = __ldcg(at), lp = __ldcg(at + kRows), Mn = fmaxf(M, m);
        const float fa = (M == -INFINITY) ? 0.f : exp2f(M - Mn), fb = (m == -INFINITY) ? 0.f : exp2f(m - Mn);
        l = fmaf(l, fa, lp * fb);
        M = Mn;
    }
    const float inv = 1.f / l;
    unsigned char *dst = static_cast<unsigned char *>(p.out) + ((((size_t)cu.b * p.N + node) * p.Hq + cu.hk * p.g + row % p.g) * kD + quarter * 32) * 2;
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
        float acc[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[x] = 0.f;
#pragma unroll 2
        for (int c = cu.c_lo; c <= cu.c_hi; ++c) {
            const float *at = part(c);
            const float m = __ldcg(at + kRows * kD + row);
            float4 v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = __ldcg(reinterpret_cast<const float4 *>(at) + (quarter * 8 + half * 4 + x) * kRows + row);
            const float w = (m == -INFINITY) ? 0.f : exp2f(m - M);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                acc[4 * x] = fmaf(v[x].x, w, acc[4 * x]);
                acc[4 * x + 1] = fmaf(v[x].y, w, acc[4 * x + 1]);
                acc[4 * x + 2] = fmaf(v[x].z, w, acc[4 * x + 2]);
                acc[4 * x + 3] = fmaf(v[x].w, w, acc[4 * x + 3]);
            }
        }
        uint32_t o[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) o[x] = pack2<kBf16>(acc[2 * x] * inv, acc[2 * x + 1] * inv);
        reinterpret_cast<uint4 *>(dst + half * 32)[0] = make_uint4(o[0], o[1], o[2], o[3]);
        reinterpret_cast<uint4 *>(dst + half * 32)[1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
}

// kPaged: the cache is a pool of pages.  kClustered: launched as clusters (p.cluster_k > 1).
template <bool kBf16, bool kPaged, bool kClustered>
__global__ void __launch_bounds__(kQ8Threads, 1)
attn_q8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Params p,
               const PagedParams pp, const Q8Params qp) {
    extern __shared__ unsigned char smem_raw[];
    SmemQ8 &sm = *reinterpret_cast<SmemQ8 *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &sm.abort;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kRawK; ++i) { mbar_init(&sm.k_full[i], 1); mbar_init(&sm.k_empty[i], kConvThreads + 1); }
        for (int i = 0; i < kRawV; ++i) { mbar_init(&sm.v_full[i], 1); mbar_init(&sm.v_empty[i], kConvThreads); }
        for (int i = 0; i < kWide; ++i) { mbar_init(&sm.w_full[i], kConvThreads); mbar_init(&sm.w_empty[i], 1); }
        mbar_init(&sm.q_empty, 1);
        mbar_init(&sm.mma_drain, 1);
        // Four of these: the converters may be two tiles, and with them two segments, ahead of the softmax.
        for (int i = 0; i < 4; ++i) { mbar_init(&sm.ref_full[i], kConvThreads); mbar_init(&sm.q_ready[i], kConvThreads); }
        // Two of each, for even and odd tiles: the softmax may be a tile ahead of the products, or the products of one tile behind,
        // and a barrier's parity tells one phase from the next only.
        for (int i = 0; i < 2; ++i) { mbar_init(&sm.s_full[i], 1); mbar_init(&sm.p_ready[i], 256); mbar_init(&sm.o_done[i], 1); }
        sm.abort = 0;
        sm.wait_kcycles = p.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32) {
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    if (warp == kCopyWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // the launch is serialized programmatically behind the kernel before it: what that one writes is read from here on
    wait_for_kernel_ahead();
    constexpr bool clustered = kClustered;
    const int group = qp.group;                                  // 1 where clustered
    const int my_pos = (int)blockIdx.x / group, my_rt = (int)blockIdx.x - my_pos * group;
    const int upl = group == 1 ? p.n_rt : 1;                      // units of a KV head in the list
    uint32_t c_rank = 0;
    RangeAsk ask;
    ask.n_pos = p.grid / group; ask.my_pos = my_pos;
    ask.cluster_k = 0; ask.cl_rank = 0; ask.cl_b = 0; ask.cl_unit = 0;
    if (clustered) {
        c_rank = cluster_ctarank();
        ask.cluster_k = p.cluster_k;                             // a power of two
        ask.cl_rank = (int)c_rank;
        const int unit = (int)blockIdx.x / p.cluster_k;
        ask.cl_b = unit / (p.Hkv * upl);
        ask.cl_unit = unit - ask.cl_b * p.Hkv * upl;
    }
    tc_fence_before();
    plan_q8(p, qp, sm, blockIdx.x == 0, kPaged, upl, ask);
    tc_fence_after();
    const uint32_t tmem = sm.tmem_base;
    const Range range = read_range(sm.plan);
    const int per = range.per, t_begin = range.t_begin, t_end = range.t_end;
    const Segment first = range.first;
    const int n = t_end - t_begin;

    if (warp == kCopyWarp) {
        // ------------------------------- copies -------------------------------
        // Contiguous cache: one thread.  Paged cache: the whole warp walks the loop, a lane per page of the tile.
        if (kPaged || lane == 0) {
            int asked_k = 0, asked_v = 0;
            TileCursor cur, cur_p;
            cur.init(t_begin, t_end, first);
            cur_p.init(t_begin, t_end, first);
            // the page ids of the next tile of the list, asked for kPgAhead tiles before the tile is fetched
            auto request_pages = [&](int jt) {
                if (cur_p.next(sm.pre, sm.nkt, p.B, upl)) {
                    const int sub = pp.page_size >= kTile ? 1 : kTile >> pp.page_shift;
                    const int at = (tile_of(sm, cur_p.s.b, cur_p.kt()) * kTile) >> pp.page_shift;
                    if (lane < sub) {
                        if (at + lane < pp.max_pages)
                            cp_async4(&sm.pg[jt % kPgTiles][lane], pp.block_table + (size_t)cur_p.s.b * pp.max_pages + at + lane);
                        else
                            sm.pg[jt % kPgTiles][lane] = -1;
                    }
                }
                cp_async_commit();
            };
            if (kPaged)
                for (int jt = 0; jt < kPgAhead; ++jt) request_pages(jt);
            uint32_t k_slot = 0, k_ph = 1, v_slot = 0, v_ph = 1;     // (a slot's first use waits for nothing)
            // Is the slot free to be armed again?  (No more copies once some wait has run out.)
            auto slot_free = [&](bool used, uint32_t bar, uint32_t ph) {
                bool ok = !used || mbar_wait_quick(bar, ph, abort_flag);
                ok = ok && *abort_flag == 0;
                return kPaged ? __all_sync(0xFFFFFFFFu, ok) != 0 : ok;
            };
            for (int j = 0; j < n; ++j) {
                cur.next(sm.pre, sm.nkt, p.B, upl);
                const int b = cur.s.b, hk = cur.s.hk, tile = tile_of(sm, b, cur.kt());
                // paged: what this lane's page is, looked up once for K and V
                long long so = (long long)b * qp.scale_b + (long long)hk * qp.scale_h + (long long)tile * kTile;
                int row0 = tile * kTile, page = b, rows = min(kTile, p.cap - tile * kTile), at = 0;      // (the capacity is a multiple of 16)
                bool mine = true;
                if (kPaged) {
                    request_pages(j + kPgAhead);
                    cp_async_wait<kPgAhead>();
                    const int ps = pp.page_size;
                    mine = lane < (ps >= kTile ? 1 : kTile >> pp.page_shift);
                    row0 = ps >= kTile ? (tile * kTile) & (ps - 1) : 0;
                    rows = min(ps, kTile);
                    at = lane << pp.page_shift;
                    if (mine) {
                        page = sm.pg[j % kPgTiles][lane];
                        if ((unsigned)page >= (unsigned)pp.n_pages) {  // page 0 in its place; reported if some row sees a key of it
                            const int key0 = tile * kTile + at;
                            if (key0 < sm.len[b] + p.N && (qp.window == 0 || key0 < qp.sinks || (long long)key0 + rows > (long long)sm.len[b] - qp.window + 1))
                                p.status[b] = HT_STATUS_BAD_PAGE;
                            page = 0;
                        }
                        so = (long long)page * qp.scale_b + (long long)hk * qp.scale_h + row0;
                    }
                }
                if (!slot_free(j >= kRawK, smem_u32(&sm.k_empty[k_slot]), k_ph)) break;
                if (lane == 0) mbar_expect_tx(&sm.k_full[k_slot], kRawBytes + 2 * (kPaged ? kTile : rows));
                if (kPaged) __syncwarp();                             // the barrier is armed before any lane's copy can complete
                if (mine) {
                    tma_load_4d(sm.raw_k[k_slot] + at * kD, &tm_k, &sm.k_full[k_slot], 0, row0, hk, page);
                    bulk_load(sm.scale[k_slot][0] + at, qp.k_scale + so, (uint32_t)rows, &sm.k_full[k_slot]);
                    bulk_load(sm.scale[k_slot][1] + at, qp.v_scale + so, (uint32_t)rows, &sm.k_full[k_slot]);
                }
                ++asked_k;
                if (!slot_free(j >= kRawV, smem_u32(&sm.v_empty[v_slot]), v_ph)) break;
                if (lane == 0) mbar_expect_tx(&sm.v_full[v_slot], kRawBytes);
                if (kPaged) __syncwarp();
                if (mine) tma_load_4d(sm.raw_v[v_slot] + at * kD, &tm_v, &sm.v_full[v_slot], 0, row0, hk, page);
                ++asked_v;
                if (++k_slot == kRawK) { k_slot = 0; k_ph ^= 1; }
                if (++v_slot == kRawV) { v_slot = 0; v_ph ^= 1; }
            }
            if (kPaged) {
                cp_async_wait<0>();
                __syncwarp();
            }
            if (lane == 0) {
                sm.plan[9] = asked_k;                      // what was asked for: should the CTA give up, the teardown waits for it
                sm.plan[10] = asked_v;
            }
        }
        if (clustered) {                                   // the two barriers of the exchange (whole warp)
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------- products -------------------------------
        const uint32_t elected = elect_one();
        // (e4m3 and fp16 are both format 0 of their kinds)
        const uint32_t idesc_qk = instr_desc(0, 0), idesc_pv = instr_desc(0, 1);
        const uint64_t q_desc = smem_desc(smem_u32(sm.q[0]), 1, 1024 >> 4), k_desc = smem_desc(smem_u32(sm.raw_k[0]), 1, 1024 >> 4);
        const uint64_t v_desc = smem_desc(smem_u32(sm.wide[0]), kSlabBytes >> 4, 1024 >> 4);
        const uint32_t bar_k_full = smem_u32(&sm.k_full[0]), bar_k_empty = smem_u32(&sm.k_empty[0]);
        const uint32_t bar_w_full = smem_u32(&sm.w_full[0]), bar_w_empty = smem_u32(&sm.w_empty[0]);
        const uint32_t bar_s_full = smem_u32(&sm.s_full[0]), bar_p_ready = smem_u32(&sm.p_ready[0]), bar_o_done = smem_u32(&sm.o_done[0]);
        const uint32_t bar_q_ready = smem_u32(&sm.q_ready[0]), bar_q_empty = smem_u32(&sm.q_empty);
        int b_hint = 0, j = 0, seg_i = 0;
        bool prev_first = false;
        bool prev_pair = false;          // does tile j - 1 send its P as a hi + lo pair?
        bool alive = true;               // false once a wait of this warp has given up: no further waits or products
        uint32_t k_slot = 0, k_ph = 0;
        auto wait = [&](uint32_t bar, uint32_t ph) {
            if (alive) alive = __all_sync(0xFFFFFFFFu, mbar_wait_quick(bar, ph, abort_flag));
        };
        auto issue_pv = [&](int jj, bool is_first, bool pair) {
            const uint32_t s = jj & 1, ph = (jj >> 1) & 1;               // (kWide is 2: V's slots alternate as the scores' buffers do)
            wait(bar_w_full + s * 8, ph);
            wait(bar_p_ready + s * 8, ph);
            if (!alive) return;
            tc_fence_after();
            const uint32_t d = tmem + 256 + s * 128, a = tmem + s * 128;
            const uint64_t v = v_desc + s * (kEntryBytes >> 4);
            if (!pair) {
                // 16 keys: 8 columns of P, 2 KiB of V; the second 64 keys' P lies 64 columns on
#pragma unroll
                for (int k = 0; k < 8; ++k) mma_pv(d, a + (k >> 2) * 64 + (k & 3) * 8, v + k * 128, idesc_pv, k > 0 || !is_first, elected);
            } else {
                // hi and lo of a chunk of 32 keys: its columns [0, 16) and [16, 32)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    mma_pv(d, a + (k >> 1) * 32 + (k & 1) * 8, v + k * 128, idesc_pv, k > 0 || !is_first, elected);
                    mma_pv(d, a + (k >> 1) * 32 + (k & 1) * 8 + 16, v + k * 128, idesc_pv, 1u, elected);
                }
            }
            commit_to(bar_w_empty + s * 8, elected);
            commit_to(bar_o_done + s * 8, elected);
        };
        for (int t = t_begin; alive && t < t_end;) {
            const Segment sg = t == t_begin ? first : locate(sm.pre, sm.nkt, p.B, upl, t, t_end, b_hint);
            const int L = sm.len[sg.b];
            wait(bar_q_ready + (seg_i & 3) * 8, (seg_i >> 2) & 1);
            for (int i = 0; alive && i < sg.len; ++i) {
                const uint32_t s = j & 1;
                wait(bar_k_full + k_slot * 8, k_ph);
                if (!alive) break;
                tc_fence_after();
                // 32 features = 32 bytes inside the swizzled row; Q's parts one after the other
                const uint64_t k = k_desc + k_slot * (kRawBytes >> 4);
#pragma unroll
                for (int x = 0; x < (kBf16 ? 8 : 12); ++x)
                    mma_codes(tmem + s * 128, q_desc + (x >> 2) * (kRawBytes >> 4) + (x & 3) * 2, k + (x & 3) * 2, idesc_qk, x > 0, elected);
                commit_to(bar_s_full + s * 8, elected);
                commit_to(bar_k_empty + k_slot * 8, elected);
                if (i == sg.len - 1) commit_to(bar_q_empty, elected);
                if (++k_slot == kRawK) { k_slot = 0; k_ph ^= 1; }
                if (j > 0) issue_pv(j - 1, prev_first, prev_pair);
                prev_first = i < 2;              // the first of its stream within the segment
                prev_pair = (tile_of(sm, sg.b, sg.kt0 + i) + 1) * kTile > L - qp.near_keys;
                ++j;
            }
            t += sg.len;
            ++seg_i;
        }
        if (j > 0) issue_pv(j - 1, prev_first, prev_pair);
        // no tensor-core operation of this CTA may be in flight when its TMEM is freed
        commit_to(smem_u32(&sm.mma_drain), elected);
        mbar_wait(&sm.mma_drain, 0, abort_flag, false);
        if (clustered) {
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();
        }
    } else if (warp >= kConvWarp && warp < kCopyWarp) {
        // ------------------------------- Q's parts, K's factors, V's tiles -------------------------------
        const int row = threadIdx.x - kConvWarp * 32;
        TileCursor cur;
        cur.init(t_begin, t_end, first);
        int seg_i = 0;
        uint32_t k_slot = 0, k_ph = 0, v_slot = 0, v_ph = 0;
        bool zero = false;                                       // of this thread's row of V tile j - 1, and its factor
        uint32_t factor = 0u;
        auto wait = [&](void *bar, uint32_t ph) { return __all_sync(0xFFFFFFFFu, mbar_wait_quick(smem_u32(bar), ph, abort_flag)) != 0; };
        for (int j = 0; j <= n; ++j) {                           // K tile j, then V tile j - 1
            bool next_zero = false;
            uint32_t next_factor = 0u;
            if (j < n) {
                cur.next(sm.pre, sm.nkt, p.B, upl);
                const int b = cur.s.b;
                if (cur.first() && seg_i++ > 0) {                // (the range's first segment: by the softmax warps)
                    const int rt = group == 1 ? cur.s.rt : my_rt, quarter = row & 3;
                    if (!wait(&sm.q_empty, (seg_i - 2) & 1)) break;
#pragma unroll 1
                    for (int r = row >> 2; r < kRows; r += kConvThreads / 4) {
                        QuarterRow<kBf16> own;
                        own.load(q_row(p, qp, cur.s, rt, r), quarter);
                        const int e = own.split(sm.q, r, quarter);
                        if (quarter == 0) sm.q_exp[(seg_i - 1) & 3][r] = e;
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    mbar_arrive(&sm.q_ready[(seg_i - 1) & 3]);
                }
                const int L = sm.len[b], tile0 = tile_of(sm, b, cur.kt()) * kTile;
                const TileRows rows = {L + p.N - tile0, qp.sinks - tile0, sm.seen[b] - tile0};
                if (!wait(&sm.k_full[k_slot], k_ph)) break;
                uint32_t keep = 0xFFFFFFFFu;
                bool data = true;
                if (!rows.all()) {
                    keep = data_bytes(rows, lane);
                    data = rows.data(row);
                }
                const int ek = sm.scale[k_slot][0][row], ev = sm.scale[k_slot][1][row];
                // K relative to the tile's largest; V seven below it, so that the largest code, 448 * 2^7, lies just within fp16
                const int ref_k = tile_exponent(sm.scale[k_slot][0], lane, keep, 0), ref_v = tile_exponent(sm.scale[k_slot][1], lane, keep, 7);
                mbar_arrive(&sm.k_empty[k_slot]);
                // A row that is not a number in K or V makes its score so, which reaches the query rows that see it and no other; V's
                // row is zero then, as the rows are that hold no data (a weight of zero times anything there is zero).
                const bool nan = ek == 255 || ev == 255;
                next_zero = !data || nan;
                sm.factor[j & 3][row] = nan ? __uint_as_float(0x7FC00000u) : pow2(min(max(ek - 127 - ref_k, -126), 0));
                if (row == 0) {
                    sm.ref[j & 3][0] = ref_k;
                    sm.ref[j & 3][1] = ref_v;
                }
                mbar_arrive(&sm.ref_full[j & 3]);
                const __half2 f = __float2half2_rn(pow2(min(max(ev - 127 - ref_v, -126), 7)));
                next_factor = *reinterpret_cast<const uint32_t *>(&f);
                if (++k_slot == kRawK) { k_slot = 0; k_ph ^= 1; }
            }
            if (j > 0) {
                const uint32_t w = (uint32_t)(j - 1) & 1;
                if (!wait(&sm.v_full[v_slot], v_ph)) break;
                if (j - 1 >= kWide && !wait(&sm.w_empty[w], (uint32_t)((j - 1) / kWide - 1) & 1)) break;
                widen_row(sm.raw_v[v_slot], sm.wide[w], row, zero, factor);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(&sm.w_full[w]);
                mbar_arrive(&sm.v_empty[v_slot]);
                if (++v_slot == kRawV) { v_slot = 0; v_ph ^= 1; }
            }
            zero = next_zero;
            factor = next_factor;
        }
        if (clustered) {
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();
        }
    } else if (warp > kMmaWarp) {
        if (clustered) {
            cluster_sync_all();
            cluster_sync_all();
        }
    } else {
        // ------------------------------- softmax -------------------------------
        // Two streams of eight warps take alternate tiles, each with its own reference, sums and accumulator; within a stream a
        // row's 128 keys are shared by two threads, in two warps that meet on the same scheduler.
        const int s = warp >> 3, h = (warp >> 2) & 1;  // stream, half of a tile's keys
        const int row = threadIdx.x & 127;             // query row within the tile = TMEM lane
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const int tid = threadIdx.x;                   // 0..511
        const int pair_id = 2 + s * 4 + (warp & 3);
        const int words = (p.N + 31) >> 5;
        if (n > 0) {                                   // Q of the range's first segment: nobody here has anything else to do yet
            QuarterRow<kBf16> own;
            own.load(q_row(p, qp, first, group == 1 ? first.rt : my_rt, tid >> 2), tid & 3);
            const int e = own.split(sm.q, tid >> 2, tid & 3);
            if ((tid & 3) == 0) sm.q_exp[0][tid >> 2] = e;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if ((tid & 3) == 0) mbar_arrive(&sm.q_ready[0]);
        }
        int b_hint = 0, J = 0, seg_i = 0;
        CutUnit cut[2];
        unsigned int ticket[2] = {0u, 0u};
        cut[0].valid = cut[1].valid = 0;
        int anc_b = -1, anc_rt = -1;
        bool dead = false;                             // a wait of this warp has run out
        for (int t = t_begin; t < t_end;) {
            const Segment sg = t == t_begin ? first : locate(sm.pre, sm.nkt, p.B, upl, t, t_end, b_hint);
            const int L = sm.len[sg.b];
            const int rt = group == 1 ? sg.rt : my_rt;
            // --- which tree rows, and from where on which context rows, the tile's rows see ---
            const int node = rt * p.rows_per_tile_nodes + row / p.g;
            const bool real = node < p.N;
            const bool warp_real = rt * p.rows_per_tile_nodes + (row & ~31) / p.g < p.N;
            if (sg.b != anc_b || rt != anc_rt) {
                softmax_sync();                        // previous segment no longer reads anc
                if (tid < kRows) {
                    const int32_t *parent = p.parent + (size_t)sg.b * p.N;         // (a few lines, in the first-level cache after the first step)
                    for (int w = 0; w < words; ++w) sm.anc[w][row] = 0u;   // padding rows see the context only; their results are dropped
                    int lo = 0;
                    if (real) {
                        int depth = 0;
                        if (qp.window > 0) {
                            for (int c = parent[node]; c >= 0; c = parent[c]) ++depth;
                            lo = (int)max(0ll, (long long)L + depth - qp.window + 1);
                        }
                        int back = 0;                  // positions from the row to its ancestor
                        for (int c = node; c >= 0; c = parent[c], ++back)
                            if (qp.window == 0 || back < qp.window || (long long)L + depth - back < qp.sinks) sm.anc[c >> 5][row] |= 1u << (c & 31);
                    }
                    sm.row_lo[row] = lo;
                }
                softmax_sync();
                anc_b = sg.b;
                anc_rt = rt;
            }
            const int row_lo = sm.row_lo[row];

            const bool complete = sg.kt0 == 0 && sg.len == sg.nkt;
            const int cut_k = (t == t_begin) ? 0 : 1;
            unsigned int delivered = 0, delivered_old = 0;
            if (!complete) {
                CutUnit &cu = cut[cut_k];
                cu.unit = (sg.b * p.Hkv + sg.hk) * p.n_rt + rt;
                cu.b = sg.b; cu.hk = sg.hk; cu.rt = rt;
                cu.t0 = sm.pre[sg.b] + (sg.hk * upl + (group == 1 ? rt : 0)) * sg.nkt;
                cu.c_lo = clustered ? 0 : cu.t0 / per;
                cu.c_hi = clustered ? 0 : (cu.t0 + sg.nkt - 1) / per;
                cu.cta_mul = group; cu.cta_add = my_rt;
            }
            bool ok = mbar_wait_quick(smem_u32(&sm.q_ready[seg_i & 3]), (seg_i >> 2) & 1, abort_flag);
            const float row_scale = p.scale_log2 * pow2(sm.q_exp[seg_i & 3][row]);
            ++seg_i;
            const int gap_at = sm.gap_at[sg.b], gap = sm.gap[sg.b];
            // Scores are held with the exponent that V's tile is taken relative to added: t = log2(e) scale q.k + ref_v.  A weight 2^(t -
            // m_ref) is then what multiplies V's fp16 values, whatever V's scales, and the sum of the weights themselves is the tile's times
            // 2^-ref_v.
            float m_ref = -INFINITY, l_sum = 0.f;      // the row's reference (alike in its two threads), this half's sum
#pragma unroll 1
            for (int i = (J ^ s) & 1; i < sg.len; i += 2) {
                const int jj = J + i;
                if (!complete && !clustered && tid == 0) {
                    delivered_old = delivered;
                    delivered = ld_relaxed_gpu(&p.tickets[cut[cut_k].unit]);
                }
                const int kt = sg.kt0 + i, tile_lo = (kt < gap_at ? kt : kt + gap) * kTile, key0 = tile_lo + h * 64;
                ok = ok && mbar_wait_quick(smem_u32(&sm.ref_full[jj & 3]), (jj >> 2) & 1, abort_flag);
                // (never zero: a masked score is -inf, and zero times that is none; scores as small are below 2^-96)
                const float tile_scale = fmaxf(row_scale * pow2(sm.ref[jj & 3][0]), 0x1p-120f), shift = (float)sm.ref[jj & 3][1];
                const float *factor = &sm.factor[jj & 3][h * 64];
                const uint32_t s_addr = tmem + lane_base + s * 128 + h * 64;
                ok = ok && mbar_wait_quick(smem_u32(&sm.s_full[s]), (jj >> 1) & 1, abort_flag);
                dead = !__all_sync(0xFFFFFFFFu, ok);
                const bool live = warp_real && !dead;
                tc_fence_after();
                const bool masked = key0 + 64 > L || (qp.window > 0 && key0 + 64 > qp.sinks && __any_sync(0xFFFFFFFFu, real && row_lo > key0));
                float mx = -INFINITY;
                unsigned long long vis = ~0ull;
                if (live) {
                    if (masked) {
                        vis = 0ull;
#pragma unroll 1
                        for (int w = 1; w >= 0; --w) {
                            const int k0 = key0 + 32 * w, cc0 = k0 - L;
                            const int wi = cc0 >> 5, sh = cc0 & 31;
                            const uint32_t lo = (wi >= 0 && wi < words) ? sm.anc[wi][row] : 0u;
                            const uint32_t hi = (wi + 1 >= 0 && wi + 1 < words) ? sm.anc[wi + 1][row] : 0u;
                            vis = vis << 32 | (__funnelshift_r(lo, hi, sh) | (low_bits(L - k0) & (~low_bits(row_lo - k0) | low_bits(qp.sinks - k0))));
                        }
                        mx = scores_max<true>(s_addr, factor, vis);
                    } else {
                        mx = scores_max<false>(s_addr, factor, vis);
                    }
                    mx = fmaf(mx, tile_scale, shift);                 // scale > 0: max commutes with scaling
                }
                // The reference rises, for the 32 rows together, only where some row's maximum leaves it 2^8 behind (or has none yet).
                // Under values that are all but zero, with an exponent down to -100, the sum of the weights themselves holds up to 2^107
                // for a key: there it rises at once, and a million such keys stay within 32 bits (2^15 did not, 2^8 behind).
                const float behind = shift < -64.f ? 0.f : kRescaleThreshold;
                if (pair_any(pair_id, mx > m_ref + behind || (m_ref == -INFINITY && mx != -INFINITY))) {
                    sm.mx[s][h][row] = mx;
                    pair_sync(pair_id);
                    const float m_new = fmaxf(m_ref, fmaxf(mx, sm.mx[s][h ^ 1][row]));
                    const float f = m_ref == -INFINITY ? 1.f : exp2f(m_ref - m_new);
                    if (live && __any_sync(0xFFFFFFFFu, f != 1.f)) {
                        // (scores of this tile being ready says that this stream's previous P V has reached the accumulator)
                        const uint32_t o_addr = tmem + lane_base + 256 + s * 128 + h * 64;
#pragma unroll 1
                        for (int c4 = 0; c4 < 4; ++c4) {
                            float o[16];
                            tmem_ld16(o_addr + c4 * 16, o);
                            tmem_ld_wait();
                            uint32_t r[16];
#pragma unroll
                            for (int c = 0; c < 16; ++c) r[c] = __float_as_uint(o[c] * f);
                            tmem_st16(o_addr + c4 * 16, r);
                        }
                        tmem_st_wait();
                        l_sum *= f;
                    }
                    m_ref = m_new;
                }
                if (live) {
                    const float lift = shift - ((m_ref == -INFINITY) ? 0.f : m_ref) + kWeightLift;
                    float sum;
                    if (tile_lo + kTile > L - qp.near_keys) sum = scores_weights<true, true>(s_addr, factor, vis, tile_scale, lift);
                    else if (masked) sum = scores_weights<true, false>(s_addr, factor, vis, tile_scale, lift);
                    else sum = scores_weights<false, false>(s_addr, factor, vis, tile_scale, lift);
                    l_sum = fmaf(sum, pow2(-(int)shift), l_sum);
                    tmem_st_wait();
                }
                tc_fence_before();
                if (!dead) mbar_arrive(&sm.p_ready[s]);
            }
            // --- segment epilogue: the streams merged, the result or a part of it written.  Maxima and sums are exchanged while the last
            // products still run. ---
            sm.sum[s][h][row] = l_sum;
            if (h == 0) sm.ref_row[s][row] = m_ref;
            if (tid == 0) {
                sm.direct = !clustered && !complete && cut[cut_k].c_hi - cut[cut_k].c_lo == 1 && delivered_old == 1u;
                if (sm.direct) p.tickets[cut[cut_k].unit] = 0u;      // zero for the next call on this workspace
            }
            softmax_sync();
            const float m0 = sm.ref_row[0][row], l0 = sm.sum[0][0][row] + sm.sum[0][1][row];
            const float m1 = sm.ref_row[1][row], l1 = sm.sum[1][0][row] + sm.sum[1][1][row];
            const bool direct = sm.direct;
            const float M = fmaxf(m0, m1);
            const float f0 = (m0 == -INFINITY) ? 0.f : exp2f(m0 - M);
            const float f1 = (m1 == -INFINITY) ? 0.f : exp2f(m1 - M);
            // (a stream that saw nothing but keys that are no numbers has a sum that is none, and no maximum)
            const float l_tot = (m0 == -INFINITY ? l0 : f0 * l0) + (m1 == -INFINITY ? l1 : f1 * l1);
            const bool has0 = sg.len >= 2 || (J & 1) == 0, has1 = sg.len >= 2 || (J & 1) == 1;      // which streams own tiles of this segment
            const int head = sg.hk * p.g + row % p.g;
            float *pslot = clustered ? nullptr : p.part + (size_t)(2 * (int)blockIdx.x + cut_k) * kSlotFloats;
            const int xk_sh = clustered ? 5 - __ffs(p.cluster_k) + 1 : 0;
            const uint32_t xrecv = smem_u32(&sm.q[0][0]) + kXchgRecvOffset;
            const float *oslot = pslot;
            float g0 = f0, g1 = f1, w_own = 0.f, w_other = 0.f, inv_two = 0.f;
            bool own_first = false;
            if (direct) {                              // merge_parts_q8's arithmetic, this CTA's part straight from the accumulators
                const CutUnit &cu = cut[cut_k];
                const int oc = (cu.c_lo == my_pos) ? cu.c_hi : cu.c_lo;
                oslot = p.part + (size_t)(2 * (oc * group + my_rt) + ((max(cu.t0, oc * per) == oc * per) ? 0 : 1)) * kSlotFloats;
                __threadfence();
                const float m_o = __ldcg(oslot + kRows * kD + row), l_o = __ldcg(oslot + kRows * kD + kRows + row);
                const float Mn = fmaxf(M, m_o);
                const float fa = (M == -INFINITY) ? 0.f : exp2f(M - Mn);
                const float fb = (m_o == -INFINITY) ? 0.f : exp2f(m_o - Mn);
                own_first = oc == cu.c_hi;
                inv_two = 1.f / (own_first ? fmaf(l_tot, fa, l_o * fb) : fmaf(l_o, fb, l_tot * fa));
                w_own = fa;
                w_other = fb;
            } else if (complete && !clustered) {
                const float inv = 1.f / l_tot;
                g0 *= inv;
                g1 *= inv;
            }
            {
                const int last_any = J + sg.len - 1;                       // the segment's last tile; x's last: same parity
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int lx = ((last_any & 1) == x) ? last_any : last_any - 1;
                    if (lx >= J) ok = ok && mbar_wait(&sm.o_done[x], (lx >> 1) & 1, abort_flag);
                }
                dead = !__all_sync(0xFFFFFFFFu, ok);
                tc_fence_after();
            }
            if (clustered) {
                __syncwarp();
                cluster_sync_all();                    // every CTA of the cluster is done with its Q buffer and rings
            }
            const bool final = (complete && !clustered) || direct;
            if (warp_real && !dead) {
#pragma unroll 1
                for (int c2 = 0; c2 < 2; ++c2) {       // 16 features at a time of this thread's 32
                    const int col0 = (s * 2 + h) * 32 + c2 * 16;
                    float x[16], y[16];
                    tmem_ld16(tmem + lane_base + 256 + col0, x);
                    tmem_ld16(tmem + lane_base + 384 + col0, y);
                    tmem_ld_wait();
                    if (!real) continue;
                    // an accumulator no tile of this segment wrote holds stale numbers (possibly NaN)
#pragma unroll
                    for (int c = 0; c < 16; ++c) x[c] = (has0 ? g0 * x[c] : 0.f) + (has1 ? g1 * y[c] : 0.f);
                    if (direct) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const float4 v = __ldcg(reinterpret_cast<const float4 *>(oslot) + (col0 / 4 + c) * kRows + row);
                            const float other[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float &mine = x[4 * c + i];
                                mine = (own_first ? fmaf(other[i], w_other, fmaf(mine, w_own, 0.f)) : fmaf(mine, w_own, fmaf(other[i], w_other, 0.f))) * inv_two;
                            }
                        }
                    }
                    if (final) {
                        uint32_t w[8];
#pragma unroll
                        for (int c = 0; c < 8; ++c) w[c] = pack2<kBf16>(x[2 * c], x[2 * c + 1]);
                        unsigned char *dst = static_cast<unsigned char *>(p.out) +
                                             ((((size_t)sg.b * p.N + node) * p.Hq + head) * kD + col0) * 2;
                        *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4 *>(dst + 16) = make_uint4(w[4], w[5], w[6], w[7]);
                    } else if (clustered) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int cg = col0 / 4 + c, xg = cg & ((1 << xk_sh) - 1);
                            st_peer_f4(map_to_peer(xrecv + (uint32_t)((((int)c_rank << xk_sh) + xg) * kRows + row) * 16u, (uint32_t)(cg >> xk_sh)),
                                       make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]));
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            reinterpret_cast<float4 *>(pslot)[(col0 / 4 + c) * kRows + row] = make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
                    }
                }
            }
            if (clustered) {
                if (real && s == 0)
                    for (int c = 0; c < p.cluster_k; ++c)
                        st_peer_f1(map_to_peer(xrecv + (uint32_t)(kRows * kD + ((int)c_rank * 2 + h) * kRows + row) * 4u, (uint32_t)c), h == 0 ? M : l_tot);
            } else if (!final && tid < kRows && real) {
                pslot[kRows * kD + row] = M;
                pslot[kRows * kD + kRows + row] = l_tot;
            }
            tc_fence_before();
            softmax_sync();                            // the accumulators and the sums are free for the next segment
            if (!final && !clustered) {
                cut[cut_k].valid = 1;
                if (tid == 0) {
                    __threadfence();
                    ticket[cut_k] = atomicAdd(&p.tickets[cut[cut_k].unit], 1u);
                }
            }
            J += sg.len;
            t += sg.len;
        }
        if (clustered) {
            if (t_end <= t_begin) {                    // an empty share still delivers a part: nothing seen
                __syncwarp();
                cluster_sync_all();
                const uint32_t xrecv = smem_u32(&sm.q[0][0]) + kXchgRecvOffset;
                if (s == 0)
                    for (int c = 0; c < p.cluster_k; ++c)
                        st_peer_f1(map_to_peer(xrecv + (uint32_t)(kRows * kD + ((int)c_rank * 2 + h) * kRows + row) * 4u, (uint32_t)c), h == 0 ? -INFINITY : 0.f);
            }
            __syncwarp();
            const int hk = ask.cl_unit / upl;
            if (s == 0) cluster_merge<kBf16>(p, &sm.q[0][0], (int)c_rank, ask.cl_b, hk, ask.cl_unit - hk * upl, sm.nkt[ask.cl_b] > 0, tid, abort_flag);
            else cluster_sync_all();                   // (the merge begins with the exchange's second barrier and is 256 threads' work)
        }
        // --- cut units: the CTA that delivers the last part of a unit merges all parts; nobody waits ---
        if (cut[0].valid || cut[1].valid) {
            if (tid == 0)
                for (int k = 0; k < 2; ++k) {
                    sm.merge_here[k] = cut[k].valid && ticket[k] == (unsigned)(cut[k].c_hi - cut[k].c_lo);
                    if (sm.merge_here[k]) p.tickets[cut[k].unit] = 0u;
                }
            softmax_sync();
            for (int k = 0; k < 2; ++k)
                if (sm.merge_here[k]) {
                    __threadfence();
                    merge_parts_q8<kBf16>(p, cut[k], per, tid);
                }
        }
    }

    // ------------------------------- teardown -------------------------------
    tc_fence_before();
    __syncthreads();
    if (sm.abort && threadIdx.x == 0) {
        for (int b = 0; b < p.B; ++b)
            if (sm.nkt[b] > 0) p.status[b] = HT_STATUS_TIMEOUT;
    }
    if (sm.abort && threadIdx.x == kCopyWarp * 32) {
        // some wait ran out: every copy that was asked for must have landed before the CTA exits
        const int asked_k = sm.plan[9], asked_v = sm.plan[10];
        for (int j = max(0, asked_k - kRawK); j < asked_k; ++j) mbar_wait(&sm.k_full[j % kRawK], (j / kRawK) & 1, abort_flag, false);
        for (int j = max(0, asked_v - kRawV); j < asked_v; ++j) mbar_wait(&sm.v_full[j % kRawV], (j / kRawV) & 1, abort_flag, false);
    }
    if (warp == kCopyWarp) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// What must be zero when the attention kernel starts: the units' arrival counters and, for a paged cache, the status words.
__global__ void prepare_kernel(unsigned int *tickets, int n_tickets, int32_t *status, int n_status) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + threadIdx.x;
    for (int i = first; i < n_tickets; i += stride) tickets[i] = 0u;
    for (int i = first; i < n_status; i += stride) status[i] = 0;
}

}  // namespace q8

// ---------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static int make_map_q8(CUtensorMap *map, const void *base, const cuuint64_t dims[4], const cuuint64_t strides_b[3], const cuuint32_t box[4]) {
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return fail(HT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
        }
        fn = reinterpret_cast<EncodeTiledFn>(ptr);
    }
    const cuuint32_t elem_strides[4] = {1, 1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(base), dims, strides_b, box, elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(HT_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d", (int)r);
    return HT_OK;
}

bool attn_q8_tc_applicable(const ht_attn_desc &d) {
    if (d.flags & HT_ATTN_FORCE_SIMT) return false;
    if (d.dtype != HT_F16 && d.dtype != HT_BF16) return false;
    if (d.D != tc::kD) return false;
    const int g = d.Hq / d.Hkv;
    if (g > tc::kRows || (g & (g - 1)) != 0) return false;
    return d.N <= tc::kMaxWords * 32 && d.B <= tc::kMaxB && d.num_splits == 0;
}

static int row_tiles_q8(const ht_attn_desc &d) { return (d.N * (d.Hq / d.Hkv) + tc::kRows - 1) / tc::kRows; }

// The units' arrival counters, in an area of a fixed size (more units than it holds: of their own size, always cleared), then
// two partial results per CTA.
constexpr size_t kTicketAreaQ8 = 64 * 1024;
static size_t ticket_bytes_q8(const ht_attn_desc &d) {
    const size_t need = ((size_t)d.B * d.Hkv * row_tiles_q8(d) * sizeof(unsigned int) + 255) / 256 * 256;
    return need > kTicketAreaQ8 ? need : kTicketAreaQ8;
}
size_t attn_q8_tc_workspace(const ht_attn_desc &d) { return ticket_bytes_q8(d) + (size_t)2 * sm_count() * tc::kSlotFloats * sizeof(float); }

typedef void (*AttnQ8Fn)(const CUtensorMap, const CUtensorMap, const tc::Params, const tc::PagedParams, const q8::Q8Params);
static AttnQ8Fn attn_q8_fn(int form) {                    // bf16, paged, clustered as bits 0, 1, 2
    static const AttnQ8Fn fns[8] = {
        q8::attn_q8_kernel<false, false, false>, q8::attn_q8_kernel<true, false, false>, q8::attn_q8_kernel<false, true, false>,
        q8::attn_q8_kernel<true, true, false>,   q8::attn_q8_kernel<false, false, true>, q8::attn_q8_kernel<true, false, true>,
        q8::attn_q8_kernel<false, true, true>,   q8::attn_q8_kernel<true, true, true>};
    return fns[form];
}
static cudaError_t raise_smem_q8(int form) {              // once per device and kernel
    static bool done[64][8];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && done[dev][form]) return cudaSuccess;
    e = cudaFuncSetAttribute(attn_q8_fn(form), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(q8::SmemQ8) + 1024);
    if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev][form] = true;
    return e;
}

// Clusters of k CTAs that the device holds at once (an SM takes one CTA, and a cluster lies within one of the groups of SMs that
// the device is made of: fewer than SMs / k).  Asked for once per device, form and size; 0 where the answer fails.
static int clusters_at_once(int form, int k) {
    static int known[64][8][4];                           // the number and one
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    int *slot = dev >= 0 && dev < 64 ? &known[dev][form][k == 8 ? 3 : (k == 4 ? 2 : 1)] : nullptr;
    if (slot && *slot) return *slot - 1;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)k;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(sm_count() / k * k));
    cfg.blockDim = dim3(q8::kQ8Threads);
    cfg.dynamicSmemBytes = sizeof(q8::SmemQ8) + 1024;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, attn_q8_fn(form), &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    if (slot) *slot = n + 1;
    return n;
}

// CTAs that share a unit (a sequence, KV head and row tile) as a cluster, where the units are so few that one CTA each would leave
// SMs idle; 0: no clusters, the list of all tiles is cut evenly, and a unit's parts meet in the workspace.  All clusters have to run
// at once (16 units by clusters of 8 on 8192 keys take 60 us, half of that when they fit).  In a cluster a CTA has its share of
// one unit, in the list an even share of everything; the list costs as much on top as some 18 tiles.  1 x 91 rows, us by clusters / by
// the list: 8 heads, KV 8192 30 / 43, 16384 44 / 63, 32768 72 / 84; 20 heads, 8192 45 / 53, 16384 74 / 85; 50 heads, 8192 74 / 84;
// 36 heads (clusters of 2), 16384 130 / 106.
static int cluster_size_q8(const ht_attn_desc &d, const ht_window_desc &w, int form) {
    const long long units = (long long)d.B * d.Hkv * row_tiles_q8(d), shown = w.window > 0 ? (long long)w.window + w.sinks + d.N : d.cap;
    const long long keys = shown < d.cap ? shown : d.cap, tiles = (keys + tc::kTile - 1) / tc::kTile;
    const int sms = sm_count();
    for (int k = 8; k >= 2; k /= 2)
        if (units * k <= sms && units <= clusters_at_once(form, k)) return (tiles + k - 1) / k <= 18 + units * tiles / sms ? k : 0;
    return 0;
}

int launch_attn_q8_tc(const ht_attn_desc &d, const ht_window_desc &w, const void *q, const void *kc, const void *vc, const Q8Scales &scales,
                      const int32_t *kv_len, const int32_t *parent, void *out, void *ws, size_t ws_bytes, int32_t *status, cudaStream_t s,
                      const ht_paged_desc *pages, const int32_t *block_table) {
    if (!ws || ws_bytes < attn_q8_tc_workspace(d))
        return fail(HT_ERR_WORKSPACE, "workspace holds %zu bytes, %zu needed", ws ? ws_bytes : 0, attn_q8_tc_workspace(d));
    const int g = d.Hq / d.Hkv;
    CUtensorMap tm_k, tm_v;
    tc::PagedParams pp{};
    {
        cuuint64_t dims[4] = {(cuuint64_t)d.D, (cuuint64_t)d.cap, (cuuint64_t)d.Hkv, (cuuint64_t)d.B};
        cuuint64_t strides[3] = {(cuuint64_t)d.D, (cuuint64_t)(d.kv_stride_h ? d.kv_stride_h : (long long)d.cap * d.D),
                                 (cuuint64_t)(d.kv_stride_b ? d.kv_stride_b : (long long)d.Hkv * d.cap * d.D)};
        cuuint32_t box[4] = {(cuuint32_t)d.D, (cuuint32_t)tc::kTile, 1, 1};
        if (pages) {                                      // [page][head][row][D]: a box is the rows of a tile that one page holds
            dims[1] = (cuuint64_t)pages->page_size;
            dims[3] = (cuuint64_t)pages->n_pages;
            strides[1] = (cuuint64_t)(pages->head_stride ? pages->head_stride : (long long)pages->page_size * d.D);
            strides[2] = (cuuint64_t)(pages->page_stride ? pages->page_stride : (long long)d.Hkv * pages->page_size * d.D);
            box[1] = (cuuint32_t)(pages->page_size < tc::kTile ? pages->page_size : tc::kTile);
            pp.block_table = block_table;
            pp.page_size = pages->page_size;
            while ((1 << pp.page_shift) < pages->page_size) ++pp.page_shift;
            pp.max_pages = pages->max_pages;
            pp.n_pages = pages->n_pages;
        }
        int rc = make_map_q8(&tm_k, kc, dims, strides, box);
        if (rc != HT_OK) return rc;
        rc = make_map_q8(&tm_v, vc, dims, strides, box);
        if (rc != HT_OK) return rc;
    }
    tc::Params p{};
    p.kv_len = kv_len; p.parent = parent; p.status = status; p.out = out; p.tickets = static_cast<unsigned int *>(ws);
    p.part = reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + ticket_bytes_q8(d));
    p.B = d.B; p.N = d.N; p.Hq = d.Hq; p.Hkv = d.Hkv; p.g = g; p.cap = d.cap;
    p.rows_per_tile_nodes = tc::kRows / g;
    p.n_rt = p.n_row_tiles = row_tiles_q8(d);
    p.scale_log2 = (d.scale > 0.f ? d.scale : 1.f / sqrtf((float)d.D)) * 1.4426950408889634f;
    p.is_bf16 = d.dtype == HT_BF16;
    p.cluster_split = 1;
    p.wait_kcycles = (d.flags & HT_ATTN_TEST_SHORT_WAITS) ? tc::kWaitKcyclesTest : tc::kWaitKcycles;
    q8::Q8Params qp{};
    qp.q = q; qp.k_scale = scales.k; qp.v_scale = scales.v; qp.scale_b = scales.stride_b; qp.scale_h = scales.stride_h;
    qp.window = w.window; qp.sinks = w.window > 0 ? w.sinks : 0;
    qp.near_keys = w.window > 0 ? tc::kTile : 0;
    const long long units = (long long)d.B * d.Hkv * p.n_rt;
    if (units > 0x7fffffffLL || units * ((d.cap + tc::kTile - 1) / tc::kTile) > 0x7fffffffLL) return fail(HT_ERR_UNSUPPORTED, "too many (sequence, head, row tile, key tile) units");
    int form = (p.is_bf16 ? 1 : 0) + (pages ? 2 : 0) + 4;
    cudaError_t e = raise_smem_q8(form);
    if (e != cudaSuccess) return fail(HT_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    const int sms = sm_count(), k = cluster_size_q8(d, w, form);
    if (k == 0) form -= 4;
    // Row tiles side by side on the same keys, where at least four such groups fit: 16 x 67 rows of 64 on 8 heads on 8192 keys take
    // 580 us, and 593 with the row tiles one after the other in the list.
    qp.group = k <= 1 && p.n_rt > 1 && p.n_rt * 4 <= sms ? p.n_rt : 1;
    p.grid = k > 1 ? (int)units * k : sms / qp.group * qp.group;
    p.cluster_k = k > 1 ? k : 0;
    const bool prepare = pages || (k <= 1 && (!(d.flags & HT_ATTN_WORKSPACE_CLEAN) || (size_t)units * sizeof(unsigned int) > kTicketAreaQ8));
    const size_t smem = offsetof(q8::SmemQ8, anc) + (size_t)((d.N + 31) / 32) * tc::kRows * sizeof(uint32_t) + 1024;
    trace("ht_tree_attention_q8 -> tcgen05 kernel, %d row tiles, %s of %d, %d CTAs", p.n_rt, k > 1 ? "clusters" : "groups", k > 1 ? k : qp.group, p.grid);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    if (prepare) {
        const int n_t = k > 1 ? 0 : (int)units, n_s = pages ? d.B : 0, most = n_t > n_s ? n_t : n_s;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((most + 255) / 256 < 64 ? (most + 255) / 256 : 64));
        cfg.blockDim = dim3(256);
        cfg.stream = s;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, q8::prepare_kernel, p.tickets, n_t, status, n_s);
    }
    if (e == cudaSuccess) e = raise_smem_q8(form);
    if (e == cudaSuccess) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)p.grid);
        cfg.blockDim = dim3(q8::kQ8Threads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = s;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)(k > 1 ? k : 1);
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = k > 1 ? 2 : 1;
        e = cudaLaunchKernelEx(&cfg, attn_q8_fn(form), tm_k, tm_v, p, pp, qp);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(HT_ERR_CUDA, "ht_tree_attention_q8 (tcgen05): %s", cudaGetErrorString(e));
    }
    return HT_OK;
}

}  // namespace ht
