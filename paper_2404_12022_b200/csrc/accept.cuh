// Acceptance on a draft tree (Fig. 2 caption; Section "Inference stage"): the longest root path whose tokens are the
// ones the model emits, given each row's emitted token.  Shared by the greedy and the sampled verification.
#pragma once
#include "ht_common.cuh"

namespace ht {

constexpr unsigned kTicket = 256u;           // arrivals are counted in units of this on the accept_len word: lengths stay below it

// pred is written by other blocks of the same launch: read through L2 when it is read from global memory
// (a generic load works for the staged copy in shared memory as well).
__device__ __forceinline__ int ld_pred(const int32_t *p) {
    return __isGlobal(p) ? __ldcg(p) : *p;
}

__device__ __forceinline__ void st_release(int32_t *p, int v) {
    asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ int ld_acquire(const int32_t *p) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// The tree of one sequence in shared memory: parents and draft tokens are inputs (staged while the logits stream, by
// every block, for the sequence of the row it works on), the rows' argmax is what the other blocks of the launch wrote
// (staged by the block that searches, once all rows have arrived).
constexpr int kStage = 1024;                 // trees of up to this many rows are staged
struct TreeSmem {
    int32_t par[kStage], tok[kStage], prd[kStage];
    int bad, root, staged_b;
    unsigned long long key[32];
};

__device__ __forceinline__ void stage_tree(TreeSmem &ts, int b, const int32_t *__restrict__ tokens, const int32_t *__restrict__ parent,
                                           const int32_t *__restrict__ root_pred, int N, int T) {
    if (ts.staged_b == b) return;                      // (uniform over the block: written behind a barrier below)
    __syncthreads();
    if (threadIdx.x == 0) {
        ts.bad = 0;
        ts.root = root_pred ? root_pred[b] : -1;
        ts.staged_b = b;
    }
    __syncthreads();
    const int32_t *par = parent + (size_t)b * N;
    for (int c = threadIdx.x; c < N; c += blockDim.x) {
        const int pc = par[c];
        if (N <= kStage) {
            ts.par[c] = pc;
            if (c < T) ts.tok[c] = tokens[(size_t)b * T + c];
        }
        if (pc < -1 || pc >= c) ts.bad = 1;
    }
}

// Path search of one sequence by one block (its tree staged by stage_tree).  Every thread walks the root path of its
// nodes (parent[c] < c makes the walk finite), checks the match rule on the way and proposes (depth, node);
// the block keeps the deepest valid node, lowest index on ties.
__device__ __forceinline__ void accept_sequence(TreeSmem &ts, const int b, const int32_t *__restrict__ tokens, const int32_t *__restrict__ parent,
              const int32_t *__restrict__ root_pred, const int32_t *pred, int N, int T,
              int max_path, int32_t *accept_len, int32_t *__restrict__ accept_path,
              int32_t *__restrict__ next_token, int32_t *__restrict__ status, const int done_mark) {
    const int32_t *par = parent + (size_t)b * N;
    const int32_t *tok = tokens + (size_t)b * T;
    const int32_t *prd = pred + (size_t)b * N;
    int32_t *path = accept_path + (size_t)b * max_path;
    // The walks below are chains of dependent reads: with the tree's three arrays in shared memory they
    // cost one round trip to L2 in all instead of one per level (trees of up to kStage rows).
    if (N <= kStage) {
        for (int c = threadIdx.x; c < N; c += blockDim.x) ts.prd[c] = __ldcg(prd + c);
        par = ts.par; tok = ts.tok; prd = ts.prd;
    }
    for (int j = threadIdx.x; j < max_path; j += blockDim.x) path[j] = -1;
    __syncthreads();
    // the word other blocks wait on (fused form) is stored with release semantics, behind everything else
    auto finish = [&](int word) {
        if (done_mark) st_release(accept_len + b, done_mark | word);
        else accept_len[b] = word;
    };
    if (ts.bad) {
        if (threadIdx.x == 0) {
            status[b] = HT_STATUS_BAD_TREE;
            next_token[b] = -1;
            finish(0);
        }
        return;
    }
    const bool has_root = root_pred != nullptr;
    const int rp = ts.root;
    // key = depth << 32 | (0xFFFFFFFF - node): max picks the deepest, then the lowest node
    unsigned long long key = 0;
    for (int n = threadIdx.x; n < T; n += blockDim.x) {
        int depth = 0;
        bool ok = true;
        for (int c = n; c >= 0; c = par[c]) {
            const int p = par[c];
            const bool m = p < 0 ? (!has_root || tok[c] == rp) : (tok[c] == ld_pred(prd + p));
            ok = ok && m;
            ++depth;
        }
        if (ok) {
            const unsigned long long k2 = ((unsigned long long)depth << 32) | (0xFFFFFFFFu - (unsigned)n);
            key = k2 > key ? k2 : key;
        }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const unsigned long long o = __shfl_xor_sync(0xffffffffu, key, off);
        key = o > key ? o : key;
    }
    if ((threadIdx.x & 31) == 0) ts.key[threadIdx.x >> 5] = key;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < (int)(blockDim.x >> 5); ++w) key = ts.key[w] > key ? ts.key[w] : key;
        const int len = (int)(key >> 32);
        const int node = (int)(0xFFFFFFFFu - (unsigned)(key & 0xFFFFFFFFu));
        if (len > max_path) {
            status[b] = HT_STATUS_PATH_TOO_LONG;
            next_token[b] = -1;
            finish(0);
        } else {
            status[b] = HT_STATUS_OK;
            if (len == 0) {
                next_token[b] = has_root ? rp : -1;
            } else {
                int j = len - 1;
                for (int c = node; c >= 0; c = par[c]) path[j--] = c;
                next_token[b] = ld_pred(prd + node);
            }
            finish(len);
        }
    }
}

}  // namespace ht
