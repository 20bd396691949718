// Operators of a step that answers several drafted tokens at once: norms of queries and keys with the position rotation,
// attention of a tree of tokens over a cache, verification of the drafts, and the accepted rows of the cache.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "drafts.h"
#include "ps_internal.h"
#include "row_math.h"

namespace ps {

namespace {

// rows first[s] .. of sequence s and how many of them count
struct SeqRows { int row0, n; };
__device__ __forceinline__ SeqRows rows_of(const int32_t *first, uint32_t s, uint32_t n_tokens, uint32_t max_tree) {
    const int a = clampi(first[s], 0, (int)n_tokens), b = clampi(first[s + 1], 0, (int)n_tokens);
    return {a, clampi(b - a, 0, (int)max_tree)};
}
__device__ __forceinline__ int parent_of(int p, int i) { return p >= 0 && p < i ? p : -1; }
__device__ __forceinline__ uint32_t byte_of(const TreeBytes &t, uint32_t i) { return t.w[i / 4] >> (i % 4 * 8) & 0xFFu; }

// ------------------------------------------------------------------------------------ norms and rotation
// Bound by memory: every element is read and written once (16384 tokens of 32 + 8 heads of 128, 336 MB: 75 us = 4.5 TB/s, where a copy
// runs at 4.9; one token 4.4 us, a launch's own time).  The angle's product and its fraction of a turn are worked out in 64 bits,
// sine and cosine of the fraction in 32.
struct Turn { float c, s; };
__device__ __forceinline__ Turn turn_of(double pos, float freq) {
    const double turns = pos * (double)freq * 0.15915494309189535;        // 1 / (2 pi)
    Turn t;
    const float f = (float)(turns - rint(turns)) * 2.f;                    // half turns, |f| <= 1
    sincospif(f, &t.s, &t.c);
    return t;
}

// head_dim and rot_dim multiples of 16 (rows may start anywhere: this machine's wide loads and stores take any element's address).  A lane
// holds 16 dimensions of a head: with halves 8 of the first half and the 8 they turn with (beyond the rotated ones: 16 of the rest),
// with pairs 16 in a row; so no value moves between lanes, and a head is a group of L = head_dim / 16 lanes (rounded up to a power of
// two), which its sum of squares goes over.  A wave takes a token, all its heads in turn or (few tokens) a share of them, the next ones
// on their way; a lane's sines and cosines, half of the arithmetic, are worked out once for all of these.
template <typename T> struct Vec8 { T v[8]; };
struct GivenPositions {
    static constexpr uint32_t kLds = 0;
    const int32_t *p;
    __device__ __forceinline__ double operator()(uint64_t t) const { return (double)p[t]; }
};
struct StackPositions {       // of a forward's tokens: see launch_stack_rotation
    static constexpr uint32_t kLds = 16;       // keeps a stack's launch off the CUs that a gather copy holds with their whole LDS
    const uint32_t *ctx_dev;
    uint32_t ctx, tree;
    TreeBytes depth;
    __device__ __forceinline__ double operator()(uint64_t t) const { return (double)((ctx_dev ? *ctx_dev : ctx) + (tree ? byte_of(depth, (uint32_t)t) : (uint32_t)t)); }
};
template <typename T, class P>
__global__ __launch_bounds__(256) void qk_norm_rope_wide_kernel(ps_qk_norm_rope_args a, P position, uint32_t L, uint32_t splits) {
    const uint32_t lane = threadIdx.x & 63, l = lane % L, groups = 64 / L, heads = a.n_q_heads + a.n_k_heads;
    const uint32_t half = a.rot_dim / 2, nrot = a.pairs ? 0 : half / 8;
    const bool live = l * 16 < a.head_dim;
    // the first dimensions of the lane's two runs of 8
    const bool across = !a.pairs && l < nrot;
    const uint32_t d0 = across ? l * 8 : l * 16, d1 = across ? half + l * 8 : l * 16 + 8;
    Vec8<T> gain[2][2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const T *g = static_cast<const T *>(w ? a.k_gain : a.q_gain);
        if (a.norm && g && live) {
            gain[w][0] = *reinterpret_cast<const Vec8<T> *>(g + d0);
            gain[w][1] = *reinterpret_cast<const Vec8<T> *>(g + d1);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) gain[w][0].v[e] = gain[w][1].v[e] = (T)1.f;
        }
    }
    auto at = [&](const void *q, const void *k, uint64_t q_token, uint64_t q_head, uint64_t k_token, uint64_t k_head, uint64_t t, uint32_t hh) {
        return hh < a.n_q_heads ? static_cast<const T *>(q) + t * q_token + hh * q_head : static_cast<const T *>(k) + t * k_token + (hh - a.n_q_heads) * k_head;
    };
    const uint64_t items = (uint64_t)a.n_tokens * splits;
    for (uint64_t item = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (uint64_t)gridDim.x * 4) {
        const uint64_t t = item / splits;
        const uint32_t h0 = (uint32_t)(item % splits) * groups + lane / L;
        Vec8<T> u, v;
        auto request = [&](uint32_t hh) {
            if (!live || hh >= heads) return;
            const T *p = at(a.q, a.k, a.q_token, a.q_head, a.k_token, a.k_head, t, hh);
            u = *reinterpret_cast<const Vec8<T> *>(p + d0);
            v = *reinterpret_cast<const Vec8<T> *>(p + d1);
        };
        request(h0);
        Turn w[8];
        if (live && half) {
            const double pos = position(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t i = a.pairs ? d0 / 2 + e : l * 8 + e;
                w[e] = i < half ? turn_of(pos, a.inv_freq[i]) : Turn{1.f, 0.f};
            }
        }
        for (uint32_t hh = h0; hh - lane / L < heads; hh += groups * splits) {      // (the same number of turns for all lanes)
            const bool on = live && hh < heads, isq = hh < a.n_q_heads;
            float x[16];
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = on ? to_f(u.v[e]) : 0.f; x[8 + e] = on ? to_f(v.v[e]) : 0.f; }
            request(hh + groups * splits);
            if (a.norm) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
                for (uint32_t o = L / 2; o; o >>= 1) ss += __shfl_xor(ss, o, 64);
                const float rinv = 1.0f / sqrtf(ss / (float)a.head_dim + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = x[e] * rinv * to_f(isq ? gain[0][0].v[e] : gain[1][0].v[e]);
                    x[8 + e] = x[8 + e] * rinv * to_f(isq ? gain[0][1].v[e] : gain[1][1].v[e]);
                }
            }
            if (!on) continue;
            if (a.pairs ? d0 < a.rot_dim : across) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = a.pairs ? x[2 * e] : x[e], q = a.pairs ? x[2 * e + 1] : x[8 + e];
                    const float pr = p * w[e].c - q * w[e].s, qr = q * w[e].c + p * w[e].s;
                    if (a.pairs) { x[2 * e] = pr; x[2 * e + 1] = qr; }
                    else { x[e] = pr; x[8 + e] = qr; }
                }
            }
            T *y = const_cast<T *>(at(a.q_out, a.k_out, a.q_out_token, a.q_out_head, a.k_out_token, a.k_out_head, t, hh));
            Vec8<T> r, z;
#pragma unroll
            for (int e = 0; e < 8; ++e) { r.v[e] = (T)x[e]; z.v[e] = (T)x[8 + e]; }
            *reinterpret_cast<Vec8<T> *>(y + d0) = r;
            *reinterpret_cast<Vec8<T> *>(y + d1) = z;
        }
    }
}

// Any other layout: a wave per (token, head), lane l holds the pairs l, l + 64, ...
template <typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(ps_qk_norm_rope_args a) {
    const uint32_t lane = threadIdx.x & 63, heads = a.n_q_heads + a.n_k_heads;
    const uint64_t items = (uint64_t)a.n_tokens * heads;
    for (uint64_t item = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (uint64_t)gridDim.x * 4) {
        const uint32_t t = (uint32_t)(item / heads), hh = (uint32_t)(item % heads);
        const bool isq = hh < a.n_q_heads;
        const uint32_t h = isq ? hh : hh - a.n_q_heads;
        const T *x = isq ? static_cast<const T *>(a.q) + t * a.q_token + h * a.q_head : static_cast<const T *>(a.k) + t * a.k_token + h * a.k_head;
        T *y = isq ? static_cast<T *>(a.q_out) + t * a.q_out_token + h * a.q_out_head : static_cast<T *>(a.k_out) + t * a.k_out_token + h * a.k_out_head;
        const T *gain = static_cast<const T *>(isq ? a.q_gain : a.k_gain);
        float rinv = 1.f;
        if (a.norm) {
            float ss = 0.f;
            for (uint32_t d = lane; d < a.head_dim; d += 64) { const float v = to_f(x[d]); ss = fmaf(v, v, ss); }
            for (int o = 32; o; o >>= 1) ss += __shfl_xor(ss, o, 64);
            rinv = 1.0f / sqrtf(ss / (float)a.head_dim + a.eps);
        }
        const uint32_t half = a.rot_dim / 2;
        const double pos = a.rot_dim ? (double)a.positions[t] : 0.0;
        for (uint32_t i = lane; i < half; i += 64) {
            const uint32_t da = a.pairs ? 2 * i : i, db = a.pairs ? 2 * i + 1 : i + half;
            const float ga = a.norm && gain ? to_f(gain[da]) : 1.f, gb = a.norm && gain ? to_f(gain[db]) : 1.f;
            const float va = to_f(x[da]) * rinv * ga, vb = to_f(x[db]) * rinv * gb;
            const Turn w = turn_of(pos, a.inv_freq[i]);
            y[da] = (T)(va * w.c - vb * w.s);
            y[db] = (T)(vb * w.c + va * w.s);
        }
        for (uint32_t d = a.rot_dim + lane; d < a.head_dim; d += 64)
            y[d] = (T)(to_f(x[d]) * rinv * (a.norm && gain ? to_f(gain[d]) : 1.f));
    }
}

template <typename T, class P>
hipError_t launch_rope_wide(const ps_qk_norm_rope_args &a, const P &position, hipStream_t st) {
    uint32_t L = 1;
    while (L * 16 < a.head_dim) L *= 2;
    // (where a launch ends, waves take more items in turn)
    // a wave to a token, and below 4096 tokens (four waves a SIMD) its heads shared out as far as that takes
    const uint32_t rounds = ((a.n_q_heads + a.n_k_heads) * L + 63) / 64, splits = (uint32_t)std::min<uint64_t>(rounds, (4095ull + a.n_tokens) / a.n_tokens);
    hipLaunchKernelGGL((qk_norm_rope_wide_kernel<T, P>), dim3((uint32_t)std::min<uint64_t>(((uint64_t)a.n_tokens * splits + 3) / 4, kMostGroups)), dim3(256), P::kLds, st, a,
                       position, L, splits);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_rope(const ps_qk_norm_rope_args &a, hipStream_t st) {
    if (a.head_dim % 16 == 0 && a.rot_dim % 16 == 0) return launch_rope_wide<T>(a, GivenPositions{a.positions}, st);
    hipLaunchKernelGGL(qk_norm_rope_kernel<T>, dim3((uint32_t)std::min<uint64_t>(((uint64_t)a.n_tokens * (a.n_q_heads + a.n_k_heads) + 3) / 4, kMostGroups)), dim3(256), 0, st, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ tree attention
// Score rows are (token, query head of the kv group) pairs.  A workgroup of four waves holds a block of NT x 16 rows of one kv
// head and a run of 32-position tiles; its waves take the tiles in turn, each with a running maximum, weight sum and value sums
// of its own, and meet in LDS at the end: no barrier in the walk.
//  scores, transposed: S^T = K Q^T, A = 16 positions x 32 dims of K straight from memory into registers, B = 16 rows of
//   queries (registers, loaded once): lane (row j, c) then holds four positions of row j for each of two tiles;
//  weights x values, transposed: O^T = V^T P^T, B = the weights exactly as the score accumulators hold them (the two
//   16-position tiles are numbered so that lane group c owns 8 consecutive positions: 4 from each), A = 16 dims x 32 positions of V
//   by LDS transpose reads of the wave's own stage; and the weights' sum by one more product, with ones.
// The next tile's K and V are requested as soon as the scores have used this one's K and its V lies in LDS.  They go through
// registers: in front of a transpose read the compiler waits for every load into LDS, the next tile's too.
// This is the kernel for up to 32 rows of a kv head, bound by the cache's bytes: 24 sequences of 2 tokens over 8192 positions (32 / 8
// heads) 147 us = 5.5 TB/s, one of 2 over 131072 (32 / 4) 70 us = 3.8, of one over 32768 35 us; few positions take a launch's and a merge's time, about 8 and 4 us.
// 16-byte piece u of a staged V row lies in slot u ^ swizzle: even swizzles keep the pair of pieces that a transpose read takes
// together, and the eight rows of half a wave (8 c + 0 .. 3) lie in different banks
template <int D> __device__ __forceinline__ uint32_t v_swizzle(uint32_t row) {
    return D == 128 ? ((row & 3u) | (((row >> 3) & 1u) << 2)) << 1 : (((row >> 1) & 1u) | (((row >> 3) & 1u) << 1)) << 1;
}

// K rows, read 16 at a time (8 (i / 4) + i % 4): their swizzles are all different (D = 64: two rows share the banks, those eight of a kind are)
template <int D> __device__ __forceinline__ uint32_t k_swizzle(uint32_t row) {
    return D == 128 ? (row & 3u) | (((row >> 3) & 3u) << 2) : ((row >> 1) & 1u) | (((row >> 3) & 3u) << 1);
}

constexpr uint32_t kTile = 32;           // positions of a tile
constexpr uint32_t kStep = 64;           // positions of a step of the kernel for many rows
constexpr uint32_t kMaskWords = PS_TREE_MAX / 32;

struct TreeDeal { uint32_t nt, blocks, nsplit, unit; };       // nt 0: the kernel for many rows; unit: positions that a split is a multiple of

constexpr uint32_t kTreeTables = PS_TREE_MAX * kMaskWords * 4 + PS_TREE_MAX * 4 + 16;
template <int D, int NT> constexpr uint32_t tree_lds() {
    const uint32_t stages = 4 * kTile * D * 2, meet = 4 * NT * 16 * (D + 4) * 4 + 4 * NT * 16 * 2 * 4;
    return std::max(stages, meet) + kTreeTables;
}
template <int D> constexpr uint32_t tree_rows_lds() { return 2 * 2 * kStep * D * 2 + kTreeTables; }

// Units of a sequence's positions: the cache's, then the tree's own; each split takes `per` of them
__device__ __forceinline__ uint32_t units_of(uint32_t ctx, uint32_t t_n, uint32_t unit) { return (ctx + unit - 1) / unit + (t_n + unit - 1) / unit; }
__device__ __forceinline__ uint32_t units_per_split(uint32_t units, uint32_t nsplit) { return (units + nsplit - 1) / nsplit; }

// Where a launch's tables are: in device memory (a batch of sequences), or in its arguments (a stack's own forward: one sequence, some
// of the model's heads, rows appended through a table of addresses)
struct BatchTrees {
    static constexpr bool kStack = false;
};
struct StackTree {
    static constexpr bool kStack = true;
    const uint64_t *home;
    uint32_t cap, heads, head0;          // query heads of the model, the launch's first one
    TreeBytes up;
};
struct TreeSeq { SeqRows rows; uint32_t ctx; };
template <class S>
__device__ __forceinline__ TreeSeq sequence_of(const ps_tree_attention_args &a, const S &, uint32_t s) {
    if constexpr (S::kStack) return {{0, (int)a.n_tokens}, a.max_context};
    else return {rows_of(a.first, s, a.n_tokens, a.max_tree), (uint32_t)clampi(a.context[s], 0, (int)a.max_context)};
}
// where the records of a token's query head start
template <class S>
__device__ __forceinline__ size_t record_of(const ps_tree_attention_args &a, const S &w, size_t token, uint32_t h, uint32_t nsplit) {
    if constexpr (S::kStack) return (token * w.heads + w.head0 + h) * nsplit;
    else return (token * a.n_q_heads + h) * nsplit;
}

// anc[token][word]: a bit for the token itself and each of its ancestors; every thread of the workgroup calls it.  Every step doubles how far back a
// token's mask reaches.  Up to 64 tokens one wave does it in registers.
template <class Where>
__device__ __forceinline__ void ancestors(const ps_tree_attention_args &a, const Where &where, const SeqRows &sr, uint32_t *anc, int *up) {
    const uint32_t tid = threadIdx.x, t_n = sr.n;
    int link = -1;
    if (tid < t_n) {
        if constexpr (Where::kStack) link = (int)byte_of(where.up, tid) - 1;
        else link = parent_of(a.parent[sr.row0 + tid], (int)tid);
    }
    if (t_n <= 64) {
        if (tid < 64) {
            uint32_t m0 = tid < 32 ? 1u << tid : 0u, m1 = tid < 32 ? 0u : 1u << (tid - 32);
            while (__any(link >= 0)) {
                const int from = max(link, 0);
                const uint32_t u0 = __shfl(m0, from, 64), u1 = __shfl(m1, from, 64);
                const int next = __shfl(link, from, 64);
                if (link >= 0) { m0 |= u0; m1 |= u1; link = next; }
            }
            if (tid < t_n) { anc[tid * kMaskWords] = m0; anc[tid * kMaskWords + 1] = m1; }
        }
        __syncthreads();
        return;
    }
    if (tid < t_n) {
#pragma unroll
        for (uint32_t w = 0; w < kMaskWords; ++w) anc[tid * kMaskWords + w] = tid / 32 == w ? 1u << (tid % 32) : 0u;
        up[tid] = link;
    }
    uint32_t m[kMaskWords];
    while (__syncthreads_or(link >= 0)) {
        int next = -1;
        if (link >= 0) {
#pragma unroll
            for (uint32_t w = 0; w < kMaskWords; ++w) m[w] = anc[link * kMaskWords + w];
            next = up[link];
        }
        __syncthreads();
        if (link >= 0) {
#pragma unroll
            for (uint32_t w = 0; w < kMaskWords; ++w) anc[tid * kMaskWords + w] |= m[w];
            up[tid] = next;
        }
        link = next;
    }
}

// rows context and up, which nobody reads: each block moves the tokens whose first row it holds
template <typename T, int D, class Where>
__device__ __forceinline__ void append_rows(const ps_tree_attention_args &a, const Where &where, uint32_t s, uint32_t hk, uint32_t ctx, uint32_t t0, uint32_t t1, const T *kn, const T *vn) {
    constexpr uint32_t kRowPieces = D / 8;
    T *kd = static_cast<T *>(a.k_cache) + s * a.k_seq + hk * a.k_head, *vd = static_cast<T *>(a.v_cache) + s * a.v_seq + hk * a.v_head;
    if constexpr (Where::kStack) {
        kd = reinterpret_cast<T *>(where.home[hk]);
        vd = kd + (size_t)where.cap * D;
    }
    for (uint32_t u = threadIdx.x; u < (t1 - t0) * kRowPieces * 2; u += 256) {
        const uint32_t t = t0 + u / (2 * kRowPieces), e = u % kRowPieces * 8;
        const bool v = u / kRowPieces & 1;
        *reinterpret_cast<u4_t *>(v ? vd + ((size_t)ctx + t) * a.v_row + e : kd + ((size_t)ctx + t) * a.k_row + e) =
            *reinterpret_cast<const u4_t *>(v ? vn + (size_t)t * a.v_new_token + e : kn + (size_t)t * a.k_new_token + e);
    }
}

template <typename T, int D, int NT, class Where>
__global__ __launch_bounds__(256, 2) void tree_attention_kernel(ps_tree_attention_args a, Where where, uint32_t blocks, uint32_t nsplit, float *part) {
    using M = Mfma<T>;
    using v8 = typename M::v8;
    constexpr int KK = D / 32, DT = D / 16, RB = NT * 16, OP = D + 4;
    constexpr uint32_t kStage = kTile * D * 2, kRowPieces = D / 8, kVLoads = kStage / 1024;
    extern __shared__ u4_t tree_lds_mem[];
    unsigned char *const lds = reinterpret_cast<unsigned char *>(tree_lds_mem);
    constexpr uint32_t kTables = tree_lds<D, NT>() - kTreeTables;
    uint32_t *const anc = reinterpret_cast<uint32_t *>(lds + kTables);           // [token][word]: itself and its ancestors
    int *const up = reinterpret_cast<int *>(anc + PS_TREE_MAX * kMaskWords);
    int *const wild = up + PS_TREE_MAX;                                          // some own value is infinite or no number

    // blocks of the same positions lie 8 workgroups apart: on one XCD, whose L2 they share
    const uint32_t units = a.n_seq * a.n_kv_heads * nsplit;
    const uint32_t unit = blockIdx.x / 8 / blocks * 8 + blockIdx.x % 8, rb = blockIdx.x / 8 % blocks;
    if (unit >= units) return;
    const uint32_t z = unit % nsplit, hk = unit / nsplit % a.n_kv_heads, s = unit / nsplit / a.n_kv_heads;
    const TreeSeq seq = sequence_of(a, where, s);
    const SeqRows sr = seq.rows;
    const uint32_t ctx = seq.ctx, t_n = sr.n, G = a.n_q_heads / a.n_kv_heads;
    const uint32_t R = t_n * G, row0 = rb * RB;
    if (row0 >= R) return;
    const uint32_t nc = (ctx + kTile - 1) / kTile, tiles = units_of(ctx, t_n, kTile), per = units_per_split(tiles, nsplit);
    const uint32_t lo = z * per, hi = min(tiles, lo + per);
    if (lo >= hi) return;               // (the merge knows how many splits a sequence has)
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t i = lane & 15, c = lane >> 4;

    const char *kc = reinterpret_cast<const char *>(static_cast<const T *>(a.k_cache) + s * a.k_seq + hk * a.k_head);
    const char *vc = reinterpret_cast<const char *>(static_cast<const T *>(a.v_cache) + s * a.v_seq + hk * a.v_head);
    const T *kn = static_cast<const T *>(a.k_new) + (size_t)sr.row0 * a.k_new_token + hk * a.k_new_head;
    const T *vn = static_cast<const T *>(a.v_new) + (size_t)sr.row0 * a.v_new_token + hk * a.v_new_head;
    unsigned char *const stage = lds + wave * kStage;
    // K: lane i of position tile Tt takes row 8 (i / 4) + i % 4 + 4 Tt; V: lane l fills slot l of four (D = 64: eight) rows
    const uint32_t krow = 8 * (i >> 2) + (i & 3), vrow = lane / kRowPieces;
    u4_t kreg[2][KK], vreg[kVLoads];
    auto request = [&](uint32_t tile) {
        const bool own = tile >= nc;
        const uint32_t P0 = (own ? tile - nc : tile) * kTile, last = min(kTile, (own ? t_n : ctx) - P0) - 1;
        const uint32_t krow_b = (uint32_t)(own ? a.k_new_token : a.k_row) * 2, vrow_b = (uint32_t)(own ? a.v_new_token : a.v_row) * 2;
        // (rows past the last lie past the buffer's range: zeros)
        const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((own ? reinterpret_cast<const char *>(kn) : kc) + (size_t)P0 * krow_b), 0,
                                                                            (int)(last * krow_b + D * 2), 0x00020000);
        const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((own ? reinterpret_cast<const char *>(vn) : vc) + (size_t)P0 * vrow_b), 0,
                                                                            (int)(last * vrow_b + D * 2), 0x00020000);
#pragma unroll
        for (int Tt = 0; Tt < 2; ++Tt)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                kreg[Tt][kk] = __builtin_bit_cast(u4_t, __builtin_amdgcn_raw_buffer_load_b128(kb, (krow + 4 * Tt) * krow_b + c * 16 + kk * 64, 0, 0));
#pragma unroll
        for (uint32_t u = 0; u < kVLoads; ++u) {
            const uint32_t row = u * (64 / kRowPieces) + vrow;
            vreg[u] = __builtin_bit_cast(u4_t, __builtin_amdgcn_raw_buffer_load_b128(vb, row * vrow_b + ((lane % kRowPieces) ^ v_swizzle<D>(row)) * 16, 0, 0));
        }
    };
    if (lo + wave < hi) request(lo + wave);

    // the block's rows of queries; a negative scale turns their signs
    const float scale_abs = fabsf(a.scale);
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    const float c2 = fmaxf(scale_abs * 1.4426950408889634f, 1e-30f);     // weights are 2^(c2 (s - m))
    const float slack = WeightRange<T>::kSlack / c2;
    uint32_t tok[NT];
    v8 q[NT][KK];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t rho = min(row0 + t * 16 + i, R - 1);
        tok[t] = rho / G;
        const T *qr = static_cast<const T *>(a.q) + ((size_t)sr.row0 + tok[t]) * a.q_token + (size_t)(hk * G + rho % G) * a.q_head + c * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            u4_t v = *reinterpret_cast<const u4_t *>(qr + kk * 32);
            v.x ^= sign; v.y ^= sign; v.z ^= sign; v.w ^= sign;
            q[t][kk] = __builtin_bit_cast(v8, v);
        }
    }
    // own tiles: which tokens each token sees
    const bool own = hi > nc;
    if (own) {
        if (tid == 0) *wild = 0;
        ancestors(a, where, sr, anc, up);
    }
    if (a.append && z == 0) append_rows<T, D>(a, where, s, hk, ctx, (row0 + G - 1) / G, min(t_n, (row0 + RB + G - 1) / G), kn, vn);

    float m_run[NT];
    f4_t O[NT][DT], L[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m_run[t] = -INFINITY;
        L[t] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[t][dt] = f4_t{0.f, 0.f, 0.f, 0.f};
    }
    v8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (T)1.f;
    uint32_t vread[DT];
    {
        const uint32_t row = 8 * c + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vread[dt] = row * (D * 2) + (((2 * dt + ((i & 3) >> 1)) ^ v_swizzle<D>(row)) << 4) + (i & 1) * 8;
    }
    for (uint32_t tile = lo + wave; tile < hi; tile += 4) {
        const bool mine = tile >= nc;                                   // (uniform) one of the tree's own tiles
        const uint32_t P0 = (mine ? tile - nc : tile) * kTile;
        f4_t S[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t][0] = S[t][1] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int Tt = 0; Tt < 2; ++Tt)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t][Tt] = M::mul(__builtin_bit_cast(v8, kreg[Tt][kk]), q[t][kk], S[t][Tt]);
        if (mine) {
            bool odd = false;
#pragma unroll
            for (uint32_t u = 0; u < kVLoads; ++u) odd |= made_finite<T>(vreg[u]);
            if (odd) *wild = 1;
        }
#pragma unroll
        for (uint32_t u = 0; u < kVLoads; ++u) *reinterpret_cast<u4_t *>(stage + u * 1024 + lane * 16) = vreg[u];
        if (tile + 4 < hi) request(tile + 4);
        if (mine) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint32_t word = anc[tok[t] * kMaskWords + P0 / 32] >> (8 * c);
#pragma unroll
                for (int e = 0; e < 8; ++e) S[t][e >> 2][e & 3] = word >> e & 1 ? S[t][e >> 2][e & 3] : -INFINITY;
            }
        } else if (ctx - P0 < kTile) {      // the cache's last tile
            asm volatile("");
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) S[t][e >> 2][e & 3] = P0 + 8 * c + e < ctx ? S[t][e >> 2][e & 3] : -INFINITY;
        }
        v8 P[NT];
        weigh<T>(S, m_run, L, O, P, c2, slack);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const v8 vr = __builtin_bit_cast(v8, transposed(stage + vread[dt], 4 * D * 2));
#pragma unroll
            for (int t = 0; t < NT; ++t) O[t][dt] = M::mul(vr, P[t], O[t][dt]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) L[t] = M::mul(ones, P[t], L[t]);
    }
    // the four waves meet
    __syncthreads();
    float *ob = reinterpret_cast<float *>(lds), *om = ob + 4 * RB * OP, *ol = om + 4 * RB;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t row = t * 16 + i;
        float *dst = ob + (wave * RB + row) * OP + 4 * c;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f4_t *>(dst + 16 * dt) = O[t][dt];
        if (c == 0) { om[wave * RB + row] = m_run[t]; ol[wave * RB + row] = L[t][0]; }
    }
    __syncthreads();
    constexpr uint32_t kPiece = 4, kPerRow = D / kPiece;
    for (uint32_t u = tid; u < RB * kPerRow; u += 256) {
        const uint32_t row = u / kPerRow, d0 = u % kPerRow * kPiece, rho = row0 + row;
        if (rho >= R) break;
        float mx = om[row];
#pragma unroll
        for (int w = 1; w < 4; ++w) mx = fmaxf(mx, om[w * RB + row]);
        float l = 0.f;
        f4_t o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = om[w * RB + row];
            // a wave that saw nothing of this row holds zeros and weighs nothing; one whose scores are no numbers holds none, and says so
            const float f = mw == -INFINITY ? (mx == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f((mw - mx) * c2);
            l = fmaf(f, ol[w * RB + row], l);
            const f4_t v = *reinterpret_cast<const f4_t *>(ob + (w * RB + row) * OP + d0);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[e], o[e]);
        }
        const uint32_t t = rho / G, h = hk * G + rho % G;
        if (own && *wild) {
            for (uint32_t j = (max(lo, nc) - nc) * kTile; j < min(t_n, (hi - nc) * kTile); ++j) {
                if (!(anc[t * kMaskWords + j / 32] >> (j % 32) & 1)) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = to_f(vn[(size_t)j * a.v_new_token + d0 + e]);
                    if (!(fabsf(v) < INFINITY)) o[e] += v;
                }
            }
        }
        const size_t token = (size_t)sr.row0 + t;
        if (nsplit > 1) {
            float *dst = part + (record_of(a, where, token, h, nsplit) + z) * OP;
            *reinterpret_cast<f4_t *>(dst + d0) = o;
            if (d0 == 0) *reinterpret_cast<float2 *>(dst + D) = make_float2(mx * c2, l);
        } else {
            T r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (T)(o[e] / l);
            *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + token * a.out_token + h * a.out_head + d0) = *reinterpret_cast<const uint2 *>(r);
        }
    }
}

// The kernel for more than 32 rows of a kv head: a workgroup of four waves with 32 rows each walks its positions in steps of 64, whose
// K and V rows all four read from LDS: a quarter of the memory traffic, which at 512 rows bounds the kernel above (16 KB a wave and tile from the L2:
// 64 tokens over 131072 positions, 8 query heads a kv head: 316 us so, 186 here = 740 TFLOP/s).  Products as above, K's operands from LDS as well.  Two stages, one barrier
// a step; a step's rows are requested two steps ahead, into registers, and written one ahead.
template <typename T, int D, class Where>
__global__ __launch_bounds__(256, 2) void tree_rows_kernel(ps_tree_attention_args a, Where where, uint32_t blocks, uint32_t nsplit, float *part) {
    using M = Mfma<T>;
    using v8 = typename M::v8;
    constexpr int KK = D / 32, DT = D / 16, NT = 2, RB = 4 * NT * 16, OP = D + 4;
    constexpr uint32_t kHalf = kStep * D * 2, kRowPieces = D / 8, kLoads = kStep * kRowPieces / 256;     // a step's K (or V) rows; pieces a thread moves of them
    extern __shared__ u4_t tree_lds_mem[];
    unsigned char *const lds = reinterpret_cast<unsigned char *>(tree_lds_mem);
    uint32_t *const anc = reinterpret_cast<uint32_t *>(lds + 4 * kHalf);
    int *const up = reinterpret_cast<int *>(anc + PS_TREE_MAX * kMaskWords);
    int *const wild = up + PS_TREE_MAX;

    const uint32_t units = a.n_seq * a.n_kv_heads * nsplit;
    const uint32_t unit = blockIdx.x / 8 / blocks * 8 + blockIdx.x % 8, rb = blockIdx.x / 8 % blocks;
    if (unit >= units) return;
    const uint32_t z = unit % nsplit, hk = unit / nsplit % a.n_kv_heads, s = unit / nsplit / a.n_kv_heads;
    const TreeSeq seq = sequence_of(a, where, s);
    const SeqRows sr = seq.rows;
    const uint32_t ctx = seq.ctx, t_n = sr.n, G = a.n_q_heads / a.n_kv_heads;
    const uint32_t R = t_n * G, row0 = rb * RB;
    if (row0 >= R) return;
    const uint32_t nc = (ctx + kStep - 1) / kStep, steps = units_of(ctx, t_n, kStep), per = units_per_split(steps, nsplit);
    const uint32_t lo = z * per, hi = min(steps, lo + per);
    if (lo >= hi) return;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t i = lane & 15, c = lane >> 4;
    const char *kc = reinterpret_cast<const char *>(static_cast<const T *>(a.k_cache) + s * a.k_seq + hk * a.k_head);
    const char *vc = reinterpret_cast<const char *>(static_cast<const T *>(a.v_cache) + s * a.v_seq + hk * a.v_head);
    const T *kn = static_cast<const T *>(a.k_new) + (size_t)sr.row0 * a.k_new_token + hk * a.k_new_head;
    const T *vn = static_cast<const T *>(a.v_new) + (size_t)sr.row0 * a.v_new_token + hk * a.v_new_head;

    u4_t kreg[kLoads], vreg[kLoads];
    auto request = [&](uint32_t step) {
        const bool mine = step >= nc;
        const uint32_t P0 = (mine ? step - nc : step) * kStep, last = min(kStep, (mine ? t_n : ctx) - P0) - 1;
        const uint32_t krow_b = (uint32_t)(mine ? a.k_new_token : a.k_row) * 2, vrow_b = (uint32_t)(mine ? a.v_new_token : a.v_row) * 2;
        // (rows past the last lie past the buffer's range: zeros)
        const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((mine ? reinterpret_cast<const char *>(kn) : kc) + (size_t)P0 * krow_b), 0,
                                                                            (int)(last * krow_b + D * 2), 0x00020000);
        const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((mine ? reinterpret_cast<const char *>(vn) : vc) + (size_t)P0 * vrow_b), 0,
                                                                            (int)(last * vrow_b + D * 2), 0x00020000);
#pragma unroll
        for (uint32_t u = 0; u < kLoads; ++u) {
            const uint32_t row = (u * 256 + tid) / kRowPieces, slot = tid % kRowPieces;
            kreg[u] = __builtin_bit_cast(u4_t, __builtin_amdgcn_raw_buffer_load_b128(kb, row * krow_b + (slot ^ k_swizzle<D>(row)) * 16, 0, 0));
            vreg[u] = __builtin_bit_cast(u4_t, __builtin_amdgcn_raw_buffer_load_b128(vb, row * vrow_b + (slot ^ v_swizzle<D>(row)) * 16, 0, 0));
        }
    };
    auto store = [&](uint32_t step, uint32_t buf) {
        if (step >= nc) {
            bool odd = false;
#pragma unroll
            for (uint32_t u = 0; u < kLoads; ++u) odd |= made_finite<T>(vreg[u]);
            if (odd) *wild = 1;
        }
        unsigned char *to = lds + buf * 2 * kHalf;
#pragma unroll
        for (uint32_t u = 0; u < kLoads; ++u) {
            *reinterpret_cast<u4_t *>(to + (u * 256 + tid) * 16) = kreg[u];
            *reinterpret_cast<u4_t *>(to + kHalf + (u * 256 + tid) * 16) = vreg[u];
        }
    };
    request(lo);
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    const float c2 = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-30f);
    const float slack = WeightRange<T>::kSlack / c2;
    const uint32_t mine0 = row0 + wave * (NT * 16);      // the wave's rows
    const bool rows = mine0 < R;
    uint32_t tok[NT], head[NT];
    v8 q[NT][KK];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t rho = min(mine0 + t * 16 + i, R - 1);
        tok[t] = rho / G;
        head[t] = hk * G + rho % G;
        const T *qr = static_cast<const T *>(a.q) + ((size_t)sr.row0 + tok[t]) * a.q_token + (size_t)head[t] * a.q_head + c * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) q[t][kk] = __builtin_bit_cast(v8, *reinterpret_cast<const u4_t *>(qr + kk * 32) ^ u4_t{sign, sign, sign, sign});
    }
    const bool own = hi > nc;
    if (own) {
        if (tid == 0) *wild = 0;
        ancestors(a, where, sr, anc, up);
    }
    if (a.append && z == 0) append_rows<T, D>(a, where, s, hk, ctx, (row0 + G - 1) / G, min(t_n, (row0 + RB + G - 1) / G), kn, vn);

    float m_run[NT];
    f4_t O[NT][DT], L[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m_run[t] = -INFINITY;
        L[t] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[t][dt] = f4_t{0.f, 0.f, 0.f, 0.f};
    }
    v8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (T)1.f;
    // LDS byte offsets of this lane's operand pieces in a stage's first tile (a tile further: 32 rows, whose swizzles are the same)
    uint32_t kread[KK], vread[DT];
    {
        const uint32_t row = 8 * (i >> 2) + (i & 3);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kread[kk] = row * (D * 2) + (((4 * kk + c) ^ k_swizzle<D>(row)) << 4);
        const uint32_t vrow = 8 * c + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vread[dt] = kHalf + vrow * (D * 2) + (((2 * dt + ((i & 3) >> 1)) ^ v_swizzle<D>(vrow)) << 4) + (i & 1) * 8;
    }
    auto meet = [] {      // everyone's LDS accesses are done (loads from memory stay on their way)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    store(lo, 0);
    if (lo + 1 < hi) request(lo + 1);
    meet();
    for (uint32_t step = lo; step < hi; ++step) {
        const bool mine = step >= nc;
        const uint32_t P0 = (mine ? step - nc : step) * kStep, left = (mine ? t_n : ctx) - P0;
        const unsigned char *st = lds + ((step - lo) & 1) * 2 * kHalf;
        if (rows) {
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                if (left <= h * kTile) break;            // (uniform)
                const unsigned char *tile = st + h * kTile * D * 2;
                f4_t S[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t][0] = S[t][1] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int Tt = 0; Tt < 2; ++Tt)
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) {
                        // (rows 4 further have the same swizzle)
                        const v8 kr = __builtin_bit_cast(v8, *reinterpret_cast<const u4_t *>(tile + kread[kk] + Tt * 4 * D * 2));
#pragma unroll
                        for (int t = 0; t < NT; ++t) S[t][Tt] = M::mul(kr, q[t][kk], S[t][Tt]);
                    }
                if (mine) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint32_t word = anc[tok[t] * kMaskWords + P0 / 32 + h] >> (8 * c);
#pragma unroll
                        for (int e = 0; e < 8; ++e) S[t][e >> 2][e & 3] = word >> e & 1 ? S[t][e >> 2][e & 3] : -INFINITY;
                    }
                } else if (left - h * kTile < kTile) {
                    asm volatile("");
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 8; ++e) S[t][e >> 2][e & 3] = h * kTile + 8 * c + e < left ? S[t][e >> 2][e & 3] : -INFINITY;
                }
                v8 P[NT];
                weigh<T>(S, m_run, L, O, P, c2, slack);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const v8 vr = __builtin_bit_cast(v8, transposed(tile + vread[dt], 4 * D * 2));
#pragma unroll
                    for (int t = 0; t < NT; ++t) O[t][dt] = M::mul(vr, P[t], O[t][dt]);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) L[t] = M::mul(ones, P[t], L[t]);
            }
        }
        if (step + 1 < hi) {
            store(step + 1, (step + 1 - lo) & 1);
            if (step + 2 < hi) request(step + 2);
        }
        meet();
    }
    if (!rows) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (mine0 + t * 16 + i >= R) continue;
        const size_t token = (size_t)sr.row0 + tok[t];
        if (own && *wild) {
            for (uint32_t j = (max(lo, nc) - nc) * kStep; j < min(t_n, (hi - nc) * kStep); ++j) {
                if (!(anc[tok[t] * kMaskWords + j / 32] >> (j % 32) & 1)) continue;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = to_f(vn[(size_t)j * a.v_new_token + 16 * dt + 4 * c + e]);
                        if (!(fabsf(v) < INFINITY)) O[t][dt][e] += v;
                    }
            }
        }
        if (nsplit > 1) {
            float *dst = part + (record_of(a, where, token, head[t], nsplit) + z) * OP;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f4_t *>(dst + 16 * dt + 4 * c) = O[t][dt];
            if (c == 0) *reinterpret_cast<float2 *>(dst + D) = make_float2(m_run[t] * c2, L[t][0]);
        } else {
            T *dst = static_cast<T *>(a.out) + token * a.out_token + (size_t)head[t] * a.out_head + 4 * c;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                T r[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = (T)(O[t][dt][e] / L[t][0]);
                *reinterpret_cast<u2_t *>(dst + 16 * dt) = *reinterpret_cast<const u2_t *>(r);
            }
        }
    }
}

// The splits' records: 4 to 5 us, a launch and two dependent loads.  A wave per (token, query head) merges the records of its sequence's splits, in their order: value sums, then maximum (in
// powers of two) and weight sum.
template <typename T, int D, class S>
__global__ __launch_bounds__(256) void tree_merge_kernel(ps_tree_attention_args a, S where, uint32_t nsplit, uint32_t unit, const float *part) {
    constexpr int E = D / 64, OP = D + 4;
    const uint32_t lane = threadIdx.x & 63, h = blockIdx.x * 4 + (threadIdx.x >> 6), t = blockIdx.y, s = blockIdx.z;
    const TreeSeq seq = sequence_of(a, where, s);
    const SeqRows sr = seq.rows;
    if (h >= a.n_q_heads || (int)t >= sr.n) return;
    const uint32_t ctx = seq.ctx;
    const uint32_t units = units_of(ctx, sr.n, unit), per = units_per_split(units, nsplit), n = (units + per - 1) / per;
    const size_t token = (size_t)sr.row0 + t;
    const float *p = part + record_of(a, where, token, h, nsplit) * OP;
    float mx = -INFINITY, l = 0.f, o[E] = {};
    for (uint32_t z0 = 0; z0 < n; z0 += 8) {
        float mv[8], lv[8], ov[8][E], m8 = mx;
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) {
            const float *r = p + (size_t)min(z0 + u, n - 1) * OP;
            mv[u] = r[D];
            lv[u] = r[D + 1];
#pragma unroll
            for (int e = 0; e < E; ++e) ov[u][e] = r[lane * E + e];
        }
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) m8 = fmaxf(m8, mv[u]);
        const float ms = m8 == -INFINITY ? 0.f : m8, resc = __builtin_amdgcn_exp2f(mx - ms);
        l *= resc;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= resc;
        mx = m8;
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) {
            const bool in = z0 + u < n;          // (a record past the last is the last again)
            const float w = mv[u] == -INFINITY ? (m8 == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(mv[u] - ms);       // as the waves above
            l = in ? fmaf(w, lv[u], l) : l;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = in ? fmaf(w, ov[u][e], o[e]) : o[e];
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) static_cast<T *>(a.out)[token * a.out_token + h * a.out_head + lane * E + e] = (T)(o[e] / l);
}

// How the work is dealt out.  Rows of a kv head: up to 16 or 32 in one block of the first kernel, more in blocks of 128 of the second (48
// rows, 8 sequences of 8190: 72 us in two blocks of the first, 62 so; with 64 rows a wave the first takes more than 256 registers, and the compiler then moves the value
// sums between its two kinds of them in every tile).  Positions: as many splits as bring the launch to the workgroups the chip holds
// at once (two per CU, by registers), none of less than four units of 32 or two of 64; for several sequences, whose lengths differ, twice as many
// (16 sequences of 17 tokens, lengths of 600 to 8190, 57 -> 48 us, 32 of 8 tokens 87 -> 82; eight of one length 62 -> 70).
// The kernels then give each split ceil(units / splits), so fewer may have work: 24 tokens over 4096 positions are 65 steps in up to 32 splits, and
// 22 of them take 3 each (176 workgroups; 80 more return at once).
TreeDeal tree_deal(const ps_tree_attention_args &a) {
    TreeDeal d;
    const uint32_t rows = std::max(1u, a.max_tree) * (a.n_q_heads / a.n_kv_heads);
    d.nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 0;
    d.unit = d.nt ? kTile : kStep;
    const uint32_t block = d.nt ? d.nt * 16 : 128;
    d.blocks = (rows + block - 1) / block;
    const uint64_t wgs = std::max<uint64_t>(1, (uint64_t)a.n_seq * a.n_kv_heads * d.blocks);
    const uint32_t units = (a.max_context + d.unit - 1) / d.unit + (a.max_tree + d.unit - 1) / d.unit, least = d.nt ? 4 : 2;
    d.nsplit = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>((a.n_seq > 1 ? 1024 : 512) / wgs, units / least));
    return d;
}

// a kernel that takes more LDS than a launch gets by itself: announced once per device
template <class K, class S>
hipError_t launch_tree_k(K kernel, uint32_t lds, std::atomic<uint64_t> &done, const ps_tree_attention_args &a, const S &where, const TreeDeal &d, float *part, hipStream_t st) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    const uint32_t units = a.n_seq * a.n_kv_heads * d.nsplit;
    hipLaunchKernelGGL(kernel, dim3((units + 7) / 8 * 8 * d.blocks), dim3(256), lds, st, a, where, d.blocks, d.nsplit, part);
    return hipGetLastError();
}
template <typename T, int D, class S>
hipError_t launch_tree(const ps_tree_attention_args &a, const S &where, const TreeDeal &d, float *part, hipStream_t st) {
    static std::atomic<uint64_t> done[3];
    if (d.nt == 0) return launch_tree_k(&tree_rows_kernel<T, D, S>, tree_rows_lds<D>(), done[0], a, where, d, part, st);
    if (d.nt == 1) return launch_tree_k(&tree_attention_kernel<T, D, 1, S>, tree_lds<D, 1>(), done[1], a, where, d, part, st);
    return launch_tree_k(&tree_attention_kernel<T, D, 2, S>, tree_lds<D, 2>(), done[2], a, where, d, part, st);
}
template <typename T, int D, class S>
hipError_t launch_merge(const ps_tree_attention_args &a, const S &where, const TreeDeal &d, const float *part, hipStream_t st) {
    hipLaunchKernelGGL((tree_merge_kernel<T, D, S>), dim3((a.n_q_heads + 3) / 4, a.max_tree, a.n_seq), dim3(256), S::kStack ? 16 : 0, st, a, where, d.nsplit, d.unit, part);
    return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_trees(const ps_tree_attention_args &a, const TreeDeal &d, float *part, hipStream_t st) {
    const hipError_t e = launch_tree<T, D>(a, BatchTrees{}, d, part, st);
    return e != hipSuccess || d.nsplit == 1 ? e : launch_merge<T, D>(a, BatchTrees{}, d, part, st);
}

// ------------------------------------------------------------------------------------ verification
// Rows are cut into chunks (rules in verify_shape).  Launches, in order:
//  verify_rows_kernel   chunk maximum and sum of exponentials of every row that a decision needs: the nodes with children, target and
//                       draft; without sampling the largest logit's index instead
//  verify_left_kernel   with drafts, for the k-th child (k = 1 ..): chunk sums W_k = sum max(p - c_k q, 0) of the nodes whose first k
//                       children are refused and that the walk may still reach
//  verify_draw_kernel   every workgroup works out the same walk; chunk sums of what is left to draw from behind its last node
//  verify_pick_kernel   the chunk that the random number falls into, and the index in it
// Sums are in 64 bits, exponentials to 4e-11 of each: with fp32's 2^-24 a border of the running sum moves by as much as a hundred thousandth of
// the vocabulary's entries weigh.  A 64-bit operation takes this machine 5.3 clocks of a wave, a 32-bit one 4.3; an exponential
// here is about 15 of them, which in a large batch takes longer than the row's bytes do.  No result depends on the order of workgroups.
// 32 trees of up to 32 nodes, two drafts a node, 128256 entries, drafts' logits: 80 + 22 + 19 + 9 us (205 MB: 42 us as bytes, about 77 as
// operations); 16 trees of given drafts 19 + 12 + 9 us; a chain of 4 drafts over 32000 5 + 9 + 8: chains of latencies (a step's loads, a few hundred
// clocks for each reduction and exponential), no longer bound by anything that more workgroups would share.
constexpr uint32_t kVerThreads = 256, kPickThreads = 512, kMaxChunks = 32;
struct RowPart { double z; float m; int best; };                 // one chunk of a row: sum of exp((x - m) k), m about its maximum (greedy: m its maximum, at `best`)
struct DrawHead { double c, ip, iq; float m, mq; int row, kind, nref, pad; };   // what is left behind the last node, for the pick
enum { DRAW_NONE = 0, DRAW_BEST = 1, DRAW_LEAF = 2, DRAW_LEFT = 3, DRAW_GIVEN = 4 };
struct VerifyShape { uint32_t chunk, nchunk, loop, dchunk, ndraw; };   // rows in chunks; what is drawn from in chunks of its own
struct VerifyWork { RowPart *parts; double *left; RowPart *recs; DrawHead *heads; int *refused; };   // [token][target, draft][chunk], [token][draw chunk], [seq][draw chunk], [seq], [seq][max_tree]

__device__ __forceinline__ double block_sum(double v, double *buf) {     // every thread gets the sum
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    return (buf[0] + buf[1]) + (buf[2] + buf[3]);
}
__device__ __forceinline__ float block_max(float v, float *buf) {
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(buf[0], buf[1]), fmaxf(buf[2], buf[3]));
}
__device__ __forceinline__ int block_min(int v, int *buf) {
    for (int o = 32; o; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    return min(min(buf[0], buf[1]), min(buf[2], buf[3]));
}
struct BlockBuf { double d[4]; float f[4]; int i[4]; };
// the numbers of the threads that `have`, in order; how many
__device__ __forceinline__ uint32_t listed(bool have, unsigned char *list, uint32_t (&cnt)[4]) {
    const uint64_t all = __ballot(have);
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) cnt[wave] = __popcll(all);
    __syncthreads();
    uint32_t at = __popcll(all & ((1ull << lane) - 1)), n = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) { at += i < wave ? cnt[i] : 0u; n += cnt[i]; }
    if (have) list[at] = (unsigned char)threadIdx.x;
    __syncthreads();
    return n;
}

// One chunk [lo, hi) of a row (see RowPart).
// A thread takes eight at a time with the next eight on their way, and keeps a running maximum and sum.
// The sum is relative to the first maximum a thread meets: 64 bits hold 2^800 times as much beside it, and only a larger value
// moves it (`slack`: how far a logit may lie above it).
__device__ __forceinline__ double sum8(const double (&r)[8]) { return ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7])); }
struct Running { float m; double z; int best; };
template <typename T>
__device__ __forceinline__ void take8(Running &r, Oct<T> &o, uint32_t i, double k, float slack, bool greedy) {
    float v[8], mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        o.take(v[e], v[e + 1]);
        mx = fmaxf(mx, fmaxf(v[e], v[e + 1]));
    }
    if (mx > r.m + slack) {
        r.z = r.m == -INFINITY ? 0.0 : r.z * weight(r.m, mx, k);
        r.m = mx;
        if (greedy)
#pragma unroll
            for (int e = 7; e >= 0; --e) r.best = v[e] == mx ? (int)(i + e) : r.best;
    }
    if (greedy) return;
    const float m = fmaxf(r.m, -kFloatMax);           // (-inf alone so far: weights of zero)
    double w[8];
    weights(v, m, k, w);
    r.z += sum8(w);
}
template <typename T>
__device__ __forceinline__ RowPart chunk_part(const T *x, uint32_t lo, uint32_t hi, double k, bool greedy, BlockBuf &b) {
    Running r{-INFINITY, 0.0, 0x7FFFFFFF};
    const float slack = greedy ? 0.f : (float)fmin(800.0 / k, 1e38);
    const uint32_t step = kVerThreads * 8;
    uint32_t i = lo + threadIdx.x * 8;
    if (i + 8 <= hi) {
        Oct<T> next;
        next.fill(x, i);
        bool more;
#pragma unroll 1
        do {
            Oct<T> o = next;
            more = i + step + 8 <= hi;
            next.fill(x, more ? i + step : i);       // (no branch around a load: behind one the next wait is for everything)
            take8(r, o, i, k, slack, greedy);
            i += step;
        } while (more);
    }
    if (i < hi) {
        Oct<T> o;
        o.fill(x, i, hi);
        take8(r, o, i, k, slack, greedy);
    }
    RowPart p{0.0, block_max(r.m, b.f), 0x7FFFFFFF};
    if (p.m == -INFINITY) return p;
    if (greedy) p.best = block_min(r.m == p.m ? r.best : 0x7FFFFFFF, b.i);
    else p.z = block_sum(r.m == -INFINITY ? 0.0 : r.z * weight(r.m, p.m, k), b.d);
    return p;
}

struct RowSum { double z; float m; int best; };
// the parts of a row put together by `g` lanes (a power of two) with one each; every lane of them gets the sum
__device__ __forceinline__ RowSum row_sum(const RowPart &mine, uint32_t g, double k, bool greedy) {
    RowSum r{0.0, mine.m, 0x7FFFFFFF};
    for (int o = g / 2; o; o >>= 1) r.m = fmaxf(r.m, __shfl_xor(r.m, o, 64));
    if (greedy) {
        r.best = mine.m == r.m && r.m != -INFINITY ? mine.best : 0x7FFFFFFF;
        for (int o = g / 2; o; o >>= 1) r.best = min(r.best, __shfl_xor(r.best, o, 64));
        return r;
    }
    r.z = mine.m == -INFINITY ? 0.0 : mine.z * weight(mine.m, r.m, k);
    for (int o = g / 2; o; o >>= 1) r.z += __shfl_xor(r.z, o, 64);
    return r;
}
__device__ __forceinline__ uint32_t lanes_for(uint32_t n) { return n <= 1 ? 1u : 1u << (32 - __clz(n - 1)); }

template <typename T>
__global__ __launch_bounds__(kVerThreads) void verify_rows_kernel(ps_verify_tree_args a, VerifyShape sh, VerifyWork w) {
    __shared__ BlockBuf b;
    __shared__ unsigned char parent[PS_TREE_MAX], list[PS_TREE_MAX];
    __shared__ uint32_t cnt[4];
    const uint32_t tid = threadIdx.x, s = blockIdx.z, chunk = blockIdx.x;
    const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
    if (sr.n < 2) return;
    const float temp = a.temperature ? a.temperature[s] : 1.f;
    const bool greedy = !(temp > 0.f);
    const double k = greedy ? 0.0 : rate_of(temp);
    parent[tid] = 0;
    __syncthreads();
    if ((int)tid < sr.n) {
        const int up = parent_of(a.parent[sr.row0 + tid], tid);
        if (up >= 0) parent[up] = 1;
    }
    __syncthreads();
    const uint32_t count = listed(parent[tid] != 0, list, cnt);
    const uint32_t lo = chunk * sh.chunk, hi = min(a.vocab, lo + sh.chunk);
    const uint32_t both = a.draft_logits && !greedy ? 2 : 1;       // target and draft rows are tasks of their own
    for (uint32_t j = blockIdx.y; j < count * both; j += gridDim.y) {
        const size_t row = (size_t)sr.row0 + list[j / both];
        const bool which = j % both;
        const T *x = which ? static_cast<const T *>(a.draft_logits) + row * a.draft_row : static_cast<const T *>(a.target_logits) + row * a.target_row;
        const RowPart p = chunk_part(x, lo, hi, k, greedy, b);
        if (tid == 0) w.parts[(row * 2 + which) * sh.nchunk + chunk] = p;
    }
}

// Decisions of a sequence's nodes, as far as they are known: by one thread for each node
struct Walk {
    RowSum p[PS_TREE_MAX], q[PS_TREE_MAX];     // of nodes with children
    double px[PS_TREE_MAX], left[PS_TREE_MAX]; // of a node as its parent's child: p(token), W (or what is left without the refused)
    double c[PS_TREE_MAX];                     // c in front of this child
    int up[PS_TREE_MAX], rank[PS_TREE_MAX], token[PS_TREE_MAX], went[PS_TREE_MAX], kids[PS_TREE_MAX];
    bool dup[PS_TREE_MAX];
    unsigned char list[PS_TREE_MAX];
    uint32_t cnt[4];
};

// known: children up to this rank are decided (their W has been summed)
template <typename T>
__device__ __forceinline__ void decide(const ps_verify_tree_args &a, const VerifyShape &sh, const VerifyWork &w, const SeqRows &sr, float temp, uint32_t known, Walk &k) {
    const int tid = threadIdx.x;
    const bool greedy = !(temp > 0.f), drafts = a.draft_logits && !greedy, in = tid < sr.n;
    const double rate = greedy ? 0.0 : rate_of(temp);
    k.kids[tid] = 0;
    k.went[tid] = 0x7FFFFFFF;
    k.left[tid] = 1.0;
    int up = -1, token = -1;
    float u = 0.f, x = -INFINITY, y = -INFINITY;
    const size_t row = (size_t)sr.row0 + tid;
    if (in) { up = parent_of(a.parent[row], tid); token = a.token[row]; u = a.u_accept[row]; }
    const bool inside = up >= 0 && token >= 0 && token < (int)a.vocab;
    if (inside) {       // (on their way while the rows are put together)
        x = to_f(static_cast<const T *>(a.target_logits)[((size_t)sr.row0 + up) * a.target_row + token]);
        if (drafts) y = to_f(static_cast<const T *>(a.draft_logits)[((size_t)sr.row0 + up) * a.draft_row + token]);
    }
    k.up[tid] = up;
    k.token[tid] = token;
    __syncthreads();
    if (up >= 0) atomicAdd(&k.kids[up], 1);
    int rank = 0;
    bool dup = false;
    if (up >= 0) {
#pragma unroll 4
        for (int j = 1; j < tid; ++j) {
            const bool same = k.up[j] == up;
            rank += same;
            dup |= same && k.token[j] == token;
        }
    }
    k.rank[tid] = rank;
    k.dup[tid] = dup;
    __syncthreads();
    // a few lanes to a row: the rows with children, target and draft; then the W of children behind a node's first
    const uint32_t rows = listed(k.kids[tid] > 0, k.list, k.cnt) * (drafts ? 2 : 1), g = lanes_for(sh.nchunk);
    for (uint32_t j0 = 0; j0 < rows; j0 += kVerThreads / g) {
        const uint32_t j = j0 + tid / g, part = tid % g;
        const int i = j < rows ? k.list[drafts ? j >> 1 : j] : 0;
        const bool which = drafts && (j & 1);
        RowPart mine{0.0, -INFINITY, 0x7FFFFFFF};
        if (j < rows && part < sh.nchunk) mine = w.parts[(((size_t)sr.row0 + i) * 2 + which) * sh.nchunk + part];
        const RowSum r = row_sum(mine, g, rate, greedy);
        if (j < rows && part == 0) (which ? k.q : k.p)[i] = r;
    }
    if (drafts && known) {
        __syncthreads();
        const uint32_t later = listed(up >= 0 && rank > 0 && rank <= (int)known && rank < (int)a.max_children, k.list, k.cnt);
        for (uint32_t j = tid >> 5; j < later; j += kVerThreads / 32) {
            const int i = k.list[j];
            double sum = (tid & 31) < (int)sh.ndraw ? w.left[((size_t)sr.row0 + i) * sh.ndraw + (tid & 31)] : 0.0;
            for (int o = 16; o; o >>= 1) sum += __shfl_xor(sum, o, 32);
            if ((tid & 31) == 0) k.left[i] = sum;
        }
    }
    __syncthreads();
    double px = 0, qx = 0;
    if (inside) {
        if (greedy) px = token == k.p[up].best ? 1.0 : 0.0;
        else if (k.p[up].m != -INFINITY) px = weight(sane(x), k.p[up].m, rate) / k.p[up].z;
        if (drafts && k.q[up].m != -INFINITY) qx = weight(sane(y), k.q[up].m, rate) / k.q[up].z;
    }
    k.px[tid] = px;
    __syncthreads();
    if (up >= 0) {
        double c = 0, rest = 1.0;
        if (drafts) {
#pragma unroll 4
            for (int j = 1; j < tid; ++j) c += k.up[j] == up ? k.left[j] : 0.0;
        } else if (!greedy) {
#pragma unroll 4
            for (int j = 1; j < tid; ++j) rest -= k.up[j] == up && !k.dup[j] ? k.px[j] : 0.0;
        }
        k.c[tid] = c;
        const bool yes = drafts ? px > (c + (double)u * k.left[tid]) * qx : (greedy || !dup) && px > (double)u * rest;
        if (yes && rank < (int)a.max_children && (!drafts || rank <= (int)known)) atomicMin(&k.went[up], tid);
    }
    __syncthreads();
}

// Eight entries i .. i + 7 of what is left to draw from: max(p - c q, 0), p without the refused, or p, times ip
template <typename T>
__device__ __forceinline__ void left8(const ps_verify_tree_args &a, const DrawHead &h, int kind, double rate, uint32_t i, uint32_t hi, const int *refused, int nref,
                                      double (&r)[8]) {
    Oct<T> p, q;
    p.fill(static_cast<const T *>(a.target_logits) + (size_t)h.row * a.target_row, i, hi);
    if (kind == DRAW_LEFT) q.fill(static_cast<const T *>(a.draft_logits) + (size_t)h.row * a.draft_row, i, hi);
    const float m = fmaxf(h.m, -kFloatMax), mq = fmaxf(h.mq, -kFloatMax);       // (rows of -inf alone: weights of zero)
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) p.take(x[e], x[e + 1]);
    weights(x, m, rate, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] *= h.ip;
    if (kind == DRAW_LEFT) {
        double w[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) q.take(x[e], x[e + 1]);
        weights(x, mq, rate, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = fmax(r[e] - w[e] * h.iq, 0.0);
    }
    if (kind == DRAW_GIVEN)
        for (int j = 0; j < nref; ++j) {
            const uint32_t at = (uint32_t)refused[j] - i;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) r[e] = at == e ? 0.0 : r[e];
        }
}
template <typename T>
__global__ __launch_bounds__(kVerThreads) void verify_left_kernel(ps_verify_tree_args a, VerifyShape sh, VerifyWork w, uint32_t k) {
    __shared__ Walk walk;
    __shared__ BlockBuf b;
    __shared__ int list[PS_TREE_MAX], n;
    const uint32_t s = blockIdx.y, chunk = blockIdx.x;
    const int tid = threadIdx.x;
    const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
    const float temp = a.temperature ? a.temperature[s] : 1.f;
    if (sr.n < 2 || !(temp > 0.f)) return;
    decide<T>(a, sh, w, sr, temp, k - 1, walk);
    if (tid == 0) n = 0;
    __syncthreads();
    // a child of rank k whose parent has accepted none before it, where no edge above is known to be refused
    bool ok = tid < sr.n && walk.up[tid] >= 0 && walk.rank[tid] == (int)k && walk.went[walk.up[tid]] == 0x7FFFFFFF;
    if (ok) {
        int i = walk.up[tid];
        for (; i > 0; i = walk.up[i]) {
            const int up = walk.up[i];
            if (up < 0 || (walk.went[up] != i && (walk.went[up] != 0x7FFFFFFF || walk.rank[i] < (int)k))) break;
        }
        ok = i == 0;
    }
    if (ok) list[atomicAdd(&n, 1)] = tid;      // (any order: each is worked on alone)
    __syncthreads();
    const double rate = rate_of(temp);
    const uint32_t lo = chunk * sh.dchunk, hi = min(a.vocab, lo + sh.dchunk);
    for (int j = 0; j < n; ++j) {
        const int child = list[j], up = walk.up[child];
        const size_t row = (size_t)sr.row0 + up;
        const RowSum p = walk.p[up], q = walk.q[up];
        // the child's c holds W of those in front of it, all known
        const double c = walk.c[child], ip = p.m == -INFINITY ? 0.0 : 1.0 / p.z, iq = q.m == -INFINITY ? 0.0 : c / q.z;
        DrawHead h{};
        h.row = row;
        h.m = p.m; h.mq = q.m; h.ip = ip; h.iq = iq;
        double sum = 0;
#pragma unroll 1
        for (uint32_t i = lo + tid * 8; i < hi; i += kVerThreads * 8) {
            double r[8];
            left8<T>(a, h, DRAW_LEFT, rate, i, hi, nullptr, 0, r);
            sum += sum8(r);
        }
        sum = block_sum(sum, b.d);
        if (tid == 0) w.left[((size_t)sr.row0 + child) * sh.ndraw + chunk] = sum;
    }
}

template <typename T>
__global__ __launch_bounds__(kVerThreads) __attribute__((amdgpu_waves_per_eu(1, 4))) void verify_draw_kernel(ps_verify_tree_args a, VerifyShape sh, VerifyWork w) {
    __shared__ Walk walk;
    __shared__ BlockBuf b;
    __shared__ int path[PS_TREE_MAX], refused[PS_TREE_MAX], n, nref, all, last;
    const uint32_t s = blockIdx.y, chunk = blockIdx.x;
    const int tid = threadIdx.x;
    const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
    if (sr.n == 0) {
        if (chunk) return;
        if (tid < (int)a.max_tree) a.path[s * a.path_seq + tid] = -1;
        if (tid == 0) { a.count[s] = 0; w.heads[s].kind = DRAW_NONE; }
        return;
    }
    const float temp = a.temperature ? a.temperature[s] : 1.f;
    const bool greedy = !(temp > 0.f), drafts = a.draft_logits && !greedy;
    const double rate = greedy ? 0.0 : rate_of(temp);
    const uint32_t lo = chunk * sh.dchunk, hi = min(a.vocab, lo + sh.dchunk);
    int kids = 0;
    if (sr.n > 1) {
        decide<T>(a, sh, w, sr, temp, a.max_children, walk);
        if (tid == 0) {
            int here = 0, m = 0;
            for (;;) {
                path[m++] = here;
                const int next = walk.went[here];
                if (next == 0x7FFFFFFF) break;
                here = next;
            }
            n = m;
            last = here;
            nref = all = 0;
        }
        __syncthreads();
        kids = walk.kids[last];
    } else {
        if (tid == 0) { path[0] = 0; n = 1; last = 0; nref = all = 0; }
        __syncthreads();
    }
    DrawHead h{};
    h.row = sr.row0 + last;
    h.m = h.mq = -INFINITY;
    if (kids) {
        const RowSum p = walk.p[last];
        h.m = p.m;
        h.kind = p.m == -INFINITY ? DRAW_NONE : greedy ? DRAW_BEST : drafts ? DRAW_LEFT : DRAW_GIVEN;
        h.ip = h.kind >= DRAW_LEAF ? 1.0 / p.z : 0.0;
        if (drafts) {      // c behind the last child tried
            const bool tried = tid < sr.n && walk.up[tid] == last && walk.rank[tid] < (int)a.max_children;
            h.c = block_sum(tried ? walk.left[tid] : 0.0, b.d);
            h.mq = walk.q[last].m;
            h.iq = h.mq == -INFINITY ? 0.0 : h.c / walk.q[last].z;
        } else if (tid < sr.n && walk.up[tid] == last && walk.rank[tid] < (int)a.max_children && !walk.dup[tid]) {
            const int x = walk.token[tid];
            if (chunk == 0) w.refused[s * a.max_tree + atomicAdd(&all, 1)] = x;
            if (x >= (int)lo && x < (int)hi) refused[atomicAdd(&nref, 1)] = x;       // (those of this chunk)
        }
        __syncthreads();
        h.nref = all;
    } else {
        h.kind = DRAW_LEAF;
    }
    if (chunk == 0) {
        if (tid < (int)a.max_tree) a.path[s * a.path_seq + tid] = tid < n ? path[tid] : -1;
        if (tid == 0) {
            a.count[s] = n;
            w.heads[s] = h;
            if (h.kind == DRAW_BEST) w.recs[s * sh.ndraw].best = walk.p[last].best;
        }
    }
    if (h.kind < DRAW_LEAF) return;
    RowPart r{0.0, h.m, 0};
    if (h.kind == DRAW_LEAF) {
        r = chunk_part(static_cast<const T *>(a.target_logits) + (size_t)h.row * a.target_row, lo, hi, rate, greedy, b);
    } else {
        double sum = 0;
#pragma unroll 1
        for (uint32_t i = lo + tid * 8; i < hi; i += kVerThreads * 8) {
            double v[8];
            left8<T>(a, h, h.kind, rate, i, hi, refused, nref, v);
            sum += sum8(v);
        }
        r.z = block_sum(sum, b.d);
    }
    if (tid == 0) w.recs[s * sh.ndraw + chunk] = r;
}

template <typename T>
__global__ __launch_bounds__(kPickThreads) __attribute__((amdgpu_waves_per_eu(1, 2))) void verify_pick_kernel(ps_verify_tree_args a, VerifyShape sh, VerifyWork w) {
    __shared__ double runs[kPickThreads / 64];
    __shared__ int refused[PS_TREE_MAX], pick[2];
    const uint32_t s = blockIdx.x;
    const int tid = threadIdx.x, half = tid & 31;
    DrawHead h = w.heads[s];
    const RowPart *recs = w.recs + s * sh.ndraw;
    RowPart mine = half < (int)sh.ndraw ? recs[half] : RowPart{0.0, -INFINITY, 0x7FFFFFFF};     // every half wave holds them all
    const int mine_refused = tid < (int)a.max_tree ? w.refused[s * a.max_tree + tid] : -1;       // (those that there are: see the head)
    if (h.kind <= DRAW_BEST) {
        if (tid == 0) a.next_token[s] = h.kind == DRAW_BEST ? mine.best : -1;
        return;
    }
    const float temp = a.temperature ? a.temperature[s] : 1.f, u = a.u_sample[s];
    const bool greedy = !(temp > 0.f);
    const double rate = greedy ? 0.0 : rate_of(temp);
    if (tid < (int)PS_TREE_MAX) refused[tid] = tid < h.nref ? mine_refused : -1;
    __syncthreads();
    const int nref = h.nref;
    int kind = h.kind;
    uint32_t chunk_len = sh.dchunk;
    if (kind == DRAW_LEAF) {
        const RowSum r = row_sum(mine, 32, rate, greedy);
        if (r.m == -INFINITY || greedy) {
            if (tid == 0) a.next_token[s] = r.m == -INFINITY ? -1 : r.best;
            return;
        }
        h.m = r.m;
        h.ip = 1.0;
        mine.z = mine.m == -INFINITY ? 0.0 : mine.z * weight(mine.m, h.m, rate);
    }
    auto running = [&](double v) {           // over the chunks, in their order
        for (int o = 1; o < 32; o <<= 1) {
            const double t = __shfl_up(v, o, 32);
            if (half >= o) v += t;
        }
        return v;
    };
    double run = running(mine.z), total = __shfl(run, 31, 32);
    if (!(total > 0)) {      // nothing left: the target's own row, whose parts are chunks of their own
        kind = DRAW_LEAF;
        h.ip = 1.0;
        chunk_len = sh.chunk;
        mine = half < (int)sh.nchunk ? w.parts[(size_t)h.row * 2 * sh.nchunk + half] : RowPart{0.0, -INFINITY, 0x7FFFFFFF};
        mine.z = mine.m == -INFINITY ? 0.0 : mine.z * weight(mine.m, h.m, rate);
        run = running(mine.z);
        total = __shfl(run, 31, 32);
    }
    // the first chunk whose running sum passes the goal (or the last one that holds anything)
    const double goal = (double)u * total;
    const uint32_t passes = (uint32_t)__ballot(run > goal && mine.z > 0), some_left = (uint32_t)__ballot(mine.z > 0);
    const int chunk = passes ? __ffs(passes) - 1 : 31 - __clz(some_left);
    const double prior_run = __shfl_up(run, 1, 32);
    const double before = chunk ? __shfl(prior_run, chunk, 32) : 0.0;
    // in it, threads take vectors of 8 entries in turn, 4096 entries at a time
    const uint32_t lo = chunk * chunk_len, hi = min(a.vocab, lo + chunk_len);
    double base = before;
    int last_some = -1;
    for (uint32_t i0 = lo; i0 < hi; i0 += kPickThreads * 8) {
        const uint32_t i = i0 + tid * 8;
        double v[8], sum = 0;
        int some = -1;
        if (i < hi) {
            left8<T>(a, h, kind, rate, i, hi, refused, nref, v);
            sum = sum8(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) some = v[e] > 0 ? (int)(i + e) : some;
        }
        double upto = sum;
        for (int o = 1; o < 64; o <<= 1) {
            const double t = __shfl_up(upto, o, 64);
            if ((tid & 63) >= o) upto += t;
        }
        __syncthreads();
        if ((tid & 63) == 63) runs[tid >> 6] = upto;
        if (tid < 2) pick[tid] = tid ? -1 : 0x7FFFFFFF;
        __syncthreads();
        double from = base;
        for (int j = 0; j < tid >> 6; ++j) from += runs[j];
        const double to = from + upto, prior = __shfl_up(upto, 1, 64);
        if (tid & 63) from += prior;
        if (to > goal && sum > 0) atomicMin(&pick[0], tid);
        if (some >= 0) atomicMax(&pick[1], some);
        __syncthreads();
        if (pick[0] != 0x7FFFFFFF) {
            if (tid != pick[0]) return;
            int found = -1;
            double r = from;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                r += v[e];
                if (found < 0 && v[e] > 0 && r > goal) found = (int)(i + e);
            }
            a.next_token[s] = found >= 0 ? found : some;
            return;
        }
        last_some = max(last_some, pick[1]);
        for (uint32_t j = 0; j < kPickThreads / 64; ++j) base += runs[j];
    }
    if (tid == 0) a.next_token[s] = last_some;      // the goal lies within the last sum's rounding
}

// Chunks are multiples of 2048 entries, 4096 at least and at most kMaxChunks of a row.  Row passes: as few chunks as keep about 2048
// workgroups, counting half of the nodes (each workgroup takes several in turn where there are more): every chunk ends in two reductions, and its part is read by
// every workgroup that works out the walk.  What is drawn from is one row of each sequence: about 1024 workgroups.
VerifyShape verify_shape(const ps_verify_tree_args &a) {
    VerifyShape sh;
    auto cut = [&](uint64_t chunks, uint32_t *len, uint32_t *n) {
        chunks = std::max<uint64_t>(1, std::min<uint64_t>(chunks, kMaxChunks));
        *len = (uint32_t)((std::max<uint64_t>(4096, (a.vocab + chunks - 1) / chunks) + 2047) / 2048 * 2048);
        *n = (a.vocab + *len - 1) / *len;
    };
    const uint64_t seqs = std::max(1u, a.n_seq), both = a.draft_logits ? 2 : 1, nodes = std::max(1u, a.max_tree / 2) * both;
    cut((2048 + seqs * nodes - 1) / (seqs * nodes), &sh.chunk, &sh.nchunk);
    cut((1024 + seqs - 1) / seqs, &sh.dchunk, &sh.ndraw);
    sh.loop = (uint32_t)std::min<uint64_t>(std::max(1u, a.max_tree - 1) * both, std::max<uint64_t>(1, 4096 / (sh.nchunk * seqs)));
    return sh;
}
uint64_t verify_work(const ps_verify_tree_args &a, const VerifyShape &sh, uint8_t *base, VerifyWork *w) {
    uint64_t off = 0;
    auto take = [&](uint64_t bytes) { uint8_t *p = base ? base + off : nullptr; off = align_up(off + bytes, kAlign); return p; };
    w->parts = reinterpret_cast<RowPart *>(take((uint64_t)a.n_tokens * 2 * sh.nchunk * sizeof(RowPart)));
    w->left = reinterpret_cast<double *>(take(a.draft_logits ? (uint64_t)a.n_tokens * sh.ndraw * 8 : 0));
    w->recs = reinterpret_cast<RowPart *>(take((uint64_t)a.n_seq * sh.ndraw * sizeof(RowPart)));
    w->heads = reinterpret_cast<DrawHead *>(take((uint64_t)a.n_seq * sizeof(DrawHead)));
    w->refused = reinterpret_cast<int *>(take((uint64_t)a.n_seq * a.max_tree * 4));
    return off;
}

template <typename T>
hipError_t launch_verify(const ps_verify_tree_args &a, const VerifyShape &sh, const VerifyWork &w, hipStream_t st) {
    if (a.n_tokens && a.max_tree > 1) {
        hipLaunchKernelGGL(verify_rows_kernel<T>, dim3(sh.nchunk, sh.loop, a.n_seq), dim3(kVerThreads), 0, st, a, sh, w);
        if (a.draft_logits)
            for (uint32_t k = 1; k < std::min(a.max_children, a.max_tree - 1); ++k)
                hipLaunchKernelGGL(verify_left_kernel<T>, dim3(sh.ndraw, a.n_seq), dim3(kVerThreads), 0, st, a, sh, w, k);
    }
    hipLaunchKernelGGL(verify_draw_kernel<T>, dim3(sh.ndraw, a.n_seq), dim3(kVerThreads), 0, st, a, sh, w);
    hipLaunchKernelGGL(verify_pick_kernel<T>, dim3(a.n_seq), dim3(kPickThreads), 0, st, a, sh, w);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ kept rows
// A wave per plane of a sequence, run of columns by run: kKeep pieces of 16 bytes a lane hold all rows of a run, and are all read before
// one is written, so rows may move onto rows that others are read from.  Rows that stay where they are are not touched.  Bound by the
// chain count, path, row, store of few waves: so two pieces a lane (46 registers, eight waves a SIMD; 48 sequences of 256 planes 9.5 us), and
// four (98, four waves; 13.3 us) only for paths that may be longer than 128.
struct BatchPlanes {
    __device__ __forceinline__ char *operator()(const ps_cache_keep_args &a, uint32_t s, uint32_t plane) const {
        return static_cast<char *>(a.cache) + s * a.seq_stride + plane * a.plane_stride;
    }
    __device__ __forceinline__ int64_t context(const ps_cache_keep_args &a, uint32_t s) const { return a.context[s]; }
};
struct StackPlanes {       // home[plane / 2]: K rows, then V rows
    const uint64_t *home;
    uint32_t ctx;
    __device__ __forceinline__ char *operator()(const ps_cache_keep_args &a, uint32_t, uint32_t plane) const {
        return reinterpret_cast<char *>(home[plane / 2]) + (plane & 1 ? (uint64_t)a.capacity * a.row_stride : 0);
    }
    __device__ __forceinline__ int64_t context(const ps_cache_keep_args &, uint32_t) const { return ctx; }
};
template <class S, uint32_t kKeep>
__global__ __launch_bounds__(256) void cache_keep_kernel(ps_cache_keep_args a, S where) {
    const uint32_t lane = threadIdx.x & 63, plane = blockIdx.x * 4 + (threadIdx.x >> 6), s = blockIdx.y;
    if (plane >= a.n_planes) return;
    const int n = clampi(a.count[s], 0, (int)a.max_tree);
    const int64_t ctx = where.context(a, s);
    const int32_t *path = a.path + s * a.path_seq;
    char *base = where(a, s, plane);
    const uint32_t units = a.row_bytes / 16;
    // columns of a run: as many (a power of two) as leave room for all rows
    const uint32_t shift = 31 - __clz(64 * kKeep / (uint32_t)max(n, 1)), seg = 1u << shift;
    if (n == 0) return;
    for (uint32_t c0 = 0; c0 < units; c0 += seg) {
        u4_t v[kKeep];
        bool ok[kKeep];
#pragma unroll
        for (uint32_t u = 0; u < kKeep; ++u) {
            const uint32_t idx = u * 64 + lane, i = idx >> shift, col = c0 + (idx & (seg - 1));
            const int node = (int)i < n && col < units ? path[i] : -1;
            const int64_t from = ctx + node, to = ctx + i;
            ok[u] = node >= 0 && node < (int)a.max_tree && node != (int)i && from >= 0 && from < a.capacity && to >= 0 && to < a.capacity;
            if (ok[u]) v[u] = *reinterpret_cast<const u4_t *>(base + from * a.row_stride + col * 16);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (uint32_t u = 0; u < kKeep; ++u) {
            const uint32_t idx = u * 64 + lane, i = idx >> shift, col = c0 + (idx & (seg - 1));
            if (ok[u]) *reinterpret_cast<u4_t *>(base + (ctx + i) * a.row_stride + col * 16) = v[u];
        }
    }
}

template <class S>
hipError_t launch_keep(const ps_cache_keep_args &a, const S &where, hipStream_t st) {
    const dim3 grid((a.n_planes + 3) / 4, a.n_seq);
    static_assert(64 * 4 >= PS_TREE_MAX, "a run of one column holds every row of a path");
    if (a.max_tree <= 128) hipLaunchKernelGGL((cache_keep_kernel<S, 2>), grid, dim3(256), 0, st, a, where);
    else hipLaunchKernelGGL((cache_keep_kernel<S, 4>), grid, dim3(256), 0, st, a, where);
    return hipGetLastError();
}

__global__ __launch_bounds__(PS_TREE_MAX) void tree_tables_kernel(int32_t *first, int32_t *parent, StackTreeNodes tree, uint32_t n) {
    const uint32_t t = threadIdx.x;
    if (t < 2) first[t] = t ? (int32_t)n : 0;
    if (t < n) parent[t] = tree.n ? (int32_t)byte_of(tree.up, t) - 1 : (int32_t)t - 1;
}

int32_t check_tree(const ps_tree_attention_args *a) {
    PS_WANT(a, "NULL argument");
    PS_WANT(a->type <= PS_TYPE_BF16, "tree attention takes fp16 or bf16 (type %u)", a->type);
    PS_WANT(a->head_dim == 64 || a->head_dim == 128, "tree attention takes head_dim 64 or 128 (got %u)", a->head_dim);
    PS_WANT(a->n_kv_heads && a->n_q_heads && a->n_q_heads % a->n_kv_heads == 0 && a->n_q_heads <= 1024,
            "%u query heads over %u kv heads: a multiple of the kv heads, at most 1024", a->n_q_heads, a->n_kv_heads);
    PS_WANT(a->max_tree <= PS_TREE_MAX, "trees of up to %u tokens (got %u)", PS_TREE_MAX, a->max_tree);
    PS_WANT(a->n_seq <= 65535 && a->n_tokens <= 0x7FFFFFFF, "%u sequences, %u tokens: too many", a->n_seq, a->n_tokens);
    PS_WANT(a->max_context <= a->capacity && a->capacity <= 0x7FFFFFFF, "a context of up to %u in a cache of %u positions", a->max_context, a->capacity);
    PS_WANT(!a->append || (uint64_t)a->max_context + a->max_tree <= a->capacity,
            "a context of up to %u and %u new tokens leave no room in a cache of %u positions", a->max_context, a->max_tree, a->capacity);
    return PS_OK;
}

}  // namespace

bool make_tree_nodes(const int32_t *parent, uint32_t n, StackTreeNodes *out) {
    *out = StackTreeNodes{};
    uint8_t *up = reinterpret_cast<uint8_t *>(out->up.w), *depth = reinterpret_cast<uint8_t *>(out->depth.w);
    for (uint32_t i = 0; i < n; ++i) {
        if (parent[i] < -1 || parent[i] >= (int32_t)i) { set_error("node %u cannot follow node %d: a parent comes before its children", i, parent[i]); return false; }
        up[i] = (uint8_t)(parent[i] + 1);
        depth[i] = parent[i] < 0 ? 0 : (uint8_t)(depth[parent[i]] + 1);
    }
    out->n = n;
    return true;
}

hipError_t launch_stack_rotation(const StackRotation &r, uint32_t layer, __half *qkv, uint32_t qkv_w, uint32_t n_q, uint32_t n_kv, uint32_t n_tokens,
                                 uint32_t ctx, const uint32_t *ctx_dev, const StackTreeNodes &tree, hipStream_t st) {
    if (n_tokens == 0) return hipSuccess;
    if (r.rot_dim % 16 || r.rot_dim > 128 || (tree.n && n_tokens > tree.n)) return hipErrorInvalidValue;
    ps_qk_norm_rope_args a{};
    a.type = PS_TYPE_F16; a.n_tokens = n_tokens; a.n_q_heads = n_q; a.n_k_heads = n_kv; a.head_dim = 128; a.rot_dim = r.rot_dim;
    a.pairs = r.pairs; a.norm = r.norm; a.eps = r.eps;
    a.q = a.q_out = qkv;
    a.k = a.k_out = qkv + (size_t)n_q * 128;
    a.q_token = a.k_token = a.q_out_token = a.k_out_token = qkv_w;
    a.q_head = a.k_head = a.q_out_head = a.k_out_head = 128;
    a.q_gain = r.q_gain ? r.q_gain + (size_t)layer * 128 : nullptr;
    a.k_gain = r.k_gain ? r.k_gain + (size_t)layer * 128 : nullptr;
    a.inv_freq = r.inv_freq;
    return launch_rope_wide<f16_t>(a, StackPositions{ctx_dev, ctx, tree.n, tree.depth}, st);
}

static ps_tree_attention_args stack_tree_call(const StackTreeArgs &s, uint32_t n_tokens, uint32_t nheads) {
    ps_tree_attention_args a{};
    const uint32_t G = s.n_q / s.n_kv;
    a.type = PS_TYPE_F16; a.n_seq = 1; a.n_tokens = a.max_tree = n_tokens; a.n_kv_heads = nheads; a.n_q_heads = nheads * G; a.head_dim = 128;
    a.max_context = s.ctx; a.capacity = s.cap; a.append = s.home ? 1 : 0; a.scale = 0.08838834764831845f;
    const uint32_t head0 = nheads == s.n_kv ? 0 : s.head0;
    a.q = s.qkv + (size_t)head0 * G * 128;
    a.k_new = s.qkv + (size_t)(s.n_q + head0) * 128;
    a.v_new = s.qkv + (size_t)(s.n_q + s.n_kv + head0) * 128;
    a.q_token = a.k_new_token = a.v_new_token = s.qkv_w;
    a.q_head = a.k_new_head = a.v_new_head = 128;
    a.k_cache = const_cast<__half *>(s.k_base);
    a.v_cache = const_cast<__half *>(s.k_base + (size_t)s.cap * 128);
    a.k_head = a.v_head = s.head_stride / 2;
    a.k_row = a.v_row = 128;
    a.out = s.out + (size_t)head0 * G * 128;
    a.out_token = (uint64_t)s.n_q * 128;
    a.out_head = 128;
    return a;
}
// (part_bytes: the plan's room for records.  Plans of kAttnOnePassTokens tokens and more have none, and their trees no splits)
uint32_t stack_tree_splits(uint32_t n_q, uint32_t n_kv, uint32_t ctx, uint32_t n_tokens, uint64_t part_bytes) {
    ps_tree_attention_args a{};
    a.n_seq = 1; a.max_tree = n_tokens; a.n_q_heads = n_q; a.n_kv_heads = n_kv; a.max_context = ctx;
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(tree_deal(a).nsplit, part_bytes / ((uint64_t)n_tokens * n_q * (128 + 4) * 4)));
}
static TreeDeal stack_deal(const StackTreeArgs &s, uint32_t n_tokens) {
    ps_tree_attention_args a{};
    a.n_seq = 1; a.max_tree = n_tokens; a.n_q_heads = s.n_q; a.n_kv_heads = s.n_kv; a.max_context = s.ctx;
    TreeDeal d = tree_deal(a);
    d.nsplit = s.splits;
    return d;
}
hipError_t launch_stack_tree(const StackTreeArgs &s, const StackTreeNodes &tree, hipStream_t st) {
    if (s.nheads == 0 || tree.n == 0) return hipSuccess;
    if (s.splits == 0 || tree.n > PS_TREE_MAX || (s.home ? (uint64_t)s.ctx + tree.n > s.cap : s.ctx > s.cap)) return hipErrorInvalidValue;
    const StackTree where{s.home ? s.home + s.head0 : nullptr, s.cap, s.n_q, s.head0 * (s.n_q / s.n_kv), tree.up};
    ps_tree_attention_args a = stack_tree_call(s, tree.n, s.nheads);
    return launch_tree<f16_t, 128>(a, where, stack_deal(s, tree.n), s.part, st);
}
hipError_t launch_stack_tree_merge(const StackTreeArgs &s, uint32_t n_tokens, hipStream_t st) {
    return launch_merge<f16_t, 128>(stack_tree_call(s, n_tokens, s.n_kv), StackTree{nullptr, s.cap, s.n_q, 0, {}}, stack_deal(s, n_tokens), s.part, st);
}
hipError_t launch_tree_tables(int32_t *first, int32_t *parent, uint32_t n, const StackTreeNodes &tree, hipStream_t st) {
    if (n > PS_TREE_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(tree_tables_kernel, dim3(1), dim3(PS_TREE_MAX), 0, st, first, parent, tree, n);
    return hipGetLastError();
}
hipError_t launch_stack_keep(const uint64_t *home, uint32_t n_homes, uint32_t cap, uint32_t ctx, uint32_t width, const int32_t *path, const int32_t *count,
                             hipStream_t st) {
    ps_cache_keep_args a{};
    a.n_seq = 1; a.n_planes = 2 * n_homes; a.capacity = cap; a.row_bytes = 256; a.max_tree = width; a.row_stride = 256;
    a.path = path; a.count = count;
    return launch_keep(a, StackPlanes{home, ctx}, st);
}
}  // namespace ps

using namespace ps;

extern "C" {

int32_t ps_qk_norm_rope(const ps_qk_norm_rope_args *a, void *stream) {
    PS_WANT(a, "NULL argument");
    PS_WANT(a->type <= PS_TYPE_F32, "unknown type %u", a->type);
    PS_WANT(a->head_dim >= 1 && a->head_dim <= 512, "head_dim 1 .. 512 (got %u)", a->head_dim);
    PS_WANT(a->rot_dim % 2 == 0 && a->rot_dim <= a->head_dim, "rot_dim must be even and at most head_dim (got %u of %u)", a->rot_dim, a->head_dim);
    PS_WANT(a->pairs <= 1 && a->norm <= 1, "pairs and norm are 0 or 1");
    PS_WANT(!a->norm || (a->eps >= 0.f && std::isfinite(a->eps)), "eps must be finite and not negative");
    PS_WANT(a->n_tokens <= 0x7FFFFFFF && a->n_q_heads <= 65535 && a->n_k_heads <= 65535, "too many tokens or heads");
    const uint64_t items = (uint64_t)a->n_tokens * (a->n_q_heads + a->n_k_heads);
    if (items == 0) return PS_OK;
    PS_WANT(items <= 0x7FFFFFFFull, "%llu heads of tokens are too many for one call", (unsigned long long)items);
    const uint32_t e = type_bytes(a->type);
    if (a->n_q_heads) {
        PS_WANT(a->q && a->q_out, "q or q_out is NULL");
        PS_WANT(aligned(a->q, e) && aligned(a->q_out, e) && aligned(a->q_gain, e), "q, q_out and q_gain must be aligned to an element");
        PS_WANT(a->q != a->q_out || (a->q_token == a->q_out_token && a->q_head == a->q_out_head), "in place: q and q_out must have the same strides");
    }
    if (a->n_k_heads) {
        PS_WANT(a->k && a->k_out, "k or k_out is NULL");
        PS_WANT(aligned(a->k, e) && aligned(a->k_out, e) && aligned(a->k_gain, e), "k, k_out and k_gain must be aligned to an element");
        PS_WANT(a->k != a->k_out || (a->k_token == a->k_out_token && a->k_head == a->k_out_head), "in place: k and k_out must have the same strides");
    }
    PS_WANT(!a->rot_dim || (a->positions && a->inv_freq && aligned(a->positions, 4) && aligned(a->inv_freq, 4)), "positions or inv_freq is NULL or unaligned");
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->type == PS_TYPE_F16) PS_TRY(launch_rope<f16_t>(*a, st));
    else if (a->type == PS_TYPE_BF16) PS_TRY(launch_rope<bf16_t>(*a, st));
    else PS_TRY(launch_rope<float>(*a, st));
    return PS_OK;
}

int32_t ps_tree_attention_workspace(const ps_tree_attention_args *a, uint64_t *bytes) {
    PS_WANT(bytes, "NULL argument");
    const int32_t rc = check_tree(a);
    if (rc) return rc;
    const TreeDeal d = tree_deal(*a);
    *bytes = d.nsplit > 1 ? align_up((uint64_t)a->n_tokens * a->n_q_heads * d.nsplit * (a->head_dim + 4) * 4, kAlign) : 0;
    return PS_OK;
}

int32_t ps_tree_attention(const ps_tree_attention_args *a, void *workspace, uint64_t workspace_bytes, void *stream) {
    uint64_t need = 0;
    const int32_t rc = ps_tree_attention_workspace(a, &need);
    if (rc) return rc;
    if (a->n_seq == 0 || a->n_tokens == 0 || a->max_tree == 0) return PS_OK;
    PS_WANT(a->q && a->k_new && a->v_new && a->out && a->first && a->context && a->parent, "NULL argument");
    PS_WANT((a->k_cache && a->v_cache) || (a->max_context == 0 && !a->append), "the cache is NULL");
    PS_WANT(std::isfinite(a->scale), "scale must be finite");
    for (const void *p : {a->q, a->k_new, a->v_new, (const void *)a->k_cache, (const void *)a->v_cache, (const void *)a->out})
        PS_WANT(aligned(p, 16), "q, k_new, v_new, the cache and out must be 16-byte aligned");
    for (uint64_t n : {a->q_token, a->q_head, a->k_new_token, a->k_new_head, a->v_new_token, a->v_new_head, a->k_seq, a->k_head, a->k_row,
                       a->v_seq, a->v_head, a->v_row, a->out_token, a->out_head})
        PS_WANT(n % 8 == 0, "strides must be multiples of 16 bytes (got %llu elements)", (unsigned long long)n);
    for (uint64_t n : {a->k_new_token, a->v_new_token, a->k_row, a->v_row})
        PS_WANT(n <= (1ull << 30) / 64, "64 rows must span less than 2 GiB (stride of %llu elements)", (unsigned long long)n);
    for (const int32_t *p : {a->first, a->context, a->parent}) PS_WANT(aligned(p, 4), "first, context and parent must be aligned to 4 bytes");
    PS_WANT(workspace_bytes >= need && (need == 0 || (workspace && aligned(workspace, kAlign))), "a workspace of %llu bytes, 256-byte aligned, is needed", (unsigned long long)need);
    const TreeDeal d = tree_deal(*a);
    PS_WANT(((uint64_t)a->n_seq * a->n_kv_heads * d.nsplit + 7) / 8 * 8 * d.blocks <= kMostGroups, "too many sequences and heads for one call");
    hipStream_t st = static_cast<hipStream_t>(stream);
    float *part = static_cast<float *>(workspace);
    if (a->type == PS_TYPE_F16) PS_TRY(a->head_dim == 64 ? (launch_trees<f16_t, 64>(*a, d, part, st)) : (launch_trees<f16_t, 128>(*a, d, part, st)));
    else PS_TRY(a->head_dim == 64 ? (launch_trees<bf16_t, 64>(*a, d, part, st)) : (launch_trees<bf16_t, 128>(*a, d, part, st)));
    return PS_OK;
}

int32_t ps_verify_tree_workspace(const ps_verify_tree_args *a, uint64_t *bytes) {
    PS_WANT(a && bytes, "NULL argument");
    PS_WANT(a->type <= PS_TYPE_F32, "unknown type %u", a->type);
    PS_WANT(a->vocab >= 1 && a->vocab <= 1u << 24, "vocab 1 .. 2^24 (got %u)", a->vocab);
    PS_WANT(a->max_tree <= PS_TREE_MAX, "trees of up to %u tokens (got %u)", PS_TREE_MAX, a->max_tree);
    PS_WANT(a->max_children >= 1 && a->max_children <= PS_TREE_MAX, "max_children 1 .. %u (got %u)", PS_TREE_MAX, a->max_children);
    PS_WANT(a->n_seq <= 65535 && a->n_tokens <= 0x7FFFFFFF, "%u sequences, %u tokens: too many", a->n_seq, a->n_tokens);
    VerifyWork w;
    *bytes = verify_work(*a, verify_shape(*a), nullptr, &w);
    return PS_OK;
}

int32_t ps_verify_tree(const ps_verify_tree_args *a, void *workspace, uint64_t workspace_bytes, void *stream) {
    uint64_t need = 0;
    const int32_t rc = ps_verify_tree_workspace(a, &need);
    if (rc) return rc;
    if (a->n_seq == 0) return PS_OK;
    PS_WANT(a->first && a->path && a->count && a->next_token, "NULL argument");
    PS_WANT(a->n_tokens == 0 || a->max_tree == 0 || (a->target_logits && a->token && a->parent && a->u_accept && a->u_sample), "NULL argument");
    PS_WANT(a->path_seq >= a->max_tree || a->n_seq == 1, "paths of %u entries lie %llu apart", a->max_tree, (unsigned long long)a->path_seq);
    const uint32_t e = type_bytes(a->type);
    PS_WANT(aligned(a->target_logits, e) && aligned(a->draft_logits, e), "logits must be aligned to an element");
    for (const void *p : {(const void *)a->first, (const void *)a->token, (const void *)a->parent, (const void *)a->u_accept, (const void *)a->u_sample,
                          (const void *)a->temperature, (const void *)a->path, (const void *)a->count, (const void *)a->next_token})
        PS_WANT(aligned(p, 4), "tables, random numbers and outputs must be aligned to 4 bytes");
    PS_WANT(workspace_bytes >= need && (need == 0 || (workspace && aligned(workspace, kAlign))), "a workspace of %llu bytes, 256-byte aligned, is needed", (unsigned long long)need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const VerifyShape sh = verify_shape(*a);
    VerifyWork w;
    verify_work(*a, sh, static_cast<uint8_t *>(workspace), &w);
    if (a->type == PS_TYPE_F16) PS_TRY(launch_verify<f16_t>(*a, sh, w, st));
    else if (a->type == PS_TYPE_BF16) PS_TRY(launch_verify<bf16_t>(*a, sh, w, st));
    else PS_TRY(launch_verify<float>(*a, sh, w, st));
    return PS_OK;
}

int32_t ps_cache_keep(const ps_cache_keep_args *a, void *stream) {
    PS_WANT(a, "NULL argument");
    PS_WANT(a->max_tree <= PS_TREE_MAX, "paths of up to %u entries (got %u)", PS_TREE_MAX, a->max_tree);
    PS_WANT(a->row_bytes >= 16 && a->row_bytes <= 4096 && a->row_bytes % 16 == 0, "row_bytes must be a multiple of 16, up to 4096 (got %u)", a->row_bytes);
    PS_WANT(a->n_seq <= 65535 && ((uint64_t)a->n_planes + 3) / 4 <= kMostGroups && a->capacity <= 0x7FFFFFFF, "too many sequences, planes or rows");
    if (a->n_seq == 0 || a->n_planes == 0 || a->max_tree == 0 || a->capacity == 0) return PS_OK;
    PS_WANT(a->cache && a->path && a->count && a->context, "NULL argument");
    PS_WANT(aligned(a->cache, 16) && a->seq_stride % 16 == 0 && a->plane_stride % 16 == 0 && a->row_stride % 16 == 0, "the cache and its strides must be multiples of 16 bytes");
    PS_WANT(a->row_stride >= a->row_bytes || a->capacity == 1, "rows of %u bytes lie %llu bytes apart", a->row_bytes, (unsigned long long)a->row_stride);
    PS_WANT(aligned(a->path, 4) && aligned(a->count, 4) && aligned(a->context, 4), "path, count and context must be aligned to 4 bytes");
    PS_TRY(launch_keep(*a, BatchPlanes{}, static_cast<hipStream_t>(stream)));
    return PS_OK;
}

}  // extern "C"
