// Operators of a step that answers several drafted tokens at once: norms of queries and keys with the position rotation,
// attention of a tree of tokens over a cache, verification of the drafts, and the accepted rows of the cache.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "ps_internal.h"

namespace ps {

namespace {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u2_t __attribute__((ext_vector_type(2)));

constexpr float kFloatMax = 3.402823466e38f;

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// rows first[s] .. of sequence s and how many of them count
struct SeqRows { int row0, n; };
__device__ __forceinline__ SeqRows rows_of(const int32_t *first, uint32_t s, uint32_t n_tokens, uint32_t max_tree) {
    const int a = clampi(first[s], 0, (int)n_tokens), b = clampi(first[s + 1], 0, (int)n_tokens);
    return {a, clampi(b - a, 0, (int)max_tree)};
}
__device__ __forceinline__ int parent_of(int p, int i) { return p >= 0 && p < i ? p : -1; }

template <typename T> __device__ __forceinline__ float to_f(T v) { return (float)v; }

// ------------------------------------------------------------------------------------ norms and rotation
// A wave per (token, head); lane l holds the pairs l, l + 64, ...
template <typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(ps_qk_norm_rope_args a) {
    const uint32_t lane = threadIdx.x & 63, heads = a.n_q_heads + a.n_k_heads;
    const uint64_t item = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item >= (uint64_t)a.n_tokens * heads) return;
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
        const double turn = pos * (double)a.inv_freq[i];
        const float c = (float)cos(turn), s = (float)sin(turn);
        y[da] = (T)(va * c - vb * s);
        y[db] = (T)(vb * c + va * s);
    }
    for (uint32_t d = a.rot_dim + lane; d < a.head_dim; d += 64)
        y[d] = (T)(to_f(x[d]) * rinv * (a.norm && gain ? to_f(gain[d]) : 1.f));
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
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef f16_t f16x8_t __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8_t __attribute__((ext_vector_type(8)));

template <typename T> struct Mfma;
template <> struct Mfma<f16_t> {
    typedef f16x8_t v8;
    static constexpr uint32_t kInf = 0x7C007C00u;
    static __device__ __forceinline__ f4_t mul(v8 a, v8 b, f4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
#else
        return c;
#endif
    }
};
template <> struct Mfma<bf16_t> {
    typedef bf16x8_t v8;
    static constexpr uint32_t kInf = 0x7F807F80u;
    static __device__ __forceinline__ f4_t mul(v8 a, v8 b, f4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
        return c;
#endif
    }
};

// A operand of 16 dims x 32 positions from rows staged in LDS: two transpose reads, four rows (hi bytes) apart
__device__ __forceinline__ u4_t transposed(const unsigned char *p, uint32_t hi) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s4_t;
    typedef __attribute__((address_space(3))) s4_t lds_s4_t;
    const u2_t a = __builtin_bit_cast(u2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t *)(p)));
    const u2_t b = __builtin_bit_cast(u2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t *)(p + hi)));
    return u4_t{a.x, a.y, b.x, b.y};
#else
    return u4_t{};
#endif
}
// largest value of the four lanes that share a row (lane, lane ^ 16, ^ 32, ^ 48)
__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
// 16-byte piece u of a staged V row lies in slot u ^ swizzle: even swizzles keep the pair of pieces that a transpose read takes
// together, and the eight rows of half a wave (8 c + 0 .. 3) lie in different banks
template <int D> __device__ __forceinline__ uint32_t v_swizzle(uint32_t row) {
    return D == 128 ? ((row & 3u) | (((row >> 3) & 1u) << 2)) << 1 : (((row >> 1) & 1u) | (((row >> 3) & 1u) << 1)) << 1;
}

constexpr uint32_t kTile = 32;           // positions of a tile
constexpr uint32_t kMaskWords = PS_TREE_MAX / 32;

struct TreeDeal { uint32_t nt, blocks, nsplit; };

template <int D, int NT> constexpr uint32_t tree_lds() {
    const uint32_t stages = 4 * kTile * D * 2, meet = 4 * NT * 16 * (D + 4) * 4 + 4 * NT * 16 * 2 * 4;
    return std::max(stages, meet) + PS_TREE_MAX * kMaskWords * 4 + PS_TREE_MAX * 4 + 16;
}

// Tiles of sequence: the cache's, then the tree's own; each split takes `per` of them
__device__ __forceinline__ uint32_t tiles_per_split(uint32_t tiles, uint32_t nsplit) { return ((tiles + nsplit - 1) / nsplit + 3) & ~3u; }

template <typename T, int D, int NT>
__global__ __launch_bounds__(256, 2) void tree_attention_kernel(ps_tree_attention_args a, uint32_t blocks, uint32_t nsplit, float *part) {
    using M = Mfma<T>;
    using v8 = typename M::v8;
    constexpr int KK = D / 32, DT = D / 16, RB = NT * 16, OP = D + 4;
    constexpr uint32_t kStage = kTile * D * 2, kRowPieces = D / 8, kVLoads = kStage / 1024;
    extern __shared__ u4_t tree_lds_mem[];
    unsigned char *const lds = reinterpret_cast<unsigned char *>(tree_lds_mem);
    constexpr uint32_t kTables = tree_lds<D, NT>() - (PS_TREE_MAX * kMaskWords * 4 + PS_TREE_MAX * 4 + 16);
    uint32_t *const anc = reinterpret_cast<uint32_t *>(lds + kTables);           // [token][word]: itself and its ancestors
    int *const up = reinterpret_cast<int *>(anc + PS_TREE_MAX * kMaskWords);
    int *const wild = up + PS_TREE_MAX;                                          // some own value is infinite or no number

    // blocks of the same positions lie 8 workgroups apart: on one XCD, whose L2 they share
    const uint32_t units = a.n_seq * a.n_kv_heads * nsplit;
    const uint32_t unit = blockIdx.x / 8 / blocks * 8 + blockIdx.x % 8, rb = blockIdx.x / 8 % blocks;
    if (unit >= units) return;
    const uint32_t z = unit % nsplit, hk = unit / nsplit % a.n_kv_heads, s = unit / nsplit / a.n_kv_heads;
    const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
    const uint32_t ctx = clampi(a.context[s], 0, (int)a.max_context), t_n = sr.n, G = a.n_q_heads / a.n_kv_heads;
    const uint32_t R = t_n * G, row0 = rb * RB;
    if (row0 >= R) return;
    const uint32_t nc = (ctx + kTile - 1) / kTile, tiles = nc + (t_n + kTile - 1) / kTile, per = tiles_per_split(tiles, nsplit);
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

    // own tiles: which tokens each token sees
    const bool own = hi > nc;
    if (own) {
        int link = -1;
        uint32_t m[kMaskWords];
        if (tid == 0) *wild = 0;
        if (tid < t_n) {
            link = parent_of(a.parent[sr.row0 + tid], (int)tid);
#pragma unroll
            for (uint32_t w = 0; w < kMaskWords; ++w) anc[tid * kMaskWords + w] = tid / 32 == w ? 1u << (tid % 32) : 0u;
            up[tid] = link;
        }
        // every step doubles how far back a token's mask reaches
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
    if (a.append && z == 0) {            // rows context and up, which nobody reads: each block moves the tokens whose first row it holds
        const uint32_t t0 = (row0 + G - 1) / G, t1 = min(t_n, (row0 + RB + G - 1) / G);
        T *kd = static_cast<T *>(a.k_cache) + s * a.k_seq + hk * a.k_head, *vd = static_cast<T *>(a.v_cache) + s * a.v_seq + hk * a.v_head;
        for (uint32_t u = tid; u < (t1 - t0) * kRowPieces * 2; u += 256) {
            const uint32_t t = t0 + u / (2 * kRowPieces), e = u % kRowPieces * 8;
            const bool v = u / kRowPieces & 1;
            *reinterpret_cast<u4_t *>(v ? vd + ((size_t)ctx + t) * a.v_row + e : kd + ((size_t)ctx + t) * a.k_row + e) =
                *reinterpret_cast<const u4_t *>(v ? vn + (size_t)t * a.v_new_token + e : kn + (size_t)t * a.k_new_token + e);
        }
    }

    // the block's rows of queries; a negative scale turns their signs
    const float scale_abs = fabsf(a.scale);
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    const float c2 = fmaxf(scale_abs * 1.4426950408889634f, 1e-30f);     // weights are 2^(c2 (s - m))
    const float slack = 8.f / c2;      // a row is rescaled only where its weights would pass 2^8
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
            // An infinite value or one that is no number must not meet the zero weight of a row that does not see it: the
            // product takes zero in its place, and rows that do see it get it at the end.
            bool odd = false;
#pragma unroll
            for (uint32_t u = 0; u < kVLoads; ++u) {
                uint32_t d[4] = {vreg[u].x, vreg[u].y, vreg[u].z, vreg[u].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool l16 = (d[e] & M::kInf & 0xFFFFu) == (M::kInf & 0xFFFFu), h16 = (d[e] & M::kInf & 0xFFFF0000u) == (M::kInf & 0xFFFF0000u);
                    odd |= l16 || h16;
                    d[e] = (l16 ? 0u : d[e] & 0xFFFFu) | (h16 ? 0u : d[e] & 0xFFFF0000u);
                }
                vreg[u] = u4_t{d[0], d[1], d[2], d[3]};
            }
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
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float mx = fmaxf(fmaxf(fmaxf(S[t][0][0], S[t][0][1]), fmaxf(S[t][0][2], S[t][0][3])), fmaxf(fmaxf(S[t][1][0], S[t][1][1]), fmaxf(S[t][1][2], S[t][1][3])));
            if (__any(mx > m_run[t] + slack)) {
                mx = row_max(mx);
                mx = mx > m_run[t] + slack ? mx : m_run[t];
                const float resc = m_run[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run[t] - mx) * c2);
                m_run[t] = mx;
                L[t] = L[t] * resc;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) O[t][dt] = O[t][dt] * resc;
            }
            const float ms = m_run[t] == -INFINITY ? 0.f : m_run[t] * c2;
#pragma unroll
            for (int e = 0; e < 8; ++e) P[t][e] = (T)__builtin_amdgcn_exp2f(fmaf(S[t][e >> 2][e & 3], c2, -ms));
        }
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
            if (mw == -INFINITY && mx != -INFINITY) continue;            // (a wave that saw nothing of this row)
            const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mw - mx) * c2);
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
            float *dst = part + ((token * a.n_q_heads + h) * nsplit + z) * OP;
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

// A wave per (token, query head) merges the records of its sequence's splits, in their order: value sums, then maximum (in
// powers of two) and weight sum.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(ps_tree_attention_args a, uint32_t nsplit, const float *part) {
    constexpr int E = D / 64, OP = D + 4;
    const uint32_t lane = threadIdx.x & 63, h = blockIdx.x * 4 + (threadIdx.x >> 6), t = blockIdx.y, s = blockIdx.z;
    const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
    if (h >= a.n_q_heads || (int)t >= sr.n) return;
    const uint32_t ctx = clampi(a.context[s], 0, (int)a.max_context);
    const uint32_t tiles = (ctx + kTile - 1) / kTile + (sr.n + kTile - 1) / kTile, per = tiles_per_split(tiles, nsplit), n = (tiles + per - 1) / per;
    const size_t token = (size_t)sr.row0 + t;
    const float *p = part + (token * a.n_q_heads + h) * nsplit * OP;
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
            const bool in = z0 + u < n && (mv[u] != -INFINITY || m8 == -INFINITY);     // left out, not weighed with zero: a sum may be infinite
            const float w = mv[u] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mv[u] - ms);
            l = in ? fmaf(w, lv[u], l) : l;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = in ? fmaf(w, ov[u][e], o[e]) : o[e];
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) static_cast<T *>(a.out)[token * a.out_token + h * a.out_head + lane * E + e] = (T)(o[e] / l);
}

// How the work is dealt out: rows in blocks of 16 or 32 (64 rows a wave take more than 256 registers, and the compiler then
// moves the value sums between its two kinds of them in every tile); positions in as many splits as bring the launch to the
// workgroups the chip holds at once (two per CU, by registers), none of less than 8 tiles
TreeDeal tree_deal(const ps_tree_attention_args &a) {
    TreeDeal d;
    const uint32_t rows = std::max(1u, a.max_tree) * (a.n_q_heads / a.n_kv_heads);
    d.nt = rows <= 16 ? 1 : 2;
    d.blocks = (rows + d.nt * 16 - 1) / (d.nt * 16);
    const uint64_t wgs = std::max<uint64_t>(1, (uint64_t)a.n_seq * a.n_kv_heads * d.blocks);
    const uint32_t tiles = (a.max_context + kTile - 1) / kTile + (a.max_tree + kTile - 1) / kTile, room = 512;
    d.nsplit = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(room / wgs, tiles / 8));
    return d;
}

template <typename T, int D, int NT>
hipError_t launch_tree_k(const ps_tree_attention_args &a, const TreeDeal &d, float *part, hipStream_t st) {
    constexpr uint32_t lds = tree_lds<D, NT>();
    static std::atomic<uint64_t> done{0};        // devices this kernel's LDS size has been announced on
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(&tree_attention_kernel<T, D, NT>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    const uint32_t units = a.n_seq * a.n_kv_heads * d.nsplit;
    hipLaunchKernelGGL((tree_attention_kernel<T, D, NT>), dim3((units + 7) / 8 * 8 * d.blocks), dim3(256), lds, st, a, d.blocks, d.nsplit, part);
    return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_tree(const ps_tree_attention_args &a, const TreeDeal &d, float *part, hipStream_t st) {
    hipError_t e = d.nt == 1 ? launch_tree_k<T, D, 1>(a, d, part, st) : launch_tree_k<T, D, 2>(a, d, part, st);
    if (e != hipSuccess || d.nsplit == 1) return e;
    hipLaunchKernelGGL((tree_merge_kernel<T, D>), dim3((a.n_q_heads + 3) / 4, a.max_tree, a.n_seq), dim3(256), 0, st, a, d.nsplit, part);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ verification
// Rows are cut into chunks (rules in verify_shape).  Launches, in order:
//  verify_rows_kernel   chunk maximum and sum of exponentials of every row that a decision needs: the nodes with children, target and
//                       draft; without sampling the largest logit's index instead
//  verify_left_kernel   with drafts, for the k-th child (k = 1 ..): chunk sums W_k = sum max(p - c_k q, 0) of the nodes whose first k
//                       children are refused and that the walk may still reach
//  verify_draw_kernel   every workgroup works out the same walk; chunk sums of what is left to draw from behind its last node
//  verify_pick_kernel   the chunk that the random number falls into, and the index in it
// Exponentials and sums are in 64 bits: with fp32's 2^-24 a border of the running sum moves by as much as a hundred thousandth of
// the vocabulary's entries weigh.  A 64-bit multiply-add costs this machine what a 32-bit one does; an exponential here is about
// 18 of them, which in a large batch takes as long as the row's bytes do.  No result depends on the order of workgroups.
constexpr uint32_t kVerThreads = 256, kMaxChunks = 32;
struct RowPart { double z; float m; int best; };                 // one chunk of a row
struct DrawHead { double c, ip, iq; float m, mq; int row, kind; };   // what is left behind the last node, for the pick
enum { DRAW_NONE = 0, DRAW_BEST = 1, DRAW_LEAF = 2, DRAW_LEFT = 3, DRAW_GIVEN = 4 };
struct VerifyShape { uint32_t chunk, nchunk, loop; };
struct VerifyWork { RowPart *parts; double *left; RowPart *recs; DrawHead *heads; };   // [token][target, draft][chunk], [token][chunk], [seq][chunk], [seq]

__device__ __forceinline__ float sane(float v) { return v != v ? -INFINITY : fminf(v, kFloatMax); }

// 2^t for t <= 0, to 3e-13 of its value: t = n + f, |f| <= 1/2, the exponential series of f ln 2 to the tenth power (the next term
// is (ln 2 / 2)^11 / 11! = 2e-13)
__device__ __forceinline__ double pow2_neg(double t) {
    t = fmax(t, -1100.0);
    const double n = rint(t), f = t - n;
    double p = 7.054911620801121e-09;                            // (ln 2)^i / i!, i = 10 .. 0
    p = fma(p, f, 1.0178086009239696e-07);
    p = fma(p, f, 1.3215486790144305e-06);
    p = fma(p, f, 1.5252733804059838e-05);
    p = fma(p, f, 1.5403530393381606e-04);
    p = fma(p, f, 1.3333558146428441e-03);
    p = fma(p, f, 9.618129107628477e-03);
    p = fma(p, f, 5.5504108664821576e-02);
    p = fma(p, f, 2.402265069591007e-01);
    p = fma(p, f, 6.931471805599453e-01);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}
// exp((x - m) / T) with k = log2(e) / T; a row of -inf alone has no probabilities
__device__ __forceinline__ double weight(float x, float m, double k) { return pow2_neg(((double)x - (double)m) * k); }
__device__ __forceinline__ double rate_of(float temp) { return 1.4426950408889634 / (double)fminf(temp, 1e30f); }

// logits i .. i + 7 of a row (past the end: -inf); rows may start anywhere
template <typename T>
__device__ __forceinline__ void load8(const T *x, uint32_t i, uint32_t end, float (&v)[8]) {
    if (i + 8 <= end) {
        T t[8];
        __builtin_memcpy(t, x + i, sizeof(t));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sane(to_f(t[e]));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = i + e < end ? sane(to_f(x[i + e])) : -INFINITY;
    }
}

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

// One chunk [lo, hi) of a row: its maximum, and the sum of exp((x - max) k), or (greedy) the first index of the maximum.
// A chunk is a multiple of 2048 long: kVec vectors of 8 to a thread at a time, all of them requested before the first is used
constexpr uint32_t kVec = 2, kSpan = kVec * kVerThreads * 8;
template <typename T>
__device__ RowPart chunk_part(const T *x, uint32_t lo, uint32_t hi, double k, bool greedy, BlockBuf &b) {
    RowPart r{0.0, -INFINITY, 0x7FFFFFFF};
    for (uint32_t s0 = lo; s0 < hi; s0 += kSpan) {
        float v[kVec][8], mx = -INFINITY;
#pragma unroll
        for (uint32_t u = 0; u < kVec; ++u) load8(x, s0 + (u * kVerThreads + threadIdx.x) * 8, hi, v[u]);
#pragma unroll
        for (uint32_t u = 0; u < kVec; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, v[u][e]);
        mx = block_max(mx, b.f);
        if (mx == -INFINITY) continue;
        if (greedy) {
            int at = 0x7FFFFFFF;
#pragma unroll
            for (uint32_t u = 0; u < kVec; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (v[u][e] == mx) at = min(at, (int)(s0 + (u * kVerThreads + threadIdx.x) * 8 + e));
            at = block_min(at, b.i);
            if (mx > r.m) r.best = at;
            r.m = fmaxf(r.m, mx);
            continue;
        }
        const float m = fmaxf(r.m, mx);
        double z = 0;
#pragma unroll
        for (uint32_t u = 0; u < kVec; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) z += weight(v[u][e], m, k);
        z = block_sum(z, b.d);
        r.z = (r.m == -INFINITY ? 0.0 : r.z * weight(r.m, m, k)) + z;
        r.m = m;
    }
    return r;
}

struct RowSum { double z; float m; int best; };
__device__ __forceinline__ RowSum row_sum(const RowPart *p, uint32_t n, double k, bool greedy) {
    RowSum r{0.0, -INFINITY, -1};
    for (uint32_t i = 0; i < n; ++i) {
        const float m = p[i].m;
        if (m > r.m) { r.m = m; r.best = p[i].best; }
    }
    if (greedy || r.m == -INFINITY) return r;
    for (uint32_t i = 0; i < n; ++i)
        if (p[i].m != -INFINITY) r.z += p[i].z * weight(p[i].m, r.m, k);
    return r;
}

template <typename T>
__global__ __launch_bounds__(kVerThreads) void verify_rows_kernel(ps_verify_tree_args a, VerifyShape sh, VerifyWork w) {
    __shared__ BlockBuf b;
    __shared__ unsigned char parent[PS_TREE_MAX];
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
    const uint32_t lo = chunk * sh.chunk, hi = min(a.vocab, lo + sh.chunk);
    uint32_t seen = 0;
    for (int i = 0; i < sr.n; ++i) {
        if (!parent[i] || seen++ % gridDim.y != blockIdx.y) continue;
        const size_t row = (size_t)sr.row0 + i;
        const RowPart p = chunk_part(static_cast<const T *>(a.target_logits) + row * a.target_row, lo, hi, k, greedy, b);
        if (tid == 0) w.parts[row * 2 * sh.nchunk + chunk] = p;
        if (!a.draft_logits || greedy) continue;
        const RowPart q = chunk_part(static_cast<const T *>(a.draft_logits) + row * a.draft_row, lo, hi, k, false, b);
        if (tid == 0) w.parts[(row * 2 + 1) * sh.nchunk + chunk] = q;
    }
}

// Decisions of a sequence's nodes, as far as they are known: by one thread for each node
struct Walk {
    RowSum p[PS_TREE_MAX], q[PS_TREE_MAX];     // of nodes with children
    double px[PS_TREE_MAX], left[PS_TREE_MAX]; // of a node as its parent's child: p(token), W (or what is left without the refused)
    double c[PS_TREE_MAX];                     // c in front of this child
    int up[PS_TREE_MAX], rank[PS_TREE_MAX], token[PS_TREE_MAX], went[PS_TREE_MAX], kids[PS_TREE_MAX];
    bool dup[PS_TREE_MAX];
};

// known: children up to this rank are decided (their W has been summed)
template <typename T>
__device__ void decide(const ps_verify_tree_args &a, const VerifyShape &sh, const VerifyWork &w, const SeqRows &sr, float temp, uint32_t known, Walk &k) {
    const int tid = threadIdx.x;
    const bool greedy = !(temp > 0.f), drafts = a.draft_logits && !greedy, in = tid < sr.n;
    const double rate = greedy ? 0.0 : rate_of(temp);
    k.kids[tid] = 0;
    k.went[tid] = 0x7FFFFFFF;
    int up = -1, token = -1;
    float u = 0.f;
    const size_t row = (size_t)sr.row0 + tid;
    if (in) { up = parent_of(a.parent[row], tid); token = a.token[row]; u = a.u_accept[row]; }
    k.up[tid] = in ? up : -1;
    k.token[tid] = token;
    __syncthreads();
    if (up >= 0) atomicAdd(&k.kids[up], 1);
    int rank = 0;
    bool dup = false;
    for (int j = 1; j < tid && up >= 0; ++j)
        if (k.up[j] == up) { ++rank; dup |= k.token[j] == token; }
    k.rank[tid] = rank;
    k.dup[tid] = dup;
    __syncthreads();
    if (in && k.kids[tid]) {
        k.p[tid] = row_sum(w.parts + row * 2 * sh.nchunk, sh.nchunk, rate, greedy);
        if (drafts) k.q[tid] = row_sum(w.parts + (row * 2 + 1) * sh.nchunk, sh.nchunk, rate, false);
    }
    double sum = 1.0;
    if (up >= 0 && drafts && rank > 0 && rank <= (int)known && rank < (int)a.max_children) {
        sum = 0;
        for (uint32_t i = 0; i < sh.nchunk; ++i) sum += w.left[row * sh.nchunk + i];
    }
    k.left[tid] = sum;
    __syncthreads();
    double px = 0, qx = 0;
    const bool inside = token >= 0 && token < (int)a.vocab;
    if (up >= 0 && inside) {
        const size_t at = (size_t)sr.row0 + up;
        if (greedy) px = token == k.p[up].best ? 1.0 : 0.0;
        else if (k.p[up].m != -INFINITY) px = weight(sane(to_f(static_cast<const T *>(a.target_logits)[at * a.target_row + token])), k.p[up].m, rate) / k.p[up].z;
        if (drafts && k.q[up].m != -INFINITY) qx = weight(sane(to_f(static_cast<const T *>(a.draft_logits)[at * a.draft_row + token])), k.q[up].m, rate) / k.q[up].z;
    }
    k.px[tid] = px;
    __syncthreads();
    if (up >= 0) {
        double c = 0, rest = 1.0;
        for (int j = 1; j < tid; ++j) {
            if (k.up[j] != up) continue;
            if (drafts) c += k.left[j];
            else if (!greedy && !k.dup[j]) rest -= k.px[j];
        }
        k.c[tid] = c;
        const bool yes = drafts ? px > (c + (double)u * k.left[tid]) * qx : (greedy || !dup) && px > (double)u * rest;
        if (yes && rank < (int)a.max_children && (!drafts || rank <= (int)known)) atomicMin(&k.went[up], tid);
    }
    __syncthreads();
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
    const uint32_t lo = chunk * sh.chunk, hi = min(a.vocab, lo + sh.chunk);
    for (int j = 0; j < n; ++j) {
        const int child = list[j], up = walk.up[child];
        const size_t row = (size_t)sr.row0 + up;
        const RowSum p = walk.p[up], q = walk.q[up];
        // the child's c holds W of those in front of it, all known
        const double c = walk.c[child], ip = p.m == -INFINITY ? 0.0 : 1.0 / p.z, iq = q.m == -INFINITY ? 0.0 : c / q.z;
        double sum = 0;
        for (uint32_t i = lo + tid * 8; i < hi; i += kVerThreads * 8) {
            float x[8], y[8];
            load8(static_cast<const T *>(a.target_logits) + row * a.target_row, i, hi, x);
            load8(static_cast<const T *>(a.draft_logits) + row * a.draft_row, i, hi, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double pv = ip > 0 ? weight(x[e], p.m, rate) * ip : 0.0, qv = iq > 0 ? weight(y[e], q.m, rate) * iq : 0.0;
                sum += fmax(pv - qv, 0.0);
            }
        }
        sum = block_sum(sum, b.d);
        if (tid == 0) w.left[((size_t)sr.row0 + child) * sh.nchunk + chunk] = sum;
    }
}

// Entries i .. i + 7 of what is left to draw from (DRAW_LEFT, DRAW_GIVEN, DRAW_LEAF with its chunk's or row's maximum in m)
template <typename T>
__device__ __forceinline__ void left8(const ps_verify_tree_args &a, const DrawHead &h, int kind, double rate, uint32_t i, uint32_t hi, const int *refused, int nref,
                                      double (&r)[8]) {
    float x[8];
    load8(static_cast<const T *>(a.target_logits) + (size_t)h.row * a.target_row, i, hi, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = weight(x[e], h.m, rate) * h.ip;
    if (kind == DRAW_LEFT) {
        load8(static_cast<const T *>(a.draft_logits) + (size_t)h.row * a.draft_row, i, hi, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = fmax(r[e] - (h.iq > 0 ? weight(x[e], h.mq, rate) * h.iq : 0.0), 0.0);
    }
    if (kind == DRAW_GIVEN)
        for (int j = 0; j < nref; ++j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = refused[j] == (int)(i + e) ? 0.0 : r[e];
        }
}

template <typename T>
__global__ __launch_bounds__(kVerThreads) void verify_draw_kernel(ps_verify_tree_args a, VerifyShape sh, VerifyWork w) {
    __shared__ Walk walk;
    __shared__ BlockBuf b;
    __shared__ int path[PS_TREE_MAX], refused[PS_TREE_MAX], n, nref, last;
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
    const uint32_t lo = chunk * sh.chunk, hi = min(a.vocab, lo + sh.chunk);
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
            nref = 0;
        }
        __syncthreads();
        kids = walk.kids[last];
    } else {
        if (tid == 0) { path[0] = 0; n = 1; last = 0; nref = 0; }
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
            // (only those of this chunk)
            const int x = walk.token[tid];
            if (x >= (int)lo && x < (int)hi) refused[atomicAdd(&nref, 1)] = x;
        }
        __syncthreads();
    } else {
        h.kind = DRAW_LEAF;
    }
    if (chunk == 0) {
        if (tid < (int)a.max_tree) a.path[s * a.path_seq + tid] = tid < n ? path[tid] : -1;
        if (tid == 0) {
            a.count[s] = n;
            w.heads[s] = h;
            if (h.kind == DRAW_BEST) w.recs[s * sh.nchunk].best = walk.p[last].best;
        }
    }
    if (h.kind < DRAW_LEAF) return;
    RowPart r{0.0, h.m, 0};
    if (h.kind == DRAW_LEAF) {
        r = chunk_part(static_cast<const T *>(a.target_logits) + (size_t)h.row * a.target_row, lo, hi, rate, greedy, b);
    } else {
        double sum = 0;
        for (uint32_t i = lo + tid * 8; i < hi; i += kVerThreads * 8) {
            double v[8];
            left8<T>(a, h, h.kind, rate, i, hi, refused, nref, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[e];
        }
        r.z = block_sum(sum, b.d);
    }
    if (tid == 0) w.recs[s * sh.nchunk + chunk] = r;
}

template <typename T>
__global__ __launch_bounds__(kVerThreads) void verify_pick_kernel(ps_verify_tree_args a, VerifyShape sh, VerifyWork w) {
    __shared__ double sums[kMaxChunks], runs[4];
    __shared__ int refused[PS_TREE_MAX], nref, pick[2];
    const uint32_t s = blockIdx.x;
    const int tid = threadIdx.x;
    DrawHead h = w.heads[s];
    if (h.kind <= DRAW_BEST) {
        if (tid == 0) a.next_token[s] = h.kind == DRAW_BEST ? w.recs[s * sh.nchunk].best : -1;
        return;
    }
    const float temp = a.temperature ? a.temperature[s] : 1.f;
    const bool greedy = !(temp > 0.f);
    const double rate = greedy ? 0.0 : rate_of(temp);
    const RowPart *recs = w.recs + s * sh.nchunk;
    int kind = h.kind;
    if (kind == DRAW_LEAF) {
        const RowSum r = row_sum(recs, sh.nchunk, rate, greedy);
        if (r.m == -INFINITY || greedy) {
            if (tid == 0) a.next_token[s] = r.m == -INFINITY ? -1 : r.best;
            return;
        }
        h.m = r.m;
        h.ip = 1.0;
    }
    auto chunk_sums = [&](const RowPart *p) {       // relative to the row's maximum
        __syncthreads();
        for (uint32_t i = tid; i < sh.nchunk; i += kVerThreads) sums[i] = p[i].m == -INFINITY ? 0.0 : kind == DRAW_LEAF ? p[i].z * weight(p[i].m, h.m, rate) : p[i].z;
        __syncthreads();
    };
    if (tid == 0) nref = 0;
    chunk_sums(recs);
    double total = 0;
    for (uint32_t i = 0; i < sh.nchunk; ++i) total += sums[i];
    if (kind == DRAW_GIVEN) {
        const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
        const int last = h.row - sr.row0;
        __shared__ int up[PS_TREE_MAX];
        up[tid] = tid < sr.n ? parent_of(a.parent[sr.row0 + tid], tid) : -1;
        __syncthreads();
        if (tid < sr.n && up[tid] == last) {
            int rank = 0;
            for (int j = 1; j < tid; ++j) rank += up[j] == last;
            if (rank < (int)a.max_children) refused[atomicAdd(&nref, 1)] = a.token[sr.row0 + tid];
        }
        __syncthreads();
    }
    if (!(total > 0)) {      // nothing left: the target's own row
        kind = DRAW_LEAF;
        h.ip = 1.0;
        chunk_sums(w.parts + (size_t)h.row * 2 * sh.nchunk);
        total = 0;
        for (uint32_t i = 0; i < sh.nchunk; ++i) total += sums[i];
    }
    const double goal = (double)a.u_sample[s] * total;
    // the first chunk whose running sum passes the goal (or the last one that holds anything)
    double run = 0, before = 0;
    uint32_t chunk = 0;
    for (uint32_t i = 0; i < sh.nchunk; ++i) {
        if (sums[i] > 0) { chunk = i; before = run; }
        run += sums[i];
        if (run > goal) break;
    }
    const uint32_t lo = chunk * sh.chunk, hi = min(a.vocab, lo + sh.chunk);
    // in it, a run of consecutive entries to a thread
    const uint32_t per = sh.chunk / kVerThreads, i0 = lo + tid * per;
    double mine = 0;
    int some = -1;
    for (uint32_t i = i0; i < min(hi, i0 + per); i += 8) {
        double v[8];
        left8<T>(a, h, kind, rate, i, hi, refused, nref, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) { mine += v[e]; some = v[e] > 0 ? (int)(i + e) : some; }
    }
    double upto = mine;
    for (int o = 1; o < 64; o <<= 1) {
        const double v = __shfl_up(upto, o, 64);
        if ((tid & 63) >= o) upto += v;
    }
    if ((tid & 63) == 63) runs[tid >> 6] = upto;
    if (tid < 2) pick[tid] = tid ? -1 : 0x7FFFFFFF;
    __syncthreads();
    double base = before;
    for (int i = 0; i < tid >> 6; ++i) base += runs[i];
    const double prior = __shfl_up(upto, 1, 64);
    const double from = (tid & 63) ? base + prior : base, to = base + upto;
    if (to > goal && mine > 0) atomicMin(&pick[0], tid);
    if (some >= 0) atomicMax(&pick[1], some);
    __syncthreads();
    if (pick[0] == 0x7FFFFFFF) {
        if (tid == 0) a.next_token[s] = pick[1];
        return;
    }
    if (tid != pick[0]) return;
    double r = from;
    int found = some;
    for (uint32_t i = i0; i < min(hi, i0 + per); i += 8) {
        double v[8];
        left8<T>(a, h, kind, rate, i, hi, refused, nref, v);
        bool done = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            r += v[e];
            if (!done && v[e] > 0 && r > goal) { found = i + e; done = true; }
        }
        if (done) break;
    }
    a.next_token[s] = found;
}

// Chunks of a multiple of 2048 entries, at most kMaxChunks: a chunk of 4096 keeps a workgroup for about 3 us, as long as a launch's ends take.
// Row passes: as many workgroups as keep the chip busy, each takes the nodes in turn.
VerifyShape verify_shape(const ps_verify_tree_args &a) {
    VerifyShape sh;
    const uint32_t unit = kSpan / kVec, want = std::max(kSpan, (a.vocab + kMaxChunks - 1) / kMaxChunks);
    sh.chunk = (want + unit - 1) / unit * unit;
    sh.nchunk = (a.vocab + sh.chunk - 1) / sh.chunk;
    sh.loop = (uint32_t)std::min<uint64_t>(std::max(1u, a.max_tree), std::max<uint64_t>(1, 4096 / std::max<uint64_t>(1, (uint64_t)sh.nchunk * a.n_seq)));
    return sh;
}
uint64_t verify_work(const ps_verify_tree_args &a, const VerifyShape &sh, uint8_t *base, VerifyWork *w) {
    uint64_t off = 0;
    auto take = [&](uint64_t bytes) { uint8_t *p = base ? base + off : nullptr; off = align_up(off + bytes, kAlign); return p; };
    w->parts = reinterpret_cast<RowPart *>(take((uint64_t)a.n_tokens * 2 * sh.nchunk * sizeof(RowPart)));
    w->left = reinterpret_cast<double *>(take(a.draft_logits ? (uint64_t)a.n_tokens * sh.nchunk * 8 : 0));
    w->recs = reinterpret_cast<RowPart *>(take((uint64_t)a.n_seq * sh.nchunk * sizeof(RowPart)));
    w->heads = reinterpret_cast<DrawHead *>(take((uint64_t)a.n_seq * sizeof(DrawHead)));
    return off;
}

template <typename T>
hipError_t launch_verify(const ps_verify_tree_args &a, const VerifyShape &sh, const VerifyWork &w, hipStream_t st) {
    if (a.n_tokens && a.max_tree > 1) {
        hipLaunchKernelGGL(verify_rows_kernel<T>, dim3(sh.nchunk, sh.loop, a.n_seq), dim3(kVerThreads), 0, st, a, sh, w);
        if (a.draft_logits)
            for (uint32_t k = 1; k < std::min(a.max_children, a.max_tree - 1); ++k)
                hipLaunchKernelGGL(verify_left_kernel<T>, dim3(sh.nchunk, a.n_seq), dim3(kVerThreads), 0, st, a, sh, w, k);
    }
    hipLaunchKernelGGL(verify_draw_kernel<T>, dim3(sh.nchunk, a.n_seq), dim3(kVerThreads), 0, st, a, sh, w);
    hipLaunchKernelGGL(verify_pick_kernel<T>, dim3(a.n_seq), dim3(kVerThreads), 0, st, a, sh, w);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ kept rows
// A wave per plane of a sequence: it reads up to 16 x 64 pieces of 16 bytes (all rows of a run of columns) before it
// writes any, so rows may move onto rows that others are read from.
__global__ __launch_bounds__(256) void cache_keep_kernel(ps_cache_keep_args a, uint32_t seg) {
    const uint32_t lane = threadIdx.x & 63, plane = blockIdx.x * 4 + (threadIdx.x >> 6), s = blockIdx.y;
    if (plane >= a.n_planes) return;
    const int n = clampi(a.count[s], 0, (int)a.max_tree);
    const int64_t ctx = a.context[s];
    const int32_t *path = a.path + s * a.path_seq;
    char *base = static_cast<char *>(a.cache) + s * a.seq_stride + plane * a.plane_stride;
    const uint32_t units = a.row_bytes / 16;
    for (uint32_t c0 = 0; c0 < units; c0 += seg) {
        u4_t v[16];
        bool ok[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const uint32_t idx = u * 64 + lane, i = idx / seg, col = c0 + idx % seg;
            ok[u] = (int)i < n && col < units;
            if (ok[u]) {
                const int node = path[i];
                const int64_t from = ctx + node, to = ctx + i;
                ok[u] = node >= 0 && node < (int)a.max_tree && from >= 0 && from < a.capacity && to >= 0 && to < a.capacity;
                if (ok[u]) v[u] = *reinterpret_cast<const u4_t *>(base + from * a.row_stride + col * 16);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const uint32_t idx = u * 64 + lane, i = idx / seg, col = c0 + idx % seg;
            if (ok[u]) *reinterpret_cast<u4_t *>(base + (ctx + i) * a.row_stride + col * 16) = v[u];
        }
    }
}

#define PS_TRY(call)                                                                                    \
    do {                                                                                                \
        const hipError_t e_ = (call);                                                                   \
        if (e_ != hipSuccess) { set_error("%s failed: %s", #call, hipGetErrorString(e_)); return PS_E_HIP; } \
    } while (0)
#define PS_WANT(cond, ...)                                        \
    do {                                                          \
        if (!(cond)) { set_error(__VA_ARGS__); return PS_E_ARG; } \
    } while (0)

uint32_t type_bytes(uint32_t type) { return type == PS_TYPE_F32 ? 4 : 2; }
bool aligned(const void *p, uint64_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

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
    const dim3 grid((uint32_t)((items + 3) / 4));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->type == PS_TYPE_F16) hipLaunchKernelGGL(qk_norm_rope_kernel<f16_t>, grid, dim3(256), 0, st, *a);
    else if (a->type == PS_TYPE_BF16) hipLaunchKernelGGL(qk_norm_rope_kernel<bf16_t>, grid, dim3(256), 0, st, *a);
    else hipLaunchKernelGGL(qk_norm_rope_kernel<float>, grid, dim3(256), 0, st, *a);
    PS_TRY(hipGetLastError());
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
    PS_WANT((uint64_t)a->n_seq * a->n_kv_heads * d.nsplit * d.blocks < 1ull << 28, "too many sequences and heads for one call");
    hipStream_t st = static_cast<hipStream_t>(stream);
    float *part = static_cast<float *>(workspace);
    if (a->type == PS_TYPE_F16) PS_TRY(a->head_dim == 64 ? (launch_tree<f16_t, 64>(*a, d, part, st)) : (launch_tree<f16_t, 128>(*a, d, part, st)));
    else PS_TRY(a->head_dim == 64 ? (launch_tree<bf16_t, 64>(*a, d, part, st)) : (launch_tree<bf16_t, 128>(*a, d, part, st)));
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
    PS_WANT(a->n_seq <= 65535 && a->n_planes <= 0x7FFFFFFF && a->capacity <= 0x7FFFFFFF, "too many sequences, planes or rows");
    if (a->n_seq == 0 || a->n_planes == 0 || a->max_tree == 0 || a->capacity == 0) return PS_OK;
    PS_WANT(a->cache && a->path && a->count && a->context, "NULL argument");
    PS_WANT(aligned(a->cache, 16) && a->seq_stride % 16 == 0 && a->plane_stride % 16 == 0 && a->row_stride % 16 == 0, "the cache and its strides must be multiples of 16 bytes");
    PS_WANT(a->row_stride >= a->row_bytes || a->capacity == 1, "rows of %u bytes lie %llu bytes apart", a->row_bytes, (unsigned long long)a->row_stride);
    PS_WANT(aligned(a->path, 4) && aligned(a->count, 4) && aligned(a->context, 4), "path, count and context must be aligned to 4 bytes");
    const uint32_t seg = std::max(1u, std::min(a->row_bytes / 16, 1024 / a->max_tree));
    hipLaunchKernelGGL(cache_keep_kernel, dim3((a->n_planes + 3) / 4, a->n_seq), dim3(256), 0, static_cast<hipStream_t>(stream), *a, seg);
    PS_TRY(hipGetLastError());
    return PS_OK;
}

}  // extern "C"
