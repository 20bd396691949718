// Operators of a step that answers several drafted tokens at once: norms of queries and keys with the position rotation,
// attention of a tree of tokens over a cache, verification of the drafts, and the accepted rows of the cache.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ps_internal.h"

namespace ps {

namespace {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;

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
// A wave per (sequence, token, query head): one position after the other, running maximum and sum.
template <typename T, int D>
__global__ __launch_bounds__(64) void tree_attention_kernel(ps_tree_attention_args a) {
    const uint32_t s = blockIdx.z, h = blockIdx.y, lane = threadIdx.x;
    const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
    const int t = blockIdx.x;
    if (t >= sr.n) return;
    const int ctx = clampi(a.context[s], 0, (int)a.max_context);
    const uint32_t hk = h / (a.n_q_heads / a.n_kv_heads);
    constexpr int E = D / 64;
    float q[E], o[E];
    const size_t row = (size_t)sr.row0 + t;
    for (int e = 0; e < E; ++e) { q[e] = to_f(static_cast<const T *>(a.q)[row * a.q_token + h * a.q_head + lane * E + e]); o[e] = 0.f; }
    float m = -INFINITY, l = 0.f;
    auto see = [&](const T *k, const T *v) {
        float d = 0.f;
        for (int e = 0; e < E; ++e) d = fmaf(q[e], to_f(k[lane * E + e]), d);
        for (int x = 32; x; x >>= 1) d += __shfl_xor(d, x, 64);
        d *= a.scale;
        const float mn = fmaxf(m, d), r = m == -INFINITY ? 0.f : __expf(m - mn), w = mn == -INFINITY ? 0.f : __expf(d - mn);
        m = mn;
        l = l * r + w;
        for (int e = 0; e < E; ++e) o[e] = o[e] * r + w * to_f(v[lane * E + e]);
    };
    const T *kc = static_cast<const T *>(a.k_cache) + s * a.k_seq + hk * a.k_head, *vc = static_cast<const T *>(a.v_cache) + s * a.v_seq + hk * a.v_head;
    for (int j = 0; j < ctx; ++j) see(kc + j * a.k_row, vc + j * a.v_row);
    for (int j = t; j >= 0; j = parent_of(a.parent[sr.row0 + j], j))
        see(static_cast<const T *>(a.k_new) + ((size_t)sr.row0 + j) * a.k_new_token + hk * a.k_new_head,
            static_cast<const T *>(a.v_new) + ((size_t)sr.row0 + j) * a.v_new_token + hk * a.v_new_head);
    for (int e = 0; e < E; ++e) static_cast<T *>(a.out)[row * a.out_token + h * a.out_head + lane * E + e] = (T)(o[e] / l);
    if (a.append && h % (a.n_q_heads / a.n_kv_heads) == 0) {
        T *kd = static_cast<T *>(a.k_cache) + s * a.k_seq + hk * a.k_head + ((size_t)ctx + t) * a.k_row;
        T *vd = static_cast<T *>(a.v_cache) + s * a.v_seq + hk * a.v_head + ((size_t)ctx + t) * a.v_row;
        for (int e = 0; e < E; ++e) {
            kd[lane * E + e] = static_cast<const T *>(a.k_new)[row * a.k_new_token + hk * a.k_new_head + lane * E + e];
            vd[lane * E + e] = static_cast<const T *>(a.v_new)[row * a.v_new_token + hk * a.v_new_head + lane * E + e];
        }
    }
}

// ------------------------------------------------------------------------------------ verification
// A workgroup per sequence walks down the tree; every row is read by the whole workgroup.
__device__ __forceinline__ float sane(float v) { return v != v ? -INFINITY : fminf(v, kFloatMax); }

constexpr int kVerThreads = 1024;

template <typename T>
struct Row { const T *x; float m; double z, k; int best; };     // probabilities exp((x - m) k) / z

__device__ double block_sum(double v, double *buf) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    double r = 0;
    for (int w = 0; w < kVerThreads / 64; ++w) r += buf[w];
    return r;
}

template <typename T>
__device__ double chance(const Row<T> &r, int x, uint32_t V, float temp) {
    if (x < 0 || x >= (int)V || r.m == -INFINITY) return 0.0;
    if (!(temp > 0.f)) return x == r.best ? 1.0 : 0.0;
    return exp(((double)sane(to_f(r.x[x])) - (double)r.m) * r.k) / r.z;
}

template <typename T>
__device__ Row<T> read_row(const T *x, uint32_t V, float temp, double *buf) {
    Row<T> r{x, -INFINITY, 0.0, 0.0, -1};
    float m = -INFINITY;
    int best = 0x7FFFFFFF;
    for (uint32_t i = threadIdx.x; i < V; i += kVerThreads) { const float v = sane(to_f(x[i])); if (v > m) { m = v; best = i; } }
    for (int o = 32; o; o >>= 1) {
        const float m2 = __shfl_xor(m, o, 64);
        const int b2 = __shfl_xor(best, o, 64);
        if (m2 > m || (m2 == m && b2 < best)) { m = m2; best = b2; }
    }
    __shared__ float wm[kVerThreads / 64];
    __shared__ int wb[kVerThreads / 64];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { wm[threadIdx.x >> 6] = m; wb[threadIdx.x >> 6] = best; }
    __syncthreads();
    for (int w = 0; w < kVerThreads / 64; ++w)
        if (w == 0 || wm[w] > m || (wm[w] == m && wb[w] < best)) { m = wm[w]; best = wb[w]; }
    r.m = m;
    r.best = best;
    r.k = 1.0 / (double)fminf(temp, 1e30f);
    if (m == -INFINITY || !(temp > 0.f)) return r;
    double z = 0;
    for (uint32_t i = threadIdx.x; i < V; i += kVerThreads) z += exp(((double)sane(to_f(x[i])) - (double)m) * r.k);
    r.z = block_sum(z, buf);
    return r;
}

template <typename T>
__global__ __launch_bounds__(kVerThreads) void verify_tree_kernel(ps_verify_tree_args a) {
    __shared__ double buf[kVerThreads / 64];
    __shared__ int up[PS_TREE_MAX], refused[PS_TREE_MAX];
    __shared__ double part[kVerThreads];
    const uint32_t s = blockIdx.x, tid = threadIdx.x, V = a.vocab;
    const SeqRows sr = rows_of(a.first, s, a.n_tokens, a.max_tree);
    int32_t *path = a.path + s * a.path_seq;
    for (uint32_t i = tid; i < a.max_tree; i += kVerThreads) path[i] = -1;
    if (sr.n == 0) {
        if (tid == 0) { a.count[s] = 0; a.next_token[s] = -1; }
        return;
    }
    for (int i = tid; i < sr.n; i += kVerThreads) up[i] = parent_of(a.parent[sr.row0 + i], i);
    __syncthreads();
    const float temp = a.temperature ? a.temperature[s] : 1.f;
    const bool greedy = !(temp > 0.f), drafts = a.draft_logits && !greedy;
    int here = 0, n = 0;
    for (;;) {
        if (tid == 0) path[n] = here;
        ++n;
        const Row<T> p = read_row(static_cast<const T *>(a.target_logits) + ((size_t)sr.row0 + here) * a.target_row, V, temp, buf);
        Row<T> q{};
        if (drafts) q = read_row(static_cast<const T *>(a.draft_logits) + ((size_t)sr.row0 + here) * a.draft_row, V, temp, buf);
        double c = 0, w = 1;
        int went = -1, nref = 0, tried = 0;
        for (int i = here + 1; i < sr.n && went < 0 && tried < (int)a.max_children; ++i) {
            if (up[i] != here) continue;
            ++tried;
            const int x = a.token[sr.row0 + i];
            const double u = a.u_accept[sr.row0 + i], px = chance(p, x, V, temp);
            if (drafts) {
                if (px > (c + u * w) * chance(q, x, V, temp)) { went = i; break; }
                c += w;
                double left = 0;
                for (uint32_t j = tid; j < V; j += kVerThreads) left += fmax(chance(p, j, V, temp) - c * chance(q, j, V, temp), 0.0);
                w = block_sum(left, buf);
            } else {
                bool again = false;
                for (int r = 0; r < nref; ++r) again |= refused[r] == x;
                if (!again && px > u * w) { went = i; break; }
                if (!again && !greedy) {
                    __syncthreads();
                    if (tid == 0) refused[nref] = x;
                    __syncthreads();
                    ++nref;
                    w -= px;
                }
            }
        }
        if (went >= 0) { here = went; continue; }
        // draw: every thread sums a run of the vocabulary, thread 0 looks for the run, then for the index
        const uint32_t per = (V + kVerThreads - 1) / kVerThreads;
        for (int again = 0; again < 2; ++again) {
            auto left = [&](uint32_t j) {
                const double v = chance(p, j, V, temp);
                if (again) return v;
                for (int r = 0; r < nref; ++r) if (refused[r] == (int)j) return 0.0;
                return drafts ? fmax(v - c * chance(q, j, V, temp), 0.0) : v;
            };
            double sum = 0;
            for (uint32_t j = tid * per; j < min(V, (tid + 1) * per); ++j) sum += left(j);
            __syncthreads();
            part[tid] = sum;
            __syncthreads();
            double total = 0;
            for (int k = 0; k < kVerThreads; ++k) total += part[k];
            if (total <= 0 && !again) continue;
            if (tid == 0) {
                int pick = -1, last = -1;
                const double goal = (double)a.u_sample[s] * total;
                double run = 0;
                for (int k = 0; k < kVerThreads && pick < 0 && total > 0; ++k) {
                    if (run + part[k] <= goal && k + 1 < kVerThreads) { run += part[k]; continue; }
                    double r = run;
                    for (uint32_t j = k * per; j < min(V, (k + 1) * per); ++j) {
                        const double v = left(j);
                        if (v > 0) last = j;
                        r += v;
                        if (r > goal) { pick = j; break; }
                    }
                    run += part[k];
                }
                a.next_token[s] = pick >= 0 ? pick : last;
                a.count[s] = n;
            }
            break;
        }
        return;
    }
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
        uint4 v[16];
        bool ok[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const uint32_t idx = u * 64 + lane, i = idx / seg, col = c0 + idx % seg;
            ok[u] = (int)i < n && col < units;
            if (ok[u]) {
                const int node = path[i];
                const int64_t from = ctx + node, to = ctx + i;
                ok[u] = node >= 0 && node < (int)a.max_tree && from >= 0 && from < a.capacity && to >= 0 && to < a.capacity;
                if (ok[u]) v[u] = *reinterpret_cast<const uint4 *>(base + from * a.row_stride + col * 16);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const uint32_t idx = u * 64 + lane, i = idx / seg, col = c0 + idx % seg;
            if (ok[u]) *reinterpret_cast<uint4 *>(base + (ctx + i) * a.row_stride + col * 16) = v[u];
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
    *bytes = 0;
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
    const dim3 grid(a->max_tree, a->n_q_heads, a->n_seq);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->type == PS_TYPE_F16) {
        if (a->head_dim == 64) hipLaunchKernelGGL((tree_attention_kernel<f16_t, 64>), grid, dim3(64), 0, st, *a);
        else hipLaunchKernelGGL((tree_attention_kernel<f16_t, 128>), grid, dim3(64), 0, st, *a);
    } else {
        if (a->head_dim == 64) hipLaunchKernelGGL((tree_attention_kernel<bf16_t, 64>), grid, dim3(64), 0, st, *a);
        else hipLaunchKernelGGL((tree_attention_kernel<bf16_t, 128>), grid, dim3(64), 0, st, *a);
    }
    PS_TRY(hipGetLastError());
    return PS_OK;
}

int32_t ps_verify_tree_workspace(const ps_verify_tree_args *a, uint64_t *bytes) {
    PS_WANT(a && bytes, "NULL argument");
    PS_WANT(a->type <= PS_TYPE_F32, "unknown type %u", a->type);
    PS_WANT(a->vocab >= 1 && a->vocab <= 1u << 24, "vocab 1 .. 2^24 (got %u)", a->vocab);
    PS_WANT(a->max_tree <= PS_TREE_MAX, "trees of up to %u tokens (got %u)", PS_TREE_MAX, a->max_tree);
    PS_WANT(a->max_children >= 1 && a->max_children <= PS_TREE_MAX, "max_children 1 .. %u (got %u)", PS_TREE_MAX, a->max_children);
    PS_WANT(a->n_seq <= 65535 && a->n_tokens <= 0x7FFFFFFF, "%u sequences, %u tokens: too many", a->n_seq, a->n_tokens);
    *bytes = 0;
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
    const dim3 grid(a->n_seq);
    if (a->type == PS_TYPE_F16) hipLaunchKernelGGL(verify_tree_kernel<f16_t>, grid, dim3(kVerThreads), 0, st, *a);
    else if (a->type == PS_TYPE_BF16) hipLaunchKernelGGL(verify_tree_kernel<bf16_t>, grid, dim3(kVerThreads), 0, st, *a);
    else hipLaunchKernelGGL(verify_tree_kernel<float>, grid, dim3(kVerThreads), 0, st, *a);
    PS_TRY(hipGetLastError());
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
