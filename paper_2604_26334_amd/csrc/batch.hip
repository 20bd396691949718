// Operators of a step that answers a batch of requests over one paged cache: places of new tokens, their rows of the cache, attention
// over shared prefixes and own positions, and the draw of the next tokens.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "ps_internal.h"
#include "row_math.h"

namespace ps {

namespace {

constexpr uint32_t kMostSeqs = 65535, kMostTableSeqs = 8192, kMostPrefixes = 4096, kMostPage = 1024;
constexpr int kMostPositions = 1 << 30;

// ------------------------------------------------------------------------------------ places of new tokens
// Every workgroup works out the running sums of all sequences in LDS (first tokens, pages that they need in front) and then the places of
// its own tokens: a token finds its sequence by bisection, and one that begins a page takes the page for the table.  Sums end at n_tokens,
// which adding with an upper end keeps independent of the order.
constexpr uint32_t kTableThreads = 512;

// running sums in front of each of v[0 .. n), ends at `most` (v: non-negative, at most `most` <= 2^30); v[n] becomes the total
__device__ __forceinline__ void running(int *v, uint32_t n, int most, int *buf) {
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (n + kTableThreads - 1) / kTableThreads;
    const uint32_t lo = min(n, tid * per), hi = min(n, lo + per);
    int sum = 0;
    for (uint32_t i = lo; i < hi; ++i) sum = min(sum + v[i], most);
    int upto = sum;
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(upto, o, 64);
        if ((int)lane >= o) upto = min(upto + t, most);
    }
    if (lane == 63) buf[wave] = upto;
    const int prior = __shfl_up(upto, 1, 64);
    int from = lane ? prior : 0;
    __syncthreads();
    for (uint32_t w = 0; w < wave; ++w) from = min(from + buf[w], most);
    for (uint32_t i = lo; i < hi; ++i) {
        const int x = v[i];
        v[i] = from;
        from = min(from + x, most);
    }
    if (tid == kTableThreads - 1) v[n] = from;
    __syncthreads();
}

__global__ __launch_bounds__(kTableThreads) void page_tables_kernel(ps_page_tables_args a, uint32_t shift) {
    extern __shared__ int table_lds[];
    __shared__ int buf[kTableThreads / 64];
    const uint32_t tid = threadIdx.x, n = a.n_seq;
    int *const first = table_lds, *const need = table_lds + n + 1;
    const int page = 1 << shift;
    for (uint32_t s = tid; s < n; s += kTableThreads) first[s] = clampi(a.new_tokens[s], 0, (int)a.n_tokens);
    __syncthreads();
    running(first, n, (int)a.n_tokens, buf);
    for (uint32_t s = tid; s < n; s += kTableThreads) {
        const int64_t room = (int64_t)a.width << shift;
        const int cached = clampi(a.cached[s], 0, kMostPositions), length = min(cached + (first[s + 1] - first[s]), kMostPositions);
        const int held = (int)((min((int64_t)cached, room) + page - 1) >> shift), full = (int)((min((int64_t)length, room) + page - 1) >> shift);
        need[s] = full - held;
        if (blockIdx.x == 0) { a.first[s] = first[s]; a.length[s] = length; }
    }
    __syncthreads();
    running(need, n, kMostPositions, buf);
    if (blockIdx.x == 0 && tid == 0) { a.first[n] = first[n]; a.taken[0] = need[n]; }
    const int64_t free_at = a.free_at ? a.free_at[0] : 0;
    for (uint32_t t = blockIdx.x * kTableThreads + tid; t < (uint32_t)first[n]; t += gridDim.x * kTableThreads) {
        uint32_t s = 0;                       // the last sequence that begins at or in front of t: one with tokens
        for (uint32_t step = 1u << (31 - __clz(n)); step; step >>= 1)
            if (s + step < n && first[s + step] <= (int)t) s += step;
        const int cached = clampi(a.cached[s], 0, kMostPositions);
        const int64_t j = (int64_t)cached + ((int)t - first[s]);
        const int held = (cached + page - 1) >> shift;
        const int64_t entry = j >> shift;
        int number = -1;
        if (j < kMostPositions && entry < a.width) {
            int32_t *row = a.table + s * a.table_seq;
            if (entry < held) number = row[entry];
            else {
                const int64_t at = free_at + need[s] + (entry - held);
                if (at >= 0 && at < a.n_free) number = a.free_pages[at];
                if (number < 0 || number >= (int)a.n_pages) number = -1;
                if ((j & (page - 1)) == 0) row[entry] = number;
            }
            if (number < 0 || number >= (int)a.n_pages) number = -1;
        }
        a.slot[t] = number < 0 ? -1 : (number << shift) + (int)(j & (page - 1));
        if (a.position) a.position[t] = (int)((uint32_t)(a.offset ? a.offset[s] : 0) + (uint32_t)j);
    }
}

// ------------------------------------------------------------------------------------ rows of new tokens
__global__ __launch_bounds__(256) void page_append_kernel(ps_page_append_args a, uint32_t shift) {
    const uint32_t units = a.row_bytes / 16;
    const uint64_t items = (uint64_t)a.n_tokens * a.n_heads * 2 * units;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (uint64_t)gridDim.x * 256) {
        const uint32_t u = (uint32_t)(i % units), v = (uint32_t)(i / units % 2), h = (uint32_t)(i / units / 2 % a.n_heads), t = (uint32_t)(i / units / 2 / a.n_heads);
        const int slot = a.slot[t];
        if (slot < 0 || (uint32_t)(slot >> shift) >= a.n_pages) continue;
        const uint64_t number = (uint32_t)slot >> shift, row = slot & ((1 << shift) - 1);
        const char *from = v ? static_cast<const char *>(a.v) + t * a.v_token + h * a.v_head : static_cast<const char *>(a.k) + t * a.k_token + h * a.k_head;
        char *to = v ? static_cast<char *>(a.v_pages) + number * a.v_page + h * a.v_page_head + row * a.v_page_row
                     : static_cast<char *>(a.k_pages) + number * a.k_page + h * a.k_page_head + row * a.k_page_row;
        *reinterpret_cast<u4_t *>(to + u * 16) = *reinterpret_cast<const u4_t *>(from + u * 16);
    }
}

// ------------------------------------------------------------------------------------ attention
// a wave per (token, query head): 64 positions at a time, a lane's whole dot product each, then the values' dimensions by lane
template <typename T, int D>
__global__ __launch_bounds__(256) void page_attention_kernel(ps_page_attention_args a, uint32_t shift) {
    constexpr int E = D / 64;
    const uint32_t lane = threadIdx.x & 63, hb = (a.n_q_heads + 3) / 4;
    const uint32_t h = blockIdx.x % hb * 4 + (threadIdx.x >> 6), i = blockIdx.x / hb % a.max_tokens, s = blockIdx.x / hb / a.max_tokens;
    const int row0 = clampi(a.first[s], 0, (int)a.n_tokens), n = clampi(a.first[s + 1], 0, (int)a.n_tokens) - row0;
    if (h >= a.n_q_heads || (int)i >= n) return;
    const int length = clampi(a.length[s], 0, (int)a.max_length);
    int group = -1;
    for (uint32_t p0 = 0; p0 < a.n_prefix && group < 0; p0 += 64) {
        const uint32_t p = p0 + lane;
        const uint64_t in = __ballot(p < a.n_prefix && a.group_first[p] <= (int)s && (int)s < a.group_first[p + 1]);
        if (in) group = (int)p0 + __ffsll((unsigned long long)in) - 1;
    }
    const uint32_t hk = h / (a.n_q_heads / a.n_kv_heads);
    const size_t token = (size_t)row0 + i;
    const T *q = static_cast<const T *>(a.q) + token * a.q_token + h * a.q_head;
    float m = -INFINITY, l = 0.f, o[E] = {};
    for (int part = 0; part < 2; ++part) {
        if (part == 0 && group < 0) continue;
        const int limit = part ? max(0, length - n + (int)i + 1) : clampi(a.prefix_length[group], 0, (int)a.max_prefix);
        const int32_t *table = part ? a.table + s * a.table_seq : a.prefix_table + group * a.prefix_seq;
        for (int p0 = 0; p0 < limit; p0 += 64) {
            const int pos = p0 + (int)lane;
            const int number = pos < limit ? table[pos >> shift] : -1;
            const bool seen = number >= 0 && number < (int)a.n_pages;
            float z = -INFINITY;
            if (seen) {
                const T *k = static_cast<const T *>(a.k_pages) + number * a.k_page + hk * a.k_head + (uint64_t)(pos & ((1 << shift) - 1)) * a.k_row;
                float dot = 0.f;
                for (int d = 0; d < D; ++d) dot = fmaf(to_f(q[d]), to_f(k[d]), dot);
                z = dot * a.scale;
            }
            float top = z;
            for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
            top = fmaxf(top, m);
            const float base = top == -INFINITY ? 0.f : top, resc = expf(m - base), w = expf(z - base);
            m = top;
            l *= resc;
            float sum = w;
            for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x, 64);
            l += sum;
            for (int e = 0; e < E; ++e) o[e] *= resc;
            for (int j = 0; j < 64; ++j) {
                if (!__shfl((int)seen, j, 64)) continue;
                const float wj = __shfl(w, j, 64);
                const int nj = __shfl(number, j, 64), pj = p0 + j;
                const T *v = static_cast<const T *>(a.v_pages) + nj * a.v_page + hk * a.v_head + (uint64_t)(pj & ((1 << shift) - 1)) * a.v_row;
                for (int e = 0; e < E; ++e) o[e] = fmaf(wj, to_f(v[lane * E + e]), o[e]);
            }
        }
    }
    T *out = static_cast<T *>(a.out) + token * a.out_token + h * a.out_head;
    for (int e = 0; e < E; ++e) out[lane * E + e] = (T)(l == 0.f ? 0.f : o[e] / l);
}

// ------------------------------------------------------------------------------------ sampling
// Sums are whole numbers, so a run of the order is known by its count and its sum whatever order it was added in.  A border
// of the order (the first entry at which count or sum pass a goal) is found digit by digit of the logits' bits.
constexpr uint32_t kSampleThreads = 1024;

// bits that order as the values do: larger for larger logits
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);        // (-0 is 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
struct SampleRow { double k, unit; float m; uint32_t vocab; };
__device__ __forceinline__ uint64_t whole(double w, const SampleRow &r) { return (uint64_t)rint(w * r.unit); }

struct Border { uint32_t key, before, equal; uint64_t sum, each; };      // entries in front of those equal to the border's, their sum; a weight of these
struct SampleLds { uint32_t cnt[256]; unsigned long long sum[256]; uint32_t digit, before; unsigned long long total; uint32_t wave[16]; float top[16]; };

template <typename T, class Cond>
__device__ Border find_border(const T *x, const SampleRow &r, SampleLds &s, Cond passes) {
    Border b{0, 0, 0, 0, 0};
    uint32_t mask = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) { s.cnt[threadIdx.x] = 0; s.sum[threadIdx.x] = 0; }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < r.vocab; i += kSampleThreads) {
            const float v = sane(to_f(x[i]));
            const uint32_t key = order_of(v);
            if (v == -INFINITY || (key & mask) != b.key) continue;
            atomicAdd(&s.cnt[key >> shift & 255], 1u);
            atomicAdd(&s.sum[key >> shift & 255], (unsigned long long)whole(weight(v, r.m, r.k), r));
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t c = b.before;
            unsigned long long t = b.sum;
            int d = 255;
            while (d > 0 && !(s.cnt[d] && passes(c + s.cnt[d], (uint64_t)(t + s.sum[d])))) { c += s.cnt[d]; t += s.sum[d]; --d; }
            s.digit = d; s.before = c; s.total = t;
        }
        __syncthreads();
        b.key |= s.digit << shift;
        b.before = s.before;
        b.sum = s.total;
        mask |= 255u << shift;
        if (shift == 0) { b.equal = s.cnt[s.digit]; b.each = b.equal ? s.sum[s.digit] / b.equal : 0; }
    }
    __syncthreads();
    return b;
}
// how many of the entries equal to a border's it takes for the sum to pass: 1 .. equal
template <class Cond>
__device__ __forceinline__ uint32_t within(const Border &b, Cond passes) {
    uint32_t lo = 1, hi = max(1u, b.equal);
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (passes(b.before + mid, b.sum + mid * b.each)) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(ps_sample_args a, double unit) {
    __shared__ SampleLds s;
    const uint32_t row = blockIdx.x, tid = threadIdx.x;
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_row;
    float top = -INFINITY;
    for (uint32_t i = tid; i < a.vocab; i += kSampleThreads) top = fmaxf(top, sane(to_f(x[i])));
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if ((tid & 63) == 0) s.top[tid >> 6] = top;
    __syncthreads();
    for (int w = 0; w < 16; ++w) top = fmaxf(top, s.top[w]);
    if (top == -INFINITY) {
        if (tid == 0) { a.token[row] = -1; if (a.kept) a.kept[row] = 0; }
        return;
    }
    const float temp = a.temperature ? a.temperature[row] : 1.f;
    const bool greedy = !(temp > 0.f);
    const SampleRow r{greedy ? 0.0 : rate_of(temp), unit, top, a.vocab};
    uint32_t kept = 1, skip = 0, key = order_of(top);        // the token: entry number `skip` of those with this key
    if (!greedy) {
        auto all = [](uint32_t, uint64_t) { return false; };
        const Border last = find_border<T>(x, r, s, all);      // the least of all kept entries
        kept = last.before + last.equal;
        uint64_t sum = last.sum + last.equal * last.each;
        if (a.top_k && a.top_k[row] > 0 && (uint32_t)a.top_k[row] < kept) {
            const uint32_t most = a.top_k[row];
            auto cond = [=](uint32_t c, uint64_t) { return c >= most; };
            const Border b = find_border<T>(x, r, s, cond);
            kept = most;
            sum = b.sum + (most - b.before) * b.each;
        }
        uint32_t n = kept;
        uint64_t total = sum;
        if (a.top_p && a.top_p[row] < 1.f) {
            const double goal = (double)a.top_p[row] * (double)sum;
            auto cond = [=](uint32_t, uint64_t t) { return (double)t >= goal; };
            const Border b = find_border<T>(x, r, s, cond);
            const uint32_t j = within(b, cond);
            if (b.before + j < n) { n = b.before + j; total = b.sum + j * b.each; }
        }
        if (a.min_p && a.min_p[row] > 0.f) {
            const double least = a.min_p[row];
            if (tid == 0) { s.before = 0; s.total = 0; }
            __syncthreads();
            for (uint32_t i = tid; i < a.vocab; i += kSampleThreads) {
                const float v = sane(to_f(x[i]));
                if (v == -INFINITY) continue;
                const double w = weight(v, top, r.k);
                if ((v == top ? 1.0 : w) >= least) { atomicAdd(&s.before, 1u); atomicAdd(&s.total, (unsigned long long)whole(w, r)); }
            }
            __syncthreads();
            if (s.before == 0) { n = 1; total = whole(weight(top, top, r.k), r); }
            else if (s.before < n) { n = s.before; total = s.total; }
        }
        kept = n;
        const double goal = (double)a.u[row] * (double)total;
        auto cond = [=](uint32_t c, uint64_t t) { return (double)t > goal || c >= n; };
        const Border b = find_border<T>(x, r, s, cond);
        key = b.key;
        skip = within(b, cond) - 1;
    }
    if (a.kept && tid == 0) a.kept[row] = (int)kept;
    for (uint32_t i0 = 0, seen = 0; i0 < a.vocab; i0 += kSampleThreads) {
        const uint32_t i = i0 + tid;
        const bool is = i < a.vocab && order_of(sane(to_f(x[i]))) == key;
        const uint64_t same = __ballot(is);
        __syncthreads();
        if ((tid & 63) == 0) s.wave[tid >> 6] = __popcll(same);
        __syncthreads();
        uint32_t at = seen + __popcll(same & ((1ull << (tid & 63)) - 1));
        for (uint32_t w = 0; w < 16; ++w) { at += w < tid >> 6 ? s.wave[w] : 0; seen += s.wave[w]; }
        if (is && at == skip) a.token[row] = (int)i;
        if (seen > skip) return;
    }
}

bool power_of_two(uint32_t v) { return v && (v & (v - 1)) == 0; }
uint32_t log2_of(uint32_t v) { return 31 - (uint32_t)__builtin_clz(v); }

int32_t check_page_attention(const ps_page_attention_args *a) {
    PS_WANT(a, "NULL argument");
    PS_WANT(a->type <= PS_TYPE_BF16, "attention over pages takes fp16 or bf16 (type %u)", a->type);
    PS_WANT(a->head_dim == 64 || a->head_dim == 128, "attention over pages takes head_dim 64 or 128 (got %u)", a->head_dim);
    PS_WANT(a->n_kv_heads && a->n_q_heads && a->n_q_heads % a->n_kv_heads == 0 && a->n_q_heads <= 1024,
            "%u query heads over %u kv heads: a multiple of the kv heads, at most 1024", a->n_q_heads, a->n_kv_heads);
    PS_WANT(power_of_two(a->page) && a->page >= 16 && a->page <= kMostPage, "pages of a power of two positions, 16 .. %u (got %u)", kMostPage, a->page);
    PS_WANT(a->n_seq <= kMostSeqs && a->n_tokens <= 0x7FFFFFFF && a->n_pages <= 0x7FFFFFFF, "%u sequences, %u tokens, %u pages: too many", a->n_seq, a->n_tokens, a->n_pages);
    PS_WANT(a->n_prefix <= kMostPrefixes, "up to %u prefixes (got %u)", kMostPrefixes, a->n_prefix);
    PS_WANT(a->max_length <= (uint32_t)kMostPositions && a->max_length <= (uint64_t)a->width * a->page, "lengths of up to %u in tables of %u pages of %u", a->max_length, a->width, a->page);
    PS_WANT(!a->n_prefix || (a->max_prefix <= (uint32_t)kMostPositions && a->max_prefix <= (uint64_t)a->prefix_width * a->page), "prefixes of up to %u in tables of %u pages of %u", a->max_prefix,
            a->prefix_width, a->page);
    return PS_OK;
}

template <typename T, int D>
hipError_t launch_page_attention(const ps_page_attention_args &a, hipStream_t st) {
    const uint64_t groups = (uint64_t)a.n_seq * a.max_tokens * ((a.n_q_heads + 3) / 4);
    if (groups > kMostGroups) return hipErrorInvalidValue;
    hipLaunchKernelGGL((page_attention_kernel<T, D>), dim3((uint32_t)groups), dim3(256), 0, st, a, log2_of(a.page));
    return hipGetLastError();
}
template <typename T>
hipError_t launch_sample(const ps_sample_args &a, hipStream_t st) {
    const uint32_t bits = a.vocab > 1 ? log2_of(a.vocab - 1) + 1 : 0;
    hipLaunchKernelGGL(sample_kernel<T>, dim3(a.n_rows), dim3(kSampleThreads), 0, st, a, std::ldexp(1.0, 62 - (int)bits));
    return hipGetLastError();
}

}  // namespace
}  // namespace ps

using namespace ps;

extern "C" {

int32_t ps_page_tables(const ps_page_tables_args *a, void *stream) {
    PS_WANT(a, "NULL argument");
    PS_WANT(power_of_two(a->page) && a->page >= 16 && a->page <= kMostPage, "pages of a power of two positions, 16 .. %u (got %u)", kMostPage, a->page);
    PS_WANT(a->n_seq <= kMostTableSeqs, "up to %u sequences (got %u)", kMostTableSeqs, a->n_seq);
    PS_WANT(a->n_tokens <= (uint32_t)kMostPositions && (uint64_t)a->n_pages * a->page <= 1ull << 31, "%u tokens, %u pages of %u: too many", a->n_tokens, a->n_pages, a->page);
    PS_WANT(a->first && a->taken, "NULL argument");
    PS_WANT(a->n_seq == 0 || (a->cached && a->new_tokens && a->length), "NULL argument");
    PS_WANT(a->n_seq == 0 || a->n_tokens == 0 || (a->slot && (a->table || !a->width) && (a->free_pages || !a->n_free)), "NULL argument");
    PS_WANT(a->table_seq >= a->width || a->n_seq <= 1, "rows of %u entries lie %llu apart", a->width, (unsigned long long)a->table_seq);
    for (const void *p : {(const void *)a->cached, (const void *)a->new_tokens, (const void *)a->offset, (const void *)a->free_pages, (const void *)a->free_at, (const void *)a->table,
                          (const void *)a->first, (const void *)a->length, (const void *)a->position, (const void *)a->slot, (const void *)a->taken})
        PS_WANT(aligned(p, 4), "tables must be aligned to 4 bytes");
    const uint32_t groups = std::min(1024u, std::max(1u, (a->n_tokens + kTableThreads - 1) / kTableThreads));
    const uint32_t lds = (a->n_seq + 1) * 2 * 4;
    static std::atomic<uint64_t> done;
    int dev = 0;
    PS_TRY(hipGetDevice(&dev));
    if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
        PS_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(&page_tables_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (kMostTableSeqs + 1) * 2 * 4));
        if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    hipLaunchKernelGGL(page_tables_kernel, dim3(groups), dim3(kTableThreads), lds, static_cast<hipStream_t>(stream), *a, log2_of(a->page));
    PS_TRY(hipGetLastError());
    return PS_OK;
}

int32_t ps_page_append(const ps_page_append_args *a, void *stream) {
    PS_WANT(a, "NULL argument");
    PS_WANT(power_of_two(a->page) && a->page >= 16 && a->page <= kMostPage, "pages of a power of two positions, 16 .. %u (got %u)", kMostPage, a->page);
    PS_WANT(a->row_bytes >= 16 && a->row_bytes <= 4096 && a->row_bytes % 16 == 0, "row_bytes must be a multiple of 16, up to 4096 (got %u)", a->row_bytes);
    PS_WANT(a->n_tokens <= (uint32_t)kMostPositions && a->n_heads <= 65535 && (uint64_t)a->n_pages * a->page <= 1ull << 31, "%u tokens, %u heads, %u pages of %u: too many", a->n_tokens,
            a->n_heads, a->n_pages, a->page);
    if (a->n_tokens == 0 || a->n_heads == 0 || a->n_pages == 0) return PS_OK;
    PS_WANT(a->k && a->v && a->k_pages && a->v_pages && a->slot, "NULL argument");
    for (const void *p : {a->k, a->v, (const void *)a->k_pages, (const void *)a->v_pages}) PS_WANT(aligned(p, 16), "k, v and the pages must be 16-byte aligned");
    for (uint64_t n : {a->k_token, a->k_head, a->v_token, a->v_head, a->k_page, a->k_page_head, a->k_page_row, a->v_page, a->v_page_head, a->v_page_row})
        PS_WANT(n % 16 == 0, "strides must be multiples of 16 bytes (got %llu)", (unsigned long long)n);
    PS_WANT(aligned(a->slot, 4), "slot must be aligned to 4 bytes");
    const uint64_t items = (uint64_t)a->n_tokens * a->n_heads * 2 * (a->row_bytes / 16);
    const uint32_t groups = (uint32_t)std::min<uint64_t>((items + 255) / 256, kMostGroups);
    hipLaunchKernelGGL(page_append_kernel, dim3(groups), dim3(256), 0, static_cast<hipStream_t>(stream), *a, log2_of(a->page));
    PS_TRY(hipGetLastError());
    return PS_OK;
}

int32_t ps_page_attention_workspace(const ps_page_attention_args *a, uint64_t *bytes) {
    PS_WANT(bytes, "NULL argument");
    const int32_t rc = check_page_attention(a);
    if (rc) return rc;
    *bytes = 0;
    return PS_OK;
}

int32_t ps_page_attention(const ps_page_attention_args *a, void *workspace, uint64_t workspace_bytes, void *stream) {
    uint64_t need = 0;
    const int32_t rc = ps_page_attention_workspace(a, &need);
    if (rc) return rc;
    if (a->n_seq == 0 || a->n_tokens == 0 || a->max_tokens == 0) return PS_OK;
    PS_WANT(a->q && a->out && a->first && a->length, "NULL argument");
    PS_WANT(!a->max_length || !a->n_pages || (a->table && a->k_pages && a->v_pages), "the table or the pages are NULL");
    PS_WANT(!a->n_prefix || (a->group_first && a->prefix_length && (!a->max_prefix || !a->n_pages || (a->prefix_table && a->k_pages && a->v_pages))), "the prefixes' tables or the pages are NULL");
    PS_WANT(std::isfinite(a->scale), "scale must be finite");
    for (const void *p : {a->q, a->k_pages, a->v_pages, (const void *)a->out}) PS_WANT(aligned(p, 16), "q, the pages and out must be 16-byte aligned");
    for (uint64_t n : {a->q_token, a->q_head, a->k_page, a->k_head, a->k_row, a->v_page, a->v_head, a->v_row, a->out_token, a->out_head})
        PS_WANT(n % 8 == 0, "strides must be multiples of 16 bytes (got %llu elements)", (unsigned long long)n);
    for (uint64_t n : {a->k_row, a->v_row}) PS_WANT(n <= (1ull << 30) / 16, "16 rows of a page must span less than 2 GiB (stride of %llu elements)", (unsigned long long)n);
    for (const int32_t *p : {a->first, a->length, a->table, a->group_first, a->prefix_length, a->prefix_table}) PS_WANT(aligned(p, 4), "tables must be aligned to 4 bytes");
    PS_WANT(workspace_bytes >= need && (need == 0 || (workspace && aligned(workspace, kAlign))), "a workspace of %llu bytes, 256-byte aligned, is needed", (unsigned long long)need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->type == PS_TYPE_F16) PS_TRY(a->head_dim == 64 ? (launch_page_attention<f16_t, 64>(*a, st)) : (launch_page_attention<f16_t, 128>(*a, st)));
    else PS_TRY(a->head_dim == 64 ? (launch_page_attention<bf16_t, 64>(*a, st)) : (launch_page_attention<bf16_t, 128>(*a, st)));
    return PS_OK;
}

int32_t ps_sample_workspace(const ps_sample_args *a, uint64_t *bytes) {
    PS_WANT(a && bytes, "NULL argument");
    PS_WANT(a->type <= PS_TYPE_F32, "unknown type %u", a->type);
    PS_WANT(a->vocab >= 1 && a->vocab <= 1u << 24, "vocab 1 .. 2^24 (got %u)", a->vocab);
    PS_WANT(a->n_rows <= 65535, "up to 65535 rows (got %u)", a->n_rows);
    *bytes = 0;
    return PS_OK;
}

int32_t ps_sample(const ps_sample_args *a, void *workspace, uint64_t workspace_bytes, void *stream) {
    uint64_t need = 0;
    const int32_t rc = ps_sample_workspace(a, &need);
    if (rc) return rc;
    if (a->n_rows == 0) return PS_OK;
    PS_WANT(a->logits && a->u && a->token, "NULL argument");
    PS_WANT(aligned(a->logits, type_bytes(a->type)), "logits must be aligned to an element");
    for (const void *p : {(const void *)a->u, (const void *)a->temperature, (const void *)a->top_k, (const void *)a->top_p, (const void *)a->min_p, (const void *)a->token, (const void *)a->kept})
        PS_WANT(aligned(p, 4), "settings, random numbers and outputs must be aligned to 4 bytes");
    PS_WANT(workspace_bytes >= need && (need == 0 || (workspace && aligned(workspace, kAlign))), "a workspace of %llu bytes, 256-byte aligned, is needed", (unsigned long long)need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->type == PS_TYPE_F16) PS_TRY(launch_sample<f16_t>(*a, st));
    else if (a->type == PS_TYPE_BF16) PS_TRY(launch_sample<bf16_t>(*a, st));
    else PS_TRY(launch_sample<float>(*a, st));
    return PS_OK;
}

}  // extern "C"
