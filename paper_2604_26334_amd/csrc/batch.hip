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
// which adding with an upper end keeps independent of the order.  Bound by its chain of latencies, two sums and a few dependent loads: 64 sequences
// of a token 4.4 us, 1000 sequences of up to 130 tokens 6.8.
constexpr uint32_t kTableThreads = 512;

// a + b, but at most `most` (each of the three 0 .. 2^30: two of them pass the signed range)
__device__ __forceinline__ int capped(int a, int b, int most) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)most); }

// running sums in front of each of v[0 .. n), ends at `most` (v: non-negative, at most `most` <= 2^30); v[n] becomes the total
__device__ __forceinline__ void running(int *v, uint32_t n, int most, int *buf) {
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (n + kTableThreads - 1) / kTableThreads;
    const uint32_t lo = min(n, tid * per), hi = min(n, lo + per);
    int sum = 0;
    for (uint32_t i = lo; i < hi; ++i) sum = capped(sum, v[i], most);
    int upto = sum;
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(upto, o, 64);
        if ((int)lane >= o) upto = capped(upto, t, most);
    }
    if (lane == 63) buf[wave] = upto;
    const int prior = __shfl_up(upto, 1, 64);
    int from = lane ? prior : 0;
    __syncthreads();
    for (uint32_t w = 0; w < wave; ++w) from = capped(from, buf[w], most);
    for (uint32_t i = lo; i < hi; ++i) {
        const int x = v[i];
        v[i] = from;
        from = capped(from, x, most);
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
        const int cached = clampi(a.cached[s], 0, kMostPositions), length = capped(cached, first[s + 1] - first[s], kMostPositions);
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
// A thread moves 16 bytes.  Bound by memory: 16384 tokens of 8 heads of 128 (134 MB) 21.5 us = 6.2 TB/s, what is written staying in the
// caches; 64 tokens 3.0 us, a launch's own time.
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
// Score rows are (token, query head of the kv group) pairs.  Two forms of a task, a workgroup of four waves each:
//  rows_few   up to NT x 16 rows over a run of positions: the waves take tiles of 32 positions in turn, each with a running maximum,
//             weight sum and value sums of its own, and meet in LDS at the end.  Bound by the cache's bytes.
//  rows_many  128 rows, 32 a wave, over a run of steps of 64 positions, whose K and V rows all four waves read from LDS (two stages, one
//             barrier a step, rows requested two steps ahead).  Bound by matrix products and exponentials.
// Products:
//  scores, transposed: S^T = K Q^T, A = 16 positions x 32 dims of K, B = 16 rows of queries: lane (row i, c) then holds four positions of
//   row i, 4 c .. 4 c + 3 of each half tile of 16;
//  weights x values, transposed: O^T = V^T P^T, B = the weights exactly as the score accumulators hold them, A = 16 dims x 32 positions of V
//   by LDS transpose reads of rows 4 c .. 4 c + 3 of each half; and the weights' sum by one more product, with ones.
// Half a tile never crosses a page (pages are multiples of 16 positions), so it has one address, and all of its rows lie in the pool: they are
// read even where the sequence ends among them (page 0 where the table names none), their scores are then hidden and their values taken as zeros.
// A wave keeps the next 64 entries of its table in a register, one a lane.
// Sequences of few tokens (up to 32 rows of a kv head): a group's prefix is walked once for all of its rows (rows_many, or rows_few where the
// whole group has few), and each sequence's own positions by rows_few; both in one launch, so that a CU holds products and loads at the
// same time, and a merge of their records.  More tokens: blocks of 128 rows walk prefix and own positions one after the other.
// Measured: own positions alone, 48 sequences of up to 8190 (16 / 8 heads of 64) 102 us = 5.3 TB/s; 64 sequences behind a prefix of 32761 (32 / 8
// heads), own lengths up to 1000, 91 us: about 60 for the prefix's products and 34 for the own positions' bytes when each runs alone; prompts, 2 of 2048
// tokens behind 16384 positions, 798 TFLOP/s, 8 of 512 behind 2048 198 to 206 us = 720 to 750: the matrix cores are busy 37 % of the CUs' time and the vector
// instructions of the softmax, which share their issue port, 46 %.
// All of a call goes one way, by its bounds: 64 sequences behind 32761 (32 / 8 heads, own 1000) take 388 us with 8 tokens each, 32 rows, and 1203 with 9.
constexpr uint32_t kTile = 32, kStep = 64;
constexpr uint32_t kFewRows = 32;

// 16-byte piece u of a staged row lies in slot u ^ swizzle, so that the rows that are read together lie in different banks: V rows 0 .. 7 (in
// pairs of pieces), K rows 0 .. 15
template <int D> __device__ __forceinline__ uint32_t v_slot(uint32_t row) { return D == 128 ? (row & 7u) << 1 : (row >> 1 & 3u) << 1; }
template <int D> __device__ __forceinline__ uint32_t k_slot(uint32_t row) { return D == 128 ? row & 15u : row >> 1 & 7u; }

struct PageDeal {
    uint32_t shared;             // 1: prefixes for all their tokens at once; 0: with each sequence's own positions
    uint32_t nt;                 // rows of a sequence, in 16; 0: in blocks of 128
    uint32_t blocks;             // of 128 rows: of all groups at most (shared), of a sequence
    uint32_t psplit, plen;       // runs of a prefix, positions of a run (shared)
    uint32_t osplit, olen;       // runs of own positions (shared), or of a sequence's tiles (nt) or steps
    uint32_t direct;             // no records: the result itself
    // Tokens that may be answered, for each of which there is a place for records.  The arrays may have room for more (rows behind the last sequence, tokens
    // beyond max_tokens): by_seq, places are then numbered by sequence and number in it, and a prefix's workgroups, as many as the tokens that may be answered fill,
    // look for blocks from `blocks` on, up to `most`.
    uint32_t tokens, by_seq, most;
};
template <int D, int NT> constexpr uint32_t few_lds() { return std::max<uint32_t>(4 * kTile * D * 2, 4 * NT * 16 * (D + 4) * 4 + 4 * NT * 16 * 2 * 4) + 16; }
template <int D> constexpr uint32_t many_lds() { return 2 * 2 * kStep * D * 2 + 16; }

struct RowSet {                                                  // rows of consecutive tokens, `group` query heads each
    int token0;
    uint32_t rows, group;
    uint32_t seq0, seqs;                                         // whose tokens they are (by_seq, of a group)
};
struct Span {                                                    // positions that one table names
    const int32_t *table;
    int entries, len;                                            // entries of the table, positions
};

// By sequence and number in it, the place of a token's records; -1: it has none.  (Below n_seq * max_tokens, whatever `first` holds)
__device__ __forceinline__ int place_of(const ps_page_attention_args &a, const RowSet &set, int token) {
    uint32_t s = set.seq0;                    // the last one that begins at or in front of the token: one with tokens
    for (uint32_t n = set.seqs; n > 1;) {
        const uint32_t half = n / 2;
        const bool behind = clampi(a.first[s + half], 0, (int)a.n_tokens) <= token;
        s = behind ? s + half : s;
        n = behind ? n - half : half;
    }
    const int i = token - clampi(a.first[s], 0, (int)a.n_tokens);
    return i >= 0 && (uint32_t)i < a.max_tokens ? (int)(s * a.max_tokens) + i : -1;
}
// The records as those of a sequence's tokens are found in them: token row0's at the sequence's first place
__device__ __forceinline__ float *records_of(const ps_page_attention_args &a, const PageDeal &d, uint32_t s, int row0, uint32_t floats, float *part) {
    return part + ((int64_t)s * a.max_tokens - row0) * a.n_q_heads * (int64_t)(d.psplit + d.osplit) * floats;
}

// page numbers of a table, 64 at a time, one a lane; -1: none
struct PageWindow {
    int number, base;
    __device__ __forceinline__ void fill(const Span &s, int entry, uint32_t n_pages) {
        base = entry;
        const int at = entry + (int)(threadIdx.x & 63);
        number = at < s.entries ? s.table[at] : -1;
        if (number < 0 || number >= (int)n_pages) number = -1;
    }
    __device__ __forceinline__ int operator()(int entry) const { return __builtin_amdgcn_readlane(number, entry - base); }
};

// Where the positions from P on of one kv head lie, as far as the page goes (strides between pages are less than 2^32 pieces of 16 bytes, a
// page's rows and 32 rows span less than 2^32 bytes)
struct PageRows {
    const char *k, *v;
    __device__ __forceinline__ PageRows(const ps_page_attention_args &a, const char *kc, const char *vc, int number, int P, uint32_t mask) {
        const uint32_t page = (uint32_t)max(number, 0), row = (uint32_t)P & mask;
        k = kc + ((uint64_t)page * (uint32_t)(a.k_page / 8) << 4) + row * (uint32_t)(a.k_row * 2);
        v = vc + ((uint64_t)page * (uint32_t)(a.v_page / 8) << 4) + row * (uint32_t)(a.v_row * 2);
    }
};
__device__ __forceinline__ u4_t piece_of(const char *rows, uint32_t offset) { return *reinterpret_cast<const u4_t *>(rows + offset); }

// Values that are infinite or no number and that a row sees: what the products had zeros for (positions from .. to - 1 of a span)
template <typename T, int N>
__device__ __forceinline__ void add_wild(const ps_page_attention_args &a, const Span &s, uint32_t shift, uint32_t hk, int from, int to, uint32_t d0, float (&o)[N]) {
    for (int j = from; j < to; ++j) {
        const int number = s.table[j >> shift];
        if (number < 0 || number >= (int)a.n_pages) continue;
        const T *v = static_cast<const T *>(a.v_pages) + (uint64_t)number * a.v_page + hk * a.v_head + (uint64_t)((uint32_t)j & ((1u << shift) - 1)) * a.v_row + d0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float x = to_f(v[e]);
            if (!(fabsf(x) < INFINITY)) o[e] += x;
        }
    }
}

// Rows of `set` (up to NT x 16) over tiles lo .. hi - 1 of a span's positions up to `end`, of which row rho sees those below limit0 + rho / group; `window` holds
// the table's entries from the wave's first tile on.  kBoth: over tiles of `prefix`, which every row sees, and then those of the span.  kSeek: records by place_of.
template <typename T, int D, int NT, bool kBoth, bool kSeek = false>
__device__ __forceinline__ void rows_few(const ps_page_attention_args &a, const RowSet &set, const Span &prefix, const Span &span, uint32_t shift, uint32_t hk, int lo, int hi, int end,
                                         int limit0, PageWindow window, uint32_t records, uint32_t z, float *part, unsigned char *lds) {
    using M = Mfma<T>;
    using v8 = typename M::v8;
    constexpr int KK = D / 32, DT = D / 16, RB = NT * 16, OP = D + 4;
    constexpr uint32_t kStage = kTile * D * 2, kRowPieces = D / 8, kVLoads = kStage / 1024;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t i = lane & 15, c = lane >> 4, R = set.rows, G = set.group, mask = (1u << shift) - 1;
    int *const wild = reinterpret_cast<int *>(lds + few_lds<D, NT>() - 16);      // some value of the last tiles is infinite or no number
    const uint32_t krow_b = (uint32_t)a.k_row * 2, vrow_b = (uint32_t)a.v_row * 2;
    const char *const kc = static_cast<const char *>(a.k_pages) + hk * a.k_head * 2, *const vc = static_cast<const char *>(a.v_pages) + hk * a.v_head * 2;
    unsigned char *const stage = lds + wave * kStage;
    const uint32_t vrow = lane / kRowPieces;
    u4_t kreg[2][KK], vreg[kVLoads];
    uint32_t gone = 0;                         // halves of the requested tile that no page holds
    const int np = kBoth ? (prefix.len + (int)kTile - 1) / (int)kTile : 0;
    int held = kBoth ? -1 : 1;                 // which table the window is of
    auto request = [&](int tile) {
        const bool mine = !kBoth || tile >= np;
        const int P = (tile - (mine ? np : 0)) * (int)kTile, last = (mine ? end : prefix.len) - 1;
        if (held != (int)mine || ((P + 31) >> shift) - window.base >= 64) {
            window.fill(mine ? span : prefix, P >> shift, a.n_pages);
            held = mine;
        }
        gone = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int number = window(min(P + h * 16, last) >> shift);
            if (number < 0) gone |= 1u << h;
            const PageRows rows(a, kc, vc, number, P + h * 16, mask);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kreg[h][kk] = piece_of(rows.k, i * krow_b + c * 16 + kk * 64);
#pragma unroll
            for (uint32_t u = h * kVLoads / 2; u < (h + 1) * kVLoads / 2; ++u) {
                const uint32_t row = u * (64 / kRowPieces) + vrow;
                vreg[u] = piece_of(rows.v, (row & 15) * vrow_b + ((lane % kRowPieces) ^ v_slot<D>(row)) * 16);
            }
        }
    };
    int tile = lo + (int)wave;
    if (tile < hi) request(tile);
    if (tid == 0) *wild = 0;
    __syncthreads();

    // the rows of queries; a negative scale turns their signs
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    const float c2 = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-30f);     // weights are 2^(c2 (s - m))
    const float slack = WeightRange<T>::kSlack / c2;
    int limit[NT];
    v8 q[NT][KK];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t rho = min(t * 16 + i, R - 1), tok = rho / G;
        limit[t] = limit0 + (int)tok;
        const T *qr = static_cast<const T *>(a.q) + ((size_t)set.token0 + tok) * a.q_token + (size_t)(hk * G + rho % G) * a.q_head + c * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) q[t][kk] = __builtin_bit_cast(v8, *reinterpret_cast<const u4_t *>(qr + kk * 32) ^ u4_t{sign, sign, sign, sign});
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
        const uint32_t row = 4 * c + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vread[dt] = row * (D * 2) + (((2 * dt + ((i & 3) >> 1)) ^ v_slot<D>(row)) << 4) + (i & 1) * 8;
    }
    const int wild0 = max(limit0, 0) & ~(int)(kTile - 1);        // from here on not every row sees every position
    for (; tile < hi; tile += 4) {
        const bool mine = !kBoth || tile >= np;
        const int P0 = (tile - (mine ? np : 0)) * (int)kTile, stop = mine ? end : prefix.len;
        const uint32_t missing = gone;
        f4_t S[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t][0] = S[t][1] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t][h] = M::mul(__builtin_bit_cast(v8, kreg[h][kk]), q[t][kk], S[t][h]);
        if (missing || P0 + (int)kTile > stop) {
            asm volatile("");
#pragma unroll
            for (uint32_t u = 0; u < kVLoads; ++u) {
                const uint32_t row = u * (64 / kRowPieces) + vrow;
                vreg[u] = P0 + (int)row < stop && !(missing >> (2 * u / kVLoads) & 1) ? vreg[u] : u4_t{0, 0, 0, 0};
            }
        }
        if (mine && P0 >= wild0) {
            bool odd = false;
#pragma unroll
            for (uint32_t u = 0; u < kVLoads; ++u) odd |= made_finite<T>(vreg[u]);
            if (odd) *wild = 1;
        }
#pragma unroll
        for (uint32_t u = 0; u < kVLoads; ++u) *reinterpret_cast<u4_t *>(stage + u * 1024 + lane * 16) = vreg[u];
        if (tile + 4 < hi) request(tile + 4);
        if (missing || P0 + (int)kTile > stop || (mine && P0 + (int)kTile > limit0)) {
            asm volatile("");
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int last = (mine ? min(stop, limit[t]) : stop) - P0 - 4 * (int)c;
#pragma unroll
                for (int e = 0; e < 8; ++e) S[t][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < last && !(missing >> (e >> 2) & 1) ? S[t][e >> 2][e & 3] : -INFINITY;
            }
        }
        v8 P[NT];
        weigh<T>(S, m_run, L, O, P, c2, slack);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const v8 vr = __builtin_bit_cast(v8, transposed(stage + vread[dt], 16 * D * 2));
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
    constexpr uint32_t kPerRow = D / 4;
    for (uint32_t u = tid; u < RB * kPerRow; u += 256) {
        const uint32_t rho = u / kPerRow, d0 = u % kPerRow * 4;
        if (rho >= R) break;
        float mx = om[rho];
#pragma unroll
        for (int w = 1; w < 4; ++w) mx = fmaxf(mx, om[w * RB + rho]);
        float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = om[w * RB + rho];
            // a wave that saw nothing of this row holds zeros and weighs nothing; one whose scores are no numbers holds none, and says so
            const float f = mw == -INFINITY ? (mx == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f((mw - mx) * c2);
            l = fmaf(f, ol[w * RB + rho], l);
            const f4_t v = *reinterpret_cast<const f4_t *>(ob + (w * RB + rho) * OP + d0);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[e], o[e]);
        }
        const uint32_t tok = rho / G, h = hk * G + rho % G;
        if (*wild) add_wild<T>(a, span, shift, hk, max((lo - np) * (int)kTile, wild0), min(min((hi - np) * (int)kTile, end), limit0 + (int)tok), d0, o);
        const size_t token = (size_t)set.token0 + tok;
        if (records) {
            const int place = kSeek ? place_of(a, set, (int)token) : 0;
            if (place < 0) continue;
            float *dst = part + (((kSeek ? (size_t)place : token) * a.n_q_heads + h) * records + z) * OP;
            *reinterpret_cast<f4_t *>(dst + d0) = f4_t{o[0], o[1], o[2], o[3]};
            if (d0 == 0) *reinterpret_cast<float2 *>(dst + D) = make_float2(mx * c2, l);
        } else {
            T r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (T)(l == 0.f ? 0.f : o[e] / l);
            *reinterpret_cast<u2_t *>(static_cast<T *>(a.out) + token * a.out_token + h * a.out_head + d0) = *reinterpret_cast<const u2_t *>(r);
        }
    }
}

// Rows row0 .. row0 + 127 of `set` over steps lo .. hi - 1: those of `prefix` (which every row sees), then those of `own` (row rho sees
// positions below limit0 + rho / group).  kOwn false: a prefix alone.  kSeek: records by place_of.
template <typename T, int D, bool kOwn, bool kSeek = false>
__device__ __forceinline__ void rows_many(const ps_page_attention_args &a, const RowSet &set, uint32_t row0, const Span &prefix, const Span &own, uint32_t shift, uint32_t hk,
                                          int lo, int hi, int limit0, uint32_t records, uint32_t z, float *part, unsigned char *lds) {
    using M = Mfma<T>;
    using v8 = typename M::v8;
    constexpr int KK = D / 32, DT = D / 16, NT = 2, OP = D + 4;
    constexpr uint32_t kHalf = kStep * D * 2, kRowPieces = D / 8, kLoads = kStep * kRowPieces / 256;     // a step's K (or V) rows; pieces a thread moves of them
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t i = lane & 15, c = lane >> 4, R = set.rows, G = set.group, mask = (1u << shift) - 1;
    int *const wild = reinterpret_cast<int *>(lds + many_lds<D>() - 16);
    const uint32_t krow_b = (uint32_t)a.k_row * 2, vrow_b = (uint32_t)a.v_row * 2;
    const char *const kc = static_cast<const char *>(a.k_pages) + hk * a.k_head * 2, *const vc = static_cast<const char *>(a.v_pages) + hk * a.v_head * 2;
    const int np = (prefix.len + (int)kStep - 1) / (int)kStep;
    const uint32_t mine0 = row0 + wave * (NT * 16);      // the wave's rows
    const bool rows = mine0 < R;
    // own positions: every row of the block sees those below `least`, none sees `own_end` and beyond, no row of the wave `wave_end`
    const int least = limit0 + (int)(row0 / G), own_end = min(own.len, limit0 + (int)(min(row0 + 127, R - 1) / G));
    const int wave_least = limit0 + (int)(min(mine0, R - 1) / G), wave_end = limit0 + (int)(min(mine0 + 31, R - 1) / G);
    const int wild0 = max(least, 0) & ~(int)(kStep - 1);

    // a thread's piece of its first row of a step (further ones: a multiple of 16 rows on, with the same swizzle)
    const uint32_t kpiece = tid / kRowPieces * krow_b + ((tid % kRowPieces) ^ k_slot<D>(tid / kRowPieces)) * 16;
    const uint32_t vpiece = tid / kRowPieces * vrow_b + ((tid % kRowPieces) ^ v_slot<D>(tid / kRowPieces)) * 16;
    u4_t kreg[kLoads], vreg[kLoads];
    PageWindow window{-1, 1 << 30};
    int held = -1;                                       // which table the window is of
    uint32_t gone = 0;                                   // halves of the requested step that no page holds
    auto request = [&](int step) {
        const bool mine = kOwn && step >= np;
        const Span &s = mine ? own : prefix;
        const int P = (mine ? step - np : step) * (int)kStep, end = mine ? own_end : prefix.len;
        if (held != (int)mine || ((P + 63) >> shift) - window.base >= 64) {
            window.fill(s, P >> shift, a.n_pages);
            held = mine;
        }
        gone = 0;
        if (shift >= 6) {               // a page holds the whole step
            const int number = window(P >> shift);
            if (number < 0) gone = 15;
            const PageRows at(a, kc, vc, number, P, mask);
#pragma unroll
            for (uint32_t u = 0; u < kLoads; ++u) {
                kreg[u] = piece_of(at.k + u * (256 / kRowPieces) * krow_b, kpiece);
                vreg[u] = piece_of(at.v + u * (256 / kRowPieces) * vrow_b, vpiece);
            }
            return;
        }
        int number[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            number[h] = window(min(P + h * 16, end - 1) >> shift);
            if (number[h] < 0) gone |= 1u << h;
        }
#pragma unroll
        for (uint32_t u = 0; u < kLoads; ++u) {
            const int h = D == 128 ? (int)u : (int)(2 * u + (wave >> 1));          // (uniform)
            const int n = D == 128 ? number[u] : wave >> 1 ? number[2 * u + 1] : number[2 * u];
            // (where rows are counted through two halves, the upper one's count from 16)
            const PageRows at(a, kc, vc, n, P + h * 16, mask);
            const uint32_t back = D == 128 ? 0u : (wave >> 1) * 16;
            kreg[u] = piece_of(at.k - back * krow_b, kpiece);
            vreg[u] = piece_of(at.v - back * vrow_b, vpiece);
        }
    };
    auto store = [&](int step, uint32_t buf) {
        const bool mine = kOwn && step >= np;
        const int P = (mine ? step - np : step) * (int)kStep, end = mine ? own_end : prefix.len;
        if (gone || P + (int)kStep > end) {
            asm volatile("");
#pragma unroll
            for (uint32_t u = 0; u < kLoads; ++u) {
                const uint32_t row = (u * 256 + tid) / kRowPieces;
                vreg[u] = P + (int)row < end && !(gone >> (row >> 4) & 1) ? vreg[u] : u4_t{0, 0, 0, 0};
            }
        }
        if (mine && P >= wild0) {
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
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    const float c2 = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-30f);
    const float slack = WeightRange<T>::kSlack / c2;
    uint32_t tok[NT], head[NT];
    v8 q[NT][KK];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t rho = min(mine0 + t * 16 + i, R - 1);
        tok[t] = rho / G;
        head[t] = hk * G + rho % G;
        const T *qr = static_cast<const T *>(a.q) + ((size_t)set.token0 + tok[t]) * a.q_token + (size_t)head[t] * a.q_head + c * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) q[t][kk] = __builtin_bit_cast(v8, *reinterpret_cast<const u4_t *>(qr + kk * 32) ^ u4_t{sign, sign, sign, sign});
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
    // LDS byte offsets of this lane's operand pieces in a stage's first tile (half a tile or a tile further the swizzles are the same)
    uint32_t kread[KK], vread[DT];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kread[kk] = i * (D * 2) + (((4 * kk + c) ^ k_slot<D>(i)) << 4);
    {
        const uint32_t row = 4 * c + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vread[dt] = kHalf + row * (D * 2) + (((2 * dt + ((i & 3) >> 1)) ^ v_slot<D>(row)) << 4) + (i & 1) * 8;
    }
    auto meet = [] {      // everyone's LDS accesses are done (loads from memory stay on their way)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (kOwn && tid == 0) *wild = 0;
    meet();
    uint32_t missing = 0, next = 0;
    // a step's rows are requested two rounds before it and written one before (one place each in the code: scalar registers are short)
    if (lo < hi)
    for (int step = lo - 2; step < hi; ++step) {
        const bool mine = kOwn && step >= np;
        const int P0 = (mine ? step - np : step) * (int)kStep, end = mine ? own_end : prefix.len;
        const unsigned char *st = lds + ((step - lo) & 1) * 2 * kHalf;
        if (rows && step >= lo && !(mine && P0 >= wave_end)) {
            f4_t S[NT][4];
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) S[t][g] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    const v8 kr = __builtin_bit_cast(v8, *reinterpret_cast<const u4_t *>(st + kread[kk] + g * 16 * D * 2));
#pragma unroll
                    for (int t = 0; t < NT; ++t) S[t][g] = M::mul(kr, q[t][kk], S[t][g]);
                }
            __builtin_amdgcn_s_setprio(0);
            if (missing || P0 + (int)kStep > end || (mine && P0 + (int)kStep > wave_least)) {
                asm volatile("");
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int last = (mine ? min(end, limit0 + (int)tok[t]) : end) - P0 - 4 * (int)c;
#pragma unroll
                    for (int e = 0; e < 16; ++e) S[t][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < last && !(missing >> (e >> 2) & 1) ? S[t][e >> 2][e & 3] : -INFINITY;
                }
            }
            v8 P[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float mx = -INFINITY;
#pragma unroll
                for (int g = 0; g < 4; ++g) mx = fmaxf(mx, fmaxf(fmaxf(S[t][g][0], S[t][g][1]), fmaxf(S[t][g][2], S[t][g][3])));
                if (__any(mx - m_run[t] > slack)) {            // (as `weigh` has it)
                    mx = row_max(mx);
                    mx = mx - m_run[t] > slack ? mx : m_run[t];
                    const float resc = m_run[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run[t] - mx) * c2);
                    m_run[t] = mx;
                    L[t] = L[t] * resc;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) O[t][dt] = O[t][dt] * resc;
                }
                const float ms = m_run[t] == -INFINITY ? 0.f : m_run[t];
#pragma unroll
                for (int e = 0; e < 16; ++e) P[t][e >> 3][e & 7] = (T)__builtin_amdgcn_exp2f(fmaf(S[t][e >> 2][e & 3] - ms, c2, WeightRange<T>::kLift));
            }
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const v8 vr = __builtin_bit_cast(v8, transposed(st + h * kTile * D * 2 + vread[dt], 16 * D * 2));
#pragma unroll
                    for (int t = 0; t < NT; ++t) O[t][dt] = M::mul(vr, P[t][h], O[t][dt]);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) L[t] = M::mul(ones, P[t][h], L[t]);
            }
            __builtin_amdgcn_s_setprio(0);
        }
        if (step + 1 >= lo && step + 1 < hi) {
            next = gone;
            store(step + 1, (step + 1 - lo) & 1);
        }
        if (step + 2 < hi) request(step + 2);
        meet();
        missing = next;
    }
    if (!rows) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (mine0 + t * 16 + i >= R) continue;
        const size_t token = (size_t)set.token0 + tok[t];
        if (kOwn && *wild) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                float o[4] = {O[t][dt][0], O[t][dt][1], O[t][dt][2], O[t][dt][3]};
                add_wild<T>(a, own, shift, hk, max(wild0, (lo - np) * (int)kStep), min(min(own_end, (hi - np) * (int)kStep), limit0 + (int)tok[t]), 16 * dt + 4 * c, o);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[t][dt][e] = o[e];
            }
        }
        if (records) {
            const int place = kSeek ? place_of(a, set, (int)token) : 0;
            if (place < 0) continue;
            float *dst = part + (((kSeek ? (size_t)place : token) * a.n_q_heads + head[t]) * records + z) * OP;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f4_t *>(dst + 16 * dt + 4 * c) = O[t][dt];
            if (c == 0) *reinterpret_cast<float2 *>(dst + D) = make_float2(m_run[t] * c2, L[t][0]);
        } else {
            T *dst = static_cast<T *>(a.out) + token * a.out_token + (size_t)head[t] * a.out_head + 4 * c;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                T r[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = (T)(L[t][0] == 0.f ? 0.f : O[t][dt][e] / L[t][0]);
                *reinterpret_cast<u2_t *>(dst + 16 * dt) = *reinterpret_cast<const u2_t *>(r);
            }
        }
    }
}

// tokens of a sequence: first row, how many there are, how many of them count
struct SeqTokens { int row0, n, answered; };
__device__ __forceinline__ SeqTokens tokens_of(const ps_page_attention_args &a, uint32_t s) {
    const int lo = clampi(a.first[s], 0, (int)a.n_tokens), hi = clampi(a.first[s + 1], 0, (int)a.n_tokens), n = max(0, hi - lo);
    return {lo, n, min(n, (int)min(a.max_tokens, 0x7FFFFFFFu))};
}
__device__ __forceinline__ int length_of(const ps_page_attention_args &a, uint32_t s) { return clampi(a.length[s], 0, (int)a.max_length); }
__device__ __forceinline__ int prefix_length_of(const ps_page_attention_args &a, int p) { return clampi(a.prefix_length[p], 0, (int)a.max_prefix); }
// the prefix that a sequence stands behind (-1: none) and its length; by a whole wave, all of it asked for at once
struct Behind { int prefix, len; };
__device__ __forceinline__ Behind prefix_behind(const ps_page_attention_args &a, uint32_t s) {
    for (uint32_t p0 = 0; p0 < a.n_prefix; p0 += 64) {
        const uint32_t p = p0 + (threadIdx.x & 63), at = min(p, a.n_prefix - 1);
        const int len = prefix_length_of(a, at), lo = a.group_first[at], hi = a.group_first[at + 1];
        const uint64_t in = __ballot(p < a.n_prefix && lo <= (int)s && (int)s < hi);
        if (in) {
            const int lane = __ffsll((unsigned long long)in) - 1;
            return {(int)p0 + lane, __builtin_amdgcn_readlane(len, lane)};
        }
    }
    return {-1, 0};
}
// the `flat`-th block of 128 rows of all groups' tokens; rows 0: there is none
struct GroupBlock { RowSet set; uint32_t prefix, block; };
__device__ __forceinline__ GroupBlock group_block(const ps_page_attention_args &a, uint32_t flat) {
    const uint32_t G = a.n_q_heads / a.n_kv_heads, lane = threadIdx.x & 63;
    uint32_t base = 0;
    for (uint32_t p0 = 0; p0 < a.n_prefix; p0 += 64) {
        const uint32_t p = p0 + lane;
        int t0 = 0, n = 0;
        if (p < a.n_prefix) {
            t0 = clampi(a.first[clampi(a.group_first[p], 0, (int)a.n_seq)], 0, (int)a.n_tokens);
            n = max(0, clampi(a.first[clampi(a.group_first[p + 1], 0, (int)a.n_seq)], 0, (int)a.n_tokens) - t0);
        }
        const uint32_t mine = (uint32_t)(((uint64_t)n * G + 127) / 128);
        uint32_t upto = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(upto, o, 64);
            if ((int)lane >= o) upto += x;
        }
        const uint64_t past = __ballot(base + upto > flat);
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            const uint32_t before = base + __builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at);
            return {{__builtin_amdgcn_readlane(t0, at), (uint32_t)__builtin_amdgcn_readlane(n, at) * G, G, 0, 0}, p0 + at, flat - before};
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    return {{0, 0, G, 0, 0}, 0, 0};
}

extern __shared__ u4_t page_lds[];

// kSeek, here and below: where the arrays have room for more tokens than may be answered (what it takes costs registers in the others: here 256 for 241, and the
// prompts' blocks 205 us for 200)
template <typename T, int D, int NT, bool kSeek>
__global__ __launch_bounds__(256, 2) void page_shared_kernel(ps_page_attention_args a, PageDeal d, uint32_t shift, uint32_t prefix8, float *part) {
    unsigned char *const lds = reinterpret_cast<unsigned char *>(page_lds);
    const uint32_t records = d.direct ? 0 : d.psplit + d.osplit, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the prefixes' workgroups first, in runs of eight (one on each XCD)
    const uint32_t run = blockIdx.x / 8;
    if (run < prefix8) {
        // blocks of the same positions follow one another on one XCD, whose L2 they share
        const uint32_t unit = run / d.blocks * 8 + blockIdx.x % 8;
        if (unit >= a.n_kv_heads * d.psplit) return;
        for (uint32_t block = run % d.blocks;;) {
            GroupBlock g = group_block(a, block);
            if (g.set.rows == 0) return;
            if (kSeek) {
                g.set.seq0 = clampi(a.group_first[g.prefix], 0, (int)a.n_seq - 1);
                g.set.seqs = max(1, clampi(a.group_first[g.prefix + 1], 0, (int)a.n_seq) - (int)g.set.seq0);
            }
            const uint32_t z = unit % d.psplit, hk = unit / d.psplit;
            const int len = prefix_length_of(a, g.prefix), lo = (int)min((uint64_t)z * d.plen, (uint64_t)len), hi = (int)min((uint64_t)lo + d.plen, (uint64_t)len);
            if (!kSeek && lo >= hi) return;
            if (lo < hi) {
                const Span span{a.prefix_table + g.prefix * a.prefix_seq, (int)min(a.prefix_width, 0x7FFFFFFFu), len};
                if (g.set.rows <= NT * 16) {
                    PageWindow window;
                    window.fill(span, (lo + (int)(wave * kTile)) >> shift, a.n_pages);
                    rows_few<T, D, NT, false, kSeek>(a, g.set, Span{nullptr, 0, 0}, span, shift, hk, lo / (int)kTile, (hi + (int)kTile - 1) / (int)kTile, hi, hi, window, records, z, part, lds);
                } else rows_many<T, D, false, kSeek>(a, g.set, g.block * 128, Span{span.table, span.entries, hi}, Span{nullptr, 0, 0}, shift, hk, lo / (int)kStep,
                                                     (hi + (int)kStep - 1) / (int)kStep, 0, records, z, part, lds);
            }
            block += d.blocks;
            if (!kSeek || block >= d.most) return;
            __syncthreads();            // (the next block's rows come to lie where this one's results were put together)
        }
    } else {
        const uint32_t unit = (run - prefix8) * 8 + blockIdx.x % 8, z = unit % d.osplit, hk = unit / d.osplit % a.n_kv_heads, s = unit / d.osplit / a.n_kv_heads;
        if (s >= a.n_seq) return;
        // (the table's entries are asked for with the lengths: one load's time less for every run)
        PageWindow window;
        window.fill(Span{a.table + s * a.table_seq, (int)min(a.width, 0x7FFFFFFFu), 0}, (int)((z * d.olen + wave * kTile) >> shift), a.n_pages);
        const SeqTokens t = tokens_of(a, s);
        const int len = length_of(a, s), lo = (int)min((uint64_t)z * d.olen, (uint64_t)len), hi = (int)min((uint64_t)lo + d.olen, (uint64_t)len);
        if (t.answered == 0 || (lo >= hi && records)) return;
        const uint32_t G = a.n_q_heads / a.n_kv_heads;
        const Span own{a.table + s * a.table_seq, (int)min(a.width, 0x7FFFFFFFu), len};
        rows_few<T, D, NT, false>(a, RowSet{t.row0, t.answered * G, G, 0, 0}, Span{nullptr, 0, 0}, own, shift, hk, lo / (int)kTile, (hi + (int)kTile - 1) / (int)kTile, hi, len - t.n + 1, window, records,
                                  d.psplit + z, kSeek ? records_of(a, d, s, t.row0, D + 4, part) : part, lds);
    }
}

// Few rows a sequence and a short prefix: the sequence's own workgroups walk its tiles, the prefix's first.  Where 128 rows' places are mostly empty, this
// kernel's reads are ahead by a tile in every wave; latencies bound it (3 sequences, 4 / 2 heads of 128, 77 + 40 positions: 8.5 us on the GPU, as a
// block of 128 rows 13.6), then memory (16 sequences, 32 / 8 heads of 128, 500 + 3000: 30.7 us a call, 4.5 TB/s, for 40.8).
template <typename T, int D, int NT, bool kSeek>
__global__ __launch_bounds__(256, 2) void page_few_kernel(ps_page_attention_args a, PageDeal d, uint32_t shift, float *part) {
    const uint32_t unit = blockIdx.x, z = unit % d.osplit, hk = unit / d.osplit % a.n_kv_heads, s = unit / d.osplit / a.n_kv_heads, G = a.n_q_heads / a.n_kv_heads;
    const SeqTokens t = tokens_of(a, s);
    const Span own{a.table + s * a.table_seq, (int)min(a.width, 0x7FFFFFFFu), length_of(a, s)};
    const Behind p = prefix_behind(a, s);
    if (t.answered == 0) return;
    const Span prefix = p.prefix < 0 ? Span{nullptr, 0, 0} : Span{a.prefix_table + p.prefix * a.prefix_seq, (int)min(a.prefix_width, 0x7FFFFFFFu), p.len};
    const int tiles = (prefix.len + (int)kTile - 1) / (int)kTile + (own.len + (int)kTile - 1) / (int)kTile;
    const int lo = (int)min((uint64_t)z * d.olen, (uint64_t)tiles), hi = (int)min((uint64_t)lo + d.olen, (uint64_t)tiles);
    if (lo >= hi && !d.direct) return;
    rows_few<T, D, NT, true>(a, RowSet{t.row0, t.answered * G, G, 0, 0}, prefix, own, shift, hk, lo, hi, own.len, own.len - t.n + 1, PageWindow{-1, 0}, d.direct ? 0 : d.osplit, z, kSeek ? records_of(a, d, s, t.row0, D + 4, part) : part,
                             reinterpret_cast<unsigned char *>(page_lds));
}

template <typename T, int D, bool kSeek>
__global__ __launch_bounds__(256, 2) void page_rows_kernel(ps_page_attention_args a, PageDeal d, uint32_t shift, float *part) {
    unsigned char *const lds = reinterpret_cast<unsigned char *>(page_lds);
    const uint32_t units = a.n_seq * a.n_kv_heads * d.osplit;
    const uint32_t unit = blockIdx.x / 8 / d.blocks * 8 + blockIdx.x % 8, block = blockIdx.x / 8 % d.blocks;
    if (unit >= units) return;
    const uint32_t z = unit % d.osplit, hk = unit / d.osplit % a.n_kv_heads, s = unit / d.osplit / a.n_kv_heads, G = a.n_q_heads / a.n_kv_heads;
    const SeqTokens t = tokens_of(a, s);
    const Span own{a.table + s * a.table_seq, (int)min(a.width, 0x7FFFFFFFu), length_of(a, s)};
    const Behind p = prefix_behind(a, s);
    if (block * 128 >= t.answered * G) return;
    const Span prefix = p.prefix < 0 ? Span{nullptr, 0, 0} : Span{a.prefix_table + p.prefix * a.prefix_seq, (int)min(a.prefix_width, 0x7FFFFFFFu), p.len};
    const RowSet set{t.row0, t.answered * G, G, 0, 0};
    const int np = (prefix.len + (int)kStep - 1) / (int)kStep, limit0 = own.len - t.n + 1;
    const int last = min(own.len, limit0 + (int)(min(block * 128 + 127, set.rows - 1) / G));
    const int steps = np + (max(last, 0) + (int)kStep - 1) / (int)kStep;
    const int lo = (int)min((uint64_t)z * d.olen, (uint64_t)steps), hi = (int)min((uint64_t)lo + d.olen, (uint64_t)steps);
    // (a run that none of the block's rows sees leaves records of nothing)
    rows_many<T, D, true>(a, set, block * 128, prefix, own, shift, hk, lo, hi, limit0, d.direct ? 0 : d.osplit, z, kSeek ? records_of(a, d, s, t.row0, D + 4, part) : part, lds);
}

// D / 4 lanes per (token, query head) put the records of its prefix's and of its sequence's runs together, in their order: value sums, then maximum
// (in powers of two) and weight sum.  Latencies: 512 tokens of 32 heads, three records each, 9 us.
template <typename T, int D>
__global__ __launch_bounds__(256) void page_merge_kernel(ps_page_attention_args a, PageDeal d, const float *part) {
    constexpr uint32_t OP = D + 4, kLanes = D / 4, kHeads = 256 / kLanes;
    const uint32_t hb = (a.n_q_heads + kHeads - 1) / kHeads, h = blockIdx.x % hb * kHeads + threadIdx.x / kLanes, e0 = threadIdx.x % kLanes * 4;
    const uint32_t i = blockIdx.x / hb % a.max_tokens, s = blockIdx.x / hb / a.max_tokens;
    // (all of these are asked for before one is waited for)
    const SeqTokens t = tokens_of(a, s);
    const int len = length_of(a, s), plen = prefix_behind(a, s).len;
    if (h >= a.n_q_heads || (int)i >= t.answered) return;
    const uint32_t np = d.shared && plen ? (plen + d.plen - 1) / d.plen : 0;
    const uint32_t unit = d.nt ? kTile : kStep, positions = d.shared ? len : (plen + unit - 1) / unit + (len + unit - 1) / unit;
    const uint32_t n = np + (positions + d.olen - 1) / d.olen;
    const size_t token = (size_t)t.row0 + i, place = d.by_seq ? (size_t)s * a.max_tokens + i : token;
    const float *r0 = part + (place * a.n_q_heads + h) * (d.psplit + d.osplit) * OP;
    float mx = -INFINITY, l = 0.f;
    f4_t o{0.f, 0.f, 0.f, 0.f};
    for (uint32_t z0 = 0; z0 < n; z0 += 8) {
        float2 ml[8];
        f4_t ov[8];
        float m8 = mx;
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) {
            const uint32_t z = min(z0 + u, n - 1);
            const float *r = r0 + (size_t)(z < np ? z : d.psplit + z - np) * OP;
            ml[u] = *reinterpret_cast<const float2 *>(r + D);
            ov[u] = *reinterpret_cast<const f4_t *>(r + e0);
        }
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) m8 = fmaxf(m8, ml[u].x);
        const float ms = m8 == -INFINITY ? 0.f : m8, resc = __builtin_amdgcn_exp2f(mx - ms);
        l *= resc;
        o = o * resc;
        mx = m8;
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) {
            const bool in = z0 + u < n;          // (a record past the last is the last again)
            const float w = ml[u].x == -INFINITY ? (m8 == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(ml[u].x - ms);       // as the waves above
            l = in ? fmaf(w, ml[u].y, l) : l;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = in ? fmaf(w, ov[u][e], o[e]) : o[e];
        }
    }
    T r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (T)(l == 0.f ? 0.f : o[e] / l);
    *reinterpret_cast<u2_t *>(static_cast<T *>(a.out) + token * a.out_token + h * a.out_head + e0) = *reinterpret_cast<const u2_t *>(r);
}

// ------------------------------------------------------------------------------------ sampling
// Launches, in order (three for rows of up to 32768 entries, whose border entries the last one picks out itself: rows of 32768, 256 of them 54 us for 60, 16 the same,
// a single one 31 for 25):
//  sample_rows_kernel   a row's chunks: largest logit and where; clears the row's bins
//  sample_bins_kernel   entries by how far they lie behind the row's largest logit, in bins of 24 / 2047 nats (the last one: all from 24 nats on):
//                       counts, and sums of weights relative to the bin's middle as whole numbers of 2^-35, so that their order does not matter
//  sample_find_kernel   running counts and sums over the bins say in which bins the borders lie (of top-k, top-p, min-p, and the drawn
//                       entry); the entries of these bins, most often a few hundred, are picked out of the row
//  sample_pick_kernel   a workgroup per row finds the borders among them, digit by digit of the logits' bits.  Where they are more than a list holds, in
//                       passes over the row instead.
// The sum of the first entries of the order is that of whole bins (64 bits, always added alike) and of a part of one, whose whole numbers are exact.
// 256 rows of 128256 fp32 logits: 22 + 35 + 37 + 16 us, where each of the first three reads the 131 MB (27 us at a copy's rate); the second has a dozen
// 64-bit operations and an addition in LDS for each entry beside.  16 rows 4 + 8 + 13 + 12 us, one of 32000 3 + 5 + 16: latencies.
// Where the borders' bins hold more than a list does, one workgroup reads its row once for each digit: rows of 128256 equal logits 254 us, of logits closer than 0.01
// 470 to 550 (with top-k and top-p 530 to 610), 16 rows hardly more, 256 rows 385 and 570 to 630.
constexpr uint32_t kBins = 2048, kRowThreads = 256, kPickThreads = 512, kBinsPad = kBins + 8, kList = 2048, kRound = kPickThreads * 8, kShortRow = 32768;
constexpr double kBinsPerNat = 2047.0 / 24.0;

struct RowTop { float m; int at; };
struct SampleShape { uint32_t top, ntop, bins, nbins, find, nfind; };       // chunks of a row for the first three launches: entries, how many
// What the borders of a row are found by, and the bins that they may lie in
struct Wanted { uint32_t most; bool by_k, by_p, by_m; double share, reach, u; int bk, p0, p1, bm, d0, d1; };
struct SampleWork {
    RowTop *tops;                  // [row][chunk]
    unsigned long long *sums;      // [row][bin]
    uint32_t *counts;              // [row][bin]
    uint32_t *listed;              // [row]
    unsigned long long *list;      // [row][kList]
    Wanted *wanted;                // [row]
    double *before_sum;            // [row][kBinsPad]: of all entries in front of a bin, and of all
    uint32_t *before_count;        // [row][kBinsPad]
};

// bits that order as the values do, and back: larger for larger logits
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);        // (-0 is 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// an entry of a list: inverted bits in front of the index (24 bits), so that it ascends as the order does
__device__ __forceinline__ unsigned long long entry_of(float v, uint32_t i) { return (unsigned long long)~order_of(v) << 24 | i; }
__device__ __forceinline__ float value_of(uint32_t key) { return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
__device__ __forceinline__ float value_in(unsigned long long entry) { return value_of(~(uint32_t)(entry >> 24)); }

// How far an entry lies behind the largest one, in bins: the nearest whole number and what remains, by adding 1.5 2^52 (a conversion takes as long as four
// operations).  Its weight, relative to that of its bin's middle, in whole numbers of 2^-35: exp(-rest / 85.3) as a polynomial of degree 4 (off by
// 6e-14 of it, the rounding by 1.5e-11).  In the last bin, which is all from 24 nats on, by the 32-bit exponential in steps of 2^-31: right to 2^-22 of e^-24
// (a step of the exponential and of its argument, 1.8e-7 at most), 9e-18 of the largest entry's weight for each, where 2^24 of them would be 1.5e-10 and the nearest entries' own
// rounding is 1.5e-11.  In 64 bits, or as the product of two table entries, 256 rows of 128256 take 43 and 6 us more.
constexpr double kWhole = 6755399441055744.0;
struct Place {
    int n;
    double rest;
    __device__ __forceinline__ int bin() const { return min(n, (int)kBins - 1); }
    __device__ __forceinline__ double value() const { return (double)n + rest; }
};
struct BinScale {
    double m, rate, least;
    float top, coarse;
    bool rough;                  // `about` says where an entry lies
    __device__ __forceinline__ Place place(float v) const {
        const double d = fmax((double)v - m, least), t = fma(d, -rate, kWhole);
        return {(int)(uint32_t)__builtin_bit_cast(uint64_t, t), fma(d, -rate, kWhole - t)};
    }
    __device__ __forceinline__ float about(float v) const { return fminf((top - v) * coarse, (float)kBins); }     // a place to within 0.01
};
__device__ __forceinline__ BinScale bin_scale(float m, float temp) {
    // (any temperature above 0: of 1e-45 the rate is 6e46, of an infinite one 0.  What a difference of two logits times the rate is in 32 bits says
    // nothing where the rate or, under a small rate, the difference passes their range)
    const double rate = kBinsPerNat / (double)temp;
    return {(double)m, rate, fmax(-1e6 / rate, -1e300), m, (float)fmin(rate, 1e30), rate >= 1e-25 && rate <= 1e30};
}
__device__ __forceinline__ unsigned long long whole_far(int n, double rest) {
    const float back = (float)(n - ((int)kBins - 1)) + (float)rest;
    return (unsigned long long)(uint32_t)(__builtin_amdgcn_exp2f(back * -0.01691484171047148f) * 2147483648.f) << 4;
}
// N in step: one after the other they are a chain of a dozen operations each
template <int N>
__device__ __forceinline__ void wholes_of(const double (&rest)[N], unsigned long long (&w)[N]) {
    constexpr double c[5] = {27.052798810934387, -9229.51319433045, 2361601.688599304, -402849888.0468979, 34359738368.0};
    double v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = c[0];
#pragma unroll
    for (int j = 1; j < 5; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = fma(v[e], rest[e], c[j]);
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = __builtin_bit_cast(uint64_t, v[e] + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
}
__device__ __forceinline__ unsigned long long whole_of(const Place &y) {
    if (y.n >= (int)kBins - 1) return whole_far(y.n, y.rest);
    const double rest[1] = {y.rest};
    unsigned long long w[1];
    wholes_of(rest, w);
    return w[0];
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void sample_rows_kernel(ps_sample_args a, SampleShape sh, SampleWork w) {
    __shared__ float top[kRowThreads / 64];
    __shared__ int where[kRowThreads / 64];
    const uint32_t tid = threadIdx.x, row = blockIdx.y, chunk = blockIdx.x;
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_row;
    const uint32_t lo = chunk * sh.top, hi = min(a.vocab, lo + sh.top);
    RowTop r{-INFINITY, 0x7FFFFFFF};
#pragma unroll 2
    for (uint32_t i = lo + tid * 8; i < hi; i += kRowThreads * 8) {
        Oct<T> o;
        o.fill(x, i, hi);
        float v[8], mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            o.take(v[e], v[e + 1]);
            mx = fmaxf(mx, fmaxf(v[e], v[e + 1]));
        }
        if (mx > r.m) {
            r.m = mx;
#pragma unroll
            for (int e = 7; e >= 0; --e) r.at = v[e] == mx ? (int)(i + e) : r.at;
        }
    }
    const uint32_t per = (kBins + sh.ntop - 1) / sh.ntop;
    for (uint32_t b = chunk * per + tid; b < min(kBins, (chunk + 1) * per); b += kRowThreads) {
        w.sums[(size_t)row * kBins + b] = 0;
        w.counts[(size_t)row * kBins + b] = 0;
    }
    if (chunk == 0 && tid == 0) w.listed[row] = 0;
    float m = r.m;
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    int at = r.m == m ? r.at : 0x7FFFFFFF;
    for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o, 64));
    if ((tid & 63) == 0) { top[tid >> 6] = m; where[tid >> 6] = at; }
    __syncthreads();
    if (tid == 0) {
        RowTop t{top[0], where[0]};
        for (uint32_t i = 1; i < kRowThreads / 64; ++i) {
            if (top[i] > t.m) t = {top[i], where[i]};
            else if (top[i] == t.m) t.at = min(t.at, where[i]);
        }
        w.tops[(size_t)row * sh.ntop + chunk] = t;
    }
}
// the largest logit of a row and its lowest index; every thread of the workgroup calls it
template <uint32_t kThreads>
__device__ __forceinline__ RowTop row_top(const RowTop *tops, uint32_t n, float *fbuf, int *ibuf) {
    const uint32_t tid = threadIdx.x;
    RowTop t{-INFINITY, 0x7FFFFFFF};
    for (uint32_t i = tid; i < n; i += kThreads) {
        const RowTop o = tops[i];
        if (o.m > t.m) t = o;
        else if (o.m == t.m) t.at = min(t.at, o.at);
    }
    for (int o = 32; o; o >>= 1) {
        const float m = __shfl_xor(t.m, o, 64);
        const int at = __shfl_xor(t.at, o, 64);
        if (m > t.m) t = {m, at};
        else if (m == t.m) t.at = min(t.at, at);
    }
    if (n <= 64) {             // (the first wave has them all)
        if (tid == 0) { fbuf[0] = t.m; ibuf[0] = t.at; }
        __syncthreads();
        return {fbuf[0], ibuf[0]};
    }
    if ((tid & 63) == 0) { fbuf[tid >> 6] = t.m; ibuf[tid >> 6] = t.at; }
    __syncthreads();
    for (uint32_t i = 0; i < kThreads / 64; ++i) {
        if (fbuf[i] > t.m) t = {fbuf[i], ibuf[i]};
        else if (fbuf[i] == t.m) t.at = min(t.at, ibuf[i]);
    }
    return t;
}

// a thread's first entries of lo .. hi - 1
template <typename T>
__device__ __forceinline__ Oct<T> first_of(const T *x, uint32_t lo, uint32_t hi) {
    Oct<T> o;
    o.fill(x, min(lo + threadIdx.x * 8, hi), hi);
    return o;
}

template <typename T>
__global__ __launch_bounds__(kPickThreads) void sample_bins_kernel(ps_sample_args a, SampleShape sh, SampleWork w) {
    __shared__ unsigned long long bins[kBins];             // sum of weights, and from bit 49 on how many: of 2^13 entries
    __shared__ float fbuf[kPickThreads / 64];
    __shared__ int ibuf[kPickThreads / 64];
    const uint32_t tid = threadIdx.x, row = blockIdx.y, chunk = blockIdx.x;
    const float temp = a.temperature ? a.temperature[row] : 1.f;
    if (!(temp > 0.f)) return;
    constexpr uint32_t kMine = kBins / kPickThreads;
    for (uint32_t j = 0; j < kMine; ++j) bins[tid + j * kPickThreads] = 0;
    const float m = row_top<kPickThreads>(w.tops + (size_t)row * sh.ntop, sh.ntop, fbuf, ibuf).m;
    if (m == -INFINITY) return;
    __syncthreads();
    const BinScale s = bin_scale(m, temp);
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_row;
    const uint32_t lo = chunk * sh.bins, hi = min(a.vocab, lo + sh.bins);
    unsigned long long sum[kMine] = {};
    uint32_t count[kMine] = {};
    Oct<T> next = first_of(x, lo, hi);
    for (uint32_t i0 = lo; i0 < hi; i0 += 2 * kRound) {
#pragma unroll
        for (uint32_t r = 0; r < 2; ++r) {
            const uint32_t i = i0 + r * kRound + tid * 8;
            Oct<T> o = next;
            if (i + kRound < hi) next.fill(x, i + kRound, hi);
            if (i < hi) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float v[4];
                    double d[4], rest[4];
                    int n[4], most = 0;
                    unsigned long long whole[4];
#pragma unroll
                    for (int e = 0; e < 4; e += 2) o.take(v[e], v[e + 1]);
                    // (as BinScale::place has it)
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] = fmax((double)v[e] - s.m, s.least);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const double t = fma(d[e], -s.rate, kWhole);
                        n[e] = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
                        rest[e] = fma(d[e], -s.rate, kWhole - t);
                        most = max(most, n[e]);
                    }
                    wholes_of(rest, whole);
                    if (most >= (int)kBins - 1)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            whole[e] = n[e] >= (int)kBins - 1 ? whole_far(n[e], rest[e]) : whole[e];
                            n[e] = min(n[e], (int)kBins - 1);
                        }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (v[e] != -INFINITY) atomicAdd(&bins[n[e]], whole[e] + (1ull << 49));
                }
            }
        }
        __syncthreads();
        for (uint32_t j = 0; j < kMine; ++j) {             // a bin has room for two rounds
            const unsigned long long v = bins[tid + j * kPickThreads];
            bins[tid + j * kPickThreads] = 0;
            sum[j] += v & ((1ull << 49) - 1);
            count[j] += (uint32_t)(v >> 49);
        }
        __syncthreads();
    }
    for (uint32_t j = 0; j < kMine; ++j)
        if (count[j]) {
            atomicAdd(&w.sums[(size_t)row * kBins + tid + j * kPickThreads], sum[j]);
            atomicAdd(&w.counts[(size_t)row * kBins + tid + j * kPickThreads], count[j]);
        }
}

// up to four runs of bins, apart and ascending
struct Runs {
    int lo[4], hi[4];
    uint32_t before[5];          // entries of the runs in front
    __device__ __forceinline__ bool has(int b) const { return (b >= lo[0] && b <= hi[0]) || (b >= lo[1] && b <= hi[1]) || (b >= lo[2] && b <= hi[2]) || (b >= lo[3] && b <= hi[3]); }
};
struct BinLds {
    double sum[kBins + 1];                 // of all entries in front of a bin, and of all
    uint32_t count[kBins + 1];             // likewise
    double dbuf[kPickThreads / 64];
    uint32_t ubuf[kPickThreads / 64];
    float fbuf[kPickThreads / 64];
    int ibuf[kPickThreads / 64], found[6];
};

// the first bin that has entries and at whose end `passes` is true, into l.found[slot] where it comes before what that holds
template <class Passes>
__device__ __forceinline__ void look(BinLds &l, int slot, Passes passes) {
#pragma unroll
    for (uint32_t j = 0; j < kBins / kPickThreads; ++j) {
        const uint32_t b = threadIdx.x + j * kPickThreads;
        const uint64_t yes = __ballot(l.count[b + 1] > l.count[b] && passes(b));
        if (yes) {
            if ((threadIdx.x & 63) == 0) atomicMin(&l.found[slot], (int)(b + __ffsll((unsigned long long)yes) - 1));
            return;
        }
    }
}

// a thread's four bins, asked for before the row's largest logit is waited for
struct FourBins {
    uint4 c;
    ulonglong2 s0, s1;
    __device__ __forceinline__ FourBins(const SampleWork &w, uint32_t row) {
        const size_t at = (size_t)row * kBins + threadIdx.x * 4;
        c = *reinterpret_cast<const uint4 *>(w.counts + at);
        s0 = *reinterpret_cast<const ulonglong2 *>(w.sums + at);
        s1 = *reinterpret_cast<const ulonglong2 *>(w.sums + at + 2);
    }
};
// Running counts and sums of a row's bins, and where its borders may lie.  By every workgroup that needs it, always added alike.
__device__ __forceinline__ Wanted analyse(const ps_sample_args &a, const FourBins &four, uint32_t row, BinLds &l) {
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = tid * 4;
    static_assert(kBins == 4 * kPickThreads, "four bins a thread");
    Wanted q{};
    {
        const uint4 c = four.c;
        const ulonglong2 s0 = four.s0, s1 = four.s1;
        const double middle = exp(-(double)b / kBinsPerNat);
        // (a bin's middle weighs 0.988 of the one before)
        const double v0 = middle * (double)s0.x, v1 = middle * 0.9883439889852305 * (double)s0.y, v2 = middle * 0.9768238405632375 * (double)s1.x, v3 = middle * 0.9654379711181429 * (double)s1.y;
        const uint32_t c1 = c.x + c.y, c2 = c1 + c.z, c3 = c2 + c.w;
        const double t1 = v0 + v1, t2 = t1 + v2, t3 = t2 + v3;
        uint32_t upto = c3;
        double sum = t3;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t xc = __shfl_up(upto, o, 64);
            const double xs = __shfl_up(sum, o, 64);
            if ((int)lane >= o) { upto += xc; sum = xs + sum; }
        }
        const uint32_t prior_c = __shfl_up(upto, 1, 64);
        const double prior_s = __shfl_up(sum, 1, 64);
        const uint64_t some = __ballot(c3 > 0);
        if (lane == 63) { l.ubuf[wave] = upto; l.dbuf[wave] = sum; }
        const int mine = c.w ? 3 : c.z ? 2 : c.y ? 1 : 0, at = some ? 63 - __clzll((long long)some) : 0;
        const int last = (int)(wave * 64 + at) * 4 + __shfl(mine, at, 64);
        if (lane == 0) l.ibuf[wave] = some ? last : -1;
        if (tid < 6) l.found[tid] = 0x7FFFFFFF;
        __syncthreads();
        uint32_t from_c = 0;
        double from_s = 0;
        for (uint32_t i = 0; i < wave; ++i) { from_c += l.ubuf[i]; from_s += l.dbuf[i]; }
        if (lane) { from_c += prior_c; from_s += prior_s; }
        l.count[b] = from_c;
        l.count[b + 1] = from_c + c.x;
        l.count[b + 2] = from_c + c1;
        l.count[b + 3] = from_c + c2;
        l.sum[b] = from_s;
        l.sum[b + 1] = from_s + v0;
        l.sum[b + 2] = from_s + t1;
        l.sum[b + 3] = from_s + t2;
        if (tid == kPickThreads - 1) { l.count[kBins] = from_c + c3; l.sum[kBins] = from_s + t3; }
    }
    __syncthreads();
    int last = -1;                              // the last bin with entries
    for (uint32_t i = 0; i < kPickThreads / 64; ++i) last = max(last, l.ibuf[i]);
    const uint32_t all = l.count[kBins];
    q.by_k = a.top_k && a.top_k[row] > 0 && (uint32_t)a.top_k[row] < all;
    q.by_p = a.top_p && a.top_p[row] < 1.f;
    q.by_m = a.min_p && a.min_p[row] > 0.f;
    q.most = q.by_k ? (uint32_t)a.top_k[row] : all;
    q.share = q.by_p ? (double)a.top_p[row] : 1.0;
    q.reach = q.by_m ? -log((double)a.min_p[row]) * kBinsPerNat : 0.0;        // weights of at least min_p lie up to this place
    q.u = fmax(fmin((double)a.u[row], 1.0 - 0x1p-24), 0.0);
    auto found = [&](int slot) { return min(l.found[slot], last); };
    double low = l.sum[kBins], high = low;      // what C(n) may be
    q.bk = q.p0 = q.p1 = q.bm = -1;
    if (q.by_k) {
        look(l, 0, [&](uint32_t j) { return l.count[j + 1] >= q.most; });
        __syncthreads();
        q.bk = found(0);
        low = l.sum[q.bk];
        high = l.sum[q.bk + 1];
    }
    if (q.by_p) {
        const double g0 = q.share * low, g1 = q.share * high;
        look(l, 1, [&](uint32_t j) { return l.sum[j + 1] >= g0; });
        look(l, 2, [&](uint32_t j) { return l.sum[j + 1] >= g1; });
        __syncthreads();
        q.p0 = found(1);
        q.p1 = max(q.p0, found(2));
        low = fmin(low, l.sum[q.p0]);
        high = fmin(high, l.sum[q.p1 + 1]);
    }
    if (q.by_m) {
        q.bm = (int)rint(fmin(fmax(q.reach, 0.0), (double)(kBins - 1)));
        low = fmin(low, l.sum[q.bm]);
        high = fmin(high, l.sum[q.bm + 1]);
    }
    const double g0 = q.u * low, g1 = q.u * high;
    look(l, 3, [&](uint32_t j) { return l.sum[j + 1] > g0; });
    look(l, 4, [&](uint32_t j) { return l.sum[j + 1] > g1; });
    __syncthreads();
    q.d0 = found(3);
    q.d1 = max(q.d0, found(4));
    return q;
}
__device__ __forceinline__ Runs runs_of(const Wanted &q, const BinLds &l) {
    Runs r{{q.by_k ? q.bk : (int)kBins, q.by_p ? q.p0 : (int)kBins, q.by_m ? q.bm : (int)kBins, q.d0}, {q.by_k ? q.bk : -1, q.by_p ? q.p1 : -1, q.by_m ? q.bm : -1, q.d1}, {}};
    auto order = [&](int i, int j) {
        if (r.lo[j] < r.lo[i]) {
            const int lo = r.lo[i], hi = r.hi[i];
            r.lo[i] = r.lo[j]; r.hi[i] = r.hi[j];
            r.lo[j] = lo; r.hi[j] = hi;
        }
    };
    order(0, 1); order(2, 3); order(0, 2); order(1, 3); order(1, 2);
    int end = -1;
    r.before[0] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.lo[i] = max(r.lo[i], end + 1);
        const bool some = r.lo[i] <= r.hi[i];
        r.before[i + 1] = r.before[i] + (some ? l.count[r.hi[i] + 1] - l.count[r.lo[i]] : 0);
        end = max(end, r.hi[i]);
    }
    return r;
}
// every entry lo .. hi - 1 of a row in one of the runs: take(value, index, place); `next`: first_of these
template <typename T, class Take>
__device__ __forceinline__ void each_in(const T *x, uint32_t lo, uint32_t hi, const BinScale &s, const Runs &r, Oct<T> next, Take take) {
    float from[4], to[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool some = r.lo[j] <= r.hi[j];
        from[j] = !some ? INFINITY : !s.rough ? -INFINITY : (float)r.lo[j] - 1.f;
        to[j] = !some ? -INFINITY : !s.rough || r.hi[j] == (int)kBins - 1 ? INFINITY : (float)r.hi[j] + 1.f;
    }
    constexpr uint32_t kStride = kPickThreads * 8;
    uint32_t i = lo + threadIdx.x * 8;
    for (; i < hi; i += kStride) {
        Oct<T> o = next;
        if (i + kStride < hi) next.fill(x, i + kStride, hi);
        float v[8], y[8];
        bool in[8] = {};
#pragma unroll
        for (int e = 0; e < 8; e += 2) o.take(v[e], v[e + 1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = s.about(v[e]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (r.lo[j] <= r.hi[j])         // (uniform)
#pragma unroll
                for (int e = 0; e < 8; ++e) in[e] |= y[e] >= from[j] && y[e] <= to[j];
        if (!(in[0] | in[1] | in[2] | in[3] | in[4] | in[5] | in[6] | in[7])) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (!in[e] || v[e] == -INFINITY) continue;
            const Place p = s.place(v[e]);
            if (r.has(p.bin())) take(v[e], i + e, p);
        }
    }
}
__device__ __forceinline__ Runs run_of(int b) { return {{b, (int)kBins, (int)kBins, (int)kBins}, {b, -1, -1, -1}, {}}; }

template <typename T>
__global__ __launch_bounds__(kPickThreads) void sample_find_kernel(ps_sample_args a, SampleShape sh, SampleWork w) {
    __shared__ BinLds l;
    __shared__ unsigned long long mine[kList];
    __shared__ uint32_t n, at;
    const uint32_t tid = threadIdx.x, row = blockIdx.y;
    const float temp = a.temperature ? a.temperature[row] : 1.f;
    if (!(temp > 0.f)) return;
    const FourBins four(w, row);
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_row;
    const uint32_t lo = blockIdx.x * sh.find, hi = min(a.vocab, lo + sh.find);
    const Oct<T> begin = first_of(x, lo, hi);
    const float m = row_top<kPickThreads>(w.tops + (size_t)row * sh.ntop, sh.ntop, l.fbuf, l.ibuf).m;
    if (m == -INFINITY) return;
    if (tid == 0) n = 0;
    __syncthreads();
    const Wanted q = analyse(a, four, row, l);
    if (blockIdx.x == 0) {                    // the last launch need not work it out again
        if (tid == 0) w.wanted[row] = q;
        for (uint32_t b = tid; b <= kBins; b += kPickThreads) {
            w.before_sum[(size_t)row * kBinsPad + b] = l.sum[b];
            w.before_count[(size_t)row * kBinsPad + b] = l.count[b];
        }
    }
    const Runs r = runs_of(q, l);
    if (r.before[4] > kList) return;
    each_in(x, lo, hi, bin_scale(m, temp), r, begin, [&](float v, uint32_t i, const Place &) {
        const uint32_t slot = atomicAdd(&n, 1u);
        if (slot < kList) mine[slot] = entry_of(v, i);
    });
    __syncthreads();
    const uint32_t count = min(n, kList);
    if (tid == 0 && count) at = atomicAdd(&w.listed[row], count);
    __syncthreads();
    for (uint32_t i = tid; i < count; i += kPickThreads)
        if (at + i < kList) w.list[(size_t)row * kList + at + i] = mine[i];
}

struct PickLds {
    BinLds bins;
    unsigned long long list[kList];
    uint16_t bin[kList];
    unsigned long long sum[256], both, any, spot_sum;
    uint32_t count[256], digit, before, equal, n;
};
// The first entries of a bin: how many, the sum of their weights, and the index of the last one
struct Spot { uint32_t count; unsigned long long sum; int index; };

template <typename T>
struct Picker {
    const T *x;
    uint32_t vocab, n;           // n: entries in the list
    bool listed;
    BinScale s;
    PickLds &l;

    __device__ __forceinline__ double sum_at(int b, unsigned long long part) const { return l.bins.sum[b] + exp(-(double)b / kBinsPerNat) * (double)part; }
    // every entry of a bin: take(entry); from the list, or where there is none from the row
    template <class Take>
    __device__ __forceinline__ void entries(int b, Take take) const {
        if (listed) {
            for (uint32_t i = threadIdx.x; i < n; i += kPickThreads)
                if (l.bin[i] == b) take(l.list[i]);
        } else {
            each_in(x, 0, vocab, s, run_of(b), first_of(x, 0, vocab), [&](float v, uint32_t i, const Place &) { take(entry_of(v, i)); });
        }
    }
    __device__ __forceinline__ unsigned long long weight_of(unsigned long long e) const { return whole_of(s.place(value_in(e))); }
    // Of the 256 digits that have been counted (l.count, l.sum), the first with entries at which passes(entries up to it, their sum) is true, or the last one with any;
    // c0 and t0 come in front.  Leaves l.digit, l.equal (its entries), l.before and l.spot_sum (all in front of it).
    template <class Passes>
    __device__ __forceinline__ void first_digit(uint32_t c0, unsigned long long t0, Passes passes) {
        const uint32_t tid = threadIdx.x;
        if (tid >= 64) return;
        uint32_t c[4], upto_c = 0;
        unsigned long long t[4], upto_t = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            c[j] = l.count[4 * tid + j];
            t[j] = l.sum[4 * tid + j];
            upto_c += c[j];
            upto_t += t[j];
        }
        uint32_t from_c = c0 - upto_c;
        unsigned long long from_t = t0 - upto_t;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t xc = __shfl_up(upto_c, o, 64);
            const unsigned long long xt = __shfl_up(upto_t, o, 64);
            if ((int)tid >= o) { upto_c += xc; upto_t += xt; }
        }
        from_c += upto_c;
        from_t += upto_t;
        int first = -1, last = -1;
        uint32_t first_c = 0, last_c = 0, first_n = 0, last_n = 0;
        unsigned long long first_t = 0, last_t = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (c[j]) {
                last = j; last_c = from_c; last_t = from_t; last_n = c[j];
                if (first < 0 && passes(from_c + c[j], from_t + t[j])) { first = j; first_c = from_c; first_t = from_t; first_n = c[j]; }
            }
            from_c += c[j];
            from_t += t[j];
        }
        const uint64_t yes = __ballot(first >= 0), some = __ballot(last >= 0);
        const int lane = yes ? __ffsll((unsigned long long)yes) - 1 : 63 - __clzll((long long)some);
        if ((int)tid == lane) {
            l.digit = 4 * tid + (yes ? first : last);
            l.before = yes ? first_c : last_c;
            l.spot_sum = yes ? first_t : last_t;
            l.equal = yes ? first_n : last_n;
        }
    }
    // The first entry of bin b (in the order) at which passes(entries of the bin up to it, their sum) is true, or its last: digit by digit of the entries' bits
    // from the first one that is not common to all.  Equal logits weigh alike, so that the value's bits say where the sum passes, and the index's
    // bits which entry it is (asked for by `which`).
    template <class Passes>
    __device__ Spot find(int b, bool which, Passes passes) {
        const uint32_t tid = threadIdx.x;
        __syncthreads();
        if (tid == 0) { l.both = ~0ull; l.any = 0; }
        __syncthreads();
        {
            unsigned long long both = ~0ull, any = 0;
            entries(b, [&](unsigned long long e) { both &= e; any |= e; });
            for (int o = 32; o; o >>= 1) { both &= __shfl_xor(both, o, 64); any |= __shfl_xor(any, o, 64); }
            if ((tid & 63) == 0 && any) { atomicAnd(&l.both, both); atomicOr(&l.any, any); }
        }
        __syncthreads();
        const unsigned long long differ = l.both ^ l.any;
        int at = differ >> 24 ? 64 - __clzll((long long)differ) : 24;         // bits from here on are known
        unsigned long long known = l.both >> at;
        uint32_t before = 0, equal = l.bins.count[b + 1] - l.bins.count[b];
        unsigned long long sum = 0;
        auto digits = [&](int bits, bool weigh, auto up_to) {
            __syncthreads();
            if (tid < 256) { l.count[tid] = 0; l.sum[tid] = 0; }
            __syncthreads();
            entries(b, [&](unsigned long long e) {
                if (e >> at != known) return;
                const uint32_t digit = (uint32_t)(e >> (at - bits)) & ((1u << bits) - 1);
                atomicAdd(&l.count[digit], 1u);
                if (weigh) atomicAdd(&l.sum[digit], weight_of(e));
            });
            __syncthreads();
            first_digit(before, sum, up_to);
            __syncthreads();
            at -= bits;
            known = known << bits | l.digit;
            before = l.before;
            sum = l.spot_sum;
            equal = l.equal;
        };
        while (at > 24) digits(min(8, at - 24), true, passes);
        const unsigned long long each = weight_of(known << 24);
        uint32_t lo = 1, hi = equal;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (passes(before + mid, sum + mid * each)) hi = mid;
            else lo = mid + 1;
        }
        Spot r{before + lo, sum + lo * each, 0};
        if (which && equal == 1) {
            __syncthreads();
            entries(b, [&](unsigned long long e) {
                if (e >> 24 == known) l.digit = (uint32_t)(e & 0xFFFFFF);
            });
            __syncthreads();
            r.index = (int)l.digit;
        } else if (which) {
            const int bits = 32 - __clz((int)(vocab - 1 | 1));
            known = known << (24 - bits);
            at = bits;
            const uint32_t want = r.count;
            while (at > 0) digits(min(8, at), false, [=](uint32_t c, unsigned long long) { return c >= want; });
            r.index = (int)(known & 0xFFFFFF);
        }
        return r;
    }
};

template <typename T>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(ps_sample_args a, SampleShape sh, SampleWork w) {
    __shared__ PickLds lds;
    BinLds &l = lds.bins;
    const uint32_t row = blockIdx.x, tid = threadIdx.x;
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_row;
    // all that earlier launches have left is asked for at once (which entries of the list there are turns out later)
    constexpr uint32_t kEach = kList / kPickThreads, kMine = kBins / kPickThreads;
    unsigned long long entry[kEach] = {};
    double sums[kMine] = {}, all_sum = 0;
    uint32_t counts[kMine] = {}, all_count = 0;
    Wanted q{};
    if (sh.nfind) {
        q = w.wanted[row];
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) entry[j] = w.list[(size_t)row * kList + tid + j * kPickThreads];
#pragma unroll
        for (uint32_t j = 0; j < kMine; ++j) {
            sums[j] = w.before_sum[(size_t)row * kBinsPad + tid + j * kPickThreads];
            counts[j] = w.before_count[(size_t)row * kBinsPad + tid + j * kPickThreads];
        }
        all_sum = w.before_sum[(size_t)row * kBinsPad + kBins];
        all_count = w.before_count[(size_t)row * kBinsPad + kBins];
    }
    const RowTop top = row_top<kPickThreads>(w.tops + (size_t)row * sh.ntop, sh.ntop, l.fbuf, l.ibuf);
    const float temp = a.temperature ? a.temperature[row] : 1.f;
    if (top.m == -INFINITY || !(temp > 0.f)) {
        if (tid == 0) {
            a.token[row] = top.m == -INFINITY ? -1 : top.at;
            if (a.kept) a.kept[row] = top.m == -INFINITY ? 0 : 1;
        }
        return;
    }
    __syncthreads();
    if (sh.nfind) {
#pragma unroll
        for (uint32_t j = 0; j < kMine; ++j) { l.sum[tid + j * kPickThreads] = sums[j]; l.count[tid + j * kPickThreads] = counts[j]; }
        if (tid == 0) { l.sum[kBins] = all_sum; l.count[kBins] = all_count; }
        __syncthreads();
    } else {
        q = analyse(a, FourBins(w, row), row, l);
    }
    const Runs runs = runs_of(q, l);
    const uint32_t n = runs.before[4];
    Picker<T> p{x, a.vocab, n, n <= kList, bin_scale(top.m, temp), lds};
    if (p.listed && sh.nfind) {
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) {
            const uint32_t i = tid + j * kPickThreads;
            if (i >= n) break;
            lds.list[i] = entry[j];
            lds.bin[i] = (uint16_t)p.s.place(value_in(entry[j])).bin();
        }
    } else if (p.listed) {                            // (a short row: picked out here)
        if (tid == 0) lds.n = 0;
        __syncthreads();
        each_in(p.x, 0, a.vocab, p.s, runs, first_of(p.x, 0, a.vocab), [&](float v, uint32_t i, const Place &y) {
            const uint32_t slot = atomicAdd(&lds.n, 1u);
            if (slot >= kList) return;
            lds.list[slot] = entry_of(v, i);
            lds.bin[slot] = (uint16_t)y.bin();
        });
    }
    auto look_again = [&](int lo, int hi, auto passes) {          // the bin of a goal that is known by now; between the two that it may lie in
        __syncthreads();
        if (tid == 0) l.found[5] = 0x7FFFFFFF;
        __syncthreads();
        look(l, 5, passes);
        __syncthreads();
        return min(max(l.found[5], lo), hi);
    };
    uint32_t kept = l.count[kBins];
    double sum = l.sum[kBins];
    if (q.by_k) {
        const uint32_t want = q.most - l.count[q.bk];
        const Spot in = p.find(q.bk, false, [=](uint32_t c, unsigned long long) { return c >= want; });
        kept = q.most;
        sum = p.sum_at(q.bk, in.sum);
    }
    if (q.by_p) {
        const double goal = q.share * sum;
        const int b = q.p0 == q.p1 ? q.p0 : look_again(q.p0, q.p1, [&](uint32_t j) { return l.sum[j + 1] >= goal; });
        const double base = l.sum[b], middle = exp(-(double)b / kBinsPerNat);
        const Spot in = p.find(b, false, [=](uint32_t, unsigned long long t) { return base + middle * (double)t >= goal; });
        if (l.count[b] + in.count < kept) { kept = l.count[b] + in.count; sum = p.sum_at(b, in.sum); }
    }
    if (q.by_m) {
        __syncthreads();
        if (tid == 0) { lds.before = 0; lds.spot_sum = 0; }
        __syncthreads();
        if (q.reach >= 0.0)
            p.entries(q.bm, [&](unsigned long long e) {
                if (p.s.place(value_in(e)).value() <= q.reach) { atomicAdd(&lds.before, 1u); atomicAdd(&lds.spot_sum, p.weight_of(e)); }
            });
        __syncthreads();
        const uint32_t c = q.reach >= 0.0 ? l.count[q.bm] + lds.before : 0;
        if (c == 0) { kept = 1; sum = 34359738368.0; }
        else if (c < kept) { kept = c; sum = p.sum_at(q.bm, lds.spot_sum); }
    }
    const double goal = q.u * sum;
    const int b = q.d0 == q.d1 ? q.d0 : look_again(q.d0, q.d1, [&](uint32_t j) { return l.sum[j + 1] > goal; });
    const double base = l.sum[b], middle = exp(-(double)b / kBinsPerNat);
    const uint32_t end = kept, ahead = l.count[b];
    const Spot in = p.find(b, true, [=](uint32_t c, unsigned long long t) { return base + middle * (double)t > goal || ahead + c >= end; });
    if (tid == 0) {
        a.token[row] = in.index;
        if (a.kept) a.kept[row] = (int)kept;
    }
}

// Chunks: as many as make about 2048 workgroups of the first launch and 1024 of the second, or 320 where rows are few
// (each leaves about a thousand atomic additions: 16 rows of 128256, 17 us with 1024, 8 with 256); of the third as few as keep about 768, each
// of which works the bins out for itself.
SampleShape sample_shape(const ps_sample_args &a) {
    SampleShape sh;
    const uint64_t rows = std::max(1u, a.n_rows);
    static_assert(2 * kRound <= 1u << 13, "two rounds in a bin: 14 bits count them");
    auto cut = [&](uint64_t groups, uint32_t multiple, uint32_t *len, uint32_t *n) {
        const uint64_t chunks = std::max<uint64_t>(1, groups / rows);
        *len = (uint32_t)(((a.vocab + chunks - 1) / chunks + multiple - 1) / multiple * multiple);
        *n = (a.vocab + *len - 1) / *len;
    };
    cut(2048, 2048, &sh.top, &sh.ntop);
    cut(rows < 128 ? 320 : 1024, kRound / 2, &sh.bins, &sh.nbins);
    sh.find = sh.nfind = 0;
    if (a.vocab > kShortRow) cut(768, kRound, &sh.find, &sh.nfind);
    return sh;
}
uint64_t sample_work(const ps_sample_args &a, const SampleShape &sh, uint8_t *base, SampleWork *w) {
    uint64_t off = 0;
    auto take = [&](uint64_t bytes) { uint8_t *p = base ? base + off : nullptr; off = align_up(off + bytes, kAlign); return p; };
    w->tops = reinterpret_cast<RowTop *>(take((uint64_t)a.n_rows * sh.ntop * sizeof(RowTop)));
    w->sums = reinterpret_cast<unsigned long long *>(take((uint64_t)a.n_rows * kBins * 8));
    w->counts = reinterpret_cast<uint32_t *>(take((uint64_t)a.n_rows * kBins * 4));
    w->listed = reinterpret_cast<uint32_t *>(take((uint64_t)a.n_rows * 4));
    w->list = reinterpret_cast<unsigned long long *>(take((uint64_t)a.n_rows * kList * 8));
    const uint64_t found = sh.nfind ? a.n_rows : 0;
    w->wanted = reinterpret_cast<Wanted *>(take(found * sizeof(Wanted)));
    w->before_sum = reinterpret_cast<double *>(take(found * kBinsPad * 8));
    w->before_count = reinterpret_cast<uint32_t *>(take(found * kBinsPad * 4));
    return off;
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
    PS_WANT((uint64_t)a->n_tokens * a->n_q_heads <= 0x7FFFFFFFull, "%u tokens of %u heads are too many for one call", a->n_tokens, a->n_q_heads);
    PS_WANT(a->n_prefix <= kMostPrefixes, "up to %u prefixes (got %u)", kMostPrefixes, a->n_prefix);
    PS_WANT(a->max_length <= (uint32_t)kMostPositions && a->max_length <= (uint64_t)a->width * a->page, "lengths of up to %u in tables of %u pages of %u", a->max_length, a->width, a->page);
    PS_WANT(!a->n_prefix || (a->max_prefix <= (uint32_t)kMostPositions && a->max_prefix <= (uint64_t)a->prefix_width * a->page), "prefixes of up to %u in tables of %u pages of %u", a->max_prefix,
            a->prefix_width, a->page);
    return PS_OK;
}

// How the work is dealt out.  Runs bring the launch to about the workgroups that the chip holds at once (two per CU).  Shared prefixes beside own
// positions: one workgroup per CU for the prefixes, which come first, so that the other place is the loads' (64 sequences, 32 / 8 heads, prefix
// 32761: own lengths to 1000 in 105 us, to 4000 in 184; with two per CU 108 and 218); two where own positions are few (lengths of 1: 76 for 93).  Own
// positions of several sequences: as many runs as places, since every run has a start of dependent loads and a record (64 sequences of up to 1000, 32 / 8 heads,
// 34 us; with 1024 runs 41, with 2048 45; only few sequences of very different lengths would rather have more: 48 of up to 8190, 16 / 8 heads of 64, 112 for 106).
PageDeal page_deal(const ps_page_attention_args &a) {
    PageDeal d{};
    const uint32_t G = a.n_q_heads / a.n_kv_heads;
    const uint64_t tokens = std::min(a.max_tokens, a.n_tokens), rows = tokens * G;
    const bool prefixes = a.n_prefix && a.max_prefix;
    // Prefixes of few positions in all are read again for each sequence sooner than joined from results of their own: 16 sequences, 32 / 8 heads of 128,
    // 500 + 500 positions 16.5 us for 25.8, 1000 + 500 19.3 for 22.3, 2000 + 100 21.8 for 20.6; 64 sequences, 250 + 250 18.3 for 21.2, 1000 + 500 35.5 for 27.9
    const bool small = prefixes && (uint64_t)a.n_seq * a.n_kv_heads * a.max_prefix <= 196608;
    d.shared = rows <= kFewRows && !small;
    // (1024 rows for 64 sequences of a token each, 32 / 8 heads behind 32761: dealt out by 1024 the prefix was one run of 16 workgroups, 620 us for 109)
    d.tokens = (uint32_t)std::min<uint64_t>(a.n_tokens, a.n_seq * tokens);
    d.by_seq = d.tokens < a.n_tokens;
    auto cut = [](uint64_t units, uint64_t want, uint64_t whole, uint64_t least, uint64_t multiple, uint32_t *n, uint32_t *len) {
        const uint64_t most = std::max<uint64_t>(1, whole / least), runs = std::min(std::max<uint64_t>(1, want / std::max<uint64_t>(1, units)), most);
        *len = (uint32_t)std::max<uint64_t>(multiple, ((whole + runs - 1) / runs + multiple - 1) / multiple * multiple);
        *n = (uint32_t)std::max<uint64_t>(1, (whole + *len - 1) / *len);
    };
    if (d.shared) {
        d.nt = rows <= 16 ? 1 : 2;
        auto blocks = [&](uint64_t n) { return prefixes ? (uint32_t)((n * G + 127ull * a.n_prefix) / 128) : 0; };
        d.blocks = blocks(d.tokens);
        d.most = blocks(a.n_tokens);
        // about how long each part takes by itself, at 700 TFLOP/s and 5 TB/s
        const double prefix_us = (double)d.tokens * a.n_q_heads * a.max_prefix * a.head_dim * 4 / 700e6, own_us = (double)a.n_seq * a.n_kv_heads * a.max_length * a.head_dim * 4 / 5e6;
        if (prefixes) cut((uint64_t)d.blocks * a.n_kv_heads, own_us * 4 > prefix_us ? 256 : 512, a.max_prefix, 256, kStep, &d.psplit, &d.plen);
        cut((uint64_t)a.n_seq * a.n_kv_heads, a.n_seq > 1 ? 512 : 1024, a.max_length, 128, 4 * kTile, &d.osplit, &d.olen);
        d.direct = d.psplit == 0 && d.osplit == 1;
    } else if (rows <= kFewRows) {
        d.nt = rows <= 16 ? 1 : 2;
        d.blocks = 1;
        const uint64_t tiles = (prefixes ? (a.max_prefix + kTile - 1) / kTile : 0) + (a.max_length + kTile - 1) / kTile;
        // (up to 1024 positions in one run: without a merge 16.5 us for 17.3, 16 sequences of 500 + 500; longer ones in runs of 512: 500 + 3000 30.7 us for 34.6)
        cut((uint64_t)a.n_seq * a.n_kv_heads, 512, tiles, tiles <= 32 ? 32 : 16, 4, &d.osplit, &d.olen);
        d.direct = d.osplit == 1;
    } else {
        d.blocks = (uint32_t)((rows + 127) / 128);
        const uint64_t steps = (prefixes ? (a.max_prefix + kStep - 1) / kStep : 0) + (a.max_length + kStep - 1) / kStep;
        // (up to four steps in one run: without a merge 17.6 us for 19, 16 sequences of 16 tokens behind 100 + 100)
        cut((uint64_t)a.n_seq * a.n_kv_heads * d.blocks, 512, steps, steps <= 4 ? 4 : 2, 1, &d.osplit, &d.olen);
        d.direct = d.osplit == 1;
    }
    return d;
}
uint64_t page_workspace(const ps_page_attention_args &a, const PageDeal &d) {
    return d.direct ? 0 : align_up((uint64_t)d.tokens * a.n_q_heads * (d.psplit + d.osplit) * (a.head_dim + 4) * 4, kAlign);
}
// workgroups of the merge for a token
uint32_t merge_groups(const ps_page_attention_args &a) { const uint32_t heads = 1024 / a.head_dim; return (a.n_q_heads + heads - 1) / heads; }
// workgroups of a call's launches, 0: more than a launch holds
uint64_t page_groups(const ps_page_attention_args &a, const PageDeal &d, uint64_t *prefix8, uint64_t *own8) {
    *prefix8 = d.shared ? ((uint64_t)a.n_kv_heads * d.psplit + 7) / 8 * d.blocks : 0;
    *own8 = ((uint64_t)a.n_seq * a.n_kv_heads * d.osplit + 7) / 8 * (d.shared ? 1 : d.blocks);
    const uint64_t groups = (*prefix8 + *own8) * 8, merge = (uint64_t)a.n_seq * std::min(a.max_tokens, a.n_tokens) * merge_groups(a);
    return groups > kMostGroups || (!d.direct && merge > kMostGroups) ? 0 : groups;
}

// a kernel that takes more LDS than a launch gets by itself: announced once per device
template <class K>
hipError_t take_lds(K kernel, uint32_t lds, std::atomic<uint64_t> &done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess || (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1))) return e;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e == hipSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}
template <typename T, int D, int NT, bool kSeek>
hipError_t launch_shared(const ps_page_attention_args &a, const PageDeal &d, uint32_t prefix8, uint32_t own8, float *part, hipStream_t st) {
    static std::atomic<uint64_t> done;
    constexpr uint32_t lds = std::max(few_lds<D, NT>(), many_lds<D>());
    const hipError_t e = take_lds(&page_shared_kernel<T, D, NT, kSeek>, lds, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((page_shared_kernel<T, D, NT, kSeek>), dim3((prefix8 + own8) * 8), dim3(256), lds, st, a, d, log2_of(a.page), prefix8, part);
    return hipGetLastError();
}
template <typename T, int D, bool kSeek>
hipError_t launch_rows(const ps_page_attention_args &a, const PageDeal &d, uint32_t own8, float *part, hipStream_t st) {
    static std::atomic<uint64_t> done;
    const hipError_t e = take_lds(&page_rows_kernel<T, D, kSeek>, many_lds<D>(), done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((page_rows_kernel<T, D, kSeek>), dim3(own8 * 8), dim3(256), many_lds<D>(), st, a, d, log2_of(a.page), part);
    return hipGetLastError();
}
template <typename T, int D, int NT, bool kSeek>
hipError_t launch_few(const ps_page_attention_args &a, const PageDeal &d, float *part, hipStream_t st) {
    static std::atomic<uint64_t> done;
    constexpr uint32_t lds = few_lds<D, NT>();
    const hipError_t e = take_lds(&page_few_kernel<T, D, NT, kSeek>, lds, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((page_few_kernel<T, D, NT, kSeek>), dim3(a.n_seq * a.n_kv_heads * d.osplit), dim3(256), lds, st, a, d, log2_of(a.page), part);
    return hipGetLastError();
}
template <typename T, int D, bool kSeek>
hipError_t launch_walk(const ps_page_attention_args &a, const PageDeal &d, float *part, hipStream_t st) {
    uint64_t prefix8, own8;
    page_groups(a, d, &prefix8, &own8);
    if (d.shared) return (d.nt == 1 ? launch_shared<T, D, 1, kSeek> : launch_shared<T, D, 2, kSeek>)(a, d, (uint32_t)prefix8, (uint32_t)own8, part, st);
    if (d.nt) return (d.nt == 1 ? launch_few<T, D, 1, kSeek> : launch_few<T, D, 2, kSeek>)(a, d, part, st);
    return launch_rows<T, D, kSeek>(a, d, (uint32_t)own8, part, st);
}
template <typename T, int D>
hipError_t launch_page_attention(const ps_page_attention_args &call, float *part, hipStream_t st) {
    ps_page_attention_args a = call;
    a.max_tokens = std::min(a.max_tokens, a.n_tokens);
    const PageDeal d = page_deal(a);
    // (where there is a page, page 0 can be read; where there are no positions, tables may be NULL)
    if (a.n_pages == 0) a.max_length = a.max_prefix = 0;
    if (a.max_length == 0) a.width = 0;
    if (a.max_prefix == 0) a.prefix_width = 0;
    const hipError_t e = d.by_seq && !d.direct ? launch_walk<T, D, true>(a, d, part, st) : launch_walk<T, D, false>(a, d, part, st);
    if (e != hipSuccess || d.direct) return e;
    hipLaunchKernelGGL((page_merge_kernel<T, D>), dim3(a.n_seq * a.max_tokens * merge_groups(a)), dim3(256), 0, st, a, d, part);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_sample(const ps_sample_args &a, const SampleShape &sh, const SampleWork &w, hipStream_t st) {
    hipLaunchKernelGGL(sample_rows_kernel<T>, dim3(sh.ntop, a.n_rows), dim3(kRowThreads), 0, st, a, sh, w);
    hipLaunchKernelGGL(sample_bins_kernel<T>, dim3(sh.nbins, a.n_rows), dim3(kPickThreads), 0, st, a, sh, w);
    if (sh.nfind) hipLaunchKernelGGL(sample_find_kernel<T>, dim3(sh.nfind, a.n_rows), dim3(kPickThreads), 0, st, a, sh, w);
    hipLaunchKernelGGL(sample_pick_kernel<T>, dim3(a.n_rows), dim3(kPickThreads), 0, st, a, sh, w);
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
    *bytes = page_workspace(*a, page_deal(*a));
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
    for (uint64_t n : {a->k_row, a->v_row}) PS_WANT(n < (1ull << 31) / std::max(32u, a->page), "a page's rows, and 32 rows, must span less than 4 GiB (stride of %llu elements)", (unsigned long long)n);
    for (uint64_t n : {a->k_page, a->v_page}) PS_WANT(n < 1ull << 35, "pages must lie less than 64 GiB apart (stride of %llu elements)", (unsigned long long)n);
    for (const int32_t *p : {a->first, a->length, a->table, a->group_first, a->prefix_length, a->prefix_table}) PS_WANT(aligned(p, 4), "tables must be aligned to 4 bytes");
    PS_WANT(workspace_bytes >= need && (need == 0 || (workspace && aligned(workspace, kAlign))), "a workspace of %llu bytes, 256-byte aligned, is needed", (unsigned long long)need);
    uint64_t prefix8, own8;
    PS_WANT(page_groups(*a, page_deal(*a), &prefix8, &own8), "too many sequences, tokens and heads for one call");
    hipStream_t st = static_cast<hipStream_t>(stream);
    float *part = static_cast<float *>(workspace);
    if (a->type == PS_TYPE_F16) PS_TRY(a->head_dim == 64 ? (launch_page_attention<f16_t, 64>(*a, part, st)) : (launch_page_attention<f16_t, 128>(*a, part, st)));
    else PS_TRY(a->head_dim == 64 ? (launch_page_attention<bf16_t, 64>(*a, part, st)) : (launch_page_attention<bf16_t, 128>(*a, part, st)));
    return PS_OK;
}

int32_t ps_sample_workspace(const ps_sample_args *a, uint64_t *bytes) {
    PS_WANT(a && bytes, "NULL argument");
    PS_WANT(a->type <= PS_TYPE_F32, "unknown type %u", a->type);
    PS_WANT(a->vocab >= 1 && a->vocab <= 1u << 24, "vocab 1 .. 2^24 (got %u)", a->vocab);
    PS_WANT(a->n_rows <= 65535, "up to 65535 rows (got %u)", a->n_rows);
    SampleWork w;
    *bytes = sample_work(*a, sample_shape(*a), nullptr, &w);
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
    const SampleShape sh = sample_shape(*a);
    PS_WANT((uint64_t)std::max({sh.ntop, sh.nbins, sh.nfind}) * a->n_rows <= kMostGroups / 2, "%u rows of %u entries are too many for one call", a->n_rows, a->vocab);
    SampleWork w;
    sample_work(*a, sh, static_cast<uint8_t *>(workspace), &w);
    if (a->type == PS_TYPE_F16) PS_TRY(launch_sample<f16_t>(*a, sh, w, st));
    else if (a->type == PS_TYPE_BF16) PS_TRY(launch_sample<bf16_t>(*a, sh, w, st));
    else PS_TRY(launch_sample<float>(*a, sh, w, st));
    return PS_OK;
}

}  // extern "C"
