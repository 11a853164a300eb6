// Rotary positions of a layer's queries and keys, and the rows that go into a paged cache with the rotation on the way.
// Both read every row once and write it once: memory, or latency for a few tokens.  Measured, in a graph: queries and keys of 18432 tokens, bf16, 302 MB, 62.5 us =
// 4.8 TB/s (a copy of as many bytes 59.4); 8192 tokens of a stack into its pages, 1074 MB, 211 us = 5.1 TB/s (206); one token for each of 8 sequences 3.2 us, a
// launch, and 6.7 us a call from Python.
//
// D / 16 threads have a row, two runs of eight channels each, so that a pair of channels meets in one thread and a rotated row
// needs nothing from other lanes.  A thread stays with a token while it goes through heads: angles depend on the token alone.
#include <algorithm>
#include <cstring>

#include "launch.h"
#include "rotary.h"

namespace zipvl {

struct Rows { char* base; int64_t b, h, t; };                // a tensor [B, H, n, d]: strides in bytes
struct RowsIn { const char* base; int64_t b, h, t; };
template <typename R> __device__ __forceinline__ auto row_of(const R& r, int b, int h, int t) { return r.base + b * r.b + h * r.h + t * r.t; }

// Tokens of all batch elements follow each other.  A workgroup has 256 D^-1 16 rows a turn: `tokens` of them (a power of two) of as many
// heads as that leaves, and goes through the heads from its first in steps of `step`.
struct Walk {
    int n, total, tokens_log2, step;                         // total = B n
    int base;                                                // the launch's first token
    uint32_t inv_n;
};

template <typename T, int D>
__global__ __launch_bounds__(256) void rotate_kernel(RowsIn Q, RowsIn K, Rows Qo, Rows Ko, int Hq, int heads, Walk w,
                                                     const int32_t* __restrict__ pos, Turns turns)
{
    constexpr int kThreads = D / 16;
    const int slot = threadIdx.x / kThreads, c = threadIdx.x % kThreads;
    const int token = w.base + (blockIdx.x << w.tokens_log2) + (slot & ((1 << w.tokens_log2) - 1));
    const int first = blockIdx.y * ((256 / kThreads) >> w.tokens_log2) + (slot >> w.tokens_log2);
    if (token >= w.total || first >= heads) return;
    const int b = divided(token, w.n, w.inv_n), t = token - b * w.n;
    const Runs runs(c, turns.pairs, turns.neighbours);
    struct Row { Run<T> a, b; };
    auto load = [&](int h) {
        const RowsIn& in = h < Hq ? Q : K;
        const T* src = reinterpret_cast<const T*>(row_of(in, b, h < Hq ? h : h - Hq, t));
        return Row{load_run(src + runs.a), load_run(src + runs.b)};
    };
    Angles at;
    if (runs.first >= 0) at.ask(turns, runs.first, pos + token, (int64_t)w.total);
    Row row = load(first);                                   // while the angles are taken
    if (runs.first >= 0) at.take(turns);
    for (int h = first; h < heads; h += w.step) {
        const Rows& out = h < Hq ? Qo : Ko;
        T* dst = reinterpret_cast<T*>(row_of(out, b, h < Hq ? h : h - Hq, t));
        if (runs.first >= 0) turn_runs(row.a, row.b, at, turns.neighbours);
        store_run(dst + runs.a, row.a);
        store_run(dst + runs.b, row.b);
        if (h + w.step < heads) row = load(h + w.step);
    }
}

constexpr int kHeadsGrid = 32768;     // workgroups on the grid's second axis; an axis has less than 65536

struct PagedRows {
    char *K, *V;
    int num_pages, page_log2, width;                         // width: pages in a unit's row of the table
    const int32_t* table;
    const int32_t* start;
    int32_t* len;                                            // NULL: another launch leaves it (advance_kernel)
    const int32_t *idx, *k;
    int per_batch;
};

__device__ __forceinline__ int paged_start(const PagedRows& p, int u) { return max(0, min(p.start[u], p.width << p.page_log2)); }
__device__ __forceinline__ int paged_count(const PagedRows& p, int u, int b, int n) { return p.k ? max(0, min(p.k[p.per_batch ? b : u], n)) : n; }
__device__ __forceinline__ int paged_len(const PagedRows& p, int start, int count) { return (int)min((int64_t)start + count, (int64_t)p.width << p.page_log2); }

// Heads [0, Hkv) are those of K and V, [Hkv, heads) of Q (as many as are given).  A row's way is two round trips to memory: where a unit starts, how
// much it brings, which token this is and its positions, all at once; then the row, and the page that it goes to, while the angles are taken.
// Every head has threads of its own: going through heads as rotate_kernel does saves angles and costs 5 to 10 % (in a graph, 64 tokens of 64 sequences: 4.1 us
// instead of 3.8, 777 tokens of 5 sequences, fp32 10.5 instead of 10.0, 8192 tokens of a stack 221 instead of 211; only where 0.4 of 18432 tokens
// are kept it is 8.6 instead of 9.0, since threads of tokens that go are there for nothing).
template <typename T, int D, bool TURN>
__global__ __launch_bounds__(256) void paged_append_kernel(RowsIn K, RowsIn V, RowsIn Q, Rows Qo, int Hkv, int G, uint32_t inv_G, int heads, Walk w, PagedRows p,
                                                           const int32_t* __restrict__ pos, Turns turns)
{
    constexpr int kThreads = D / 16;
    const int slot = threadIdx.x / kThreads, c = threadIdx.x % kThreads;
    const int token = w.base + (blockIdx.x << w.tokens_log2) + (slot & ((1 << w.tokens_log2) - 1));
    if (token >= w.total) return;
    const int b = divided(token, w.n, w.inv_n), i = token - b * w.n;         // row i of what a unit brings
    const Runs runs(c, TURN ? turns.pairs : 0, TURN ? turns.neighbours : 0);
    Angles at;
    const bool turn = TURN && runs.first >= 0;
    if (turn && !p.idx) at.ask(turns, runs.first, pos + token, (int64_t)w.total);
    const int h = (blockIdx.z * kHeadsGrid + blockIdx.y) * ((256 / kThreads) >> w.tokens_log2) + (slot >> w.tokens_log2);
    if (h >= heads) return;
    const bool query = h >= Hkv;
    const int g = query ? divided(h - Hkv, G, inv_G) : h, u = b * Hkv + g, set = p.per_batch ? b : u;
    int brings = w.n, starts = 0, which = i;
    if (p.k) brings = p.k[set];
    if (!query) starts = p.start[u];                         // only the threads of a row of K may read it: len may stand there
    if (p.idx) which = p.idx[(int64_t)set * w.n + i];
    asm volatile("" : "+v"(brings), "+v"(starts), "+v"(which));              // here they are waited for, all three at once
    const int count = max(0, min(brings, w.n)), start = max(0, min(starts, p.width << p.page_log2)), t = max(0, min(which, w.n - 1));
    if (!query && i == 0 && c == 0 && p.len) p.len[u] = paged_len(p, start, count);
    if (i >= count) return;
    if (query) {
        const T* src = reinterpret_cast<const T*>(row_of(Q, b, h - Hkv, t));
        T* dst = reinterpret_cast<T*>(row_of(Qo, b, h - Hkv, t));
        Run<T> ra = load_run(src + runs.a), rb = load_run(src + runs.b);
        if (turn) {
            at.take(turns);
            turn_runs(ra, rb, at, turns.neighbours);
        }
        store_run(dst + runs.a, ra);
        store_run(dst + runs.b, rb);
        return;
    }
    const int64_t row = (int64_t)start + i;
    if (row >> p.page_log2 >= p.width) return;               // behind the table
    if (turn && p.idx) at.ask(turns, runs.first, pos + (int64_t)b * w.n + t, (int64_t)w.total);
    const int page = p.table[(int64_t)u * p.width + (row >> p.page_log2)];
    const T* ks = reinterpret_cast<const T*>(row_of(K, b, g, t));
    const T* vs = reinterpret_cast<const T*>(row_of(V, b, g, t));
    Run<T> ra = load_run(ks + runs.a), rb = load_run(ks + runs.b);
    const Run<T> va = load_run(vs + runs.a), vb = load_run(vs + runs.b);
    asm volatile("" ::: "memory");                           // the rows are asked for before it is known that there is a page for them
    if (turn) {
        at.take(turns);
        turn_runs(ra, rb, at, turns.neighbours);
    }
    if ((unsigned)page >= (unsigned)p.num_pages) return;
    const int64_t at_row = (((int64_t)page << p.page_log2) + (row & ((1 << p.page_log2) - 1))) * D;
    T *kd = reinterpret_cast<T*>(p.K) + at_row, *vd = reinterpret_cast<T*>(p.V) + at_row;
    store_run(kd + runs.a, ra);
    store_run(kd + runs.b, rb);
    store_run(vd + runs.a, va);
    store_run(vd + runs.b, vb);
}

// len of every unit, where it stands in the place of start and several workgroups of the append read that
__global__ __launch_bounds__(256) void advance_kernel(PagedRows p, int32_t* len, int units, int Hkv, int n) {
    const int u = blockIdx.x * 256 + threadIdx.x;
    if (u < units) len[u] = paged_len(p, paged_start(p, u), paged_count(p, u, u / Hkv, n));
}

static Turns turns_of(const zipvl_rope* r, bool inverse) {
    Turns t = {};
    if (!r) return t;
    t.axes = r->axes;
    t.pairs = r->pairs;
    t.neighbours = r->layout == ZIPVL_ROPE_NEIGHBOURS;
    t.backwards = inverse ? 0x80000000u : 0u;
    for (int i = 0; i < r->pairs; ++i) {                     // in whole numbers of 64 bits and their products: long double took 2 to 8 us of a call
        uint64_t bits;
        std::memcpy(&bits, &r->freq[i], sizeof(bits));
        const int shift = 1077 - (int)(bits >> 52 & 0x7FF);  // |freq| = m 2^(2 - shift), below 8
        const uint64_t m = (bits & 0xFFFFFFFFFFFFFull) | 1ull << 52;
        const uint64_t part = shift < 128 ? (uint64_t)((unsigned __int128)m * 0xA2F9836E4E441529ull >> shift) : 0;     // 2^66 / (2 pi)
        t.turn[i] = r->freq[i] < 0 ? 0 - part : part;
        t.axis[i] = (uint8_t)r->axis[i];
    }
    return t;
}

static RowsIn rows_in(const void* p, const int64_t (&s)[3], int e) { return {(const char*)p, s[0] * e, s[1] * e, s[2] * e}; }
static Rows rows_out(void* p, const int64_t (&s)[3], int e) { return {(char*)p, s[0] * e, s[1] * e, s[2] * e}; }

// `apart`: every head has threads of its own; else about kRotateGrid workgroups, each with several heads of its tokens, whose angles it takes once
// (18432 tokens: 62.5 us; with 2048 65.4, with 4096 63.1, with 16384 63.9).
constexpr int kRotateGrid = 8192;
static dim3 walk_of(const zipvl_dims& d, int heads, bool apart, Walk& w) {
    const int rows = 4096 / d.d;                             // of a workgroup, a turn
    w.n = d.n;
    w.total = d.B * d.n;
    w.tokens_log2 = 0;
    while ((1 << w.tokens_log2) < rows && (1 << w.tokens_log2) < w.total) ++w.tokens_log2;
    const int lanes = rows >> w.tokens_log2, tiles = (w.total + (1 << w.tokens_log2) - 1) >> w.tokens_log2;
    const int most = (heads + lanes - 1) / lanes;
    const int parts = apart ? most : std::min(most, (kRotateGrid + tiles - 1) / tiles);
    w.step = parts * lanes;
    w.inv_n = inverse(d.n);
    return dim3(tiles, std::min(parts, kHeadsGrid), (parts + kHeadsGrid - 1) / kHeadsGrid);
}

// An axis of a grid has fewer than 2^32 threads: what goes beyond 2^23 workgroups of tokens is another launch.
constexpr int kTokenGrid = 1 << 23;
template <typename F> static void over_tokens(Walk& w, dim3 grid, F&& launch) {
    const int most = kTokenGrid << w.tokens_log2;
    for (w.base = 0; w.base < w.total; w.base += most) {
        grid.x = (std::min(w.total - w.base, most) + (1 << w.tokens_log2) - 1) >> w.tokens_log2;
        launch(grid);
    }
}

int launch_rotate(const void* Q, const void* K, const zipvl_dims& d, const int32_t* pos, const zipvl_rope& rope, int flags, void* Qo, void* Ko,
                  const zipvl_dims& out, hipStream_t st)
{
    const int e = d.dtype == ZIPVL_BF16 ? 2 : 4;
    const int Hq = Q ? d.Hq : 0, heads = Hq + (K ? d.Hkv : 0);
    Walk w;
    const dim3 grid = walk_of(d, heads, false, w);
    const Turns turns = turns_of(&rope, flags & ZIPVL_ROTATE_INVERSE);
    KernelTimer tm(ZIPVL_K_ROTATE, st);
    over_tokens(w, grid, [&](dim3 grid) {
#define ZIPVL_ROTATE(T, D)                                                                                                         \
    hipLaunchKernelGGL((rotate_kernel<T, D>), grid, dim3(256), 0, st, rows_in(Q, d.q_strides, e), rows_in(K, d.k_strides, e), \
                       rows_out(Qo, out.q_strides, e), rows_out(Ko, out.k_strides, e), Hq, heads, w, pos, turns)
    if (d.dtype == ZIPVL_BF16) { if (d.d == 128) ZIPVL_ROTATE(__bf16, 128); else ZIPVL_ROTATE(__bf16, 64); }
    else { if (d.d == 128) ZIPVL_ROTATE(float, 128); else ZIPVL_ROTATE(float, 64); }
#undef ZIPVL_ROTATE
    });
    return check_launch("rotate");
}

int launch_paged_append(const void* K, const void* V, const zipvl_dims& d, const int32_t* idx, const int32_t* k, const int32_t* pos,
                        const zipvl_rope* rope, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* start,
                        int32_t* len, const void* Q, void* Qo, int flags, hipStream_t st)
{
    const int e = d.dtype == ZIPVL_BF16 ? 2 : 4;
    const int heads = d.Hkv + (Q ? d.Hq : 0);
    Walk w;
    const dim3 grid = walk_of(d, heads, true, w);
    const Turns turns = turns_of(rope, false);
    const bool in_place = len == start && d.n > 1;           // one token: the threads that read a start are one wave, and its store comes after
    PagedRows p = {(char*)pages.K, (char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table_pages, table, start, in_place ? nullptr : len,
                   idx, k, (flags & ZIPVL_T_PER_BATCH) ? 1 : 0};
    const int64_t qo[3] = {(int64_t)d.Hq * d.n * d.d, (int64_t)d.n * d.d, d.d};
    {
        KernelTimer tm(ZIPVL_K_PAGED_APPEND, st);
        over_tokens(w, grid, [&](dim3 grid) {
#define ZIPVL_APPEND(T, D, TURN)                                                                                                           \
    hipLaunchKernelGGL((paged_append_kernel<T, D, TURN>), grid, dim3(256), 0, st, rows_in(K, d.k_strides, e), rows_in(V, d.v_strides, e),  \
                       rows_in(Q, d.q_strides, e), rows_out(Qo, qo, e), d.Hkv, d.Hq / d.Hkv, inverse(d.Hq / d.Hkv), heads, w, p, pos, turns)
#define ZIPVL_APPEND_T(T, D) do { if (rope) ZIPVL_APPEND(T, D, true); else ZIPVL_APPEND(T, D, false); } while (0)
        if (d.dtype == ZIPVL_BF16) { if (d.d == 128) ZIPVL_APPEND_T(__bf16, 128); else ZIPVL_APPEND_T(__bf16, 64); }
        else { if (d.d == 128) ZIPVL_APPEND_T(float, 128); else ZIPVL_APPEND_T(float, 64); }
#undef ZIPVL_APPEND_T
#undef ZIPVL_APPEND
        });
    }
    const int rc = check_launch("paged_append");
    if (rc || !in_place) return rc;
    const int units = d.B * d.Hkv;
    KernelTimer tm(ZIPVL_K_PAGED_ADVANCE, st);
    hipLaunchKernelGGL(advance_kernel, dim3((units + 255) / 256), dim3(256), 0, st, p, len, units, d.Hkv, d.n);
    return check_launch("paged_append lengths");
}

}  // namespace zipvl
