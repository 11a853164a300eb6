// Attention of several new tokens to a paged cache (Eq. (2) / Eq. (5) with a causal end): pieces of prompts, questions about a cached
// image, drafted tokens.
//
// A unit (batch element, KV head) has c G rows of queries, the G heads of its group token by token, so that a key that is met serves all heads of the group.
// They go in tiles of rows against the prefix of the unit's group and then its own rows, up to the row that the tile's last token stands in.
// Two forms:
//   few     up to 32 rows a unit, not packed: memory-bound.  Each wave has all of them and tiles of 32 keys of its own (wavepart.h, as decode).  Four tokens each of 16 conversations of up to 33 000
//           rows, bf16: 78 us for 341 MB, 4.4 TB/s.
//   many    128 rows a workgroup, 32 a wave; tiles of keys in LDS are shared by the four waves, two deep, or three where whole tiles of bf16 follow each other (piped).  2048 tokens of 28
//           heads on 4 behind 16 384, bf16: 492 us, 1.0 PFLOP/s, the matrix units busy 54 % of the time, of a large product 1.14 (543 us two deep throughout, 506 with the third).
// S^T = K Q^T and O^T += V^T P^T on matrix tiles, so that a lane has one row of queries and its statistics are scalars.
//
// The rows of a group's units may go together against its prefix (packed rows): eight questions of 6 tokens of 7 heads about 7200 rows 33 us and not 38 a unit at a time, 55 tokens 75 and not 88.
//
// How the keys are cut up is decided on the device, where the lengths are (find_place): every workgroup adds up the tiles of keys that all tiles of rows see
// and takes a piece; a tile of rows whose keys are many gets several workgroups, and their parts are joined by a second launch.  To know its place takes a workgroup 4 us of a chain of
// loads and barriers; that all see how long each is, and not only its unit, took five prompts of unequal length from 65 to 46 us.
#include <algorithm>
#include <atomic>

#include "launch.h"
#include "planes.h"
#include "wavepart.h"

namespace zipvl {

constexpr int kRowsMany = 128;
constexpr int kLeastMany = 4, kLeastFew = 4;                 // tiles of keys (64, or 32 of fp32; 32) that a piece has at least: packed rows with 4, 8, 12, 16 took 28, 33, 37, 43 us (94 rows, 4964 keys), few rows of 616 keys with 4, 8 13.3, 14.7
constexpr int kScanItems = 2048;                             // more tiles of rows than this get a workgroup each, whatever their keys

// 8-byte fields and pairs of others only: it is read again as a row of 32-bit numbers
struct Chunk {
    const char *K, *V;
    int num_pages, page_log2;
    const int32_t* table; int width; const int32_t *len, *cnt;
    const int32_t* prefix_table; int prefix_width; const int32_t *prefix_len, *group_begin; int groups;
    int B, Hq, Hkv, G, n, units;
    uint32_t inv_Hkv, inv_G;
    const char* Q; int64_t q[3];
    char* O; int64_t o[3];
    float* lse;
    float c;                                                 // scale log2(e)
    int slots;                                               // packed: tiles of rows that a KV head's groups may have; 0: rows are not packed
};

// Parts of tiles of rows that were cut: rows of D sums and (offset, sum) each.  pieces: of a tile (those of packed rows first), its first row here and into how many its keys were
// cut; shared: of a unit, the first tile of its group's packed rows (-1: none) and its first row among them.
struct ChunkParts { float* o; float* ml; int2* pieces; int2* shared; int rows; };

__device__ __forceinline__ int between(int v, int low, int high) { return max(low, min(v, high)); }

// the group that batch element b is in, -1: none.  begin: groups + 1 numbers that ascend
__device__ __forceinline__ int group_with(const int32_t* begin, int groups, int B, int b) {
    int lo = 0, hi = groups;
    while (lo < hi) {                                        // the first group that ends behind b
        const int mid = (lo + hi) >> 1;
        if (between(begin[mid + 1], 0, B) > b) hi = mid;
        else lo = mid + 1;
    }
    return lo < groups && between(begin[lo], 0, B) <= b ? lo : -1;
}

struct ChunkUnit {
    int b, g, rows, cnt, len, group, prefix, prefix_rows;    // rows of queries; prefix: row of prefix_table
    // own rows that the last token of rows of queries up to r sees
    __device__ __forceinline__ int seen(const Chunk& p, int r) const { return between(len - cnt + divided(min(r, rows - 1), p.G, p.inv_G) + 1, 0, len); }
};
__device__ __forceinline__ int tokens_of(const Chunk& p, int u) { return p.cnt ? between(p.cnt[u], 0, p.n) : p.n; }
__device__ __forceinline__ int prefix_rows_of(const Chunk& p, int prefix) { return between(p.prefix_len[prefix], 0, p.prefix_width << p.page_log2); }
__device__ __forceinline__ ChunkUnit chunk_unit(const Chunk& p, int u, const int32_t* begin) {
    ChunkUnit x;
    x.b = divided(u, p.Hkv, p.inv_Hkv);
    x.g = u - x.b * p.Hkv;
    x.cnt = tokens_of(p, u);
    x.rows = x.cnt * p.G;
    x.len = between(p.len[u], 0, p.width << p.page_log2);
    x.prefix = x.prefix_rows = 0;
    x.group = -1;
    if (p.groups) {
        x.group = group_with(begin, p.groups, p.B, x.b);
        if (x.group >= 0) {
            x.prefix = x.group * p.Hkv + x.g;
            x.prefix_rows = prefix_rows_of(p, x.prefix);
        }
    }
    return x;
}

// What a workgroup has: keys `piece` of `pieces` of tile t of unit u's rows, or of the rows of KV head u that group `group` has packed (-1: a unit's).  record: its first row among the
// parts, -1: it has all that its rows see.
struct Place { int u, t, piece, pieces, record, group; };
struct PlaceShared {
    int32_t begin[kScanItems + 1], keys[kScanItems], before[kScanItems];        // before: packed rows of the unit's group in front of its own
    unsigned long long total[4];
    int4 sums[4];
    Place place;
};

// Packed rows: those of all units of a group and KV head follow each other, so that a prefix meets as few tiles as can.  Tile 0 of a group's is item first_slot() of the head's.
template <int BM>
__device__ __forceinline__ int first_slot(const Chunk& p, const int32_t* begin, int group) { return between(begin[group], 0, p.B) * (p.n * p.G) / BM + group; }
struct Packed { int group, tile, rows; };
template <int BM>
__device__ __forceinline__ Packed packed_tile(const Chunk& p, const PlaceShared& sh, int g, int slot) {
    int lo = 0, hi = p.groups - 1;
    while (lo < hi) {                                        // the last group that begins there or before
        const int mid = (lo + hi + 1) >> 1;
        if (first_slot<BM>(p, sh.begin, mid) <= slot) lo = mid;
        else hi = mid - 1;
    }
    const int b0 = between(sh.begin[lo], 0, p.B), b1 = between(sh.begin[lo + 1], 0, p.B) - 1;
    return {lo, slot - first_slot<BM>(p, sh.begin, lo), b1 < b0 ? 0 : sh.before[b1 * p.Hkv + g] + tokens_of(p, b1 * p.Hkv + g) * p.G};
}
// the unit and its row that packed row r of a group and head is
__device__ __forceinline__ int2 packed_row(const Chunk& p, const PlaceShared& sh, int group, int g, int r) {
    int lo = between(sh.begin[group], 0, p.B), hi = max(lo, between(sh.begin[group + 1], 0, p.B) - 1);
    while (lo < hi) {                                        // the last element whose rows begin there or before; those without rows have the one behind them
        const int mid = (lo + hi + 1) >> 1;
        if (sh.before[mid * p.Hkv + g] <= r) lo = mid;
        else hi = mid - 1;
    }
    return make_int2(lo, between(r - sh.before[lo * p.Hkv + g], 0, p.n * p.G - 1));
}

// BM rows of queries and BN keys a tile.  Workgroups that have neighbouring tiles of rows, and so the same keys, follow each other on one XCD (workgroups go to the eight in turn).
template <int BM, int BN, bool PACKS>
__device__ __forceinline__ bool find_place(const Chunk& p, PlaceShared& sh, const ChunkParts& out, int log2_wgs, int least, int direct, Place& x) {
    const int tid = threadIdx.x, lane = tid & 63, w = scalar(tid >> 6), rows = p.n * p.G;
    const int most = (rows + BM - 1) / BM, packed = PACKS ? p.Hkv * p.slots : 0, items = packed + p.units * most;        // tiles of rows of a unit, of packed rows, all
    if (direct) {
        const int per = gridDim.x / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
        if (id >= items) return false;
        x = {id / most, most - 1 - id % most, 0, 1, -1, -1};
        return true;
    }
    for (int i = tid; i <= p.groups && p.groups; i += 256) sh.begin[i] = p.group_begin[i];
    if (tid == 0) sh.place.pieces = 0;
    __syncthreads();
    if (packed) {
        for (int u = tid; u < p.units; u += 256) {
            const int b = divided(u, p.Hkv, p.inv_Hkv), group = group_with(sh.begin, p.groups, p.B, b);
            int before = 0;
            if (group >= 0) {
#pragma unroll 8
                for (int y = between(sh.begin[group], 0, p.B); y < b; ++y) before += tokens_of(p, y * p.Hkv + u - b * p.Hkv);
            }
            sh.before[u] = before * p.G;
        }
        __syncthreads();
    }
    // tiles of keys of each: packed rows first, and a unit's tile of rows `most` - 1, the longest; -1: there are fewer rows
    int mine = 0;                                            // of 8 items at most
    for (int e = tid; e < items; e += 256) {
        int N = -1;
        if (e < packed) {
            const int g = e / p.slots;
            const Packed x = packed_tile<BM>(p, sh, g, e - g * p.slots);
            if (x.tile >= 0 && x.tile * BM < x.rows) N = (prefix_rows_of(p, x.group * p.Hkv + g) + BN - 1) / BN;
            if (N == 0) N = -1;
        } else {
            const int u = (e - packed) / most, r0 = (most - 1 - (e - packed) % most) * BM;
            const ChunkUnit v = chunk_unit(p, u, sh.begin);
            if (r0 < v.rows) N = (v.seen(p, r0 + BM - 1) + BN - 1) / BN + (packed ? 0 : (v.prefix_rows + BN - 1) / BN);
        }
        mine += max(N, 0);
        sh.keys[e] = N;
    }
    {
        // 32 bits may not hold the sum of all: high and low halves apart
        const int low = wave_sum(mine & 0xFFFF), high = wave_sum(mine >> 16);
        if (lane == 0) sh.total[w] = ((unsigned long long)high << 16) + low;
    }
    __syncthreads();
    // A tile of rows is cut into as many pieces as it has loads q, rounded down.  With the average load all pieces fit the chip at once, but for tiles that have less than one: where they
    // are many, loads are made larger, until the workgroups suffice (14 go to waste: two kinds of pieces are dealt to eight XCDs).  A workgroup for every piece that there might be
    // would find nothing to do most of the time, and look for it as long as others: 8 units' 1022 packed rows took 210 us so, and 156 now.
    const int limit = gridDim.x - 14;
    int q = max(least, (int)min((unsigned long long)INT32_MAX, (sh.total[0] + sh.total[1] + sh.total[2] + sh.total[3] + (1 << log2_wgs) - 1) >> log2_wgs));
    // how many workgroups all tiles take; then whose tile this one's is: each thread has some that follow each other
    const int some = (items + 255) / 256, e0 = tid * some, e1 = min(items, e0 + some);
    auto pieces = [&](int e) { const int N = sh.keys[e]; return N < 0 ? 0 : max(1, N / q); };
    // A piece's part has so many rows.  Of tiles that are not cut, those of packed rows have one, and of packed prefixes those of the units' rows (also of units without such a prefix,
    // which leave theirs).
    const int part = min(rows, BM);
    auto parts = [&](int e, int s) { return e < packed ? s * BM : s > 1 || packed ? s * part : 0; };
    int a, a0, r0, used, first;                              // first: pieces of packed rows
    for (int round = 0;; ++round) {
        int records = 0, of_packed = 0;
        a = 0;
        for (int e = e0; e < e1; ++e) {
            const int s = pieces(e);
            a += s;
            records += parts(e, s);
            if (e < packed) of_packed += s;
        }
        const int a_upto = wave_scan(a), r_upto = wave_scan(records);
        if (PACKS) of_packed = wave_sum(of_packed);
        if (lane == 63) sh.sums[w] = int4{a_upto, r_upto, of_packed, 0};
        __syncthreads();
        a0 = a_upto - a;
        r0 = r_upto - records;
        used = first = 0;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int4 v = sh.sums[y];
            if (y < w) { a0 += v.x; r0 += v.y; }
            used += v.x;
            first += v.z;
        }
        used = scalar(used);
        first = PACKS ? scalar(first) : 0;
        if (used <= limit || round == 4) break;
        q = round < 3 ? (int)fminf((float)q * used / limit, 1e9f) + 1 : INT32_MAX;      // the last: one piece a tile
        __syncthreads();
    }
    // each XCD has its share of the packed rows' and of the units' pieces, which are shorter
    const int per = (first + 7) / 8, rest = (used - first + 7) / 8, at = blockIdx.x >> 3, xcd = blockIdx.x & 7;
    const int own = at < per ? xcd * per + at : first + xcd * rest + at - per;
    if (at < per ? own >= first : at - per >= rest || own >= used) return false;
    if (a0 <= own && own < a0 + a)
        for (int e = e0; e < e1; ++e) {
            const int s = pieces(e);
            if (own < a0 + s) {
                const int piece = own - a0;
                if (e < packed) {
                    const int g = e / p.slots;
                    const Packed x = packed_tile<BM>(p, sh, g, e - g * p.slots);
                    sh.place = {g, x.tile, piece, s, r0 + piece * BM, x.group};
                } else {
                    const int u = (e - packed) / most, t = most - 1 - (e - packed) % most;
                    bool whole = s == 1;
                    if (packed) {
                        const ChunkUnit v = chunk_unit(p, u, sh.begin);
                        if (v.prefix_rows) whole = false;
                        if (piece == 0) out.shared[u] = v.prefix_rows ? make_int2(v.g * p.slots + first_slot<BM>(p, sh.begin, v.group), sh.before[u]) : make_int2(-1, 0);
                    }
                    sh.place = {u, t, piece, s, whole ? -1 : r0 + piece * part, -1};
                }
                if (piece == 0) out.pieces[e < packed ? e : packed + (e - packed) / most * most + sh.place.t] = make_int2(sh.place.record, s);
                break;
            }
            a0 += s;
            r0 += parts(e, s);
        }
    __syncthreads();
    x = sh.place;
    x.u = scalar(x.u); x.t = scalar(x.t); x.piece = scalar(x.piece); x.pieces = scalar(x.pieces); x.record = scalar(x.record); x.group = scalar(x.group);
    __syncthreads();
    return x.pieces > 0;
}

__device__ __forceinline__ float log_sum(float m, float l) { return l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY; }

template <typename T> __device__ __forceinline__ void store4(T* dst, floatx4 v);
template <> __device__ __forceinline__ void store4<float>(float* dst, floatx4 v) { *reinterpret_cast<floatx4*>(dst) = v; }
template <> __device__ __forceinline__ void store4<__bf16>(__bf16* dst, floatx4 v) { *reinterpret_cast<uintx2*>(dst) = uintx2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }

// Row r of a unit: token r / G, head r % G of the group.
struct RowAt { int token, head; };
__device__ __forceinline__ RowAt row_at(const Chunk& p, int g, int r) {
    const int i = divided(r, p.G, p.inv_G);
    return {i, g * p.G + r - i * p.G};
}
template <typename T>
__device__ __forceinline__ T* out_row(const Chunk& p, int b, RowAt x) {
    return reinterpret_cast<T*>(p.O) + b * p.o[0] + x.head * p.o[1] + x.token * p.o[2];
}
template <typename T>
__device__ __forceinline__ const T* query_row(const Chunk& p, int b, RowAt x) {
    return reinterpret_cast<const T*>(p.Q) + b * p.q[0] + x.head * p.q[1] + x.token * p.q[2];
}
__device__ __forceinline__ float* lse_at(const Chunk& p, int b, RowAt x) { return p.lse + ((int64_t)b * p.Hq + x.head) * p.n + x.token; }

// ---------------------------------------------------------------- few rows
template <typename T, int D, int COLS>
__global__ __launch_bounds__(256, (PartCfg<T, D>::PER_CU)) void chunk_few_kernel(Chunk p, ChunkParts out, int log2_wgs, int direct) {
    using C = PartCfg<T, D>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    static_assert(sizeof(PlaceShared) <= C::LDS, "the keys' numbers stand where tiles come later");
    __shared__ float2 ml[kPartWaves][kCols];
    Place x;
    if (!find_place<COLS, kTileRows, false>(p, *reinterpret_cast<PlaceShared*>(smem), out, log2_wgs, kLeastFew, direct, x)) return;
    const ChunkUnit v = chunk_unit(p, x.u, p.group_begin);
    if (v.rows == 0) return;
    const int w = scalar(threadIdx.x >> 6);
    char* const mine = smem + w * C::WAVE;
    const int tp = (v.prefix_rows + kTileRows - 1) / kTileRows, all = tp + (v.len + kTileRows - 1) / kTileRows;
    const int t0 = (int)((int64_t)all * x.piece / x.pieces), t1 = (int)((int64_t)all * (x.piece + 1) / x.pieces);
    WavePart<T, D, COLS> part;
    const int col = part.col();
    const RowAt at = row_at(p, v.g, min(col, v.rows - 1));
    part.load_queries(query_row<T>(p, v.b, at), col < v.rows);
    const int last = v.len - v.cnt + at.token;               // own row that the lane's token stands in
    const int32_t *own = p.table + (int64_t)x.u * p.width, *pre = p.prefix_table + (int64_t)v.prefix * p.prefix_width;
    auto pass = [&](auto again) {
        constexpr bool AGAIN = decltype(again)::value;
        part.reset();
        if (t0 < tp) part.template tiles<AGAIN, false, false>(p, pre, v.prefix_rows, t0 + w, kPartWaves, min(t1, tp), p.c, mine);
        if (t1 > tp) {
            const int first = max(t0 - tp, 0);
            part.template tiles<AGAIN, true, false>(p, own, v.len, first + ((w - max(tp - t0, 0)) & 3), kPartWaves, t1 - tp, p.c, mine, last);
        }
    };
    pass(std::false_type{});
    if (part.spoilt()) pass(std::true_type{});
    part.sum_groups();
    // the parts of the four waves meet in LDS: [channel][column], columns turned by the channel so that neither way through meets conflicts
    const int lane = part.here(), i = lane & (COLS - 1), group = lane / COLS;
    if (group == 0) ml[w][i] = make_float2(part.m, part.l);
    __syncthreads();
    float M = -INFINITY;
#pragma unroll
    for (int y = 0; y < kPartWaves; ++y) M = fmaxf(M, ml[y][i].x);
    const float a = M > -INFINITY ? fast_exp2(part.m - M) : 0.f;
    float* mo = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int b = 0; b < part.kO; ++b)
#pragma unroll
        for (int r = 0; r < part.kRegs; ++r) {
            const int ch = part.channel(b, r, group);
            mo[ch * kCols + (i ^ (ch & 31))] = part.o[b][r] * a;
        }
    __syncthreads();
    const int tid = w * 64 + lane, ch = tid % (D / 4) * 4;
    for (int r = tid / (D / 4); r < v.rows; r += 1024 / D) {
        const float* base = reinterpret_cast<const float*>(smem);
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
        float top = -INFINITY, L = 0.f;
#pragma unroll
        for (int y = 0; y < kPartWaves; ++y) top = fmaxf(top, ml[y][r].x);
#pragma unroll
        for (int y = 0; y < kPartWaves; ++y) {
            if (top > -INFINITY) L += fast_exp2(ml[y][r].x - top) * ml[y][r].y;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += base[y * (C::WAVE / 4) + (ch + e) * kCols + (r ^ ((ch + e) & 31))];
        }
        if (x.record < 0) {
            const RowAt to = row_at(p, v.g, r);
            s *= L > 0.f ? 1.f / L : 0.f;
            store4(out_row<T>(p, v.b, to) + ch, s);
            if (p.lse && ch == 0) *lse_at(p, v.b, to) = log_sum(top, L);
        } else {
            const int64_t rec = x.record + r;
            *reinterpret_cast<floatx4*>(out.o + rec * D + ch) = s;
            if (ch == 0) *reinterpret_cast<float2*>(out.ml + 2 * rec) = make_float2(top, L);
        }
    }
}

// ---------------------------------------------------------------- many rows
template <typename T, int D>
struct ChunkCfg {
    static constexpr int RB = D * (int)sizeof(T);
    static constexpr int BN = sizeof(T) == 2 ? 64 : 32, NBK = BN / 32;          // keys a tile, blocks of 32 of them
    static constexpr int TILE = BN * RB, NL = TILE / 4096, RPL = 1024 / RB;     // loads of 1 KiB per wave and tile, rows per load
    static constexpr int CH = D / Elem<T>::kPerChunk, ODB = D / 32;
    static constexpr int CHP = sizeof(T) == 4 ? D / 16 : 1;  // operands of three planes of a row of queries
    static constexpr bool KEPT = D == 64;                    // planes of queries are kept; of longer rows they are made for every tile, or operands spill
    static constexpr int LDS = 4 * TILE + 64 + (sizeof(T) == 4 ? 8 * kRowsMany : 0);     // two tiles of K, two of V, the workgroup's place for the end, of fp32 where the rows of queries are
    __device__ static __forceinline__ int k_swizzle(int r) { return k_row_swizzle<RB>(r); }
    __device__ static __forceinline__ int v_swizzle(int r) { return PartCfg<T, D>::v_swizzle(r); }
};

// Where a tile of keys stands: 16 rows each in row 16 at0 ... of the pages (which hold 16 or more), -1: in no page.  Numbers of their own, in scalar registers: an array that
// loops walk over would stay in memory.  whole: all rows are there.
struct KeyTile {
    int32_t at0, at1, at2, at3;
    bool whole;
    __device__ __forceinline__ int32_t at(int x) const { return x == 0 ? at0 : x == 1 ? at1 : x == 2 ? at2 : at3; }
};

// What planes are off by where a number is small (planes.h), 2^-134, is nothing in an output, times the sum of its weights, beside kOutLow, where values are off, and beside
// kOutLowOfMost times the largest value, where weights are.  A piece with smaller outputs is done again.
constexpr float kOutLow = 0x1p-80f, kOutLowOfMost = 0x1p-90f;
// Sums of the offset that stays, outside which the tiles are repeated with running maxima.
constexpr float kSumLow = 0x1p-64f, kSumHigh = 0x1p64f;

// A tile of rows of one unit against the keys of its piece.
template <typename T, int D>
struct Many {
    using C = ChunkCfg<T, D>;
    static constexpr uint64_t kWhole = C::BN == 64 ? ~0ull : 0xFFFFFFFFull;
    const char *K, *V;
    int num_pages, page_log2;
    float c;
    char* const smem;
    const int32_t *own_table, *pre_table;
    int prefix_rows, seen, tp;                               // rows of the prefix, own rows that a token of the tile sees, tiles of the prefix
    int wave_first, wave_last, r_first, r_last, before, G;   // the own rows that the wave's first and last row of queries see up to (-2: the wave has none); own rows before the new ones
    uint32_t inv_G;
    int w, lane, i, h;
    uintx4 qf[C::CH];
    Planes qp[C::KEPT ? C::CHP : 1];                         // fp32, instead
    floatx16 o[C::ODB];
    float m, l, l_rounded;                                   // l: sum of the weights; as V was weighed by them
    float most;                                              // fp32: the largest number, at least, that went into planes
    int entry[C::BN / 16];                                   // of the table, for the tile that look() was last called for: asked for a step before they are used

    __device__ __forceinline__ void look(int j) {
        using scalar_table = const __attribute__((address_space(4))) int32_t*;
        const bool own = j >= tp;
        const int first = (own ? j - tp : j) * C::BN, end = own ? seen : prefix_rows;
        const scalar_table table = (scalar_table)(own ? own_table : pre_table);
#pragma unroll
        for (int x = 0; x < C::BN / 16; ++x) entry[x] = table[min(first + 16 * x, end - 1) >> page_log2];
    }
    __device__ __forceinline__ bool own(int j) const { return j >= tp; }
    __device__ __forceinline__ int first(int j) const { return (own(j) ? j - tp : j) * C::BN; }
    __device__ __forceinline__ int left(int j) const { return (own(j) ? seen : prefix_rows) - first(j); }
    __device__ __forceinline__ KeyTile locate(int j) const {
        KeyTile k = {0, 0, 0, 0, left(j) >= C::BN};
        const int row = first(j);
        auto where = [&](int x) {
            const bool there = (unsigned)entry[x] < (unsigned)num_pages;
            k.whole = k.whole && there;
            return there ? (entry[x] << (page_log2 - 4)) + (((row + 16 * x) & ((1 << page_log2) - 1)) >> 4) : -1;
        };
        k.at0 = where(0);
        k.at1 = where(1);
        if constexpr (C::BN == 64) {
            k.at2 = where(2);
            k.at3 = where(3);
        }
        return k;
    }
    // Own tiles that all tokens of the workgroup's rows see whole.
    __device__ __forceinline__ int clean_own() const { return between(before + divided(r_first - 32 * w, G, inv_G) + 1, 0, seen) / C::BN; }
    // Whether some of the rows of tiles j0 ... j1 - 1 are in no page.
    __device__ __forceinline__ bool lacks_pages(int j0, int j1) const {
        bool lacks = false;
        auto table = [&](const int32_t* t, int a, int b) {   // rows a ... b - 1
            if (a < b)
                for (int e = (a >> page_log2) + lane; e <= (b - 1) >> page_log2; e += 64) lacks |= (unsigned)t[e] >= (unsigned)num_pages;
        };
        table(pre_table, min(j0 * C::BN, prefix_rows), min(j1 * C::BN, prefix_rows));
        table(own_table, max(j0 - tp, 0) * C::BN, min(max(j1 - tp, 0) * C::BN, seen));
        return __any(lacks);
    }
    // the rows that there are, as bits
    __device__ __forceinline__ uint64_t rows(const KeyTile& k, int j) const {
        uint64_t x = left(j) >= C::BN ? kWhole : (1ull << left(j)) - 1;
        if (k.at0 < 0) x &= ~0xFFFFull;
        if (k.at1 < 0) x &= ~(0xFFFFull << 16);
        if (k.at2 < 0) x &= ~(0xFFFFull << 32);
        if (k.at3 < 0) x &= ~(0xFFFFull << 48);
        return x;
    }

    // Load q of the wave of a whole tile of K (V): a lane's offset is the same in all of them, but for the row of the pages.
    template <bool IS_V>
    __device__ __forceinline__ int lane_offset() const {
        const int lr = lane / (C::RB / 16), row = w * C::RPL + lr;
        return (row & 15) * C::RB + (((lane % (C::RB / 16)) ^ (IS_V ? C::v_swizzle(row) : C::k_swizzle(row))) << 4);
    }
    template <bool IS_V>
    __device__ __forceinline__ const char* load_base(const KeyTile& k, int q) const {
        constexpr int kRows = 4 * C::RPL;                    // of the four waves' loads together: 8, 16 or 32
        const int32_t at = kRows == 16 ? k.at(q) : kRows == 32 ? (w < 2 ? k.at(2 * q) : k.at(2 * q + 1)) : k.at(q / 2);
        return scalar_ptr((IS_V ? V : K) + ((int64_t)at * 16 + (kRows == 8 ? q % 2 * 8 : 0)) * C::RB);
    }
    __device__ __forceinline__ char* buffer(bool v, int buf) const { return smem + (v ? 2 * C::TILE : 0) + buf * C::TILE; }

    // A tile of K (V) to LDS; rows that are not there take one that is: they are masked, and their values weigh nothing
    template <bool IS_V>
    __device__ __forceinline__ void request(const KeyTile& k, int j, int buf) const {
        char* const to = buffer(IS_V, buf) + w * 1024;
        if (k.whole) {
            const int off = lane_offset<IS_V>();
#pragma unroll
            for (int q = 0; q < C::NL; ++q) load_kib_to_lds(load_base<IS_V>(k, q), C::RPL == 2 && q % 2 ? off ^ 128 : off, lds_address(to) + q * 4096);      // rows of 512 bytes: the swizzle of 8 rows on
        } else if (const uint64_t there = rows(k, j); there == 0) {
            for (int q = 0; q < C::NL; ++q) *reinterpret_cast<uintx4*>(to + q * 4096 + lane * 16) = uintx4{0, 0, 0, 0};
        } else {
            const int safe = __builtin_ctzll(there), ck = lane % (C::RB / 16);
#pragma unroll 1
            for (int q = 0; q < C::NL; ++q) {
                const int row = (q * 4 + w) * C::RPL + lane / (C::RB / 16), from = there >> row & 1 ? row : safe;
                load_kib_to_lds_at((IS_V ? V : K) + ((int64_t)k.at(from >> 4) * 16 + (from & 15)) * C::RB + ((ck ^ (IS_V ? C::v_swizzle(row) : C::k_swizzle(row))) << 4), lds_address(to) + q * 4096);
            }
        }
    }

    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int db = 0; db < C::ODB; ++db) o[db] = floatx16{0};
        m = -INFINITY;
        l = l_rounded = 0.f;
    }
    // fp32 numbers go as three planes of bf16, six products for one that takes sixteen times as long, where none is too large for them (kPlaneHigh).  Five pieces of up to 777 tokens, d = 64:
    // 38.6 us, 43.4 in fp32 products; 8 units of 168 rows about 7200 shared ones, d = 128: 196 and 213 (planes of queries kept, 54 registers spilled: 270).
    __device__ __forceinline__ Planes split(const uintx4& a, const uintx4& b) {
#pragma unroll
        for (int e = 0; e < 4; ++e) asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(most) : "v"(a[e]), "v"(b[e]));
        return split8(a, b);
    }
    __device__ __forceinline__ void load_planes(const T* row) {
        most = 0.f;
#pragma unroll
        for (int cc = 0; cc < C::CHP; ++cc) {
            const uintx4 a = load16(row + 16 * cc + 8 * h), b = load16(row + 16 * cc + 8 * h + 4);
            if constexpr (C::KEPT) qp[cc] = split(a, b);
            else {
                qf[2 * cc] = a;
                qf[2 * cc + 1] = b;
            }
        }
    }
    __device__ __forceinline__ void load_queries(const T* row) {
#pragma unroll
        for (int cc = 0; cc < C::CH; ++cc) qf[cc] = load16(row + (2 * cc + h) * Elem<T>::kPerFrag);
    }
    using Scores = floatx16[C::NBK];
    __device__ __forceinline__ void plane_scores(const char* kb, Scores& s) {
        int at = lane;
        if constexpr (!C::KEPT) asm volatile("" : "+v"(at));  // nor are addresses through all tiles
        const int i = at & 31, h = at >> 5;
        const char* const row = kb + i * C::RB;
        s[0] = floatx16{0};
#pragma unroll
        for (int cc = 0; cc < C::CHP; ++cc) {
            const Planes k = split(load16(row + swz_chunk(4 * cc + 2 * h, C::k_swizzle(i))), load16(row + swz_chunk(4 * cc + 2 * h + 1, C::k_swizzle(i))));
            if constexpr (C::KEPT) s[0] = mma_planes(k, qp[cc], s[0]);
            else {
                uintx4 a = qf[2 * cc], b = qf[2 * cc + 1];
                asm volatile("" : "+v"(a), "+v"(b));         // not made once for all tiles
                s[0] = mma_planes(k, split(a, b), s[0]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // channels 32 db ... of eight keys, a channel a lane
    __device__ __forceinline__ Planes v_planes(const char* vb, int s2, int db) {
        uintx4 x[2];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
            const int k = acc_row(8 * s2 + y, h);
            x[y / 4][y % 4] = *reinterpret_cast<const uint32_t*>(vb + k * C::RB + swz_chunk(8 * db + (i >> 2), C::v_swizzle(k)) + (i & 3) * 4);
        }
        return split(x[0], x[1]);
    }
    __device__ __forceinline__ void scores(const char* kb, Scores& s) const {
#pragma unroll
        for (int blk = 0; blk < C::NBK; ++blk) {
            s[blk] = floatx16{0};
#pragma unroll
            for (int cc = 0; cc < C::CH; ++cc) {
                const uintx4 kf = *reinterpret_cast<const uintx4*>(kb + (32 * blk + i) * C::RB + swz_chunk(2 * cc + h, C::k_swizzle(i)));
                s[blk] = mma_frag<T>(kf, qf[cc], s[blk]);
                if (sizeof(T) == 2 && cc & 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    __device__ __forceinline__ void mask(const KeyTile& k, int j, Scores& s) const {
        if (!k.whole) {
            const uint64_t there = rows(k, j) >> 4 * h;
#pragma unroll
            for (int blk = 0; blk < C::NBK; ++blk)
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                    if (!(there >> (32 * blk + acc_row(y, 0)) & 1)) s[blk][y] = -INFINITY;
                    __builtin_amdgcn_sched_barrier(0);       // one condition at a time: all 32 at once are 64 scalar registers
                }
        }
        if (own(j) && first(j) + C::BN - 1 > wave_first) {
            int tid = threadIdx.x;                           // the lane's own row, said anew: it is not kept for this
            asm volatile("" : "+v"(tid));
            const int upto = before + divided(min(r_first + (tid & 31), r_last), G, inv_G) - first(j) - 4 * (tid >> 5 & 1);        // against numbers that the lane does not come into: those would be kept in registers
#pragma unroll
            for (int blk = 0; blk < C::NBK; ++blk)
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                    if (32 * blk + acc_row(y, 0) > upto) s[blk][y] = -INFINITY;
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
    }
    __device__ __forceinline__ float largest(const Scores& s) const {
        float mx = s[0][0];
#pragma unroll
        for (int blk = 0; blk < C::NBK; ++blk)
#pragma unroll
            for (int y = 0; y < 16; ++y) mx = fmaxf(mx, s[blk][y]);
        return mx * c;
    }
    // Where a lane's address of V stands in a tile: channels 32 db ... of key 4 h + e, for the transposing reads
    __device__ __forceinline__ int v_lane(int db) const {
        const int e = (lane >> 2) & 3, q = lane & 3, row = 4 * h + e;
        return row * C::RB + swz_chunk(4 * db + 2 * ((lane >> 4) & 1) + (q >> 1), C::v_swizzle(row)) + (q & 1) * 8;
    }
    __device__ static __forceinline__ uintx4 v_frag(const char* a0) {
        typedef short shortx4 __attribute__((ext_vector_type(4)));
        using lds_ptr = __attribute__((address_space(3))) shortx4*;
        const uintx2 f0 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)a0));
        const uintx2 f1 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(a0 + 8 * C::RB)));
        return uintx4{f0[0], f0[1], f1[0], f1[1]};
    }

    // Tiles j0 ... j1 - 1, one after the other, the offset of the exponentials behind the running maximum: any tiles, any logits
    template <bool PLANES>
    __device__ __forceinline__ void plain(int j0, int j1) {
        if (j0 >= j1) return;
        look(j0);
        KeyTile cur = locate(j0), nxt = cur;
        request<false>(cur, j0, 0);
        request<true>(cur, j0, 0);
        if (j0 + 1 < j1) look(j0 + 1);
        for (int j = j0, buf = 0; j < j1; ++j, buf ^= 1) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __syncthreads();                                 // the tile is there for all waves, and all have read the one before
            if (j + 1 < j1) {
                nxt = locate(j + 1);
                request<false>(nxt, j + 1, buf ^ 1);
                request<true>(nxt, j + 1, buf ^ 1);
                if (j + 2 < j1) look(j + 2);
            }
            const KeyTile here = cur;
            cur = nxt;
            if (wave_last < (own(j) ? first(j) : -1)) continue;      // nothing that the wave's rows see, or no rows
            const char* vb = buffer(true, buf);
            Scores s;
            if constexpr (PLANES) plane_scores(buffer(false, buf), s);
            else scores(buffer(false, buf), s);
            mask(here, j, s);
            float mx = largest(s);
            if (__any(mx > m + kLazy)) {
                mx = over_groups<32>(mx, [](float a, float b) { return fmaxf(a, b); });
                const float m_new = fmaxf(m, mx), a = m_new > -INFINITY ? fast_exp2(m - m_new) : 1.f;
                l *= a;
                l_rounded *= a;
#pragma unroll
                for (int db = 0; db < C::ODB; ++db)
#pragma unroll
                    for (int y = 0; y < 16; ++y) o[db][y] *= a;
                m = m_new;
            }
            const float ms = m > -INFINITY ? m : 0.f;
#pragma unroll
            for (int blk = 0; blk < C::NBK; ++blk) {
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                    s[blk][y] = fast_exp2(fmaf(s[blk][y], c, -ms));
                    l += s[blk][y];
                }
                if constexpr (sizeof(T) == 2) {
                    // Rounded to bf16, and what they are divided by is the sum of the rounded ones: three planes, as few queries have them, would be four products where these are two.  Of an output
                    // the weights' roundings leave 0.7e-3 to 1.4e-3 (2-norm), its own 1.67e-3.
#pragma unroll
                    for (int s2 = 0; s2 < 2; ++s2) {
                        uintx4 pf;
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            pf[y] = pack_bf16x2(s[blk][8 * s2 + 2 * y], s[blk][8 * s2 + 2 * y + 1]);
                            l_rounded = add_bf16x2(pf[y], l_rounded);
                        }
#pragma unroll
                        for (int db = 0; db < C::ODB; ++db) o[db] = mma_frag<__bf16>(v_frag(vb + v_lane(db) + (32 * blk + 16 * s2) * C::RB), pf, o[db]);
                    }
                } else if constexpr (PLANES) {
#pragma unroll
                    for (int s2 = 0; s2 < 2; ++s2) {
                        uintx4 x[2];
#pragma unroll
                        for (int y = 0; y < 8; ++y) x[y / 4][y % 4] = __float_as_uint(s[0][8 * s2 + y]);
                        const Planes weights = split8(x[0], x[1]);
#pragma unroll
                        for (int db = 0; db < C::ODB; ++db) {
                            o[db] = mma_planes(v_planes(vb, s2, db), weights, o[db]);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                } else {
#pragma unroll
                    for (int y = 0; y < 16; ++y) {
                        const int k = 32 * blk + acc_row(y, h);
#pragma unroll
                        for (int db = 0; db < C::ODB; ++db) {
                            const float vv = *reinterpret_cast<const float*>(vb + k * C::RB + swz_chunk(8 * db + (i >> 2), C::v_swizzle(k)) + (i & 3) * 4);
                            o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv, s[blk][y], o[db], 0, 0, 0);
                        }
                    }
                }
            }
        }
        __syncthreads();
    }

    // bf16: n tiles from j0, an even number of 4 or more, all rows of which are there and seen by all queries, three tiles deep.  A step multiplies P V of tile t - 1 and takes half
    // of the exponentials of tile t in its first half, multiplies K Q^T of tile t + 1 and takes the other half in its second: nothing in a step waits for anything
    // else in it, and the order of instructions is written out - behind every product its share of the vector work, in front of it the reads of an operand three products
    // ahead, the requests (K of tile t + 2, V of t + 1) one at a time.  The offset of the exponentials stays, or is the first tile's maximum if there was no
    // tile before: right as long as no sum leaves the middle of the fp32 range, which the caller asks strayed() about.
    // The steps are a loop of their own without any other way through them: with one for tiles that lack rows beside it, operands spilled in both.
    static constexpr int kAhead = 3;
    __device__ __forceinline__ void piped(int j0, int n) {
        static_assert(sizeof(T) == 2, "");
        using Probs = uintx4[2][2];
        const int koff = lane_offset<false>(), voff = lane_offset<true>(), vl = v_lane(0);      // V of channel block db: the swizzle takes its number by exclusive or
        Scores sa, sb;
        Probs pa, pb;
        auto exps = [&](int blk, Scores& sc, Probs& pc) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float e0 = fast_exp2(fmaf(sc[blk][r], c, -m)), e1 = fast_exp2(fmaf(sc[blk][r + 1], c, -m));
                const uint32_t pk = pack_bf16x2(e0, e1);
                pc[blk][r >> 3][(r & 7) >> 1] = pk;
                l_rounded = add_bf16x2(pk, l_rounded);
                l += e0 + e1;
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto weighted = [&](const char* vb, Probs& pp) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 4 * C::ODB; ++j) {
                o[j % C::ODB] = mma_frag<__bf16>(v_frag(vb + (vl ^ (j % C::ODB) << 6) + (32 * (j / (2 * C::ODB)) + 16 * (j / C::ODB & 1)) * C::RB), pp[j / (2 * C::ODB)][j / C::ODB & 1], o[j % C::ODB]);
                if (j & 1) __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto all_there = [&]() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); __syncthreads(); };
        auto look_or_last = [&](int t) { look(j0 + min(t, n - 1)); };                // behind the last tile that again, unread
        look(j0);
        KeyTile next, after;                                 // tiles t + 1, t + 2 of step t
        {
            const KeyTile c0 = locate(j0);
            look(j0 + 1);
            const KeyTile c1 = locate(j0 + 1);
            look(j0 + 2);
            request<false>(c0, j0, 0);
            request<false>(c1, j0 + 1, 1);
            request<true>(c0, j0, 0);
            all_there();
            scores(buffer(false, 0), sa);
            if (__any(m == -INFINITY)) {
                const float mx = over_groups<32>(largest(sa), [](float a, float b) { return fmaxf(a, b); });
                if (m == -INFINITY) m = mx;                  // of lanes that have met none: no sums yet
            }
            exps(0, sa, pb);
            exps(1, sa, pb);
            scores(buffer(false, 1), sb);
            all_there();                                     // K of both has been read by all
            next = locate(j0 + 2);
            request<false>(next, j0 + 2, 0);
            request<true>(c1, j0 + 1, 1);
            look_or_last(3);
        }
        auto half = [&](auto half_tag, const char* src, Scores& sc, Scores& sn, Probs& pp, Probs& pc, const KeyTile& k, unsigned to) __attribute__((always_inline)) {
            constexpr int HALF = decltype(half_tag)::value, NM = HALF == 0 ? 4 * C::ODB : 2 * C::CH, PPM = 16 / NM;
            uintx4 frag[NM];
            float e[16];
            auto read = [&](int j) __attribute__((always_inline)) {
                if constexpr (HALF == 0) frag[j] = v_frag(src + (vl ^ (j % C::ODB) << 6) + (32 * (j / (2 * C::ODB)) + 16 * (j / C::ODB & 1)) * C::RB);
                else frag[j] = *reinterpret_cast<const uintx4*>(src + (32 * (j & 1) + i) * C::RB + swz_chunk(2 * (j >> 1) + h, C::k_swizzle(i)));
            };
            auto vector = [&](int q) __attribute__((always_inline)) {       // 16 pieces: half a pair of keys each
                const int r = q & ~1;
                if ((q & 1) == 0) {
                    e[r] = fast_exp2(fmaf(sc[HALF][r], c, -m));
                    e[r + 1] = fmaf(sc[HALF][r + 1], c, -m);
                } else {
                    e[r + 1] = fast_exp2(e[r + 1]);
#pragma unroll
                    for (int L = 0; L < C::NL; ++L)
                        if (q == (((2 * L + 1) * 16 / (2 * C::NL)) | 1)) {
                            unsigned pin = __float_as_uint(e[r + 1]);
                            load_kib_to_lds_pinned(load_base<HALF == 1>(k, L), HALF == 0 ? koff : voff, to + L * 4096, pin);
                            e[r + 1] = __uint_as_float(pin);
                        }
                    const uint32_t pk = pack_bf16x2(e[r], e[r + 1]);
                    pc[HALF][r >> 3][(r & 7) >> 1] = pk;
                    l_rounded = add_bf16x2(pk, l_rounded);
                    l += e[r] + e[r + 1];
                }
            };
#pragma unroll
            for (int j = 0; j < kAhead; ++j) read(j);
#pragma unroll
            for (int j = 0; j < NM; ++j) {
                if (j + kAhead < NM) read(j + kAhead);
                if constexpr (HALF == 0) o[j % C::ODB] = mma_frag<__bf16>(frag[j], pp[j / (2 * C::ODB)][j / C::ODB & 1], o[j % C::ODB]);
                else sn[j & 1] = mma_frag<__bf16>(frag[j], qf[j >> 1], j < 2 ? floatx16{0} : sn[j & 1]);
#pragma unroll
                for (int q = 0; q < PPM; ++q) vector(j * PPM + q);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto wait = [&]() __attribute__((always_inline)) {   // all but the last two requests of tiles have landed, and the wave's LDS reads
            __builtin_amdgcn_s_waitcnt(0x0070 | ((2 * C::NL) & 15) | (((2 * C::NL) >> 4) << 14));
            __syncthreads();
        };
        // V of tile t - 1, K of tile t + 1 are there or on their way, V of tile t behind them; ODD: t is
        auto step = [&](auto odd_tag, int t, Scores& sc, Scores& sn, Probs& pp, Probs& pc) __attribute__((always_inline)) {
            constexpr int ODD = decltype(odd_tag)::value;
            after = locate(j0 + min(t + 2, n - 1));
            look_or_last(t + 3);
            half(std::integral_constant<int, 0>{}, buffer(true, !ODD), sc, sn, pp, pc, after, lds_address(buffer(false, ODD)) + w * 1024);
            wait();                                          // K of tile t + 1 is there
            half(std::integral_constant<int, 1>{}, buffer(false, !ODD), sc, sn, pp, pc, next, lds_address(buffer(true, !ODD)) + w * 1024);
            wait();                                          // V of tile t is there
            next = after;
        };
        for (int t = 1; t < n - 1; t += 2) {
            step(std::integral_constant<int, 1>{}, t, sb, sa, pb, pa);
            step(std::integral_constant<int, 0>{}, t + 1, sa, sb, pa, pb);
        }
        weighted(buffer(true, 0), pb);                       // tile n - 2
        all_there();
        exps(0, sb, pa);
        exps(1, sb, pa);
        weighted(buffer(true, 1), pa);
        __syncthreads();
    }
    // Right behind piped(), before a running maximum scales the sums: whether one of the wave's is no number, infinite, or of weights that are far from 1.  Sums of V leave the range
    // before those of the weights where V is large.
    __device__ __forceinline__ bool strayed() const {
        float probe[4] = {fmaf(l_rounded, 0.f, 0.f), 0.f, 0.f, 0.f};                 // no number if a sum is not finite
#pragma unroll
        for (int db = 0; db < C::ODB; ++db)
#pragma unroll
            for (int y = 0; y < 16; ++y) probe[y & 3] = fmaf(o[db][y], 0.f, probe[y & 3]);
        const float weights = over_groups<32>(l, [](float a, float b) { return a + b; });
        return __any(!(weights >= kSumLow && weights <= kSumHigh) || probe[0] + probe[1] + probe[2] + probe[3] != 0.f);
    }
    // fp32, behind plain<true>(): whether numbers were larger, or outputs are smaller, than planes hold with all bits.  Outputs of 0 pass: of values that are 0.
    __device__ __forceinline__ bool exceeds_planes() const {
        Least least;
#pragma unroll
        for (int db = 0; db < C::ODB; ++db)
#pragma unroll
            for (int y = 0; y < 16; ++y) least.add(__float_as_uint(o[db][y]));
        const float weights = over_groups<32>(l, [](float a, float b) { return a + b; });
        return __any(!(most < kPlaneHigh) || least.below(fmaxf(kOutLow, kOutLowOfMost * wave_max(most)) * fmaxf(weights, 1.f)));
    }
};

// The kernel's arguments, read again: kept in scalar registers through the tiles they spilled.
template <typename A>
__device__ __forceinline__ A read_again(int offset) {
    typedef const __attribute__((address_space(4))) char* const_ptr;
    const_ptr at = (const_ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    A x;
    static_assert(sizeof(A) % 4 == 0, "");
    uint32_t* to = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
    for (int i = 0; i < (int)sizeof(A) / 4; ++i) to[i] = reinterpret_cast<const __attribute__((address_space(4))) uint32_t*>(at + offset)[i];
    return x;
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void chunk_many_kernel(Chunk p_, ChunkParts out_, int log2_wgs, int direct) {
    using C = ChunkCfg<T, D>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    // of the workgroup, for the end; behind the tiles, which then begin where LDS does: their addresses fit an instruction's offset
    struct Held { Place x; int b, g, rows, again; };
    static_assert(sizeof(Held) <= 64, "");
    Held& held = *reinterpret_cast<Held*>(smem + 4 * C::TILE);
    static_assert(sizeof(PlaceShared) <= 4 * C::TILE, "the keys' numbers stand where tiles come later");
    const T** const query_at = reinterpret_cast<const T**>(smem + 4 * C::TILE + 64);
    Many<T, D> many = {p_.K, p_.V, p_.num_pages, p_.page_log2, p_.c, smem};
    int j0, j1, r0;
    {
        const Chunk p = read_again<Chunk>(0);
        const ChunkParts out = read_again<ChunkParts>(sizeof(Chunk));
        Place x;
        PlaceShared& sh = *reinterpret_cast<PlaceShared*>(smem);
        if (!find_place<kRowsMany, C::BN, true>(p, sh, out, log2_wgs, kLeastMany, direct, x)) return;
        ChunkUnit v;
        if (x.group >= 0) {                                  // packed rows, which see all of their prefix and nothing else
            v = {0, x.u, packed_tile<kRowsMany>(p, sh, x.u, first_slot<kRowsMany>(p, sh.begin, x.group)).rows, 0, 0, x.group, x.group * p.Hkv + x.u, 0};
            v.prefix_rows = prefix_rows_of(p, v.prefix);
        } else {
            v = chunk_unit(p, x.u, p.group_begin);
            if (p.slots) v.prefix_rows = 0;
        }
        r0 = x.t * kRowsMany;
        if (r0 >= v.rows) return;
        const int tid = threadIdx.x;
        many.w = scalar(tid >> 6);
        many.lane = tid & 63;
        many.i = tid & 31;
        many.h = tid >> 5 & 1;
        many.r_first = r0 + 32 * many.w;
        many.r_last = scalar(min(r0 + kRowsMany, v.rows) - 1);
        many.before = scalar(v.len - v.cnt);
        many.G = p.G;
        many.inv_G = p.inv_G;
        many.own_table = p.table + (int64_t)(x.group >= 0 ? 0 : x.u) * p.width;
        many.pre_table = p.prefix_table + (int64_t)scalar(v.prefix) * p.prefix_width;
        many.prefix_rows = scalar(v.prefix_rows);
        many.seen = scalar(v.seen(p, many.r_last));
        many.tp = scalar((v.prefix_rows + C::BN - 1) / C::BN);
        many.wave_first = scalar(many.before + divided(min(many.r_first, many.r_last), p.G, p.inv_G));
        many.wave_last = many.r_first > many.r_last ? -2 : max(-1, scalar(many.before + divided(min(many.r_first + 31, many.r_last), p.G, p.inv_G)));
        const int all = many.tp + scalar((many.seen + C::BN - 1) / C::BN);
        j0 = scalar((int)((int64_t)all * x.piece / x.pieces));
        j1 = scalar((int)((int64_t)all * (x.piece + 1) / x.pieces));
        if (tid == 0) held = {x, v.b, v.g, v.rows, 0};
        int r = min(many.r_first + many.i, many.r_last);
        if (x.group >= 0) {
            const int2 at = packed_row(p, sh, x.group, v.g, r);
            v.b = at.x;
            r = at.y;
        }
        __syncthreads();                                     // `before` has been read: tiles may come there
        const T* row = query_row<T>(p, v.b, row_at(p, v.g, r));
        if constexpr (sizeof(T) == 4) {
            many.load_planes(row);
            if (many.h == 0) query_at[32 * many.w + many.i] = row;
        } else many.load_queries(row);
    }
    auto both = [](float a) { return over_groups<32>(a, [](float p, float q) { return p + q; }); };
    // What follows the tiles goes by numbers read and said anew: registers are scarce among them.
    struct End { Place x; int b, g, i, h, r, r_last, token; };
    auto end = [&](const Chunk& p) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        End e;
        e.x = held.x;
        e.b = held.b;
        e.g = held.g;
        e.i = tid & 31;
        e.h = tid >> 5 & 1;
        e.r = held.x.t * kRowsMany + 32 * (tid >> 6) + e.i;
        e.r_last = min((held.x.t + 1) * kRowsMany, held.rows) - 1;
        e.token = divided(min(e.r, e.r_last), p.G, p.inv_G);
        return e;
    };
    if constexpr (sizeof(T) == 2) {
        for (bool safe = many.lacks_pages(j0, j1);; safe = true) {
            many.reset();
            int j = j0;
#pragma unroll 1
            for (int own = 0; own < 2; ++own) {              // the prefix, then the unit's rows: first the tiles that have all rows and are seen by all, then others up to the next such
                const int clean = own ? max(j, many.tp + many.clean_own()) : many.prefix_rows / C::BN, n = max(0, min(clean, j1) - j) & ~1;
                if (!safe && n >= 4) {
                    many.piped(j, n);
                    if (many.wave_last != -2 && many.strayed() && threadIdx.x % 64 == 0) held.again = 1;       // of waves that have rows
                    j += n;
                }
                const int upto = own ? j1 : min(j1, max(j, many.tp));
                many.template plain<false>(j, upto);
                j = upto;
            }
            if (safe) break;
            __syncthreads();
            if (!scalar(held.again)) break;
        }
    } else {
        many.reset();
        many.template plain<true>(j0, j1);
        if (many.exceeds_planes() && threadIdx.x % 64 == 0) held.again = 1;
        __syncthreads();
        if (scalar(held.again)) {                            // in fp32 products
            many.load_queries(query_at[threadIdx.x / 64 * 32 + threadIdx.x % 32]);
            many.reset();
            many.template plain<false>(j0, j1);
        }
    }
    const Chunk p = read_again<Chunk>(0);
    const float m = many.m, l = both(many.l), weight = sizeof(T) == 2 ? both(many.l_rounded) : l;      // what V was weighed by
    const End e = end(p);
    if (e.r > e.r_last) return;
    const RowAt at = {e.token, e.g * p.G + e.r - e.token * p.G};
    auto four = [&](int db, int a) { return floatx4{many.o[db][4 * a], many.o[db][4 * a + 1], many.o[db][4 * a + 2], many.o[db][4 * a + 3]}; };
    if (e.x.record < 0) {
        const float inv = weight > 0.f ? 1.f / weight : 0.f;
        T* row = out_row<T>(p, e.b, at);
#pragma unroll
        for (int db = 0; db < C::ODB; ++db)
#pragma unroll
            for (int a = 0; a < 4; ++a) store4(row + 32 * db + 8 * a + 4 * e.h, four(db, a) * inv);
        if (p.lse && e.h == 0) *lse_at(p, e.b, at) = log_sum(m, l);
    } else {
        // the sums to the part's own unrounded one, so that parts are joined by one number
        const ChunkParts out = read_again<ChunkParts>(sizeof(Chunk));
        const float f = weight > 0.f ? l / weight : 0.f;
        const int64_t rec = e.x.record + e.r % kRowsMany;
#pragma unroll
        for (int db = 0; db < C::ODB; ++db)
#pragma unroll
            for (int a = 0; a < 4; ++a) *reinterpret_cast<floatx4*>(out.o + rec * D + 32 * db + 8 * a + 4 * e.h) = four(db, a) * f;
        if (e.h == 0) *reinterpret_cast<float2*>(out.ml + 2 * rec) = make_float2(l > 0.f ? m : -INFINITY, l);
    }
}

// ---------------------------------------------------------------- parts of cut rows -> rows
// 1024 / D rows at a time, D / 4 lanes a row; `per` rows a workgroup.  Parts are asked for eight or sixteen at a time: a row is a chain of few loads, not of as many as it has parts.
template <typename T, int D, int BM>
__global__ __launch_bounds__(256) void chunk_join_kernel(Chunk p, ChunkParts in, int per) {
    const int u = blockIdx.y, b = divided(u, p.Hkv, p.inv_Hkv), g = u - b * p.Hkv, rows = tokens_of(p, u) * p.G;
    const int most = (p.n * p.G + BM - 1) / BM, part = min(p.n * p.G, BM), packed = p.Hkv * p.slots, r_end = min(rows, ((int)blockIdx.x + 1) * per);
    const int ch = threadIdx.x % (D / 4) * 4;
    for (int r = blockIdx.x * per + threadIdx.x / (D / 4); r < r_end; r += 1024 / D) {
        const int2 own = in.pieces[packed + u * most + r / BM], shared = packed ? in.shared[u] : make_int2(-1, 0);
        if (own.x < 0 || own.y < 1 || own.x + own.y * part > in.rows) continue;          // nothing to join
        int2 first = {0, 0};
        const int packed_r = shared.y + r;
        if (shared.x >= 0 && shared.x + packed_r / BM < packed) first = in.pieces[shared.x + packed_r / BM];
        if (first.x < 0 || first.y < 0 || first.x + first.y * BM > in.rows) continue;
        const int s = first.y + own.y;                       // parts
        auto record = [&](int y) { return (int64_t)(y < first.y ? first.x + y * BM + packed_r % BM : own.x + (y - first.y) * part + r % BM); };
        float M = -INFINITY, L = 0.f;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
        auto parts = [&](auto at_once, int y0) __attribute__((always_inline)) {
            constexpr int N = decltype(at_once)::value;
            float2 ml[N];
            floatx4 o[N];
#pragma unroll
            for (int y = 0; y < N; ++y) {
                const int64_t rec = record(min(y0 + y, s - 1));
                ml[y] = *reinterpret_cast<const float2*>(in.ml + 2 * rec);
                o[y] = *reinterpret_cast<const floatx4*>(in.o + rec * D + ch);
            }
            float top = M;
#pragma unroll
            for (int y = 0; y < N; ++y) top = fmaxf(top, ml[y].x);
            if (top == -INFINITY) return;
            const float f = fast_exp2(M - top);
            L *= f;
            acc *= f;
#pragma unroll
            for (int y = 0; y < N; ++y) {
                const float a = y0 + y < s ? fast_exp2(ml[y].x - top) : 0.f;
                L += a * ml[y].y;
                acc += a * o[y];
            }
            M = top;
        };
        int y0 = 0;
        for (; s - y0 > 8; y0 += 16) parts(std::integral_constant<int, 16>{}, y0);
        if (y0 < s) parts(std::integral_constant<int, 8>{}, y0);
        const RowAt at = row_at(p, g, r);
        acc *= L > 0.f ? 1.f / L : 0.f;
        store4(out_row<T>(p, b, at) + ch, acc);
        if (p.lse && ch == 0) *lse_at(p, b, at) = log_sum(M, L);
    }
}

// ---------------------------------------------------------------- host
constexpr int kFewRows = 32;
// Rows of a unit up to which those of a group are packed, where tiles that are not full are a part of all that counts.  Eight units, 7200 shared rows, us, packed and not: 42 rows 33, 38; 168
// rows 48, 56 (two a group); 259 rows 64, 73; 385 rows 75, 88; 511 rows 90, 89.  Not for groups whose rows fit a wave: 28 rows in two units are read twice, from L2.
constexpr int kRowsPacked = 4 * kRowsMany;
struct ChunkPlan { int few, direct, wgs, rows, bm, slots; int64_t grid; size_t ml, pieces, shared, total; };
// keys: that the tables of a unit and its prefix can hold
static ChunkPlan chunk_plan(const zipvl_dims& d, int64_t keys, int groups) {
    ChunkPlan x;
    const int64_t rows = (int64_t)d.n * (d.Hq / d.Hkv), units = (int64_t)d.B * d.Hkv;
    x.few = rows <= kFewRows;
    x.slots = 0;
    int64_t items = 0;
    if (groups > 0 && 2 * groups <= d.B && rows <= kRowsPacked && rows * d.B / groups > kFewRows) {
        const int64_t slots = d.B * rows / kRowsMany + groups + 1;
        items = units * ((rows + kRowsMany - 1) / kRowsMany) + d.Hkv * slots;
        if (items <= kScanItems) {
            x.slots = (int)slots;
            x.few = 0;
        }
    }
    x.bm = x.few ? (rows <= 16 ? 16 : 32) : kRowsMany;
    const int bn = x.few || d.dtype == ZIPVL_F32 ? 32 : 64;
    const int64_t tiles = (keys + bn - 1) / bn + 1;
    if (!x.slots) items = units * ((rows + x.bm - 1) / x.bm);
    x.wgs = x.few && d.dtype == ZIPVL_F32 && d.d == 128 ? kCus : 2 * kCus;
    const int64_t least = x.few ? kLeastFew : kLeastMany, part = std::min<int64_t>(rows, x.bm);
    x.direct = !x.slots && (items > kScanItems || tiles < 2 * least);      // the last: nothing can be cut
    x.grid = x.direct ? items / 8 * 8 + 8 : std::max<int64_t>(x.wgs + 64, (items + 21) / 8 * 8);
    x.rows = x.direct ? 0 : x.slots ? (int)(x.wgs * x.bm + units * ((rows + x.bm - 1) / x.bm) * part + (int64_t)d.Hkv * x.slots * x.bm) : (int)(x.wgs * part);
    x.ml = (size_t)x.rows * d.d * sizeof(float);
    x.pieces = x.ml + (size_t)x.rows * 2 * sizeof(float);
    x.shared = x.pieces + (x.direct ? 0 : items * sizeof(int2));
    x.total = x.shared + (x.slots ? units * sizeof(int2) : 0);
    return x;
}

// For any number of groups: of those whose rows are packed, the most take most.
size_t chunk_attn_workspace_bytes(const zipvl_dims& d, int64_t keys) {
    const int64_t rows = (int64_t)d.n * (d.Hq / d.Hkv), left = (kScanItems - (int64_t)d.B * d.Hkv * ((rows + kRowsMany - 1) / kRowsMany)) / d.Hkv - d.B * rows / kRowsMany - 1;
    const int64_t groups = std::min<int64_t>(std::min<int64_t>(d.B / 2, left), d.B * rows / (kFewRows + 1));
    return std::max<size_t>(std::max<size_t>(16, chunk_plan(d, keys, 0).total), groups > 0 ? chunk_plan(d, keys, (int)groups).total : 0);
}

template <typename Kernel>
static int allow_lds(Kernel kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;                                             // more than 64 KB of LDS has to be asked for, on every device
    if (hipGetDevice(&dev) != hipSuccess) return set_error(ZIPVL_EHIP, "chunk_attn_paged: no current device");
    if (dev > 63 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess)
            return set_error(ZIPVL_EHIP, "chunk_attn_paged: %d bytes of LDS are refused", bytes);
        if (dev <= 63) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    return ZIPVL_OK;
}

template <typename T, int D, int BM>
static int launch_join(const Chunk& p, const ChunkParts& parts, const ChunkPlan& x, hipStream_t st) {
    const int64_t rows = (int64_t)p.n * p.G, step = 1024 / D;
    int64_t per = step;                                      // about 2048 workgroups at most
    while (p.units * ((rows + per - 1) / per) > 2048 && per < rows) per *= 2;
    KernelTimer tm(ZIPVL_K_CHUNK_JOIN, st);
    hipLaunchKernelGGL((chunk_join_kernel<T, D, BM>), dim3((unsigned)((rows + per - 1) / per), p.units), dim3(256), 0, st, p, parts, (int)per);
    return check_launch("chunk_attn_paged parts");
}

template <typename T, int D, int COLS>
static int launch_few(const Chunk& p, const ChunkParts& parts, const ChunkPlan& x, hipStream_t st) {
    static std::atomic<uint64_t> done{0};
    int rc = allow_lds(&chunk_few_kernel<T, D, COLS>, PartCfg<T, D>::LDS, done);
    if (rc) return rc;
    {
        KernelTimer tm(ZIPVL_K_CHUNK_ATTN, st);
        hipLaunchKernelGGL((chunk_few_kernel<T, D, COLS>), dim3((unsigned)x.grid), dim3(256), (PartCfg<T, D>::LDS), st, p, parts, __builtin_ctz(x.wgs), x.direct);
        if ((rc = check_launch("chunk_attn_paged"))) return rc;
    }
    return !x.direct ? launch_join<T, D, COLS>(p, parts, x, st) : ZIPVL_OK;
}

template <typename T, int D>
static int launch_chunk_t(const Chunk& p, const ChunkParts& parts, const ChunkPlan& x, hipStream_t st) {
    if (x.few) return x.bm == 16 ? launch_few<T, D, 16>(p, parts, x, st) : launch_few<T, D, 32>(p, parts, x, st);
    static std::atomic<uint64_t> done{0};
    int rc = allow_lds(&chunk_many_kernel<T, D>, ChunkCfg<T, D>::LDS, done);
    if (rc) return rc;
    {
        KernelTimer tm(ZIPVL_K_CHUNK_ATTN, st);
        hipLaunchKernelGGL((chunk_many_kernel<T, D>), dim3((unsigned)x.grid), dim3(256), (ChunkCfg<T, D>::LDS), st, p, parts, __builtin_ctz(x.wgs), x.direct);
        if ((rc = check_launch("chunk_attn_paged"))) return rc;
    }
    return !x.direct ? launch_join<T, D, kRowsMany>(p, parts, x, st) : ZIPVL_OK;
}

int launch_chunk_attn_paged(const void* Q, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* len, const int32_t* k,
                            const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_len, const int32_t* group_begin, int32_t groups,
                            const zipvl_dims& d, float scale, void* O, const int64_t* o_strides, float* lse, void* ws, hipStream_t st)
{
    const int G = d.Hq / d.Hkv;
    Chunk p = {(const char*)pages.K, (const char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table, table_pages, len, k,
                     prefix_table, prefix_pages, prefix_len, group_begin, groups, d.B, d.Hq, d.Hkv, G, d.n, d.B * d.Hkv, inverse(d.Hkv), inverse(G),
                     (const char*)Q, {d.q_strides[0], d.q_strides[1], d.q_strides[2]}, (char*)O, {o_strides[0], o_strides[1], o_strides[2]}, lse, scale * kLog2e, 0};
    const ChunkPlan x = chunk_plan(d, ((int64_t)table_pages + prefix_pages) * pages.page, groups);
    p.slots = x.slots;
    if (x.grid >= 1 << 24) return set_error(ZIPVL_ESHAPE, "zipvl_chunk_attn_paged: %lld tiles of queries are more than one grid takes", (long long)x.grid);
    const ChunkParts parts = {(float*)ws, (float*)((char*)ws + x.ml), (int2*)((char*)ws + x.pieces), (int2*)((char*)ws + x.shared), x.rows};
    if (d.dtype == ZIPVL_BF16) return d.d == 128 ? launch_chunk_t<__bf16, 128>(p, parts, x, st) : launch_chunk_t<__bf16, 64>(p, parts, x, st);
    return d.d == 128 ? launch_chunk_t<float, 128>(p, parts, x, st) : launch_chunk_t<float, 64>(p, parts, x, st);
}

}  // namespace zipvl
