// Decode attention over pages, with prefixes that several batch elements share (Eq. (5); Algorithm 2).
//
// Memory-bound for as long as few queries meet a row.  An item is a unit (batch element, KV head) with its own rows and the G queries of its
// group of heads, or a (prefix, KV head) with the G queries of every batch element that shares it, in blocks of 32: a row of a prefix is read once
// for 32 queries instead of once for every batch element.  Both are the same work: 32 columns of queries (those that an item lacks are
// zero) against tiles of 32 rows, S^T = K Q^T and O^T += V^T P^T on 32x32 matrix tiles, so that a lane has one query and the softmax
// statistics are scalars of a lane.
//
// How the work is cut up is decided on the device, where the lengths are: every item weighs its tiles and a little for its start, the weights of all
// items follow each other on a line, and the workgroups take equal pieces of that line.  However unequal the lengths, no workgroup has more than
// another; a long item gets many workgroups and several short ones share one.  Every workgroup sums up the weights by itself (B Hkv +
// groups Hkv lengths, a microsecond), nothing is read back and no launch is spent on it.
// Parts (max, sum, weighted sum of rows) of an item that was cut are joined by a second launch.
#include <algorithm>
#include <atomic>

#include "launch.h"
#include "ldsload.h"

namespace zipvl {

constexpr int kTileRows = 32, kCols = 32, kPartWaves = 4;
constexpr int kStart = 2;            // what starting an item weighs, in tiles: its queries, its first rows, its part
constexpr int kLeast = 8;            // weight below which a workgroup is not worth its part
constexpr int kSolo = 4;             // tiles up to which one wave takes an item alone
constexpr int kPartGrid = 512;       // two workgroups a CU
constexpr float kLazy = 8.f;         // how far (log2) a logit may exceed the offset of the exponentials before that moves

struct PagedRead {
    const char *K, *V;
    int num_pages, page_log2;
    const int32_t* table; int width; const int32_t* len;
    const int32_t* prefix_table; int prefix_width; const int32_t* prefix_len;
    const int32_t* group_begin; int groups;
    int B, Hq, Hkv, G;
};

// Parts: a record is D floats and (max, sum).  Records 2 (b Hq + h) + {0: prefix, 1: own} are those of items that one workgroup had whole;
// behind them every workgroup has 32 for the piece of an item that began before it and 32 for one that goes on after it.  `pieces` says of
// every own item and every block of a prefix which workgroups had it.
struct Parts {
    float* o; float* ml; int2* pieces; int rows;             // rows = B Hq
    __device__ __forceinline__ int64_t whole(int row, int own) const { return 2 * (int64_t)row + own; }
    __device__ __forceinline__ int64_t piece(int wg, int begins, int col) const { return 2 * (int64_t)rows + ((int64_t)wg * 2 + begins) * kCols + col; }
};
// Blocks of a prefix are counted from begin G / 32 + p: no two groups meet, and B G / 32 + groups + 1 are enough.
__host__ __device__ __forceinline__ int piece_slots(const PagedRead& p) { return (int)((int64_t)p.B * p.G / kCols) + p.groups + 1; }
__device__ __forceinline__ int piece_own(const PagedRead& p, int u) { return u; }
__device__ __forceinline__ int piece_prefix(const PagedRead& p, int group, int begin, int block, int g) {
    return p.B * p.Hkv + (begin * p.G / kCols + group + block) * p.Hkv + g;
}

__device__ __forceinline__ int clamped(int v, int low, int high) { return max(low, min(v, high)); }
struct Group { int begin, end; };
__device__ __forceinline__ Group group_of(const PagedRead& p, int i) {
    const int begin = clamped(p.group_begin[i], 0, p.B);
    return {begin, clamped(p.group_begin[i + 1], begin, p.B)};
}
__device__ __forceinline__ int own_rows(const PagedRead& p, int u) { return clamped(p.len[u], 0, p.width << p.page_log2); }
__device__ __forceinline__ int prefix_rows(const PagedRead& p, int i) { return clamped(p.prefix_len[i], 0, p.prefix_width << p.page_log2); }

// Items: (prefix, KV head) first, then (batch element, KV head).
struct Item {
    int rows, blocks, begin;                                 // rows of the cache; blocks of queries; first batch element
    __device__ __forceinline__ int tiles() const { return (rows + kTileRows - 1) / kTileRows; }
    __device__ __forceinline__ int weight_of_block() const { return rows ? tiles() + kStart : 0; }
    __device__ __forceinline__ double weight() const { return (double)blocks * weight_of_block(); }       // whole numbers below 2^53
};
__device__ __forceinline__ Item item_of(const PagedRead& p, int i) {
    const int prefixes = p.groups * p.Hkv;
    if (i >= prefixes + p.B * p.Hkv) return {0, 0, 0};
    if (i >= prefixes) return {own_rows(p, i - prefixes), 1, (i - prefixes) / p.Hkv};
    const Group g = group_of(p, i / p.Hkv);
    return {prefix_rows(p, i), ((g.end - g.begin) * p.G + kCols - 1) / kCols, g.begin};
}

// sums of lanes 0 ... own
__device__ __forceinline__ double wave_scan(double v) {
    v += lane_moved<0x111, 0xF>(v, 0.0);
    v += lane_moved<0x112, 0xF>(v, 0.0);
    v += lane_moved<0x114, 0xF>(v, 0.0);
    v += lane_moved<0x118, 0xF>(v, 0.0);
    v += lane_moved<0x142, 0xA>(v, 0.0);
    v += lane_moved<0x143, 0xC>(v, 0.0);
    return v;
}

__device__ __forceinline__ float other_half(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

template <typename T, int D>
struct PartCfg {
    static constexpr int RB = D * (int)sizeof(T);            // bytes per row
    static constexpr int TILE = kTileRows * RB;
    static constexpr int NL = TILE / 1024, RPL = 1024 / RB;  // loads of 1 KiB per tile, rows per load
    static constexpr int WAVE = 2 * TILE;                    // a wave's LDS: a tile of K, one of V
    static constexpr int CH = D / Elem<T>::kPerChunk, ODB = D / 32;
    static constexpr int MB = WAVE >= 2 * 32 * 33 * 4 ? 2 : 1;       // blocks of 32 channels joined at a time
    static constexpr int LDS = kPartWaves * WAVE;
    static constexpr int PER_CU = LDS > 80 * 1024 ? 1 : 2;
    // swizzle of row r's 16-byte chunks: K is read 32 rows at a time at one chunk, V of bf16 by transposing reads
    __device__ static __forceinline__ int k_swizzle(int r) { return k_row_swizzle<RB>(r); }
    __device__ static __forceinline__ int v_swizzle(int r) {
        if constexpr (sizeof(T) == 2) return ((r & 3) >> (RB == 128 ? 1 : 0)) << 2;
        else return k_row_swizzle<RB>(r);
    }
};

// A wave's queries against tiles of one item.
template <typename T, int D>
struct WavePart {
    using C = PartCfg<T, D>;
    uintx4 qf[C::CH];
    floatx16 o[C::ODB];
    float m, l;                                              // l: of the lane's half of the keys, until `finish`

    struct Tile { const char *k0, *k1, *v0, *v1; uint32_t rows; };      // of its first and second 16 rows; which of the 32 there are

    __device__ __forceinline__ void reset() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int db = 0; db < C::ODB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
    }
    __device__ __forceinline__ void load_queries(const T* row, bool there) {     // of column lane % 32
        const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
        for (int cc = 0; cc < C::CH; ++cc) {
            qf[cc] = uintx4{0, 0, 0, 0};
            if (there) qf[cc] = load16(row + (2 * cc + h) * Elem<T>::kPerFrag);
        }
    }

    // Rows that are not there take a row that is: its scores are masked, and what weighs nothing must be finite.
    template <bool V>
    __device__ static __forceinline__ void fetch(const char* g0, const char* g1, uint32_t rows, unsigned lds) {
        const int lane = threadIdx.x & 63, lr = lane / (C::RB / 16), p = lane % (C::RB / 16);
        if (rows == 0xFFFFFFFFu) {
#pragma unroll
            for (int q = 0; q < C::NL; ++q) {
                const int off = lr * C::RB + ((p ^ (V ? C::v_swizzle(q * C::RPL + lr) : C::k_swizzle(q * C::RPL + lr))) << 4);
                const char* base = q < C::NL / 2 ? g0 + q * 1024 : g1 + (q - C::NL / 2) * 1024;
                load_kib_to_lds(base, off, lds + q * 1024);
            }
        } else {
            const int safe = __builtin_ctz(rows);
#pragma unroll 1
            for (int q = 0; q < C::NL; ++q) {
                const int r = q * C::RPL + lr, chunk = (p ^ (V ? C::v_swizzle(r) : C::k_swizzle(r))) << 4;
                const int rr = rows >> r & 1 ? r : safe;
                load_kib_to_lds_at((rr < 16 ? g0 + rr * C::RB : g1 + (rr - 16) * C::RB) + chunk, lds + q * 1024);
            }
        }
    }

    __device__ __forceinline__ floatx16 scores(const char* kb) const {
        const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
        floatx16 s = {0};
#pragma unroll
        for (int cc = 0; cc < C::CH; ++cc) {
            const uintx4 kf = *reinterpret_cast<const uintx4*>(kb + i * C::RB + swz_chunk(2 * cc + h, C::k_swizzle(i)));
            s = mma_frag<T>(kf, qf[cc], s);
        }
        return s;
    }

    // scores -> weights; the offset m follows the running maximum lazily
    __device__ __forceinline__ void weigh(floatx16& s, uint32_t rows, float c) {
        const int h = (threadIdx.x >> 5) & 1;
        if (rows != 0xFFFFFFFFu) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!(rows >> acc_row(r, h) & 1)) s[r] = -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        mx *= c;
        if (__any(mx > m + kLazy)) {
            mx = fmaxf(mx, other_half(mx));
            const float m_new = fmaxf(m, mx), a = m_new > -INFINITY ? fast_exp2(m - m_new) : 1.f;
            l *= a;
#pragma unroll
            for (int db = 0; db < C::ODB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[db][r] *= a;
            m = m_new;
        }
        const float ms = m > -INFINITY ? m : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = fast_exp2(fmaf(s[r], c, -ms));
            l += s[r];
        }
    }

    // O^T += V^T P^T.  The accumulators of S^T are the operand of P^T as they are (contraction slot t of a lane = key 16 s2 + 8 (t / 4) + 4 h + t % 4).
    // bf16: the weights as two planes, 16 bits of each: one plane alone is off by 2^-9 of a weight, as much as the output's own rounding where a
    // few rows have all the weight, and costs as much memory time.
    __device__ __forceinline__ void weighted_rows(const char* vb, const floatx16& s) {
        const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            typedef short shortx4 __attribute__((ext_vector_type(4)));
            using lds_ptr = __attribute__((address_space(3))) shortx4*;
            const int grp = (lane >> 4) & 1, e = (lane >> 2) & 3, q = lane & 3, row = 4 * h + e;
            uintx4 hi[2], lo[2];
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float a = s[8 * s2 + 2 * x], b = s[8 * s2 + 2 * x + 1];
                    const uint32_t w = pack_bf16x2(a, b);
                    hi[s2][x] = w;
                    lo[s2][x] = pack_bf16x2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xFFFF0000u));
                }
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int db = 0; db < C::ODB; ++db) {
                    const char* a0 = vb + (row + 16 * s2) * C::RB + swz_chunk(4 * db + 2 * grp + (q >> 1), C::v_swizzle(row)) + (q & 1) * 8;
                    const uintx2 f0 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)a0));
                    const uintx2 f1 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(a0 + 8 * C::RB)));
                    const uintx4 vf = {f0[0], f0[1], f1[0], f1[1]};
                    o[db] = mma_frag<__bf16>(vf, lo[s2], o[db]);
                    o[db] = mma_frag<__bf16>(vf, hi[s2], o[db]);
                }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = acc_row(r, h);
#pragma unroll
                for (int db = 0; db < C::ODB; ++db) {
                    const float v = *reinterpret_cast<const float*>(vb + key * C::RB + swz_chunk(8 * db + (i >> 2), C::v_swizzle(key)) + (i & 3) * 4);
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[r], o[db], 0, 0, 0);
                }
            }
        }
    }

    // Tiles first, first + step, ... below `end` of an item with `rows` rows and this row of a table.  K of the next tile is requested when K of this one
    // has been read, V of the next when V of this one has: a wave has one tile of each in LDS and one on the way at any time.
    __device__ __forceinline__ void run(const PagedRead& p, const int32_t* table, int rows, int first, int step, int end, float c, char* mine) {
        const int lane = threadIdx.x & 63, n = first < end ? (end - first + step - 1) / step : 0;
        const bool small = p.page_log2 == 4;                 // a tile is two pages
        int from = 0, e0 = -1, e1 = -1;                      // entries of the tiles from .. from + 63, one a lane
        auto entries = [&]() {
            const int t = first + min(from + lane, n - 1) * step;
            e0 = table[t * kTileRows >> p.page_log2];
            if (small) e1 = t * kTileRows + 16 < rows ? table[2 * t + 1] : -1;
        };
        int at = -1;
        auto next = [&](Tile& x) {                           // the next tile of which there is a row; false: none
            for (++at; at < n; ++at) {
                if (at == from + 64) { from = at; entries(); }
                const int t = first + at * step, left = rows - t * kTileRows;
                const int a = __builtin_amdgcn_readlane(e0, at - from);
                x.rows = left >= kTileRows ? 0xFFFFFFFFu : (1u << left) - 1;
                const bool there = (unsigned)a < (unsigned)p.num_pages;
                const int64_t at0 = (((int64_t)(there ? a : 0) << p.page_log2) + (t * kTileRows & ((1 << p.page_log2) - 1))) * C::RB;
                int64_t at1 = at0 + 16 * C::RB;
                if (small) {
                    const int b = __builtin_amdgcn_readlane(e1, at - from);
                    if (!there) x.rows &= 0xFFFF0000u;
                    if ((unsigned)b >= (unsigned)p.num_pages) x.rows &= 0x0000FFFFu;
                    at1 = ((int64_t)((unsigned)b < (unsigned)p.num_pages ? b : 0) << 4) * C::RB;
                } else if (!there) x.rows = 0;
                if (x.rows == 0) continue;
                x.k0 = scalar_ptr(p.K + at0);
                x.k1 = scalar_ptr(p.K + at1);
                x.v0 = scalar_ptr(p.V + at0);
                x.v1 = scalar_ptr(p.V + at1);
                x.rows = __builtin_amdgcn_readfirstlane(x.rows);
                return true;
            }
            return false;
        };
        if (n <= 0) return;
        entries();
        char *kb = mine, *vb = mine + C::TILE;
        const unsigned klds = lds_address(kb), vlds = lds_address(vb);
        Tile cur, nxt;
        bool have = next(cur);
        if (!have) return;
        fetch<false>(cur.k0, cur.k1, cur.rows, klds);
        fetch<true>(cur.v0, cur.v1, cur.rows, vlds);
        while (have) {
            const bool more = next(nxt);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::NL) : "memory");             // all but V of this tile
            floatx16 s = scores(kb);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                       // K has been read
            if (more) fetch<false>(nxt.k0, nxt.k1, nxt.rows, klds);
            weigh(s, cur.rows, c);
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::NL) : "memory");   // all but K of the next
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            weighted_rows(vb, s);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) fetch<true>(nxt.v0, nxt.v1, nxt.rows, vlds);
            cur = nxt;
            have = more;
        }
    }
};

template <typename T, int D>
__global__ __launch_bounds__(64 * kPartWaves, (PartCfg<T, D>::PER_CU)) void paged_part_kernel(const T* __restrict__ q, PagedRead p, float c, Parts out) {
    using C = PartCfg<T, D>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ double sums[kPartWaves];
    __shared__ double found_base;
    __shared__ int found_item;
    __shared__ float2 ml[kPartWaves][kCols];
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i = lane & 31, h = lane >> 5;
    const int items = (p.groups + p.B) * p.Hkv, per = (items + 255) / 256;
    char* const mine = smem + w * C::WAVE;

    // where on the line of weights this workgroup's piece is
    double sum = 0.0;
    for (int x = 0; x < per; ++x) sum += item_of(p, tid * per + x).weight();
    const double upto = wave_scan(sum);
    if (lane == 63) sums[w] = upto;
    if (tid == 0) found_item = items;
    __syncthreads();
    double total = 0.0, base = upto - sum;
    for (int x = 0; x < kPartWaves; ++x) {
        if (x < w) base += sums[x];
        total += sums[x];
    }
    const int64_t all = (int64_t)total;
    const int64_t wgs = max((int64_t)1, min((int64_t)gridDim.x, all / kLeast));
    if (blockIdx.x >= wgs || all == 0) return;
    const int64_t lo = all * blockIdx.x / wgs, hi = all * (blockIdx.x + 1) / wgs;
    if (base <= (double)lo && (double)lo < base + sum) { found_item = tid * per; found_base = base; }
    __syncthreads();

    int item = __builtin_amdgcn_readfirstlane(found_item), window = item;
    int64_t pos = lo, start = (int64_t)found_base;           // start: of `item` on the line
    Item seen = item_of(p, window + lane);                   // of 64 items, one a lane
    int ordinal = 0;                                         // of short items, which the waves take in turn
    while (pos < hi && item < items) {                       // the items end where the line does, unless lengths change meanwhile
        if (item == window + 64) {
            window = item;
            seen = item_of(p, window + lane);
        }
        Item it;
        it.rows = __builtin_amdgcn_readlane(seen.rows, item - window);
        it.blocks = __builtin_amdgcn_readlane(seen.blocks, item - window);
        it.begin = __builtin_amdgcn_readlane(seen.begin, item - window);
        const int tiles = it.tiles(), wb = it.weight_of_block();
        const int64_t weight = (int64_t)it.blocks * wb;
        if (pos >= start + weight) { start += weight; ++item; continue; }
        const int block = (int)(pos - start) / wb;            // an item weighs less than 2^31
        const int64_t block_start = start + (int64_t)block * wb;
        const int x0 = (int)(pos - block_start), x1 = (int)min((int64_t)wb, hi - block_start);
        pos = block_start + x1;
        const int ta = min(x0, tiles), tb = min(x1, tiles);
        if (ta >= tb) continue;                              // nothing but the item's start
        const bool own = item >= p.groups * p.Hkv, begins = ta == 0, ends = tb == tiles, whole = begins && ends;
        const int unit = own ? item - p.groups * p.Hkv : item, g = unit % p.Hkv, group = own ? 0 : item / p.Hkv;
        const Group members = own ? Group{it.begin, it.begin + 1} : group_of(p, group);
        const int cols = min(kCols, (members.end - members.begin) * p.G - block * kCols);
        int2* const piece = out.pieces + (own ? piece_own(p, unit) : piece_prefix(p, group, members.begin, block, g));
        if (tid == 0) {
            if (begins) piece->x = blockIdx.x;
            if (ends) piece->y = blockIdx.x;
        }
        const bool solo = tb - ta <= kSolo;
        if (solo && ordinal++ % kPartWaves != w) continue;

        const int col = block * kCols + min(i, cols - 1);    // row of the output that lane i has
        const int row = (members.begin + col / p.G) * p.Hq + g * p.G + col % p.G;
        WavePart<T, D> part;
        part.reset();
        part.load_queries(q + (int64_t)row * D, i < cols);
        const int32_t* table = own ? p.table + (int64_t)unit * p.width : p.prefix_table + (int64_t)unit * p.prefix_width;
        part.run(p, table, it.rows, solo ? ta : ta + w, solo ? 1 : kPartWaves, tb, c, mine);
        part.l += other_half(part.l);
        auto record = [&](int of_col, int of_row) { return whole ? out.whole(of_row, own) : out.piece(blockIdx.x, begins, of_col); };
        if (solo) {
            if (i < cols) {
                const int64_t rec = record(i, row);
                float* dst = out.o + rec * D;
#pragma unroll
                for (int db = 0; db < C::ODB; ++db)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        *reinterpret_cast<floatx4*>(dst + 32 * db + 8 * x + 4 * h) = floatx4{part.o[db][4 * x], part.o[db][4 * x + 1], part.o[db][4 * x + 2], part.o[db][4 * x + 3]};
                if (h == 0) *reinterpret_cast<float2*>(out.ml + 2 * rec) = make_float2(part.m, part.l);
            }
            continue;
        }
        // the waves' parts meet in LDS, a few channels at a time, rows of 33 so that both ways through are free of conflicts
        if (h == 0) ml[w][i] = make_float2(part.m, part.l);
        __syncthreads();
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int x = 0; x < kPartWaves; ++x) M = fmaxf(M, ml[x][i].x);
#pragma unroll
        for (int x = 0; x < kPartWaves; ++x) L += M > -INFINITY ? fast_exp2(ml[x][i].x - M) * ml[x][i].y : 0.f;
        const float a = M > -INFINITY ? fast_exp2(part.m - M) : 0.f;
        if (w == 0 && h == 0 && i < cols) *reinterpret_cast<float2*>(out.ml + 2 * record(i, row)) = make_float2(M, L);
        constexpr int kChannels = 32 * C::MB;
        for (int pass = 0; pass < C::ODB / C::MB; ++pass) {
            float* mo = reinterpret_cast<float*>(mine);
#pragma unroll
            for (int db = 0; db < C::ODB; ++db)
                if (db / C::MB == pass)
#pragma unroll
                    for (int r = 0; r < 16; ++r) mo[(32 * (db % C::MB) + acc_row(r, h)) * 33 + i] = part.o[db][r] * a;
            __syncthreads();
            for (int x = tid; x < cols * kChannels; x += 64 * kPartWaves) {
                const int cc = x / kChannels, ch = x % kChannels;
                float v = 0.f;
#pragma unroll
                for (int y = 0; y < kPartWaves; ++y) v += reinterpret_cast<const float*>(smem + y * C::WAVE)[ch * 33 + cc];
                const int r = block * kCols + cc;
                out.o[record(cc, (members.begin + r / p.G) * p.Hq + g * p.G + r % p.G) * D + pass * kChannels + ch] = v;
            }
            __syncthreads();
        }
    }
}

// The parts of one query head: those of its group's prefix, then its own -> its output row.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedRead p, Parts in, T* __restrict__ o, int wgs) {
    constexpr int kPer = D / 4, kAt = 256 / kPer;            // threads per part, parts at a time
    __shared__ floatx4 sum[256];
    const int row = blockIdx.x, b = row / p.Hq, head = row - b * p.Hq, g = head / p.G, u = b * p.Hkv + g;
    const int tid = threadIdx.x, lane = tid & 63;
    int group = -1, begin = 0;
    for (int x = 0; x < p.groups; x += 64) {
        const Group m = x + lane < p.groups ? group_of(p, x + lane) : Group{0, 0};
        const uint64_t in_it = __ballot(m.begin <= b && b < m.end);
        if (in_it) {
            const int who = __builtin_ctzll(in_it);
            group = x + who;
            begin = __shfl(m.begin, who);
            break;
        }
    }
    int2 pre = {0, -1}, own = {0, -1};
    int col = 0;
    if (group >= 0 && prefix_rows(p, group * p.Hkv + g) > 0) {
        col = (b - begin) * p.G + head - g * p.G;
        pre = in.pieces[piece_prefix(p, group, begin, col / kCols, g)];
        col %= kCols;
    }
    if (own_rows(p, u) > 0) own = in.pieces[piece_own(p, u)];
    pre.x = max(pre.x, 0), pre.y = min(pre.y, wgs - 1), own.x = max(own.x, 0), own.y = min(own.y, wgs - 1);
    const int n_pre = max(0, pre.y - pre.x + 1), n = n_pre + max(0, own.y - own.x + 1);
    auto record = [&](int s) {
        const bool is_own = s >= n_pre;
        const int2 x = is_own ? own : pre;
        const int wg = x.x + (is_own ? s - n_pre : s);
        return x.x == x.y ? in.whole(row, is_own) : in.piece(wg, wg == x.x, is_own ? head - g * p.G : col);
    };
    float M = -INFINITY, L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += 64) {                     // 64 parts at a time, every wave all of their maxima and sums
        const int count = min(64, n - s0);
        float2 v = make_float2(-INFINITY, 0.f);
        int64_t rec = 0;
        if (lane < count) {
            rec = record(s0 + lane);
            v = *reinterpret_cast<const float2*>(in.ml + 2 * rec);
        }
        const float M_new = fmaxf(M, wave_max(v.x));
        const float a = M_new > -INFINITY ? fast_exp2(v.x - M_new) : 0.f, before = M_new > -INFINITY ? fast_exp2(M - M_new) : 0.f;
        L = L * before + wave_sum(a * v.y);
        acc *= before;
        M = M_new;
        for (int x0 = 0; x0 < count; x0 += kAt) {            // all lanes to the end: a lane that has left answers no other
            const int x = x0 + tid / kPer;
            const float weight = __shfl(a, min(x, 63));
            const int64_t r = __shfl(rec, min(x, 63));
            if (x < count) acc += weight * *reinterpret_cast<const floatx4*>(in.o + r * D + tid % kPer * 4);
        }
    }
    sum[tid] = acc;
    __syncthreads();
    if (tid < kPer) {
        for (int x = 1; x < min(kAt, n); ++x) acc += sum[x * kPer + tid];
        const float inv = L > 0.f ? 1.f / L : 0.f;
        T* dst = o + (int64_t)row * D + tid * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) dst[e] = (T)(acc[e] * inv);
    }
}

struct PagedLayout { size_t o, ml, pieces, total; };
static PagedLayout paged_layout(const zipvl_dims& d, int groups) {
    const size_t records = 2 * (size_t)d.B * d.Hq + 2 * (size_t)kPartGrid * kCols;
    PagedLayout l;
    l.o = 0;
    l.ml = l.o + records * d.d * sizeof(float);
    l.pieces = l.ml + records * 2 * sizeof(float);
    const size_t blocks = (size_t)d.B * (d.Hq / d.Hkv) / kCols + groups + 1;
    l.total = l.pieces + ((size_t)d.B + blocks) * d.Hkv * sizeof(int2);
    return l;
}

// a call with a prefix has at most B groups
size_t decode_paged_workspace_bytes(const zipvl_dims& d, int own, int prefix) { return paged_layout(d, prefix ? d.B : 0).total; }

template <typename T, int D>
static int launch_paged_t(const T* q, const PagedRead& p, const zipvl_dims& d, float scale, T* o, char* ws, hipStream_t st) {
    using C = PartCfg<T, D>;
    const PagedLayout l = paged_layout(d, p.groups);
    const Parts parts = {(float*)(ws + l.o), (float*)(ws + l.ml), (int2*)(ws + l.pieces), d.B * d.Hq};
    // what all lengths at their greatest would weigh
    const int64_t own = (int64_t)d.B * d.Hkv * (((int64_t)p.width << p.page_log2) / kTileRows + 1 + kStart);
    const int64_t pre = p.groups ? ((int64_t)d.B * p.G / kCols + p.groups) * d.Hkv * (((int64_t)p.prefix_width << p.page_log2) / kTileRows + 1 + kStart) : 0;
    const int wgs = (int)std::max<int64_t>(1, std::min<int64_t>(kPartGrid, (own + pre) / kLeast));
    static std::atomic<uint64_t> lds_set{0};                 // more than 64 KB of LDS has to be asked for, on every device
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return set_error(ZIPVL_EHIP, "decode_attn_paged: no current device");
    if (dev > 63 || !(lds_set.load(std::memory_order_relaxed) >> dev & 1)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_part_kernel<T, D>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS) != hipSuccess)
            return set_error(ZIPVL_EHIP, "decode_attn_paged: %d bytes of LDS are refused", (int)C::LDS);
        if (dev <= 63) lds_set.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    {
        KernelTimer tm(ZIPVL_K_PAGED_PARTIAL, st);
        hipLaunchKernelGGL((paged_part_kernel<T, D>), dim3(wgs), dim3(64 * kPartWaves), C::LDS, st, q, p, scale * kLog2e, parts);
        const int rc = check_launch("decode_attn_paged");
        if (rc) return rc;
    }
    KernelTimer tm(ZIPVL_K_PAGED_COMBINE, st);
    hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3(d.B * d.Hq), dim3(256), 0, st, p, parts, o, wgs);
    return check_launch("decode_attn_paged parts");
}

int launch_decode_attn_paged(const void* q, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* len,
                             const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_len, const int32_t* group_begin,
                             int32_t groups, const zipvl_dims& d, float scale, void* o, void* ws, hipStream_t st)
{
    const PagedRead p = {(const char*)pages.K, (const char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table, table_pages, len,
                         prefix_table, prefix_pages, prefix_len, group_begin, groups, d.B, d.Hq, d.Hkv, d.Hq / d.Hkv};
    if (d.dtype == ZIPVL_BF16)
        return d.d == 128 ? launch_paged_t<__bf16, 128>((const __bf16*)q, p, d, scale, (__bf16*)o, (char*)ws, st)
                          : launch_paged_t<__bf16, 64>((const __bf16*)q, p, d, scale, (__bf16*)o, (char*)ws, st);
    return d.d == 128 ? launch_paged_t<float, 128>((const float*)q, p, d, scale, (float*)o, (char*)ws, st)
                      : launch_paged_t<float, 64>((const float*)q, p, d, scale, (float*)o, (char*)ws, st);
}

}  // namespace zipvl
