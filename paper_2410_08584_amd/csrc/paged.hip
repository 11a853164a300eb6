// Decode attention over pages, with prefixes that several batch elements share (Eq. (5); Algorithm 2).
//
// Memory-bound for as long as few queries meet a row.  An item is a unit (batch element, KV head) with its own rows and the G queries of its
// group of heads, or a (prefix, KV head) with the G queries of every batch element that shares it, in blocks of 128: a row of a prefix comes from
// memory once for 128 queries instead of once for every batch element.  Both are the same work: columns of queries (those that an item
// lacks are zero) against tiles of 32 rows, S^T = K Q^T and O^T += V^T P^T on matrix tiles, so that a lane has one query and the
// softmax statistics are scalars of a lane.  A wave has 32 columns, or 16, and tiles of its own in LDS.  Items of up to 16 queries are cut by waves; of the others
// a workgroup has a block: its four waves take four tiles in turn (up to 32 queries), two and two the same two (up to 64), or all the same one, which
// comes from L2 for all but the first.
//
// How the work is cut up is decided on the device, where the lengths are (Line).  Nothing is read back and no launch is spent on it: every
// workgroup goes over the B Hkv + groups Hkv lengths by itself, a microsecond.
// Parts (max, sum, weighted sum of rows) of an item that was cut are joined by a second launch.
//
// Measured, in a graph, both launches, bf16, d = 128: 64 questions about four videos of up to 18432 tokens, 437 MB, 107 us = 4.1 TB/s (reading that much and
// nothing else: 71); 16 sequences with nothing shared, 353 MB, 75 us = 4.7 TB/s (58).  Two questions about one image, fp32: 11.7 us, which is two launches,
// finding the pieces and one tile after the other, not bytes.
// The constants below were measured over 29 calls, each in a graph: the listed cases of decode in perf/operators.py and the first 24 that its
// draw(random.Random(7)) gives of them.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "launch.h"
#include "ldsload.h"

namespace zipvl {

constexpr int kTileRows = 32, kCols = 32, kPartWaves = 4, kBlock = kCols * kPartWaves;
// What starting an item weighs: its queries, its first rows, its part.  Of items that waves cut, bf16: 3; with 6 the 29 calls take 2.0 % longer, with 1 4.3 %.  fp32
// tiles last longer and a start is 2 of them (two questions about an image: 11.7 us, with 3 12.8).  Of blocks: 12; with 6 2.2 % longer, with 24 0.4 %.
constexpr int kStartPrefix = 12, kStartWave = 3;
// Queries up to which waves cut a prefix, as they cut own rows.  Blocks of workgroups for all prefixes: the 29 calls take 12 % longer, and those where many prefixes
// are short twice as long (four of 246 rows with 32 KV heads: 29.9 us instead of 13.3).  More than 16 columns would need the wider tile.
constexpr int kLight = 16;
// Weight below which a workgroup is not worth its part; a tile of a block may weigh as much and no piece may be shorter.  fp32 without blocks: half of it, a tile
// for each wave, since such a tile is 2 us (with 8: 1.1 % longer over the 29 calls, 13.0 us instead of 11.7 for two questions about an image); bf16 with 6: as long.
constexpr int kLeast = 8;
constexpr int kCus = 256;
constexpr float kLazy = 8.f;         // how far (log2) a logit may exceed the offset of the exponentials before that moves (0: 0.5 % longer over the 29 calls)

// a wave-uniform number in scalar registers
__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct PagedRead {
    const char *K, *V;
    int num_pages, page_log2;
    const int32_t* table; int width; const int32_t* len;
    const int32_t* prefix_table; int prefix_width; const int32_t* prefix_len;
    const int32_t* group_begin; int groups;
    int B, Hq, Hkv, G;
    uint32_t inv_Hkv, inv_G, inv_Hq;
    int wide, least;
    __device__ __forceinline__ int prefixes() const { return groups * Hkv; }
    __device__ __forceinline__ int items() const { return (groups + B) * Hkv; }
};

// Parts: a record is D floats and (max, sum).  Records 2 (b Hq + h) + {0: prefix, 1: own} are those of items that were not cut.  Behind them are those
// of pieces: for every workgroup `cols` of a prefix that began before it and as many of one that goes on after it, then for every
// wave `wave_cols` and as many in the same way.  `pieces` says of every own item and every block of a prefix from which to which
// workgroup, or wave, its pieces are.
struct Parts {
    float* o; float* ml; int2* pieces; int rows, cols, wave_cols, grid;      // rows = B Hq
    __device__ __forceinline__ int whole(int row, int own) const { return 2 * row + own; }
    __device__ __forceinline__ int piece(int by_wave, int who, int begins, int col) const {  // below 2^20
        return 2 * rows + (by_wave ? 2 * grid * cols + (who * 2 + begins) * wave_cols : (who * 2 + begins) * cols) + col;
    }
};
// On the numbers of pieces: of waves; of a long item; of the first wave, for its whole workgroup.
constexpr int kByWave = 1 << 30, kLong = 1 << 29, kEntire = 1 << 28, kNumber = kEntire - 1;
// A workgroup all of whose piece is of one item joins its four waves' parts if the item is long: more than 16 workgroups' pieces (parts are fewer for the second launch:
// one sequence of 60000 rows among 63 of 200, 32 heads on 1, 28.7 us instead of 41.0; from 4 on: 2.1 % longer over the 29 calls), or any item where pieces are 32 tiles
// and more (its waves then read side by side: 16 unshared sequences 75.9 us instead of 77.9).  For short pieces meeting in LDS costs more than it saves (all items: 3.9 %).
constexpr int kLongWorkgroups = 16, kLongPiece = 32;
// Blocks of a prefix are counted from begin G / kBlock + p: no two groups meet, and B G / kBlock + groups + 1 are enough.
__device__ __forceinline__ int piece_own(const PagedRead& p, int u) { return u; }
__device__ __forceinline__ int piece_prefix(const PagedRead& p, int group, int begin, int block, int g) {
    return p.B * p.Hkv + (begin * p.G / kBlock + group + block) * p.Hkv + g;
}

__device__ __forceinline__ int clamped(int v, int low, int high) { return max(low, min(v, high)); }
struct Group { int begin, end; };
__device__ __forceinline__ Group group_of(const PagedRead& p, int i) {
    const int begin = clamped(p.group_begin[i], 0, p.B);
    return {begin, clamped(p.group_begin[i + 1], begin, p.B)};
}
__device__ __forceinline__ int own_rows(const PagedRead& p, int u) { return clamped(p.len[u], 0, p.width << p.page_log2); }
__device__ __forceinline__ int prefix_rows(const PagedRead& p, int i) { return clamped(p.prefix_len[i], 0, p.prefix_width << p.page_log2); }

// Items: (prefix, KV head) first, then (batch element, KV head).  A wave's tile is one unit of weight: a tile of a block weighs 1, 2 or 4 by
// the waves that have it; of fp32 rows twice that where it takes 32 columns, not 16 (`wide`: matrix time is what fp32 tiles last).
struct Item {
    int rows;                                                // of the cache
    uint32_t who;                                            // queries | first batch element << 16: both below 2^16
    __device__ __forceinline__ int cols() const { return who & 0xFFFF; }
    __device__ __forceinline__ int begin() const { return who >> 16; }
    __device__ __forceinline__ int tiles() const { return (rows + kTileRows - 1) / kTileRows; }
    __device__ __forceinline__ int blocks() const { return rows ? (cols() + kBlock - 1) / kBlock : 0; }
    __device__ __forceinline__ int waves_log2(int block) const {            // that have the same tile
        const int left = cols() - block * kBlock;
        return left <= kCols ? 0 : left <= 2 * kCols ? 1 : 2;
    }
    __device__ __forceinline__ int tile_log2(int block, int wide) const {   // weight of a tile: up to 8
        return waves_log2(block) + (cols() - block * kBlock > 16 ? wide : 0);
    }
    __device__ __forceinline__ int weight_of_full_block(int wide) const { return (tiles() << (2 + wide)) + kStartPrefix; }
    // Items of few queries are cut by waves (find_piece); the others' blocks by workgroups.
    __device__ __forceinline__ bool light() const { return cols() <= kLight; }
    __device__ __forceinline__ int weight(bool by_wave, int wide) const {
        const int n = blocks();
        if (by_wave) return n ? (tiles() << (cols() > 16 ? wide : 0)) + kStartWave - wide : 0;
        return n ? (n - 1) * weight_of_full_block(wide) + (tiles() << tile_log2(n - 1, wide)) + kStartPrefix : 0;
    }
};
__device__ __forceinline__ Item own_item(const PagedRead& p, int u, int length) {
    return {clamped(length, 0, p.width << p.page_log2), (uint32_t)p.G | (uint32_t)divided(u, p.Hkv, p.inv_Hkv) << 16};
}
__device__ __forceinline__ Item prefix_item(const PagedRead& p, int length, int g0, int g1) {
    const int begin = clamped(g0, 0, p.B), members = clamped(g1, begin, p.B) - begin;
    return {clamped(length, 0, p.prefix_width << p.page_log2), (uint32_t)(members * p.G) | (uint32_t)begin << 16};
}
__device__ __forceinline__ Item item_of(const PagedRead& p, int i) {
    if (i >= p.items()) return {0, 0};
    if (i >= p.prefixes()) return own_item(p, i - p.prefixes(), p.len[i - p.prefixes()]);
    const int group = divided(i, p.Hkv, p.inv_Hkv);
    return prefix_item(p, p.prefix_len[i], p.group_begin[group], p.group_begin[group + 1]);
}

// sums of lanes 0 ... own
__device__ __forceinline__ int wave_scan(int v) {
    v += lane_moved<0x111, 0xF>(v, 0);
    v += lane_moved<0x112, 0xF>(v, 0);
    v += lane_moved<0x114, 0xF>(v, 0);
    v += lane_moved<0x118, 0xF>(v, 0);
    v += lane_moved<0x142, 0xA>(v, 0);
    v += lane_moved<0x143, 0xC>(v, 0);
    return v;
}

// Over the groups of lanes that have one column each (lanes l and l ^ 32; for columns of 16 also l ^ 16), by register swaps.
template <int COLS, typename F>
__device__ __forceinline__ float over_groups(float v, F&& f) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    if constexpr (COLS == 16) {
        const unsigned x = __float_as_uint(v);
        const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        v = f(__uint_as_float(y[0]), __uint_as_float(y[1]));
    }
    return v;
}

template <typename T, int D>
struct PartCfg {
    static constexpr int RB = D * (int)sizeof(T);            // bytes per row
    static constexpr int TILE = kTileRows * RB;
    static constexpr int NL = TILE / 1024, RPL = 1024 / RB;  // loads of 1 KiB per tile, rows per load
    static constexpr int WAVE = 2 * TILE;                    // a wave's LDS: a tile of K, one of V
    static constexpr int CH = D / Elem<T>::kPerChunk, ODB = D / 32;
    static_assert(WAVE >= D * kCols * 4, "room for a wave's sums");
    static constexpr int LDS = kPartWaves * WAVE;
    // workgroups: of bf16 rows of 64 channels two as well, three take 0.5 % longer over the 29 calls (61 questions about 19382 rows: 63.8 us instead of 60.5); one
    // for all: 3.6 % longer, 64 questions about videos 125 us instead of 107
    static constexpr int PER_CU = LDS > 80 * 1024 ? 1 : 2;
    static constexpr int GRID = kCus * PER_CU;
    // swizzle of row r's 16-byte chunks: K is read 32 rows at a time at one chunk, V of bf16 by transposing reads
    __device__ static __forceinline__ int k_swizzle(int r) { return k_row_swizzle<RB>(r); }
    __device__ static __forceinline__ int v_swizzle(int r) {
        if constexpr (sizeof(T) == 2) return ((r & 3) >> (RB == 128 ? 1 : 0)) << 2;
        else return k_row_swizzle<RB>(r);
    }
};

// A wave's queries, in 32 columns or in 16, against tiles of one item.  With 16 a tile is two of 16x16: half the matrix cycles and half the
// exponentials, which is what a few tiles on their own last (fp32 products: 2 us a tile of d = 128, 4 with 32 columns; 32 columns for all: 7 % longer over the 29
// calls, two questions about an image 13.3 us instead of 11.7).
// Lane l has column l % COLS; the 64 / COLS groups of lanes share its keys and channels.
template <typename T, int D, int COLS>
struct WavePart {
    using C = PartCfg<T, D>;
    static constexpr int kGroups = 64 / COLS, kFrags = C::RB / 16 / kGroups, kKeys = kTileRows / kGroups;
    static constexpr int kPer = D / 16;                      // fp32, 16 columns: channels of a row that a lane has (weighted_rows)
    static constexpr int kO = D / COLS;                      // blocks of COLS channels
    using Acc = std::conditional_t<COLS == 32, floatx16, floatx4>;
    uintx4 qf[kFrags];
    Acc o[kO];
    float m, l;                                              // l: of the lane's share of the keys while tiles come

    struct Tile { const char *k0, *k1, *v0, *v1; uint32_t rows; };      // of its first and second 16 rows; which of the 32 there are

    // The lane, said anew: what follows from it is not worked out before the tiles and kept through them (it took 40 registers and spilled).
    __device__ static __forceinline__ int here() {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        return lane;
    }
    __device__ static __forceinline__ int col() { return threadIdx.x & (COLS - 1); }
    __device__ static __forceinline__ int group() { return (threadIdx.x & 63) / COLS; }
    __device__ static __forceinline__ int key(int r) {      // of score r
        if constexpr (COLS == 32) return acc_row(r, group());
        else return 16 * (r >> 2) + 4 * group() + (r & 3);
    }
    static constexpr int kRegs = COLS == 32 ? 16 : 4;        // sums of a block in a lane
    __device__ static __forceinline__ int channel(int b, int r, int group) {         // of o[b][r]
        if constexpr (COLS == 32) return 32 * b + acc_row(r, group);
        else if constexpr (sizeof(T) == 2) return 16 * b + 4 * group + r;
        else return kPer * (4 * group + r) + b;
    }

    __device__ __forceinline__ void reset() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int b = 0; b < kO; ++b)
#pragma unroll
            for (int r = 0; r < kRegs; ++r) o[b][r] = 0.f;
    }
    __device__ __forceinline__ void load_queries(const T* row, bool there) {     // of the lane's column
#pragma unroll
        for (int cc = 0; cc < kFrags; ++cc) {
            qf[cc] = uintx4{0, 0, 0, 0};
            if (there) qf[cc] = load16(row + (kGroups * cc + group()) * Elem<T>::kPerFrag);
        }
    }

    // Rows that are not there take a row that is: its scores are masked, and its values, which weigh nothing, are finite (or clear_absent takes them).
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

    __device__ static __forceinline__ floatx4 mma16(const uintx4& a, const uintx4& b, floatx4 acc) {
        if constexpr (sizeof(T) == 2) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
        else {
            const floatx4 fa = __builtin_bit_cast(floatx4, a), fb = __builtin_bit_cast(floatx4, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], acc, 0, 0, 0);
            return acc;
        }
    }

    // fp32 sums go in short chains that are added pairwise: with one through all channels the output is off by 6.2e-7 to 1.2e-6 of itself over the eight calls
    // of the 29 that are fp32, with these by 2.9e-7 to 5.1e-7, for up to 3 % of the time.
    __device__ __forceinline__ void scores(const char* kb, float (&s)[kKeys]) const {
        const int lane = threadIdx.x & 63, i = lane & (COLS - 1);
        if constexpr (COLS == 32) {
            constexpr int kChains = sizeof(T) == 4 ? 4 : 1;
            floatx16 x[kChains];
#pragma unroll
            for (int y = 0; y < kChains; ++y) x[y] = floatx16{0};
#pragma unroll
            for (int cc = 0; cc < kFrags; ++cc) {
                const uintx4 kf = *reinterpret_cast<const uintx4*>(kb + i * C::RB + swz_chunk(2 * cc + group(), C::k_swizzle(i)));
                x[cc * kChains / kFrags] = mma_frag<T>(kf, qf[cc], x[cc * kChains / kFrags]);
            }
#pragma unroll
            for (int half = kChains / 2; half; half >>= 1)
#pragma unroll
                for (int y = 0; y < half; ++y) x[y] += x[y + half];
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = x[0][r];
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                constexpr int kChains = sizeof(T) == 4 ? kFrags : 1;
                floatx4 x[kChains];
#pragma unroll
                for (int y = 0; y < kChains; ++y) x[y] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int cc = 0; cc < kFrags; ++cc) {
                    const uintx4 kf = *reinterpret_cast<const uintx4*>(kb + (16 * t + i) * C::RB + swz_chunk(4 * cc + group(), C::k_swizzle(16 * t + i)));
                    x[cc * kChains / kFrags] = mma16(kf, qf[cc], x[cc * kChains / kFrags]);
                }
#pragma unroll
                for (int half = kChains / 2; half; half >>= 1)
#pragma unroll
                    for (int y = 0; y < half; ++y) x[y] += x[y + half];
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * t + r] = x[0][r];
            }
        }
    }

    // scores -> weights; the offset m follows the running maximum lazily
    __device__ __forceinline__ void weigh(float (&s)[kKeys], uint32_t rows, float c) {
        if (rows != 0xFFFFFFFFu) {
#pragma unroll
            for (int r = 0; r < kKeys; ++r)
                if (!(rows >> key(r) & 1)) s[r] = -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < kKeys; ++r) mx = fmaxf(mx, s[r]);
        mx *= c;
        if (__any(mx > m + kLazy)) {
            mx = over_groups<COLS>(mx, [](float a, float b) { return fmaxf(a, b); });
            const float m_new = fmaxf(m, mx), a = m_new > -INFINITY ? fast_exp2(m - m_new) : 1.f;
            l *= a;
#pragma unroll
            for (int b = 0; b < kO; ++b)
#pragma unroll
                for (int r = 0; r < kRegs; ++r) o[b][r] *= a;
            m = m_new;
        }
        const float ms = m > -INFINITY ? m : 0.f;
#pragma unroll
        for (int r = 0; r < kKeys; ++r) {
            s[r] = fast_exp2(fmaf(s[r], c, -ms));
            l += s[r];
        }
    }

    // O^T += V^T P^T.  A lane's weights are the operand of P^T as they are: contraction slot t of a lane = its key t.
    // bf16: the weights as three planes, whose sum they are exactly (PLANES), or one value after the other in fp32 products.  With two planes, 16 bits, a sum that
    // nearly cancels was off by 64 times what fp32 rounds, and 1.9e-3 of the outputs of 16 unshared sequences were not the nearest bf16 numbers (4e-4 with three;
    // 1e-3 of fp32 sums by library calls); 1.3 % less time over the 29 calls.
    template <bool PLANES>
    __device__ __forceinline__ void weighted_rows(const char* vb, const float (&s)[kKeys]) {
        const int lane = threadIdx.x & 63, i = lane & (COLS - 1);
        if constexpr (sizeof(T) == 2 && !PLANES) {
#pragma unroll
            for (int r = 0; r < kKeys; ++r) {
                const int k = key(r);
#pragma unroll
                for (int b = 0; b < kO; ++b) {
                    const int ch = COLS * b + i;
                    const float v = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(vb + k * C::RB + swz_chunk(ch >> 3, C::v_swizzle(k)) + (ch & 7) * 2) << 16);
                    if constexpr (COLS == 32) o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[r], o[b], 0, 0, 0);
                    else o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[r], o[b], 0, 0, 0);
                }
            }
        } else if constexpr (sizeof(T) == 2) {
            typedef short shortx4 __attribute__((ext_vector_type(4)));
            using lds_ptr = __attribute__((address_space(3))) shortx4*;
            // Channel l of four keys for every lane l of 16, which give the addresses of four consecutive channels each: lane 4 e + q of key e.
            const int e = (lane >> 2) & 3, q = lane & 3, row = 4 * group() + e;
#pragma unroll
            for (int y = 0; y < kKeys / 8; ++y) {
                uintx4 plane[3];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float a = s[8 * y + 2 * x], b = s[8 * y + 2 * x + 1];
#pragma unroll
                    for (int z = 0; z < 3; ++z) {
                        const uint32_t w = pack_bf16x2(a, b);
                        plane[z][x] = w;
                        a -= __uint_as_float(w << 16);
                        b -= __uint_as_float(w & 0xFFFF0000u);
                    }
                }
                // 16 columns: four blocks side by side, so that a product does not wait for the one before it (20 sequences of 278 rows 17.3 us, one block
                // after the other 17.6).  Those of 32 columns last long enough (61 questions about 19382 rows of 64 channels: 60.7 us side by side, 59.9 so).
                constexpr int kSide = COLS == 16 ? 4 : 1;
#pragma unroll
                for (int b0 = 0; b0 < kO; b0 += kSide) {
                    uintx4 vf[kSide];
#pragma unroll
                    for (int x = 0; x < kSide; ++x) {
                        const int b = b0 + x, chunk = COLS == 32 ? 4 * b + 2 * ((lane >> 4) & 1) + (q >> 1) : 2 * b + (q >> 1);
                        const char* a0 = vb + (row + 16 * y) * C::RB + swz_chunk(chunk, C::v_swizzle(row)) + (q & 1) * 8;
                        const uintx2 f0 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)a0));
                        const uintx2 f1 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(a0 + (COLS == 32 ? 8 : 16) * C::RB)));
                        vf[x] = uintx4{f0[0], f0[1], f1[0], f1[1]};
                    }
#pragma unroll
                    for (int z = 2; z >= 0; --z)
#pragma unroll
                        for (int x = 0; x < kSide; ++x) {
                            if constexpr (COLS == 32) o[b0 + x] = mma_frag<__bf16>(vf[x], plane[z], o[b0 + x]);
                            else o[b0 + x] = mma16(vf[x], plane[z], o[b0 + x]);
                        }
                }
            }
        } else if constexpr (COLS == 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k = key(r);
#pragma unroll
                for (int b = 0; b < kO; ++b) {
                    const float v = *reinterpret_cast<const float*>(vb + k * C::RB + swz_chunk(8 * b + (i >> 2), C::v_swizzle(k)) + (i & 3) * 4);
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[r], o[b], 0, 0, 0);
                }
            }
        } else {
            // a lane reads its kPer channels of a row as they stand; channel kPer i + b is row i of block b
#pragma unroll
            for (int r = 0; r < kKeys; ++r) {
                const int k = key(r);
#pragma unroll
                for (int x = 0; x < kPer / 4; ++x) {
                    const floatx4 v = *reinterpret_cast<const floatx4*>(vb + k * C::RB + swz_chunk(kPer / 4 * i + x, C::v_swizzle(k)));
#pragma unroll
                    for (int y = 0; y < 4; ++y) o[4 * x + y] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[y], s[r], o[4 * x + y], 0, 0, 0);
                }
            }
        }
    }

    // Values of rows that are not there become zeros.
    __device__ static __forceinline__ void clear_absent(char* vb, uint32_t rows) {
        const int lane = here(), lr = lane / (C::RB / 16);
#pragma unroll 1
        for (int q = 0; q < C::NL; ++q)
            if (!(rows >> (q * C::RPL + lr) & 1)) *reinterpret_cast<uintx4*>(vb + q * 1024 + lane * 16) = uintx4{0, 0, 0, 0};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    // The lane's sums to a record of D floats.
    __device__ __forceinline__ void store(float* dst) const {
        const int group = here() / COLS;
        if constexpr (COLS == 16 && sizeof(T) == 4) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int x = 0; x < kPer / 4; ++x) *reinterpret_cast<floatx4*>(dst + channel(4 * x, r, group)) = floatx4{o[4 * x][r], o[4 * x + 1][r], o[4 * x + 2][r], o[4 * x + 3][r]};
        } else {
#pragma unroll
            for (int b = 0; b < kO; ++b)
#pragma unroll
                for (int r = 0; r < kRegs; r += 4) *reinterpret_cast<floatx4*>(dst + channel(b, r, group)) = floatx4{o[b][r], o[b][r + 1], o[b][r + 2], o[b][r + 3]};
        }
    }

    // Tiles first, first + step, ... below `end` of an item with `rows` rows and this row of a table.  K of the next tile is requested when K of this one
    // has been read, V of the next when V of this one has: a wave has one tile of each in LDS and one on the way at any time.
    template <bool AGAIN>
    __device__ __forceinline__ void tiles(const PagedRead& p, const int32_t* table, int rows, int first, int step, int end, float c, char* mine) {
        first = scalar(first);
        step = scalar(step);
        end = scalar(end);
        rows = scalar(rows);
        const int lane = threadIdx.x & 63, n = first < end ? (end - first + step - 1) / step : 0;
        const bool small = p.page_log2 == 4;                 // a tile is two pages
        int from = 0, e0 = -1, e1 = -1;                      // entries of the tiles from .. from + 63, one a lane
        auto entries = [&]() {
            const int t = first + min(from + lane, n - 1) * step;
            e0 = table[t * kTileRows >> p.page_log2];
            if (small) e1 = t * kTileRows + 16 < rows ? table[2 * t + 1] : -1;
            asm volatile("" : "+v"(e0), "+v"(e1));           // here they are waited for, and not, with all requested rows, where a tile looks at them
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
                x.k0 = p.K + at0;
                x.k1 = p.K + at1;
                x.v0 = p.V + at0;
                x.v1 = p.V + at1;
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
            float s[kKeys];
            scores(kb, s);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                       // K has been read
            if (more) fetch<false>(nxt.k0, nxt.k1, nxt.rows, klds);
            weigh(s, cur.rows, c);
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::NL) : "memory");   // all but K of the next
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (AGAIN && cur.rows != 0xFFFFFFFFu) clear_absent(vb, cur.rows);
            weighted_rows<!AGAIN>(vb, s);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) fetch<true>(nxt.v0, nxt.v1, nxt.rows, vlds);
            cur = nxt;
            have = more;
        }
        l = over_groups<COLS>(l, [](float a, float b) { return a + b; });
    }

    // The part of the lane's column.  An infinity in V is no number times a plane of 0, or where it stands for a row that is not there: a wave whose sums are not
    // finite takes its tiles again, without either.  Looking at the sums of each piece: 0.8 % of the time over the 29 calls.
    __device__ __forceinline__ void run(const PagedRead& p, const int32_t* table, int rows, int first, int step, int end, float c, char* mine) {
        tiles<false>(p, table, rows, first, step, end, c, mine);
        float probe[4] = {};                                 // no number if a sum is not finite
#pragma unroll
        for (int b = 0; b < kO; ++b)
#pragma unroll
            for (int r = 0; r < kRegs; ++r) probe[r & 3] = fmaf(o[b][r], 0.f, probe[r & 3]);
        if (__builtin_expect(__any(probe[0] + probe[1] + probe[2] + probe[3] != 0.f), 0)) {
            reset();
            tiles<true>(p, table, rows, first, step, end, c, mine);
        }
    }
};

// a / b for 0 <= a < 2^22, b > 0 (512 * 512 is less): the quotient in fp32 is off by less than one.  The compiler's division
// of whole numbers is some 40 instructions.
__device__ __forceinline__ int quotient(int a, int b) {
    const int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b)), left = a - q * b;
    return q + (left >= b) - (left < 0);
}


// The line of work: the weights of all items follow each other and the workgroups take equal pieces, so that however unequal the lengths, no
// workgroup has more than another; a long item gets many workgroups and several short ones share one.  First come the blocks of
// prefixes, which the waves of a workgroup share; then what waves cut, light prefixes and own rows: a workgroup's piece of those is cut again into equal ones for
// each wave, which then wait for nobody.
struct Line {
    int item;                                                // of the workgroup's first position
    int start;                                               // of that item on the line, which is shorter than 2^31
    int lo, hi;                                              // the workgroup's piece
    int waves;                                               // where the items begin that waves cut
    int least;                                               // weight of a piece that four waves share
    int longer;                                              // tiles that make an item a long one
    int me;                                                  // the workgroup's number on the line
};

struct LineShared {
    int4 sums[kPartWaves];                                   // of prefixes that workgroups cut, that waves cut, of own items
    int item, base;
};
constexpr int kSeen = 4096;          // items whose sizes are left in LDS

// What a thread has of a kind of items: `per` of them from `from`.
struct Share { int from, end; };
__device__ __forceinline__ Share share_of(int n) {
    const int per = (n + 255) / 256, from = min(n, (int)threadIdx.x * per);
    return {from, min(n, from + per)};
}

__device__ __forceinline__ bool find_piece(const PagedRead& p, LineShared& sh, Item* seen, Line& line) {
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, prefixes = p.prefixes();
    const Share pre = share_of(prefixes), own = share_of(p.B * p.Hkv);
    int pre_sum = 0, light_sum = 0, own_sum = 0;
    int length[4];                                           // four are asked for at once, and the first four before those of prefixes are there
    auto ask = [&](int u0) {
#pragma unroll
        for (int x = 0; x < 4; ++x) length[x] = p.len[clamped(u0 + x, 0, p.B * p.Hkv - 1)];
    };
    ask(own.from);
    for (int i = pre.from; i < pre.end; ++i) {
        const Item it = item_of(p, i);
        if (it.light()) light_sum += it.weight(true, p.wide);
        else pre_sum += it.weight(false, p.wide);
        if (i < kSeen) seen[i] = it;
    }
    for (int u0 = own.from; u0 < own.end; u0 += 4) {
        if (u0 != own.from) ask(u0);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (u0 + x >= own.end) break;
            const Item it = own_item(p, u0 + x, length[x]);
            own_sum += it.weight(true, p.wide);
            if (prefixes + u0 + x < kSeen) seen[prefixes + u0 + x] = it;
        }
    }
    const int pre_upto = wave_scan(pre_sum), light_upto = wave_scan(light_sum), own_upto = wave_scan(own_sum);
    if (lane == 63) sh.sums[w] = make_int4(pre_upto, light_upto, own_upto, 0);
    if (tid == 0) sh.item = p.items();
    __syncthreads();
    int pre_base = pre_upto - pre_sum, light_base = light_upto - light_sum, own_base = own_upto - own_sum, pre_all = 0, light_all = 0, own_all = 0;
#pragma unroll
    for (int x = 0; x < kPartWaves; ++x) {
        const int4 v = sh.sums[x];
        if (x < w) { pre_base += v.x; light_base += v.y; own_base += v.z; }
        pre_all += v.x;
        light_all += v.y;
        own_all += v.z;
    }
    const int total = scalar(pre_all + light_all + own_all);
    if (total == 0) return false;
    line.me = blockIdx.x;
    line.waves = scalar(pre_all);
    line.least = line.waves == 0 ? p.least : kLeast;
    const int wgs = max(1, min((int)gridDim.x, total / line.least));     // a piece is longer than a tile of any item: none is without a tile
    if (line.me >= wgs) return false;
    const int each = scalar(total / wgs), more = total - each * wgs;
    line.longer = each >= kLongPiece ? 0 : kLongWorkgroups * each;
    light_base += pre_all;
    own_base += pre_all + light_all;
    line.lo = line.me * each + quotient(line.me * more, wgs);
    line.hi = (line.me + 1) * each + quotient((line.me + 1) * more, wgs);
    line.lo = scalar(line.lo);
    line.hi = scalar(line.hi);
    if (pre_base <= line.lo && line.lo < pre_base + pre_sum) {
        sh.item = pre.from;
        sh.base = pre_base;
    }
    if (light_base <= line.lo && line.lo < light_base + light_sum) {
        sh.item = pre.from;
        sh.base = light_base;
    }
    if (own_base <= line.lo && line.lo < own_base + own_sum) {
        sh.item = prefixes + own.from;
        sh.base = own_base;
    }
    __syncthreads();
    line.item = scalar(sh.item);
    line.start = scalar(sh.base);
    return true;
}

// What a workgroup, or a wave, has of an item.
struct Piece { int item, block, ta, tb; bool own; Item it; };

// The pieces on [pos, hi) of the line one after the other, from `item`, which starts at `start`.
struct Walker {
    const PagedRead& p;
    const Item* in_lds;                                      // NULL: no longer
    int item, window;
    int start, pos, hi;                                      // below 2^31
    bool by_wave;                                            // among the items that waves cut; the others have no weight there
    Item seen;                                               // 64 items from `window`, one a lane
    __device__ __forceinline__ void look() {
        const int i = window + (int)(threadIdx.x & 63);
        if (in_lds && p.items() <= kSeen) seen = i < p.items() ? in_lds[i] : Item{0, 0};
        else seen = item_of(p, i);
    }
    // On to the item that `pos` is in: its weight; 0: there is none (the items end where the line does, unless lengths change meanwhile).
    __device__ __forceinline__ int skip(Item& it) {
        for (; item < p.items(); ++item) {
            if (item >= window + 64) {
                window = item;
                look();
            }
            it.rows = __builtin_amdgcn_readlane(seen.rows, item - window);
            it.who = __builtin_amdgcn_readlane(seen.who, item - window);
            const int weight = (item >= p.prefixes() || it.light()) == by_wave ? it.weight(by_wave, p.wide) : 0;
            if (pos - start < weight) return weight;
            start += weight;
        }
        return 0;
    }
    __device__ __forceinline__ bool next(Piece& x) {
        while (pos < hi) {
            Item& it = x.it;
            const int weight = skip(it);
            if (weight == 0) return false;
            x.item = item;
            x.own = item >= p.prefixes();
            const int tiles = it.tiles(), n = it.blocks();
            const int off = max(0, pos - start);             // a walker that was set back may stand before its item
            const int full = it.weight_of_full_block(p.wide);
            x.block = n > 1 ? min(off / full, n - 1) : 0;
            const int block_start = start + x.block * full, x0 = off - x.block * full, x1 = min((x.block < n - 1 ? full : weight - x.block * full), hi - block_start);
            pos = block_start + x1;
            const int shift = it.tile_log2(x.block, p.wide), last = (1 << shift) - 1;
            x.ta = clamped((x0 + last) >> shift, 0, tiles);  // a tile is whose piece it begins in
            x.tb = min((x1 + last) >> shift, tiles);
            if (x.ta < x.tb) return true;                    // else: nothing but an item's start
        }
        return false;
    }
};

// What the waves of a workgroup have of a block of queries: `phases` waves the same columns and every phases-th tile.
struct Block {
    int unit, g, first, block, cols;                         // first: batch element; of the group, if it is a prefix
    int phases, phase, first_col;
    int who;                                                 // among those that cut such items
    bool by_wave, own, begins, whole;
};

// All waves of the workgroup, or, with one phase, any.
template <typename T, int D, int COLS>
__device__ __forceinline__ void shared_piece(const T* __restrict__ q, const PagedRead& p, float c, const Parts& out, const Piece& x, const Block& k,
                                             char* smem, float2 (&ml)[kPartWaves][kCols])
{
    using C = PartCfg<T, D>;
    const int w = scalar(threadIdx.x >> 6);
    char* const mine = smem + w * C::WAVE;
    const int in_wave = min(COLS, k.cols - k.first_col);     // columns; none where a block has three times 32
    auto row_of = [&](int col) {                             // column of the block -> row of the output
        const int r = k.block * kBlock + col, s = divided(r, p.G, p.inv_G);
        return (k.first + s) * p.Hq + k.g * p.G + r - s * p.G;
    };
    auto record = [&](int col) { return k.whole ? out.whole(row_of(col), k.own) : out.piece(k.by_wave, k.who, k.begins, col); };
    WavePart<T, D, COLS> part;
    part.load_queries(q + (int64_t)row_of(k.first_col + max(0, min(part.col(), in_wave - 1))) * D, part.col() < in_wave);
    const int32_t* table = k.own ? p.table + (int64_t)k.unit * p.width : p.prefix_table + (int64_t)k.unit * p.prefix_width;
    part.reset();
    if (in_wave > 0) part.run(p, table, x.it.rows, x.ta + k.phase, k.phases, x.tb, c, mine);
    if (k.phases == 1) {
        const int i = part.here() & (COLS - 1);
        if (i < in_wave) {
            const int64_t rec = record(k.first_col + i);
            part.store(out.o + rec * D);
            if (part.group() == 0) *reinterpret_cast<float2*>(out.ml + 2 * rec) = make_float2(part.m, part.l);
        }
        return;
    }
    // The parts of waves with the same columns meet in LDS: [channel][column], columns turned by the channel so that neither way through meets conflicts.
    const int lane = part.here(), i = lane & (COLS - 1), group = lane / COLS;
    if (group == 0) ml[w][i] = make_float2(part.m, part.l);
    __syncthreads();
    float M = -INFINITY, L = 0.f;
    const int w0 = w - k.phase;
    for (int y = 0; y < k.phases; ++y) M = fmaxf(M, ml[w0 + y][i].x);
    for (int y = 0; y < k.phases; ++y) L += M > -INFINITY ? fast_exp2(ml[w0 + y][i].x - M) * ml[w0 + y][i].y : 0.f;
    const float a = M > -INFINITY ? fast_exp2(part.m - M) : 0.f;
    if (k.phase == 0 && group == 0 && i < in_wave) *reinterpret_cast<float2*>(out.ml + 2 * (int64_t)record(k.first_col + i)) = make_float2(M, L);
    float* mo = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int b = 0; b < part.kO; ++b)
#pragma unroll
        for (int r = 0; r < part.kRegs; ++r) {
            const int ch = part.channel(b, r, group);
            mo[ch * kCols + (i ^ (ch & 31))] = part.o[b][r] * a;
        }
    __syncthreads();
    const int tid = w * 64 + lane, ch = tid % (D / 4) * 4, rec0 = k.whole ? 0 : out.piece(k.by_wave, k.who, k.begins, 0);
#pragma unroll 4
    for (int cc = tid / (D / 4); cc < k.cols; cc += 64 * kPartWaves / (D / 4)) {
        const float* base = reinterpret_cast<const float*>(smem + cc / kCols * k.phases * C::WAVE);
        floatx4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = base[(ch + e) * kCols + ((cc % kCols) ^ ((ch + e) & 31))];
        for (int z = 1; z < k.phases; ++z)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += base[z * (C::WAVE / 4) + (ch + e) * kCols + ((cc % kCols) ^ ((ch + e) & 31))];
        *reinterpret_cast<floatx4*>(out.o + (int64_t)(k.whole ? out.whole(row_of(cc), k.own) : rec0 + cc) * D + ch) = v;
    }
    __syncthreads();
}

// OWN: columns for the queries of a group of heads.  With 16, blocks of up to 16 queries of a prefix have 16 too.
template <typename T, int D, int OWN>
__global__ __launch_bounds__(64 * kPartWaves, (PartCfg<T, D>::PER_CU)) void paged_part_kernel(const T* __restrict__ q, PagedRead p, float c, Parts out) {
    using C = PartCfg<T, D>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ LineShared sh;
    __shared__ float2 ml[kPartWaves][kCols];
    const int tid = threadIdx.x, w = scalar(tid >> 6);
    Line line;
    static_assert(kSeen * sizeof(Item) <= C::LDS, "the items' sizes stand where tiles come later");
    if (!find_piece(p, sh, reinterpret_cast<Item*>(smem), line)) return;
    // Of all waves: blocks of prefixes, then, if one long item that waves cut is all of the workgroup's piece, that.  Else each wave has a quarter of what
    // is left; of less than `least` (the first workgroup with such items) the last wave has all: the pieces of an item are those of waves that follow
    // each other.  One loop for all three: a launch comes to cold code, and what it does not need costs as much as what it needs.
    enum { kBlocks, kOneItem, kWaves } stage = kBlocks;
    const int prefixes = p.prefixes(), from = max(line.lo, line.waves), all = line.hi - from;
    Walker walk = {p, reinterpret_cast<const Item*>(smem), line.item, line.item, line.start, line.lo, line.hi, line.lo >= line.waves, {0, 0}};
    auto quarters = [&]() {
        const int quarter = all / kPartWaves, rest = all % kPartWaves;
        walk.by_wave = true;
        walk.pos = all < line.least ? from : from + w * quarter + min(w, rest);
        walk.hi = all < line.least ? (w == kPartWaves - 1 ? line.hi : from) : walk.pos + quarter + (w < rest);
        stage = kWaves;
    };
    walk.look();
    if (walk.by_wave) {
        Item it;
        const int weight = walk.skip(it);
        if (it.tiles() > line.longer && walk.start + weight >= line.hi) stage = kOneItem;
        else quarters();
    } else walk.hi = min(line.hi, line.waves);
    walk.in_lds = nullptr;
    __syncthreads();                                         // tiles may come

    Piece x;
    for (;;) {
        if (!walk.next(x)) {
            if (stage != kBlocks || all <= 0) return;
            quarters();
            walk.item = walk.window = 0;                     // it stands behind the items that workgroups cut: back to the first item
            walk.start = line.waves;
            walk.look();
            continue;
        }
        const bool ends = x.tb == x.it.tiles();
        Block k;
        k.own = x.own;
        k.begins = x.ta == 0;
        k.whole = k.begins && ends;
        k.unit = x.own ? x.item - prefixes : x.item;
        const int group = x.own ? 0 : divided(k.unit, p.Hkv, p.inv_Hkv);
        k.g = x.own ? k.unit - x.it.begin() * p.Hkv : k.unit - group * p.Hkv;
        k.first = x.it.begin();
        k.block = x.block;
        k.cols = min(kBlock, x.it.cols() - x.block * kBlock);
        const int waves = x.it.waves_log2(x.block);          // 0 of what waves cut
        k.phases = stage == kWaves ? 1 : kPartWaves >> waves;
        k.phase = w & (k.phases - 1);
        k.first_col = (w >> (2 - waves)) * kCols;
        k.by_wave = stage != kBlocks;
        k.who = k.by_wave ? line.me * kPartWaves + (stage == kWaves ? w : 0) : line.me;
        if ((stage == kWaves ? tid & 63 : tid) == 0) {
            int2* const piece = out.pieces + (x.own ? piece_own(p, k.unit) : piece_prefix(p, group, k.first, x.block, k.g));
            const int number = k.who | (k.by_wave ? kByWave | (x.it.tiles() > line.longer ? kLong : 0) : 0) | (stage == kOneItem ? kEntire : 0);
            if (k.begins) piece->x = number;
            if (ends) piece->y = number;
        }
        if (OWN == 16 && k.cols <= 16) shared_piece<T, D, 16>(q, p, c, out, x, k, smem, ml);
        else shared_piece<T, D, 32>(q, p, c, out, x, k, smem, ml);
    }
}

// Whose an item's parts are: x .. y, workgroups or waves, within the workspace whatever stands in `pieces` (nothing, where groups overlap and weigh more than the
// line holds).  Of a long item: waves from x of the first workgroup (or all four at once), one part of each
// workgroup between, which has nothing else, and waves up to y of the last (or all four at once).
struct Span {
    int head, mid, tail;                                     // parts
    int x, between, last;                                    // part i is of x + i, between + 4 i or last + i
    int base, cols;                                          // of records
    __device__ __forceinline__ int count() const { return head + mid + tail; }
    __device__ __forceinline__ int record(int i) const {
        const int who = i < head ? x + i : i < head + mid ? between + kPartWaves * i : last + i;
        return base + (2 * who + (i == 0)) * cols;
    }
};
__device__ __forceinline__ Span span_of(const Parts& in, int2 v, int row, int own, int col) {
    static_assert(kPartWaves == 4, "");
    const bool by_wave = v.x & kByWave;
    const int cols = by_wave ? in.wave_cols : in.cols;
    const int x = min(v.x & kNumber, in.grid * kPartWaves - 1), y = v.y < 0 ? -1 : min(v.y & kNumber, in.grid * (by_wave ? kPartWaves : 1) - 1);
    Span s = {max(0, y - x + 1), 0, 0, x, 0, 0, in.piece(by_wave, 0, 0, min(col, cols - 1)), cols};
    if (v.x & kLong && x >> 2 < y >> 2) {
        s.head = v.x & kEntire ? 1 : 4 - (x & 3);
        s.mid = (y >> 2) - (x >> 2) - 1;
        s.tail = v.y & kEntire ? 1 : (y & 3) + 1;
        s.between = (x | 3) + 1 - 4 * s.head;
        s.last = (y & ~3) - s.head - s.mid;
    }
    if (x == y) {
        s.base = in.whole(row, own);
        s.cols = 0;
    }
    return s;
}

// The parts of one query head: those of its group's prefix, then its own.  Found by a chain of loads, each for the address of the next: groups, pieces (with the lengths).
struct RowParts {
    Span pre, own;
    __device__ __forceinline__ RowParts(const PagedRead& p, const Parts& in, int row) {
        const int lane = threadIdx.x & 63;
        const int b = divided(row, p.Hq, p.inv_Hq), head = row - b * p.Hq, g = divided(head, p.G, p.inv_G), u = b * p.Hkv + g;
        const int2 own_pieces = in.pieces[piece_own(p, u)];
        const int own_len = own_rows(p, u);
        int2 of_pre = {0, -1}, of_own = {0, -1};
        int col = 0;
        for (int x = 0; x < p.groups; x += 64) {
            const Group m = x + lane < p.groups ? group_of(p, x + lane) : Group{0, 0};
            const uint64_t in_it = __ballot(m.begin <= b && b < m.end);
            if (in_it) {
                const int who = __builtin_ctzll(in_it), group = x + who, begin = __builtin_amdgcn_readlane(m.begin, who);
                col = (b - begin) * p.G + head - g * p.G;
                const int2 pieces = in.pieces[piece_prefix(p, group, begin, col / kBlock, g)];
                if (prefix_rows(p, group * p.Hkv + g) > 0) of_pre = pieces;
                col %= kBlock;
                break;
            }
        }
        if (own_len > 0) of_own = own_pieces;
        pre = span_of(in, of_pre, row, 0, col);
        own = span_of(in, of_own, row, 1, head - g * p.G);
    }
    __device__ __forceinline__ int count() const { return pre.count() + own.count(); }
    __device__ __forceinline__ int record(int i) const {
        const int n = pre.count();
        return i < n ? pre.record(i) : own.record(i - n);
    }
};

// They are joined by a wave, or by all four of a workgroup (then with a barrier) -> the output row.
template <typename T, int D, int WAVES>
__device__ __forceinline__ void join_row(const RowParts& parts, const Parts& in, int row, floatx4 (&sum)[256], T* __restrict__ o) {
    constexpr int kPer = D / 4, kAt = 64 * WAVES / kPer, kAtOnce = WAVES == 1 ? 4 : 64 / kAt;        // threads per part, parts at a time, loads on the way
    const int lane = threadIdx.x & 63, tid = WAVES == 1 ? lane : threadIdx.x;                        // among the row's threads
    const int n = parts.count();
    float M = -INFINITY, L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += 64) {                     // 64 parts at a time, every wave all of their maxima and sums
        const int count = min(64, n - s0);
        float2 v = make_float2(-INFINITY, 0.f);
        const int rec = parts.record(s0 + min(lane, count - 1));
        if (lane < count) v = *reinterpret_cast<const float2*>(in.ml + 2 * (int64_t)rec);
        floatx4 part[kAtOnce];
        auto ask = [&](int y0) {
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y)
                if ((y0 + y) * kAt < count) part[y] = *reinterpret_cast<const floatx4*>(in.o + (int64_t)__shfl(rec, (y0 + y) * kAt + tid / kPer) * D + tid % kPer * 4);
        };
        ask(0);
        const float M_new = fmaxf(M, wave_max(v.x));
        const float a = M_new > -INFINITY ? fast_exp2(v.x - M_new) : 0.f, before = M_new > -INFINITY ? fast_exp2(M - M_new) : 0.f;
        L = L * before + wave_sum(a * v.y);
        acc *= before;
        M = M_new;
        for (int y0 = 0; y0 * kAt < count; y0 += kAtOnce) {
            if (y0) ask(y0);
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y)
                if ((y0 + y) * kAt < count) {                // all lanes: a lane that is not there answers no other
                    const float weight = __shfl(a, (y0 + y) * kAt + tid / kPer);
                    if ((y0 + y) * kAt + tid / kPer < count) acc += weight * part[y];
                }
        }
    }
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int off = kPer; off < 64; off <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], off);
    } else {
        sum[tid] = acc;
        __syncthreads();
        if (tid < kPer)
            for (int x = 1; x < min(kAt, n); ++x) acc += sum[x * kPer + tid];
    }
    if (tid < kPer) {
        acc *= L > 0.f ? 1.f / L : 0.f;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uintx2*>(o + (int64_t)row * D + tid * 4) = uintx2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
        else *reinterpret_cast<floatx4*>(o + (int64_t)row * D + tid * 4) = acc;
    }
}

// Four waves a row, or, where rows are many, one: most rows have a few parts then and dispatching a workgroup for each is what lasts (from kManyRows on; 2000 sequences
// of 40 rows, 8 heads on 1 35.4 us with four, 22.9 with one; 64 questions about 160 rows, 32 heads on 8 18.2, 16.1; always one: 8 questions about a video
// 23.6 instead of 20.4).  Rows of more parts than a wave sees at once are joined by the whole workgroup then as well, and the rows of a workgroup are far
// apart, since the heads of one long item follow each other (one sequence of 60000 rows among 63 of 200, 32 heads on 1: 41.3 us by one wave, 28.7 so, 28.6 with four for
// all rows; from 32 parts on: two prefixes of 9000 rows, 64 channels 32.6 us instead of 28.0).
constexpr int kFew = 64, kManyRows = 1536;
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(256, 4) void paged_join_kernel(PagedRead p, Parts in, T* __restrict__ o) {
    __shared__ floatx4 sum[256];
    if constexpr (WAVES == 4) {
        const int row = blockIdx.x;
        join_row<T, D, 4>(RowParts(p, in, row), in, row, sum, o);
    } else {
        __shared__ int many[4];
        const int w = scalar(threadIdx.x >> 6), row = w * (int)gridDim.x + (int)blockIdx.x;
        bool mine = false;
        if (row < in.rows) {
            const RowParts parts(p, in, row);
            mine = parts.count() > kFew;
            if (!mine) join_row<T, D, 1>(parts, in, row, sum, o);
        }
        if ((threadIdx.x & 63) == 0) many[w] = mine;
        __syncthreads();
        for (int x = 0; x < 4; ++x)
            if (many[x]) {
                const int row = x * (int)gridDim.x + (int)blockIdx.x;
                join_row<T, D, 4>(RowParts(p, in, row), in, row, sum, o);
                __syncthreads();
            }
    }
}

struct PagedLayout { size_t o, ml, pieces, total; int cols, wave_cols; };
static PagedLayout paged_layout(const zipvl_dims& d, bool prefixes, int grid) {
    const int G = d.Hq / d.Hkv;
    PagedLayout l;
    l.cols = prefixes ? std::min(kBlock, (d.B * G + kCols - 1) / kCols * kCols) : kCols;     // that a workgroup may have
    l.wave_cols = prefixes ? std::max(G, kLight) : G;
    const size_t records = 2 * (size_t)d.B * d.Hq + 2 * (size_t)grid * (l.cols + kPartWaves * l.wave_cols);
    l.o = 0;
    l.ml = l.o + records * d.d * sizeof(float);
    l.pieces = l.ml + records * 2 * sizeof(float);
    const size_t blocks = prefixes ? (size_t)d.B * G / kBlock + d.B + 1 : 0;         // at most B groups
    l.total = l.pieces + ((size_t)d.B + blocks) * d.Hkv * sizeof(int2);
    return l;
}

// What all lengths at their greatest would weigh, and more.
static int64_t most_weight(const zipvl_dims& d, int64_t own, int64_t prefix, int groups) {
    auto tiles = [](int64_t rows) { return (rows + kTileRows - 1) / kTileRows; };
    const int64_t pre = groups ? ((int64_t)d.B * (d.Hq / d.Hkv) / kBlock + groups) * d.Hkv * (8 * tiles(prefix) + kStartPrefix) : 0;
    return (int64_t)d.B * d.Hkv * (2 * tiles(own) + kStartWave) + pre;
}
// No more workgroups than can have a piece (find_piece).
static int grid_of(int most, int64_t weight) { return (int)std::max<int64_t>(1, std::min<int64_t>(most, weight / (kLeast / 2))); }

size_t decode_paged_workspace_bytes(const zipvl_dims& d, int own, int prefix) {
    const int most = d.dtype == ZIPVL_BF16 ? (d.d == 128 ? PartCfg<__bf16, 128>::GRID : PartCfg<__bf16, 64>::GRID) : d.d == 128 ? PartCfg<float, 128>::GRID : PartCfg<float, 64>::GRID;
    return paged_layout(d, prefix > 0, grid_of(most, most_weight(d, own, prefix, prefix > 0 ? d.B : 0))).total;
}

template <typename T, int D, int OWN>
static int launch_paged_t(const T* q, const PagedRead& p, const zipvl_dims& d, float scale, T* o, char* ws, hipStream_t st) {
    using C = PartCfg<T, D>;
    const int64_t weight = most_weight(d, (int64_t)p.width << p.page_log2, (int64_t)p.prefix_width << p.page_log2, p.groups);
    if (weight >= (int64_t)1 << 31)                          // positions on the line are below that
        return set_error(ZIPVL_ESHAPE, "zipvl_decode_attn_paged: tables of %d units and %d prefixes of %d and %d pages hold too many rows (2^35)", d.B * d.Hkv, p.groups * d.Hkv, p.width, p.prefix_width);
    const int wgs = grid_of(C::GRID, weight);
    const PagedLayout l = paged_layout(d, p.groups > 0, wgs);
    const Parts parts = {(float*)(ws + l.o), (float*)(ws + l.ml), (int2*)(ws + l.pieces), d.B * d.Hq, l.cols, l.wave_cols, wgs};
    static std::atomic<uint64_t> lds_set{0};                 // more than 64 KB of LDS has to be asked for, on every device
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return set_error(ZIPVL_EHIP, "decode_attn_paged: no current device");
    if (dev > 63 || !(lds_set.load(std::memory_order_relaxed) >> dev & 1)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_part_kernel<T, D, OWN>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS) != hipSuccess)
            return set_error(ZIPVL_EHIP, "decode_attn_paged: %d bytes of LDS are refused", (int)C::LDS);
        if (dev <= 63) lds_set.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    {
        KernelTimer tm(ZIPVL_K_PAGED_PARTIAL, st);
        hipLaunchKernelGGL((paged_part_kernel<T, D, OWN>), dim3(wgs), dim3(64 * kPartWaves), C::LDS, st, q, p, scale * kLog2e, parts);
        const int rc = check_launch("decode_attn_paged");
        if (rc) return rc;
    }
    KernelTimer tm(ZIPVL_K_PAGED_COMBINE, st);
    if (parts.rows >= kManyRows) hipLaunchKernelGGL((paged_join_kernel<T, D, 1>), dim3((parts.rows + 3) / 4), dim3(256), 0, st, p, parts, o);
    else hipLaunchKernelGGL((paged_join_kernel<T, D, 4>), dim3(parts.rows), dim3(256), 0, st, p, parts, o);
    return check_launch("decode_attn_paged parts");
}

int launch_decode_attn_paged(const void* q, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* len,
                             const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_len, const int32_t* group_begin,
                             int32_t groups, const zipvl_dims& d, float scale, void* o, void* ws, hipStream_t st)
{
    const PagedRead p = {(const char*)pages.K, (const char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table, table_pages, len,
                         prefix_table, prefix_pages, prefix_len, group_begin, groups, d.B, d.Hq, d.Hkv, d.Hq / d.Hkv,
                         inverse(d.Hkv), inverse(d.Hq / d.Hkv), inverse(d.Hq), d.dtype == ZIPVL_BF16 ? 0 : 1,
                         d.dtype == ZIPVL_F32 && d.Hq / d.Hkv <= 16 ? kLeast / 2 : kLeast};
#define ZIPVL_PAGED(T, D)                                                                              \
    return p.G <= 16 ? launch_paged_t<T, D, 16>((const T*)q, p, d, scale, (T*)o, (char*)ws, st)       \
                     : launch_paged_t<T, D, 32>((const T*)q, p, d, scale, (T*)o, (char*)ws, st)
    if (d.dtype == ZIPVL_BF16) { if (d.d == 128) ZIPVL_PAGED(__bf16, 128); ZIPVL_PAGED(__bf16, 64); }
    if (d.d == 128) ZIPVL_PAGED(float, 128);
    ZIPVL_PAGED(float, 64);
#undef ZIPVL_PAGED
}

}  // namespace zipvl
