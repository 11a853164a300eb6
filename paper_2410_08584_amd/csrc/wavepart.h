// A wave's queries against rows of a paged cache, 32 at a time: what decode over pages and pieces of few queries are made of.
#pragma once
#include <type_traits>

#include "common.h"
#include "ldsload.h"

namespace zipvl {

constexpr int kTileRows = 32, kCols = 32, kPartWaves = 4, kBlock = kCols * kPartWaves;
constexpr int kCus = 256;
constexpr float kLazy = 8.f;         // how far (log2) a logit may exceed the offset of the exponentials before that moves (0: 0.5 % longer over the 29 calls of paged.hip)

// a wave-uniform number in scalar registers
__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }

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

    struct Tile { const char *k0, *k1, *v0, *v1; uint32_t rows; int first; };      // of its first and second 16 rows; which of the 32 there are

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

    // scores -> weights; the offset m follows the running maximum lazily.  CAUSAL: keys of the tile up to `last`, which is the lane's own.
    template <bool CAUSAL>
    __device__ __forceinline__ void weigh(float (&s)[kKeys], uint32_t rows, float c, int last) {
        if (rows != 0xFFFFFFFFu) {
#pragma unroll
            for (int r = 0; r < kKeys; ++r)
                if (!(rows >> key(r) & 1)) s[r] = -INFINITY;
        }
        if constexpr (CAUSAL)
            if (__any(last < kTileRows - 1)) {
#pragma unroll
                for (int r = 0; r < kKeys; ++r)
                    if (key(r) > last) s[r] = -INFINITY;
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
    // `cache` says where pages are (K, V, num_pages, page_log2).  CAUSAL: the lane's query sees rows up to `last`.  LAST: no tiles come behind these, sum_groups().
    template <bool AGAIN, bool CAUSAL, bool LAST, typename Cache>
    __device__ __forceinline__ void tiles(const Cache& p, const int32_t* table, int rows, int first, int step, int end, float c, char* mine, int last = 0) {
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
                x.first = t * kTileRows;
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
            weigh<CAUSAL>(s, cur.rows, c, last - cur.first);
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::NL) : "memory");   // all but K of the next
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (AGAIN && cur.rows != 0xFFFFFFFFu) clear_absent(vb, cur.rows);
            weighted_rows<!AGAIN>(vb, s);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) fetch<true>(nxt.v0, nxt.v1, nxt.rows, vlds);
            cur = nxt;
            have = more;
        }
        if constexpr (LAST) sum_groups();
    }
    __device__ __forceinline__ void sum_groups() { l = over_groups<COLS>(l, [](float a, float b) { return a + b; }); }       // behind the last tile

    // Whether a sum is not finite, in any lane.
    __device__ __forceinline__ bool spoilt() const {
        float probe[4] = {};                                 // no number if a sum is not finite
#pragma unroll
        for (int b = 0; b < kO; ++b)
#pragma unroll
            for (int r = 0; r < kRegs; ++r) probe[r & 3] = fmaf(o[b][r], 0.f, probe[r & 3]);
        return __builtin_expect(__any(probe[0] + probe[1] + probe[2] + probe[3] != 0.f), 0);
    }

    // The part of the lane's column.  An infinity in V is no number times a plane of 0, or where it stands for a row that is not there: a wave whose sums are not
    // finite takes its tiles again, without either.  Looking at the sums of each piece: 0.8 % of the time over the 29 calls.
    template <typename Cache>
    __device__ __forceinline__ void run(const Cache& p, const int32_t* table, int rows, int first, int step, int end, float c, char* mine) {
        tiles<false, false, true>(p, table, rows, first, step, end, c, mine);
        if (spoilt()) {
            reset();
            tiles<true, false, true>(p, table, rows, first, step, end, c, mine);
        }
    }
};

}  // namespace zipvl
