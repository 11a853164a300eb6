// The attention weight that cached rows get from new queries: weight[u, r] = before[u, r] + sum over heads and tokens of exp(scale q.k - lse).
//
// Keys stay, queries come: a wave has 32 keys in registers, S = K Q^T on matrix tiles gives a lane one query and 16 keys of each 32, whose exponentials it
// adds up over all queries; the 32 lanes, and the waves that share keys, meet once, at the end.  No sum crosses workgroups and no wave waits for another before that, so no order of
// arrival changes a result.  Queries come through LDS, tiles ahead.
// fp32 numbers go as three planes of bf16 (planes.h): six products instead of one that takes sixteen times as long.
// Few queries (a decode step) are bound by the read of K, many by products, the exponentials between them (64 queries over a video's cache, bf16: the matrix units are busy 23 % of 20 us, the exponentials and
// their sums take 5 us of vector instructions) and the rest by a barrier a tile and by workgroups that are not a whole number a CU.
#include <atomic>

#include "launch.h"
#include "planes.h"
#include "wavepart.h"

namespace zipvl {

struct Weigh {
    const char* K;
    int num_pages, page_log2;
    const int32_t* table; int width; const int32_t *len, *cnt;
    const char* Q; int64_t q[3];
    const float* lse; int64_t lse_pitch;
    const float* before; float* weight;
    int Hq, Hkv, G, n;
    uint32_t inv_Hkv, inv_G;
    float scale;
    int units, blocks; uint32_t inv_blocks;                  // blocks: workgroups of a unit; 0: the grid's x, and the units its y
};

// Operands of 16 channels of 32 rows, a row a lane (halves of the wave: 8 channels each).
template <typename T> struct Rows;
template <> struct Rows<__bf16> {
    using Raw = uintx4;
    using Frag = uintx4;
    __device__ static __forceinline__ Frag split(const Raw& x) { return x; }
    __device__ static __forceinline__ floatx16 mma(const Frag& a, const Frag& b, floatx16 acc) { return mma_frag<__bf16>(a, b, acc); }
    __device__ static __forceinline__ float largest(const Raw&, float most) { return most; }
    __device__ static __forceinline__ Raw load(const char* row, int cc, int h) { return load16(row + 32 * cc + 16 * h); }
    template <int RB> __device__ static __forceinline__ Raw from_lds(const char* row, int r, int cc, int h) { return load16(row + swz_chunk(2 * cc + h, k_row_swizzle<RB>(r))); }
};
template <> struct Rows<float> {
    struct Raw { uintx4 a, b; };
    using Frag = Planes;
    __device__ static __forceinline__ Frag split(const Raw& x) { return split8(x.a, x.b); }
    __device__ static __forceinline__ floatx16 mma(const Frag& a, const Frag& b, floatx16 acc) { return mma_planes(a, b, acc); }
    __device__ static __forceinline__ float largest(const Raw& x, float most) {
#pragma unroll
        for (int e = 0; e < 4; ++e) asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(most) : "v"(x.a[e]), "v"(x.b[e]));
        return most;
    }
    __device__ static __forceinline__ Raw load(const char* row, int cc, int h) { return {load16(row + 64 * cc + 32 * h), load16(row + 64 * cc + 32 * h + 16)}; }
    template <int RB> __device__ static __forceinline__ Raw from_lds(const char* row, int r, int cc, int h) {
        const int sw = k_row_swizzle<RB>(r);
        return {load16(row + swz_chunk(4 * cc + 2 * h, sw)), load16(row + swz_chunk(4 * cc + 2 * h + 1, sw))};
    }
};
// 32 keys a wave.  QW = 1: the four waves have keys of their own and share tiles of queries; 4: they have the same keys and take every fourth tile, each from LDS of its own.
// A tile is of queries that follow each other head by head, token by token, or, WIDE, of tokens of one head: its rows are then at one distance and asked for without a
// vector instruction, and n is long enough that a last tile with few tokens is no loss.
template <typename T, int D, int QW, bool WIDE>
struct WeighCfg {
    static constexpr int RB = D * (int)sizeof(T), CH = D / 16, KEYS = 32 * (4 / QW);
    static constexpr int QT = QW == 1 && sizeof(T) == 2 ? 64 : 32, SHARE = 4 / QW;       // queries a tile, waves that share it
    static constexpr int TILE = QT * RB, NL = TILE / 1024 / SHARE, RPL = 1024 / RB;  // loads of 1 KiB a wave, rows a load
    static constexpr int BUF = TILE + 256 * SHARE;                                   // a tile, and each wave's copy of its lse
    // Tiles on the way, beside the one that is read.  A wave that has its tiles to itself takes one into registers and asks for the next into its place, where
    // there are registers for it (511 tokens of three prompts, fp32: 55.3 us, with two buffers 57.3).
    static constexpr int AHEAD = QW > 1 && RB <= 256 ? 0 : QW > 1 ? 1 : 2;
    static constexpr int LDS = (AHEAD + 1) * BUF * QW;
};

// The unit and the block of a workgroup where the queries of all are more than the L2s hold.  Workgroups go to the eight XCDs in turn, and all of a unit's read the same queries: eight
// units at a time have an XCD's L2 each, then, of those that are left, four at a time two XCDs each, two four, one eight.
// bf16, 3091 tokens of 3392 rows: 16 units of 4 heads (50 MB of queries) 157 us and not 383, 8 (25 MB) 95 and not 203.  But unequal units load XCDs unequally, which costs where L2 is no bound:
// 14 units of 7 heads, fp32, 511 tokens (13 MB) 131 us and not 94.
constexpr int64_t kQueriesAlone = 24 << 20;
__device__ __forceinline__ bool place_of(const Weigh& p, int& u, int& block) {
    const int xcd = block & 7, whole = (p.units >> 3) * p.blocks;
    int j = block >> 3;
    if (j < whole) {
        const int at = divided(j, p.blocks, p.inv_blocks);
        u = at * 8 + xcd;
        block = j - at * p.blocks;
        return true;
    }
    j -= whole;
    u = p.units & ~7;
#pragma unroll
    for (int log2 = 2; log2 >= 0; --log2)
        if (p.units >> log2 & 1) {
            const int n = (p.blocks + (8 >> log2) - 1) >> (3 - log2);
            if (j < n) {
                u += xcd & ((1 << log2) - 1);
                block = (j << (3 - log2)) + (xcd >> log2);
                return block < p.blocks;
            }
            j -= n;
            u += 1 << log2;
        }
    return false;
}

template <typename T, int D, int QW, bool WIDE>
__global__ __launch_bounds__(256, 2) void paged_weigh_kernel(Weigh p) {
    using R = Rows<T>;
    using C = WeighCfg<T, D, QW, WIDE>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ float meet[4][32];
    int u = blockIdx.y, block = blockIdx.x;
    if (p.blocks && !place_of(p, u, block)) return;
    const int k0 = block * C::KEYS, room = p.width << p.page_log2;
    const int tid = threadIdx.x, w = scalar(tid >> 6), lane = tid & 63, i = lane & 31, h = lane >> 5;
    const int key0 = k0 + 32 * (w / QW), qw = w % QW;
    // All that a workgroup goes by is asked for at once: the table's entries also of rows behind the length, if it has room for them.
    const int len_there = p.len[u], cnt_there = p.cnt ? p.cnt[u] : p.n;
    const int entry = p.table[(int64_t)u * p.width + (min(key0 + i, room - 1) >> p.page_log2)];
    const int64_t at0 = (int64_t)u * room + key0;
    const float was = p.before && qw == 0 && lane < 32 && key0 + lane < room ? p.before[at0 + lane] : 0.f;        // of row lane of the wave
    const int len = scalar(max(0, min(len_there, room))), cnt = scalar(max(0, min(cnt_there, p.n)));
    if (k0 >= len) return;
    const int b = divided(u, p.Hkv, p.inv_Hkv), g = u - b * p.Hkv, rows = cnt * p.G, first = len - cnt;        // token i stands in row first + i
    // The lane's row of keys.  One that is not there reads row 0 of the pages and gets nothing.
    const int key = key0 + i;
    const bool there = key < len && (unsigned)entry < (unsigned)p.num_pages;
    const char* const key_row = p.K + (there ? ((int64_t)entry << p.page_log2) + (key & ((1 << p.page_log2) - 1)) : 0) * C::RB;
    const char* const queries = p.Q + (b * p.q[0] + (int64_t)g * p.G * p.q[1]) * (int64_t)sizeof(T);
    const char* const lses = reinterpret_cast<const char*>(p.lse + ((int64_t)b * p.Hq + g * p.G) * p.lse_pitch);
    const int64_t token_bytes = p.q[2] * (int64_t)sizeof(T), head_bytes = p.q[1] * (int64_t)sizeof(T), pitch = p.lse_pitch * 4;
    char* const ring = smem + (QW == 1 ? 0 : w * (C::AHEAD + 1) * C::BUF);
    const int part = QW == 1 ? w : 0;                        // of a shared tile
    // Tiles from the first token that sees a key of those that share them, qw tiles on for each wave of the same keys.
    const int skipped = max(0, (QW == 1 ? k0 : key0) - first);
    const int t0 = (WIDE ? skipped / C::QT * p.G : skipped * p.G / C::QT) + qw, t1 = WIDE ? (cnt + C::QT - 1) / C::QT * p.G : (rows + C::QT - 1) / C::QT;
    // !WIDE: row r: token r / G, head r % G.  The rows that a lane asks for, one in each load and one lse, are QT QW rows on with every tile, which is `tokens` tokens and
    // `heads` heads, and where those run over a token more: sums, since products of numbers of 64 bits took as long as the tile's own.
    const int tokens = C::QT * QW / p.G, heads = C::QT * QW - tokens * p.G;
    const int64_t row_step = tokens * token_bytes + heads * head_bytes, row_carry = token_bytes - p.G * head_bytes;
    const int64_t lse_step = tokens * 4 + heads * pitch, lse_carry = 4 - p.G * pitch;
    struct Walk { const char* at; int r, head; };
    Walk row[WIDE ? 1 : C::NL], number;
    auto begin = [&](Walk& x, int r, const char* from, int64_t token_step, int64_t head_step) {
        const int token = divided(r, p.G, p.inv_G);
        x.r = r;
        x.head = r - token * p.G;
        x.at = from + token * token_step + x.head * head_step;
    };
    auto walk = [&](Walk& x, const char* from, int64_t step, int64_t carry) {        // where it stands, in the first row for rows that are not there; and on
        const char* at = x.r < rows ? x.at : from;
        x.r += C::QT * QW;
        x.head += heads;
        x.at += step;
        if (x.head >= p.G) {
            x.head -= p.G;
            x.at += carry;
        }
        return at;
    };
    auto in_tile = [&](int x) { return (x * C::SHARE + part) * C::RPL + lane / (C::RB / 16); };  // the lane's row of load x
    auto chunk = [&](int x) { return swz_chunk(lane % (C::RB / 16), k_row_swizzle<C::RB>(in_tile(x))); };
    auto request = [&](int t, int buf) {
        const unsigned to = lds_address(ring) + buf * C::BUF;
        if constexpr (WIDE) {
            const int block = divided(t, p.G, p.inv_G), head = t - block * p.G, token = block * C::QT, left = cnt - 1 - token;
            const char* from = scalar_ptr(queries + head * head_bytes + token * token_bytes);
            const char* numbers = scalar_ptr(lses + head * pitch + token * 4);
#pragma unroll
            for (int x = 0; x < C::NL; ++x) {
                const int at = left >= C::QT - 1 ? in_tile(x) : min(in_tile(x), left);
                load_kib_to_lds(from, at * (int)token_bytes + chunk(x), to + (x * C::SHARE + part) * 1024);
            }
            load_dwords_to_lds(numbers, 4 * min(C::QT == 64 ? lane : i, left), to + C::TILE + part * 256);
        } else {
#pragma unroll
            for (int x = 0; x < C::NL; ++x) load_kib_to_lds_at(walk(row[x], queries, row_step, row_carry) + chunk(x), to + (x * C::SHARE + part) * 1024);
            load_dwords_to_lds_at(walk(number, lses, lse_step, lse_carry), to + C::TILE + part * 256);
        }
    };
    const float c = p.scale * kLog2e;
    float sum[16];
    // exp(x - lse) = 2^(x log2 e - whole) * 2^(whole - lse log2 e), with a whole number near lse log2 e: the second factor is one a query, and no logit loses bits to lse.
    struct Base { float whole, factor; };
    auto base_of = [&](float lse) {
        const float whole = rintf(lse * kLog2e);
        Base x = {whole, fast_exp2(fmaf(-lse, kLog2e, whole))};
        if (__builtin_isinf(lse)) x = {INFINITY, 0.f};       // a query that sees nothing weighs nothing, whatever its logits are
        return x;
    };
    auto add = [&](const floatx16& s, const Base& base, auto whole, int last) __attribute__((always_inline)) {
        const int upto = last - key0 - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float e = fast_exp2(fmaf(s[r], c, -base.whole));
            if (!decltype(whole)::value && acc_row(r, 0) > upto) e = 0.f;
            sum[r] = fmaf(e, base.factor, sum[r]);
        }
    };
    // the token of query `at` of a tile, cnt or more where there is none
    auto token_of = [&](int t, int at) {
        if constexpr (WIDE) return divided(t, p.G, p.inv_G) * C::QT + at;
        else return t * C::QT + at < rows ? divided(t * C::QT + at, p.G, p.inv_G) : cnt;
    };
    auto last_of = [&](int token) { return token < cnt ? first + token : -1; };      // own row that a token stands in
    auto clear = [&]() {
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[r] = 0.f;
    };
    float most = 0.f;
    clear();
    if (t0 < t1) {
        if constexpr (!WIDE) {
#pragma unroll
            for (int x = 0; x < C::NL; ++x) begin(row[x], t0 * C::QT + in_tile(x), queries, token_bytes, head_bytes);
            begin(number, t0 * C::QT + (C::QT == 64 ? lane : i), lses, 4, pitch);
        }
#pragma unroll
        for (int x = 0; x < max(C::AHEAD, 1); ++x)
            if (t0 + x * QW < t1) request(t0 + x * QW, x);
        typename R::Frag kf[C::CH];
#pragma unroll
        for (int cc = 0; cc < C::CH; ++cc) {
            const typename R::Raw x = R::load(key_row, cc, h);
            if (there) most = R::largest(x, most);
            kf[cc] = R::split(x);
        }
        int buf = 0;
        for (int t = t0; t < t1; t += QW) {
            if (C::AHEAD > 1 && t + QW < t1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::NL + 1) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if constexpr (QW == 1) __syncthreads();          // the tile is there for all waves, and all have read the one before
            else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const char* tile = ring + buf * C::BUF;
            typename R::Raw held[C::AHEAD ? 1 : C::CH];
            float held_lse = 0.f;
            if constexpr (C::AHEAD > 0) {
                if (t + C::AHEAD * QW < t1) request(t + C::AHEAD * QW, buf == 0 ? C::AHEAD : buf - 1);
            } else {
                static_assert(C::AHEAD || C::QT == 32, "");
#pragma unroll
                for (int cc = 0; cc < C::CH; ++cc) held[cc] = R::template from_lds<C::RB>(tile + i * C::RB, i, cc, h);
                held_lse = *reinterpret_cast<const float*>(tile + C::TILE + part * 256 + i * 4);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (t + QW < t1) request(t + QW, 0);
            }
            auto weigh_tile = [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
                for (int x = 0; x < C::QT / 32; ++x) {
                    if (!WIDE && x && t * C::QT + 32 * x >= rows) break;             // of few queries
                    const int r = 32 * x + i;
                    const Base base = base_of(C::AHEAD ? *reinterpret_cast<const float*>(tile + C::TILE + part * 256 + r * 4) : held_lse);
                    floatx16 s = {0};
#pragma unroll
                    for (int cc = 0; cc < C::CH; ++cc) {
                        typename R::Raw raw;
                        if constexpr (C::AHEAD > 0) raw = R::template from_lds<C::RB>(tile + r * C::RB, i, cc, h);
                        else raw = held[cc];
                        most = R::largest(raw, most);
                        const typename R::Frag qf = R::split(raw);
                        s = R::mma(kf[cc], qf, s);
                    }
                    const int last = decltype(whole)::value ? 0 : last_of(token_of(t, r));
                    add(s, base, whole, last);
                    if (C::CH >= 8) __builtin_amdgcn_sched_barrier(0);          // one after the other: side by side they took 60 registers more, and a workgroup of a CU
                }
            };
            // whether every query of the tile sees every key of the wave
            if (first + token_of(t, 0) >= key0 + 31 && token_of(t, C::QT - 1) < cnt) weigh_tile(std::true_type{});
            else weigh_tile(std::false_type{});
            buf = buf == C::AHEAD ? 0 : buf + 1;
        }
    }
    const int at = acc_row(i >> 1, h);                       // the row whose sum the lane ends with
    float mine;
#pragma unroll 1
    for (bool again = false;; again = true) {
        if (again) {
            clear();
            for (int t = t0; t < t1; t += QW)
                for (int x = 0; x < C::QT; x += 32) {
                    const int token = token_of(t, x + i), safe = min(token, cnt - 1);
                    const int head = WIDE ? t - divided(t, p.G, p.inv_G) * p.G : min(t * C::QT + x + i, rows - 1) - safe * p.G;
                    const char* q = queries + head * head_bytes + safe * token_bytes;
                    const Base base = base_of(*reinterpret_cast<const float*>(lses + head * pitch + safe * 4));
                    floatx16 s = {0};
#pragma unroll 1
                    for (int c16 = 16 * h; c16 < C::RB; c16 += 32) s = mma_frag<T>(load16(key_row + c16), load16(q + c16), s);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = base.factor == 0.f ? 0.f : s[r];
                    add(s, base, std::false_type{}, last_of(token));
                }
        }
        // Over the 32 lanes of a half, half as many numbers a step: lane i ends with number i / 2.
#pragma unroll
        for (int off = 16, n = 8; n; off >>= 1, n >>= 1)
#pragma unroll
            for (int r = 0; r < n; ++r) {
                const float low = sum[r], high = sum[r + n];
                sum[r] = (i & off ? high : low) + __shfl_xor(i & off ? low : high, off);
            }
        mine = sum[0] + __shfl_xor(sum[0], 1);
        if (!__shfl((int)there, at)) mine = 0.f;
        // Once more, with operands from memory: numbers that planes do not hold, in fp32 products; and a sum that is not finite, since a query that weighs nothing may have logits that are
        // not, and 0 times their exponentials is no number.
        if (again || !__any(!(most < kPlaneHigh) || mine * 0.f != 0.f)) break;
    }
    if ((i & 1) == 0) meet[w][at] = mine;
    if (QW > 1) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (qw == 0 && lane < 32 && key0 + lane < len) {
        float v = 0.f;
#pragma unroll
        for (int y = 0; y < QW; ++y) v += meet[w + y][lane];
        p.weight[at0 + lane] = was + v;
    }
}

template <typename T, int D, int QW, bool WIDE>
static void launch_weigh_as(Weigh p, int units, hipStream_t st) {
    using C = WeighCfg<T, D, QW, WIDE>;
    static std::atomic<uint64_t> set{0};                     // more than 64 KB of LDS has to be asked for, on every device
    int dev = 0;
    if (C::LDS + 1024 > 64 * 1024 && hipGetDevice(&dev) == hipSuccess && (dev > 63 || !(set.load(std::memory_order_relaxed) >> dev & 1))) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_weigh_kernel<T, D, QW, WIDE>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS) == hipSuccess && dev <= 63)
            set.fetch_or(1ull << dev, std::memory_order_relaxed);        // the launch says so if it was refused
    }
    const int64_t blocks = (((int64_t)p.width << p.page_log2) + C::KEYS - 1) / C::KEYS;
    dim3 grid((unsigned)blocks, units);
    if ((int64_t)units * p.G * p.n * C::RB >= kQueriesAlone && units * blocks < 1 << 23) {       // 2^32 threads
        p.units = units;
        p.blocks = (int)blocks;
        p.inv_blocks = inverse(p.blocks);
        int64_t rounds = units / 8 * blocks;
        for (int log2 = 2; log2 >= 0; --log2)
            if (units >> log2 & 1) rounds += (blocks + (8 >> log2) - 1) >> (3 - log2);
        grid = dim3((unsigned)(8 * rounds));
    }
    hipLaunchKernelGGL((paged_weigh_kernel<T, D, QW, WIDE>), grid, dim3(256), C::LDS, st, p);
}
template <typename T, int D>
static int launch_weigh_t(const Weigh& p, int units, hipStream_t st) {
    const int64_t keys = (int64_t)units * p.width << p.page_log2;
    constexpr int kTile = WeighCfg<T, D, 1, true>::QT;
    const bool wide = p.n >= 64 && p.q[2] * (int64_t)sizeof(T) < 1 << 24;            // offsets of a tile's rows fit 32 bits
    KernelTimer tm(ZIPVL_K_PAGED_WEIGH, st);
    // Four waves on the same keys where waves of 32 keys each would leave the chip idle or unequal work to the last of them.  bf16, d = 128, us, four and one: 53 000 keys, 3091 tokens 157, 241;
    // 37 000, 256 tokens 23, 27; 74 000, 64 tokens 28, 20; 110 000, 512 tokens 92, 71.
    if (wide && keys / 32 < 2048) launch_weigh_as<T, D, 4, true>(p, units, st);
    // Tiles of one head where their last ones are nearly full.  131 000 keys of groups of 7, us, of one head and of all: 64 tokens 24, 27; 100 (of 128 that two tiles have) 34, 30; 160 (of 192) 46, 44.
    else if (wide && (p.n + kTile - 1) / kTile * kTile <= p.n + p.n / 8) launch_weigh_as<T, D, 1, true>(p, units, st);
    else launch_weigh_as<T, D, 1, false>(p, units, st);
    return check_launch("paged_weigh");
}

int launch_paged_weigh(const void* Q, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* len, const int32_t* k,
                       const float* lse, int64_t lse_pitch, const zipvl_dims& d, float scale, const float* before, float* weight, hipStream_t st)
{
    const int G = d.Hq / d.Hkv;
    const Weigh p = {(const char*)pages.K, pages.num_pages, __builtin_ctz(pages.page), table, table_pages, len, k, (const char*)Q,
                     {d.q_strides[0], d.q_strides[1], d.q_strides[2]}, lse, lse_pitch, before, weight, d.Hq, d.Hkv, G, d.n, inverse(d.Hkv), inverse(G), scale, 0, 0, 0};
    if (d.dtype == ZIPVL_BF16) return d.d == 128 ? launch_weigh_t<__bf16, 128>(p, d.B * d.Hkv, st) : launch_weigh_t<__bf16, 64>(p, d.B * d.Hkv, st);
    return d.d == 128 ? launch_weigh_t<float, 128>(p, d.B * d.Hkv, st) : launch_weigh_t<float, 64>(p, d.B * d.Hkv, st);
}

}  // namespace zipvl
