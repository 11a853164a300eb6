// Attention of several new tokens to a paged cache (Eq. (2) / Eq. (5) with a causal end): pieces of prompts, questions about a cached
// image, drafted tokens.
//
// A unit (batch element, KV head) has c G rows of queries, the G heads of its group token by token, so that a key that is met serves all heads of the group.
// They go in tiles of rows against the prefix of the unit's group and then its own rows, up to the row that the tile's last token stands in.
// Two forms:
//   few     up to 32 rows a unit: memory-bound.  Each wave has all of them and tiles of 32 keys of its own (wavepart.h, as decode).
//   many    128 rows a workgroup, 32 a wave; tiles of keys in LDS, double-buffered, are shared by the four waves.
// S^T = K Q^T and O^T += V^T P^T on matrix tiles, so that a lane has one row of queries and its statistics are scalars.
//
// How the keys are cut up is decided on the device, where the lengths are (find_place): every workgroup adds up what all units
// weigh and takes a piece; a tile of rows whose keys are many gets several workgroups, and their parts are joined by a second launch.
#include <algorithm>
#include <atomic>

#include "launch.h"
#include "wavepart.h"

namespace zipvl {

constexpr int kRowsMany = 128;
constexpr int kLeastMany = 4, kLeastFew = 8;                 // tiles of keys (64, or 32 of fp32; 32) that a piece has at least
constexpr int kScanUnits = 2048;                             // more units than this go one workgroup a tile of rows, whatever their lengths

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
};

// Parts of tiles of rows that were cut: `rows` rows of D sums and (offset, sum) each.  pieces: the first record of a unit and into how many its keys were cut.
struct ChunkParts { float* o; float* ml; int2* pieces; };

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
    int b, g, rows, cnt, len, prefix, prefix_rows;           // rows of queries; prefix: row of prefix_table
    __device__ __forceinline__ int tiles(int bn) const { return (len + bn - 1) / bn + (prefix_rows + bn - 1) / bn; }
};
__device__ __forceinline__ ChunkUnit chunk_unit(const Chunk& p, int u, const int32_t* begin) {
    ChunkUnit x;
    x.b = divided(u, p.Hkv, p.inv_Hkv);
    x.g = u - x.b * p.Hkv;
    x.cnt = p.cnt ? between(p.cnt[u], 0, p.n) : p.n;
    x.rows = x.cnt * p.G;
    x.len = between(p.len[u], 0, p.width << p.page_log2);
    x.prefix = x.prefix_rows = 0;
    if (p.groups) {
        const int group = group_with(begin, p.groups, p.B, x.b);
        if (group >= 0) {
            x.prefix = group * p.Hkv + x.g;
            x.prefix_rows = between(p.prefix_len[x.prefix], 0, p.prefix_width << p.page_log2);
        }
    }
    return x;
}

// What a workgroup has: keys `piece` of `pieces` of tile t of `tiles` of unit u's rows; its record, if pieces > 1.
struct Place { int u, t, tiles, piece, pieces, record; };
struct PlaceShared {
    int32_t begin[kScanUnits + 1];
    unsigned long long total;
    int2 sums[4];
    Place place;
};

// BM rows of queries and BN keys a tile.  Workgroups of one unit that have the same keys follow each other on one XCD (workgroups go to the eight in turn).
template <int BM, int BN>
__device__ __forceinline__ bool find_place(const Chunk& p, PlaceShared& sh, const ChunkParts& out, int wgs, int least, int direct, Place& x) {
    const int tid = threadIdx.x, lane = tid & 63, w = scalar(tid >> 6);
    if (direct) {
        const int per = gridDim.x / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3), most = (p.n * p.G + BM - 1) / BM;
        if (id >= p.units * most) return false;
        x = {id / most, most - 1 - id % most, 0, 0, 1, 0};
        return true;
    }
    for (int i = tid; i <= p.groups && p.groups; i += 256) sh.begin[i] = p.group_begin[i];
    if (tid == 0) { sh.total = 0; sh.place.pieces = 0; }
    __syncthreads();
    int T = 0, N = 0;
    unsigned long long mine = 0;
    auto sizes = [&](int u) {
        T = N = 0;
        if (u < p.units) {
            const ChunkUnit v = chunk_unit(p, u, sh.begin);
            T = (v.rows + BM - 1) / BM;
            N = v.tiles(BN);
        }
    };
    for (int u0 = 0; u0 < p.units; u0 += 256) {
        sizes(u0 + tid);
        mine += (unsigned long long)T * N;
    }
    if (mine) atomicAdd(&sh.total, mine);
    __syncthreads();
    // A tile of rows is cut into as many pieces as it has average loads, rounded down: then all pieces fit the chip at once
    const int q = max(least, (int)min((unsigned long long)INT32_MAX, (sh.total + wgs - 1) / wgs));
    // how many workgroups all tiles take, first; then whose unit this one's is
    int used = 0, own = 0;
    for (int round = 0; round < 2; ++round) {
        int at = 0, record = 0;
        for (int u0 = 0; u0 < p.units; u0 += 256) {
            if (p.units > 256) sizes(u0 + tid);
            const int s = max(1, N / q), a = T * s, r = s > 1 ? a : 0;
            const int a_upto = wave_scan(a), r_upto = wave_scan(r);
            __syncthreads();
            if (lane == 63) sh.sums[w] = make_int2(a_upto, r_upto);
            __syncthreads();
            int a0 = at + a_upto - a, r0 = record + r_upto - r;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int2 v = sh.sums[y];
                if (y < w) { a0 += v.x; r0 += v.y; }
                at += v.x;
                record += v.y;
            }
            if (round && a0 <= own && own < a0 + a) {
                const int rest = own - a0;
                sh.place = {u0 + tid, T - 1 - rest % T, T, rest / T, s, r0};
                if (rest == 0) out.pieces[u0 + tid] = make_int2(r0, s);
            }
        }
        if (round) break;
        used = scalar(at);
        const int per = (used + 7) / 8;
        own = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
        if ((int)(blockIdx.x >> 3) >= per || own >= used) return false;
    }
    __syncthreads();
    x = sh.place;
    x.u = scalar(x.u); x.t = scalar(x.t); x.tiles = scalar(x.tiles); x.piece = scalar(x.piece); x.pieces = scalar(x.pieces); x.record = scalar(x.record);
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
__global__ __launch_bounds__(256, (PartCfg<T, D>::PER_CU)) void chunk_few_kernel(Chunk p, ChunkParts out, int wgs, int direct) {
    using C = PartCfg<T, D>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ PlaceShared sh;
    __shared__ float2 ml[kPartWaves][kCols];
    Place x;
    if (!find_place<COLS, kTileRows>(p, sh, out, wgs, kLeastFew, direct, x)) return;
    const ChunkUnit v = chunk_unit(p, x.u, p.group_begin);
    if (v.rows == 0) return;
    const int w = scalar(threadIdx.x >> 6);
    char* const mine = smem + w * C::WAVE;
    const int tp = (v.prefix_rows + kTileRows - 1) / kTileRows, all = v.tiles(kTileRows);
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
        if (x.pieces == 1) {
            const RowAt to = row_at(p, v.g, r);
            s *= L > 0.f ? 1.f / L : 0.f;
            store4(out_row<T>(p, v.b, to) + ch, s);
            if (p.lse && ch == 0) *lse_at(p, v.b, to) = log_sum(top, L);
        } else {
            const int64_t rec = (int64_t)(x.record + x.piece) * COLS + r;
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
    static constexpr int LDS = 4 * TILE;                     // two tiles of K, two of V
    __device__ static __forceinline__ int k_swizzle(int r) { return k_row_swizzle<RB>(r); }
    __device__ static __forceinline__ int v_swizzle(int r) { return PartCfg<T, D>::v_swizzle(r); }
};

// Where a tile of keys stands: rows of a table from `first`, those that there are as bits, and 64 of the table's entries, one a lane.
struct KeyTile { int first; bool own; uint64_t rows; };
struct KeyWindow {
    int entry, from;                                         // of the table's pages from ... from + 63
    bool own;
};

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void chunk_many_kernel(Chunk p, ChunkParts out, int wgs, int direct) {
    using C = ChunkCfg<T, D>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    static_assert(sizeof(PlaceShared) <= C::LDS, "the lengths' sums stand where tiles come later");
    Place x;
    if (!find_place<kRowsMany, C::BN>(p, *reinterpret_cast<PlaceShared*>(smem), out, wgs, kLeastMany, direct, x)) return;
    const ChunkUnit v = chunk_unit(p, x.u, p.group_begin);
    const int r0 = x.t * kRowsMany;
    if (r0 >= v.rows) return;
    const int tid = threadIdx.x, w = scalar(tid >> 6), lane = tid & 63, i = lane & 31, h = lane >> 5;
    const int r = r0 + 32 * w + i, r_last = min(r0 + kRowsMany, v.rows) - 1;
    const RowAt at = row_at(p, v.g, min(r, r_last));
    const int before = v.len - v.cnt, last = before + at.token;                  // own row that the lane's token stands in
    const int seen = scalar(between(before + row_at(p, v.g, r_last).token + 1, 0, v.len));         // own rows that a token of the tile sees
    const int wave_first = scalar(before + row_at(p, v.g, min(r0 + 32 * w, r_last)).token);        // up to this row no lane's mask begins
    const int tp = scalar((v.prefix_rows + C::BN - 1) / C::BN), all = tp + scalar((seen + C::BN - 1) / C::BN);
    const int j0 = (int)((int64_t)all * x.piece / x.pieces), j1 = (int)((int64_t)all * (x.piece + 1) / x.pieces);
    const int32_t *own_table = p.table + (int64_t)x.u * p.width, *pre_table = p.prefix_table + (int64_t)v.prefix * p.prefix_width;
    const int prefix_rows = scalar(v.prefix_rows);

    uintx4 qf[C::CH];
    {
        const T* row = query_row<T>(p, v.b, at);
#pragma unroll
        for (int cc = 0; cc < C::CH; ++cc) qf[cc] = load16(row + (2 * cc + h) * Elem<T>::kPerFrag);
    }
    floatx16 o[C::ODB];
#pragma unroll
    for (int db = 0; db < C::ODB; ++db) o[db] = floatx16{0};
    float m = -INFINITY, l = 0.f, l_rounded = 0.f;

    KeyWindow win = {-1, 0, false};
    bool empty = true;
    const int page_mask = (1 << p.page_log2) - 1;
    auto locate = [&](int j) {
        KeyTile k;
        k.own = j >= tp;
        k.first = (k.own ? j - tp : j) * C::BN;
        const int left = (k.own ? seen : prefix_rows) - k.first;
        k.rows = left >= 64 ? ~0ull : (1ull << left) - 1;
        if (C::BN == 32) k.rows &= 0xFFFFFFFFull;
        const int a = k.first >> p.page_log2, b = (k.first + min(left, C::BN) - 1) >> p.page_log2;
        if (empty || win.own != k.own || b >= win.from + 64) {
            const int width = k.own ? p.width : p.prefix_width;
            win = {(k.own ? own_table : pre_table)[min(a + lane, width - 1)], a, k.own};
            empty = false;
            asm volatile("" : "+v"(win.entry));              // waited for here
        }
        for (int e = a; e <= b; ++e)
            if ((unsigned)__builtin_amdgcn_readlane(win.entry, e - win.from) >= (unsigned)p.num_pages) {
                const int f0 = max((e << p.page_log2) - k.first, 0), f1 = min(((e + 1) << p.page_log2) - k.first, C::BN);
                k.rows &= ~((f1 >= 64 ? ~0ull : (1ull << f1) - 1) & ~((1ull << f0) - 1));
            }
        return k;
    };
    constexpr uint64_t kWhole = C::BN == 64 ? ~0ull : 0xFFFFFFFFull;
    // a tile of K (V) to LDS; rows that are not there take one that is: they are masked, and their values weigh nothing
    auto request = [&](const KeyTile& k, auto v_tag, unsigned lds, char* at_lds) {
        constexpr bool V = decltype(v_tag)::value;
        const char* pool = V ? p.V : p.K;
        const int lr = lane / (C::RB / 16), ck = lane % (C::RB / 16);
        if (k.rows == kWhole) {
#pragma unroll
            for (int q = 0; q < C::NL; ++q) {
                const int row = (q * 4 + w) * C::RPL, key = k.first + row;
                const int64_t e = __builtin_amdgcn_readlane(win.entry, (key >> p.page_log2) - win.from);
                const char* base = scalar_ptr(pool + ((e << p.page_log2) + (key & page_mask)) * C::RB);
                load_kib_to_lds(base, lr * C::RB + ((ck ^ (V ? C::v_swizzle(row + lr) : C::k_swizzle(row + lr))) << 4), lds + (q * 4 + w) * 1024);
            }
        } else if (k.rows == 0) {
            for (int q = 0; q < C::NL; ++q) *reinterpret_cast<uintx4*>(at_lds + (q * 4 + w) * 1024 + lane * 16) = uintx4{0, 0, 0, 0};
        } else {
            const int safe = __builtin_ctzll(k.rows);
#pragma unroll 1
            for (int q = 0; q < C::NL; ++q) {
                const int row = (q * 4 + w) * C::RPL + lr, there = k.rows >> row & 1 ? row : safe, key = k.first + there;
                const int64_t e = __shfl(win.entry, (key >> p.page_log2) - win.from);
                load_kib_to_lds_at(pool + ((e << p.page_log2) + (key & page_mask)) * C::RB + ((ck ^ (V ? C::v_swizzle(row) : C::k_swizzle(row))) << 4),
                                   lds + (q * 4 + w) * 1024);
            }
        }
    };
    char *const kbuf = smem, *const vbuf = smem + 2 * C::TILE;
    auto request_both = [&](const KeyTile& k, int buf) {
        request(k, std::false_type{}, lds_address(kbuf) + buf * C::TILE, kbuf + buf * C::TILE);
        request(k, std::true_type{}, lds_address(vbuf) + buf * C::TILE, vbuf + buf * C::TILE);
    };

    KeyTile cur = {}, nxt = {};
    if (j0 < j1) {
        cur = locate(j0);
        request_both(cur, 0);
    }
    for (int j = j0, buf = 0; j < j1; ++j, buf ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();                                     // the tile is there for all waves, and all have read the one before
        if (j + 1 < j1) {
            nxt = locate(j + 1);
            request_both(nxt, buf ^ 1);
        }
        const char *kb = kbuf + buf * C::TILE, *vb = vbuf + buf * C::TILE;
        floatx16 s[C::NBK];
#pragma unroll
        for (int blk = 0; blk < C::NBK; ++blk) {
            s[blk] = floatx16{0};
#pragma unroll
            for (int cc = 0; cc < C::CH; ++cc) {
                const uintx4 kf = *reinterpret_cast<const uintx4*>(kb + (32 * blk + i) * C::RB + swz_chunk(2 * cc + h, C::k_swizzle(32 * blk + i)));
                s[blk] = mma_frag<T>(kf, qf[cc], s[blk]);
            }
        }
        if (cur.rows != kWhole) {
#pragma unroll
            for (int blk = 0; blk < C::NBK; ++blk)
#pragma unroll
                for (int y = 0; y < 16; ++y)
                    if (!(cur.rows >> (32 * blk + acc_row(y, h)) & 1)) s[blk][y] = -INFINITY;
        }
        if (cur.own && cur.first + C::BN - 1 > wave_first) {
#pragma unroll
            for (int blk = 0; blk < C::NBK; ++blk)
#pragma unroll
                for (int y = 0; y < 16; ++y)
                    if (cur.first + 32 * blk + acc_row(y, h) > last) s[blk][y] = -INFINITY;
        }
        // the offset of the exponentials follows the running maximum lazily
        float mx = s[0][0];
#pragma unroll
        for (int blk = 0; blk < C::NBK; ++blk)
#pragma unroll
            for (int y = 0; y < 16; ++y) mx = fmaxf(mx, s[blk][y]);
        mx *= p.c;
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
                s[blk][y] = fast_exp2(fmaf(s[blk][y], p.c, -ms));
                l += s[blk][y];
            }
            if constexpr (sizeof(T) == 2) {
                typedef short shortx4 __attribute__((ext_vector_type(4)));
                using lds_ptr = __attribute__((address_space(3))) shortx4*;
                const int e = (lane >> 2) & 3, q = lane & 3, row = 4 * h + e;
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) {
                    uintx4 pf;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        pf[y] = pack_bf16x2(s[blk][8 * s2 + 2 * y], s[blk][8 * s2 + 2 * y + 1]);
                        l_rounded = add_bf16x2(pf[y], l_rounded);
                    }
#pragma unroll
                    for (int db = 0; db < C::ODB; ++db) {
                        const char* a0 = vb + (32 * blk + 16 * s2 + row) * C::RB + swz_chunk(4 * db + 2 * ((lane >> 4) & 1) + (q >> 1), C::v_swizzle(row)) + (q & 1) * 8;
                        const uintx2 f0 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)a0));
                        const uintx2 f1 = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(a0 + 8 * C::RB)));
                        o[db] = mma_frag<__bf16>(uintx4{f0[0], f0[1], f1[0], f1[1]}, pf, o[db]);
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
        cur = nxt;
    }
    auto both = [](float a) { return over_groups<32>(a, [](float p, float q) { return p + q; }); };
    l = both(l);
    const float weight = sizeof(T) == 2 ? both(l_rounded) : l;       // what V was weighed by
    if (r > r_last) return;
    if (x.pieces == 1) {
        const float inv = weight > 0.f ? 1.f / weight : 0.f;
        T* row = out_row<T>(p, v.b, at);
#pragma unroll
        for (int db = 0; db < C::ODB; ++db)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                store4(row + 32 * db + 8 * a + 4 * h, floatx4{o[db][4 * a], o[db][4 * a + 1], o[db][4 * a + 2], o[db][4 * a + 3]} * inv);
        if (p.lse && h == 0) *lse_at(p, v.b, at) = log_sum(m, l);
    } else {
        // the sums to the part's own unrounded one, so that parts are joined by one number
        const float f = weight > 0.f ? l / weight : 0.f;
        const int64_t rec = (int64_t)(x.record + x.piece * x.tiles + x.t) * kRowsMany + 32 * w + i;
#pragma unroll
        for (int db = 0; db < C::ODB; ++db)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<floatx4*>(out.o + rec * D + 32 * db + 8 * a + 4 * h) = floatx4{o[db][4 * a], o[db][4 * a + 1], o[db][4 * a + 2], o[db][4 * a + 3]} * f;
        if (h == 0) *reinterpret_cast<float2*>(out.ml + 2 * rec) = make_float2(m, l);
    }
}

// ---------------------------------------------------------------- parts of cut rows -> rows
// 1024 / D rows at a time, D / 4 lanes a row; `per` rows a workgroup.
template <typename T, int D, int BM>
__global__ __launch_bounds__(256) void chunk_join_kernel(Chunk p, ChunkParts in, int per, int records) {
    const int u = blockIdx.y;
    const ChunkUnit v = chunk_unit(p, u, p.group_begin);
    const int2 piece = in.pieces[u];
    const int s = piece.y, tiles = (v.rows + BM - 1) / BM, r_end = min(v.rows, ((int)blockIdx.x + 1) * per);
    if (v.rows == 0 || s <= 1 || piece.x < 0 || piece.x + tiles * s > records) return;
    const int ch = threadIdx.x % (D / 4) * 4;
    for (int r = blockIdx.x * per + threadIdx.x / (D / 4); r < r_end; r += 1024 / D) {
        const int64_t rec0 = (int64_t)(piece.x + r / BM) * BM + r % BM, step = (int64_t)tiles * BM;
        float M = -INFINITY, L = 0.f;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int y = 0; y < s; ++y) M = fmaxf(M, in.ml[2 * (rec0 + y * step)]);
        if (M > -INFINITY) {
#pragma unroll 4
            for (int y = 0; y < s; ++y) {
                const float2 ml = *reinterpret_cast<const float2*>(in.ml + 2 * (rec0 + y * step));
                const float a = fast_exp2(ml.x - M);
                L += a * ml.y;
                acc += a * *reinterpret_cast<const floatx4*>(in.o + (rec0 + y * step) * D + ch);
            }
        }
        const RowAt at = row_at(p, v.g, r);
        acc *= L > 0.f ? 1.f / L : 0.f;
        store4(out_row<T>(p, v.b, at) + ch, acc);
        if (p.lse && ch == 0) *lse_at(p, v.b, at) = log_sum(M, L);
    }
}

// ---------------------------------------------------------------- host
constexpr int kFewRows = 32;
struct ChunkPlan { int few, direct, wgs, records, bm, join; int64_t grid; size_t ml, pieces, total; };
// keys: that the tables of a unit and its prefix can hold
static ChunkPlan chunk_plan(const zipvl_dims& d, int64_t keys) {
    ChunkPlan x;
    const int64_t rows = (int64_t)d.n * (d.Hq / d.Hkv), units = (int64_t)d.B * d.Hkv;
    x.few = rows <= kFewRows;
    x.bm = x.few ? (rows <= 16 ? 16 : 32) : kRowsMany;
    const int bn = x.few || d.dtype == ZIPVL_F32 ? 32 : 64;
    const int64_t tiles = (keys + bn - 1) / bn + 1, items = units * ((rows + x.bm - 1) / x.bm);
    x.wgs = x.few && d.dtype == ZIPVL_F32 && d.d == 128 ? kCus : 2 * kCus;
    const int64_t least = x.few ? kLeastFew : kLeastMany;
    x.direct = units > kScanUnits || tiles < 2 * least;      // nothing can be cut
    x.join = !x.direct;
    x.grid = (x.direct ? items : items + x.wgs) / 8 * 8 + 8;
    x.records = x.direct ? 0 : x.wgs;
    x.ml = (size_t)x.records * x.bm * d.d * sizeof(float);
    x.pieces = x.ml + (size_t)x.records * x.bm * 2 * sizeof(float);
    x.total = x.pieces + (x.direct ? 0 : units * sizeof(int2));
    return x;
}

size_t chunk_attn_workspace_bytes(const zipvl_dims& d, int64_t keys) { return std::max<size_t>(16, chunk_plan(d, keys).total); }

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
    hipLaunchKernelGGL((chunk_join_kernel<T, D, BM>), dim3((unsigned)((rows + per - 1) / per), p.units), dim3(256), 0, st, p, parts, (int)per, x.records);
    return check_launch("chunk_attn_paged parts");
}

template <typename T, int D, int COLS>
static int launch_few(const Chunk& p, const ChunkParts& parts, const ChunkPlan& x, hipStream_t st) {
    static std::atomic<uint64_t> done{0};
    int rc = allow_lds(&chunk_few_kernel<T, D, COLS>, PartCfg<T, D>::LDS, done);
    if (rc) return rc;
    {
        KernelTimer tm(ZIPVL_K_CHUNK_ATTN, st);
        hipLaunchKernelGGL((chunk_few_kernel<T, D, COLS>), dim3((unsigned)x.grid), dim3(256), (PartCfg<T, D>::LDS), st, p, parts, x.wgs, x.direct);
        if ((rc = check_launch("chunk_attn_paged"))) return rc;
    }
    return x.join ? launch_join<T, D, COLS>(p, parts, x, st) : ZIPVL_OK;
}

template <typename T, int D>
static int launch_chunk_t(const Chunk& p, const ChunkParts& parts, const ChunkPlan& x, hipStream_t st) {
    if (x.few) return x.bm == 16 ? launch_few<T, D, 16>(p, parts, x, st) : launch_few<T, D, 32>(p, parts, x, st);
    static std::atomic<uint64_t> done{0};
    int rc = allow_lds(&chunk_many_kernel<T, D>, ChunkCfg<T, D>::LDS, done);
    if (rc) return rc;
    {
        KernelTimer tm(ZIPVL_K_CHUNK_ATTN, st);
        hipLaunchKernelGGL((chunk_many_kernel<T, D>), dim3((unsigned)x.grid), dim3(256), (ChunkCfg<T, D>::LDS), st, p, parts, x.wgs, x.direct);
        if ((rc = check_launch("chunk_attn_paged"))) return rc;
    }
    return x.join ? launch_join<T, D, kRowsMany>(p, parts, x, st) : ZIPVL_OK;
}

int launch_chunk_attn_paged(const void* Q, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* len, const int32_t* k,
                            const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_len, const int32_t* group_begin, int32_t groups,
                            const zipvl_dims& d, float scale, void* O, const int64_t* o_strides, float* lse, void* ws, hipStream_t st)
{
    const int G = d.Hq / d.Hkv;
    const Chunk p = {(const char*)pages.K, (const char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table, table_pages, len, k,
                     prefix_table, prefix_pages, prefix_len, group_begin, groups, d.B, d.Hq, d.Hkv, G, d.n, d.B * d.Hkv, inverse(d.Hkv), inverse(G),
                     (const char*)Q, {d.q_strides[0], d.q_strides[1], d.q_strides[2]}, (char*)O, {o_strides[0], o_strides[1], o_strides[2]}, lse, scale * kLog2e};
    const ChunkPlan x = chunk_plan(d, ((int64_t)table_pages + prefix_pages) * pages.page);
    if (x.grid >= 1 << 24) return set_error(ZIPVL_ESHAPE, "zipvl_chunk_attn_paged: %lld tiles of queries are more than one grid takes", (long long)x.grid);
    const ChunkParts parts = {(float*)ws, (float*)((char*)ws + x.ml), (int2*)((char*)ws + x.pieces)};
    if (d.dtype == ZIPVL_BF16) return d.d == 128 ? launch_chunk_t<__bf16, 128>(p, parts, x, st) : launch_chunk_t<__bf16, 64>(p, parts, x, st);
    return d.d == 128 ? launch_chunk_t<float, 128>(p, parts, x, st) : launch_chunk_t<float, 64>(p, parts, x, st);
}

}  // namespace zipvl
