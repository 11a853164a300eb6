// Rows leave a paged cache by the attention weight that they have got.
//
// Keys are stored rotated, so the order of a unit's rows means nothing to attention: what stays need not move up.  With k rows to stay, a row below k that
// stays is where it is; the i-th row at or behind k that stays goes to the i-th row below k that leaves.  No row is both read and written, as few move as
// can, and all of them at once.
//   select   a workgroup a unit: the k-th largest key by a radix descent (protected rows above all others, then by weight), ties to the lower row, weights
//            and tokens in their new places, and the list of moves
//   move     K and V of the rows on the lists; where a unit can have few, the first kernel's workgroup does it
// Bounded by the latency of a chain of steps over a unit's weights, then by the bytes that move.
#include <algorithm>

#include "launch.h"
#include "wavepart.h"

namespace zipvl {

constexpr int kDigit = 11, kDigits = 1 << kDigit;            // a key of 32 bits goes in digits of 11, 11 and 10
constexpr int kMovesHere = 64;                               // moves of a unit up to which the first kernel does them

struct Late { int row, token; float weight; int unused; };   // a row at or behind k that stays
struct Evict {
    const int32_t* len; const int32_t* k;
    const float* weight; const int32_t* tokens;
    int budget, sinks, recent, room;
    int32_t* len_out; float* weight_out; int32_t* tokens_out;
    int32_t *count, *gap; Late* late; int64_t most;          // moves of a unit; rows that leave below k; `most` of both a unit
    int here;                                                // the moves are done here
    char *K, *V; int num_pages, page_log2; const int32_t* table; int width;
};

// Order of a weight: its bits; what has the sign bit set or is no number counts as 0.
__device__ __forceinline__ uint32_t weight_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return b > 0x7F800000u ? 0u : b;
}

// Moves j = first, first + step, ... below `end` of a unit, RB / 16 threads each.
template <int RB>
__device__ __forceinline__ void move_rows(char* K, char* V, int num_pages, int page_log2, const int32_t* table, const int32_t* gap, const Late* late, int first, int step, int end) {
    const int c = threadIdx.x % (RB / 16) * 16, page = (1 << page_log2) - 1;
#pragma unroll 4
    for (int j = first; j < end; j += step) {
        const int to = gap[j], from = late[j].row;
        const int pt = table[to >> page_log2], pf = table[from >> page_log2];
        if ((unsigned)pt >= (unsigned)num_pages || (unsigned)pf >= (unsigned)num_pages) continue;
        const int64_t x = (((int64_t)pt << page_log2) + (to & page)) * RB + c, y = (((int64_t)pf << page_log2) + (from & page)) * RB + c;
        const uintx4 kk = load16(K + y), vv = load16(V + y);
        store16(K + x, kk);
        store16(V + x, vv);
    }
}

template <int WAVES>
struct EvictShared {
    uint32_t hist[kDigits];
    int sums[WAVES];
    uint32_t digit, equal;
    int above, newest;
};

// Exclusive sum over the workgroup's threads, and the total.
template <int WAVES>
__device__ __forceinline__ int block_scan_of(int v, int (&sums)[WAVES], int& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, upto = wave_scan(v);
    __syncthreads();
    if (lane == 63) sums[w] = upto;
    __syncthreads();
    int before = upto - v;
    total = 0;
#pragma unroll
    for (int y = 0; y < WAVES; ++y) {
        const int s = sums[y];
        if (y < w) before += s;
        total += s;
    }
    return before;
}

// The digit at which rows counted from the largest key on reach k, of a histogram of `digits` (sh.hist): sh.digit, sh.above (rows above it), sh.equal (rows with it).
template <int WAVES>
__device__ __forceinline__ void crossing_digit(EvictShared<WAVES>& sh, int digits, int above, int k) {
    constexpr int kPer = kDigits / (64 * WAVES);
    uint32_t mine[kPer];
    int sum = 0, total;
    const int top = digits - 1 - (int)threadIdx.x * kPer;    // thread t has the digits from there down
#pragma unroll
    for (int x = 0; x < kPer; ++x) sum += mine[x] = top - x >= 0 ? sh.hist[top - x] : 0;
    int before = above + block_scan_of<WAVES>(sum, sh.sums, total);
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
        if (before < k && k <= before + (int)mine[x]) {
            sh.digit = top - x;
            sh.above = before;
            sh.equal = mine[x];
        }
        before += mine[x];
    }
    __syncthreads();
}

// What a unit's workgroup goes by.
struct EvictUnit {
    const float* weight; const int32_t* tokens; float* weight_out; int32_t* tokens_out;
    int32_t* gap; Late* late;
    int len, k;
};
__device__ __forceinline__ EvictUnit evict_unit(const Evict& p, int u) {
    const int64_t at = (int64_t)u * p.room;
    EvictUnit x = {p.weight + at, p.tokens ? p.tokens + at : nullptr, p.weight_out + at, p.tokens ? p.tokens_out + at : nullptr,
                   p.gap + u * p.most, p.late + u * p.most, max(0, min(p.len[u], p.room)), 0};
    x.k = min(x.len, p.budget);
    if (p.k) x.k = max(0, min(x.k, p.k[u]));
    return x;
}

// Behind the list of moves: the moved rows' weights and tokens, and where moves are done here, their K and V.
template <int RB>
__device__ __forceinline__ void finish_unit(const Evict& p, const EvictUnit& x, int u, int moves, int threads) {
    __syncthreads();
    for (int j = threadIdx.x; j < moves; j += threads) {
        const int r = x.gap[j];
        const Late from = x.late[j];
        x.weight_out[r] = from.weight;
        if (x.tokens) x.tokens_out[r] = from.token;
    }
    if (p.here) move_rows<RB>(p.K, p.V, p.num_pages, p.page_log2, p.table + (int64_t)u * p.width, x.gap, x.late, threadIdx.x / (RB / 16), threads / (RB / 16), moves);
    if (threadIdx.x == 0) {
        p.count[u] = moves;
        p.len_out[u] = x.k;
    }
}

// Up to KPT rows a thread, their keys in registers: row c 64 WAVES + t is thread t's c-th.  Ranks in the order of rows come from ballots: the counts of
// (c, wave) stand in LDS and one scan adds them up, two barriers for all rows of a kind.
template <int WAVES, int KPT, int RB>
__global__ __launch_bounds__(64 * WAVES) void evict_select_kernel(Evict p) {
    constexpr int kThreads = 64 * WAVES, kCells = KPT * WAVES, kPer = (kCells + kThreads - 1) / kThreads;
    __shared__ EvictShared<WAVES> sh;
    __shared__ int cells[KPT][WAVES];
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = scalar(tid >> 6);
    const EvictUnit x = evict_unit(p, u);
    int len = scalar(x.len);
    const int k = scalar(x.k), rounds = (len + kThreads - 1) / kThreads;
    auto row = [&](int c) { return c * kThreads + tid; };
    // Said anew before each loop over the rows: which of them there are (two scalar registers a row) is not kept from one for the next (it spilled).
    auto afresh = [&]() { asm volatile("" : "+s"(len)); };
    // cells -> what all cells before hold; the total
    auto scan_cells = [&]() {
        __syncthreads();
        int v[kPer], sum = 0, total;
#pragma unroll
        for (int y = 0; y < kPer; ++y) {
            const int cell = tid * kPer + y;
            sum += v[y] = cell < rounds * WAVES ? (&cells[0][0])[cell] : 0;
        }
        int before = block_scan_of<WAVES>(sum, sh.sums, total);
#pragma unroll
        for (int y = 0; y < kPer; ++y) {
            const int cell = tid * kPer + y;
            if (cell < rounds * WAVES) (&cells[0][0])[cell] = before;
            before += v[y];
        }
        __syncthreads();
        return total;
    };
    auto below = [&](uint64_t bits) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0)); };

    uint64_t sure = 0;                                       // bit c: row c is protected
    if (x.tokens) {
        // the newest token: rows without one (negative) are new and follow each other behind it
        int32_t token[KPT];
#pragma unroll
        for (int c = 0; c < KPT; ++c) {
            token[c] = 0;
            if (c < rounds && row(c) < len) token[c] = x.tokens[row(c)];
        }
        if (tid == 0) sh.newest = -1;
        int newest = -1;
        afresh();
#pragma unroll
        for (int c = 0; c < KPT; ++c)
            if (c < rounds) {
                if (row(c) < len) newest = max(newest, token[c]);
                const uint64_t fresh = __ballot(token[c] < 0);
                if (lane == 0) cells[c][w] = __popcll(fresh);
            }
        __syncthreads();
        newest = wave_reduce(newest, -1, [](int a, int b) { return max(a, b); });
        if (lane == 0) atomicMax(&sh.newest, newest);
        const int fresh = scan_cells();
        newest = sh.newest;
        const int last = newest + fresh;
#pragma unroll
        for (int c = 0; c < KPT; ++c)
            if (c < rounds) {
                const int rank = below(__ballot(token[c] < 0));
                if (token[c] < 0) {
                    token[c] = newest + 1 + cells[c][w] + rank;
                    x.tokens_out[row(c)] = token[c];         // where it is looked up again below
                }
                sure |= (uint64_t)(token[c] < p.sinks || token[c] > last - p.recent) << c;
            }
        __syncthreads();
    }
    uint32_t key[KPT];
    {
        float weight[KPT];
        afresh();
#pragma unroll
        for (int c = 0; c < KPT; ++c) {
            weight[c] = 0.f;
            if (c < rounds && row(c) < len) weight[c] = x.weight[row(c)];
        }
#pragma unroll
        for (int c = 0; c < KPT; ++c) {
            const bool first = x.tokens ? sure >> c & 1 : row(c) < p.sinks || row(c) > len - 1 - p.recent;
            key[c] = weight_key(weight[c]) | (first ? 0x80000000u : 0u);
        }
    }
    // the k-th largest key, how many rows have a larger one and how many have it
    uint32_t prefix = 0, mask = 0;
    int above = 0, equal = 0;
    if (k > 0 && k < len)
        for (int shift : {32 - kDigit, 32 - 2 * kDigit, 0}) {
            const uint32_t digits = shift ? kDigits : 1u << (32 - 2 * kDigit);
            for (int y = tid; y < kDigits; y += kThreads) sh.hist[y] = 0;
            __syncthreads();
            afresh();
#pragma unroll
            for (int c = 0; c < KPT; ++c)
                if (c < rounds && row(c) < len && (key[c] & mask) == prefix) atomicAdd(&sh.hist[key[c] >> shift & (digits - 1)], 1u);
            __syncthreads();
            crossing_digit<WAVES>(sh, (int)digits, above, k);
            prefix |= sh.digit << shift;
            mask |= (digits - 1) << shift;
            above = sh.above;
            equal = sh.equal;
            __syncthreads();
        }
    const int ties = k - above;                              // of the rows with that key, the first ones stay
    // 0 leaves, 1 stays, of rows with the k-th key those that come first
    const bool all = k == len, some = k > 0 && k < len, count_ties = some && ties < equal;
    if (count_ties) {
        afresh();
#pragma unroll
        for (int c = 0; c < KPT; ++c)
            if (c < rounds) {
                const uint64_t tie = __ballot(row(c) < len && key[c] == prefix);
                if (lane == 0) cells[c][w] = __popcll(tie);
            }
        scan_cells();
    }
    uint64_t stays = 0;                                      // bit c: of row c
    afresh();
#pragma unroll
    for (int c = 0; c < KPT; ++c)
        if (c < rounds) {
            const bool there = row(c) < len, tie = there && some && key[c] == prefix;
            bool in = there && (all || (some && key[c] >= prefix));
            if (count_ties) {
                const int rank = cells[c][w] + below(__ballot(tie));
                if (tie) in = rank < ties;
            }
            stays |= (uint64_t)in << c;
        }
    static_assert(KPT <= 64, "a bit for each row of a thread");
    __syncthreads();
    // moves: rows below k that leave, rows from k on that stay; both kinds counted in one number
    afresh();
#pragma unroll
    for (int c = 0; c < KPT; ++c)
        if (c < rounds) {
            const bool in = stays >> c & 1, there = row(c) < len;
            const uint64_t out = __ballot(there && row(c) < k && !in), come = __ballot(row(c) >= k && in);
            if (lane == 0) cells[c][w] = __popcll(out) | __popcll(come) << 16;
        }
    static_assert(KPT * 64 * WAVES < 1 << 17, "at most half of the rows are of either kind: 16 bits each");
    const int total = scan_cells();
    const int moves = (int)min<int64_t>(min(total & 0xFFFF, (int)((uint32_t)total >> 16)), p.most);
    afresh();
#pragma unroll
    for (int c = 0; c < KPT; ++c)
        if (c < rounds) {
            const int r = row(c);
            const bool in = stays >> c & 1, there = r < len, out = there && r < k && !in, come = r >= k && in;
            const uint32_t base = cells[c][w];
            const int gap_rank = (base & 0xFFFF) + below(__ballot(out)), late_rank = (base >> 16) + below(__ballot(come));
            if (there && in) {
                const float weight = x.weight[r];
                int token = r;
                if (x.tokens) {
                    token = x.tokens[r];
                    if (token < 0) token = x.tokens_out[r];
                }
                if (come && late_rank < p.most) x.late[late_rank] = {r, token, weight, 0};
                if (r < k) {
                    x.weight_out[r] = weight;
                    if (x.tokens) x.tokens_out[r] = token;
                }
            }
            if (out && gap_rank < p.most) x.gap[gap_rank] = r;
            if (there && r >= k) {
                x.weight_out[r] = 0.f;
                if (x.tokens) x.tokens_out[r] = -1;
            }
        }
    finish_unit<RB>(p, x, u, moves, kThreads);
}

// Units of any length, whose keys do not stay in registers: the same, in sweeps over the rows, 1024 at a time.
template <int RB>
__global__ __launch_bounds__(1024) void evict_sweep_kernel(Evict p) {
    constexpr int kWaves = 16, kThreads = 1024;
    __shared__ EvictShared<kWaves> sh;
    const int u = blockIdx.x, tid = threadIdx.x;
    const EvictUnit x = evict_unit(p, u);
    const int len = scalar(x.len), k = scalar(x.k);
    // ranks of the threads' flags, from `base` on, which moves on by their number
    auto ranks = [&](bool flag, int& base) {
        int total;
        const int rank = base + block_scan_of<kWaves>(flag, sh.sums, total);
        base += total;
        return rank;
    };
    int newest = -1, fresh = 0;
    if (x.tokens) {
        if (tid == 0) sh.newest = -1;
        __syncthreads();
        for (int r = tid; r < len; r += kThreads) newest = max(newest, x.tokens[r]);
        atomicMax(&sh.newest, newest);
        __syncthreads();
        newest = sh.newest;
        for (int r0 = 0; r0 < len; r0 += kThreads) ranks(r0 + tid < len && x.tokens[r0 + tid] < 0, fresh);
    }
    const int last = x.tokens ? newest + fresh : len - 1;
    // f(row, there, weight, key, token) for every row, in order, by all threads
    auto sweep = [&](auto&& f) {
        int fresh_before = 0;
        for (int r0 = 0; r0 < len; r0 += kThreads) {
            const int r = r0 + tid;
            const bool there = r < len;
            int token = r;
            if (x.tokens) {
                token = there ? x.tokens[r] : 0;
                const int rank = ranks(token < 0, fresh_before);
                if (token < 0) token = newest + 1 + rank;
            }
            const float weight = there ? x.weight[r] : 0.f;
            f(r, there, weight, weight_key(weight) | (token < p.sinks || token > last - p.recent ? 0x80000000u : 0u), token);
        }
    };
    uint32_t prefix = 0, mask = 0;
    int above = 0;
    if (k > 0 && k < len)
        for (int shift : {32 - kDigit, 32 - 2 * kDigit, 0}) {
            const uint32_t digits = shift ? kDigits : 1u << (32 - 2 * kDigit);
            for (int y = tid; y < kDigits; y += kThreads) sh.hist[y] = 0;
            __syncthreads();
            sweep([&](int, bool there, float, uint32_t key, int) {
                if (there && (key & mask) == prefix) atomicAdd(&sh.hist[key >> shift & (digits - 1)], 1u);
            });
            __syncthreads();
            crossing_digit<kWaves>(sh, (int)digits, above, k);
            prefix |= sh.digit << shift;
            mask |= (digits - 1) << shift;
            above = sh.above;
            __syncthreads();
        }
    const int ties = k - above;
    int tied = 0, gaps = 0, lates = 0;
    sweep([&](int r, bool there, float weight, uint32_t key, int token) {
        const bool tie = there && k > 0 && k < len && key == prefix;
        const int tie_rank = ranks(tie, tied);
        const bool stays = there && (k == len || (k > 0 && (key > prefix || (tie && tie_rank < ties))));
        const bool out = there && r < k && !stays, come = r >= k && stays;
        const int gap_rank = ranks(out, gaps), late_rank = ranks(come, lates);
        if (out && gap_rank < p.most) x.gap[gap_rank] = r;
        if (come && late_rank < p.most) x.late[late_rank] = {r, token, weight, 0};
        if (there && (r >= k || stays)) {
            x.weight_out[r] = r < k ? weight : 0.f;
            if (x.tokens) x.tokens_out[r] = r < k ? token : -1;
        }
    });
    finish_unit<RB>(p, x, u, (int)min<int64_t>(min(gaps, lates), p.most), kThreads);
}

constexpr int kMoveRows = 32;                                // a workgroup
template <int RB>
__global__ __launch_bounds__(256) void evict_move_kernel(Evict p) {
    const int u = blockIdx.y, moves = p.count[u], j0 = blockIdx.x * kMoveRows;
    if (j0 >= moves) return;
    move_rows<RB>(p.K, p.V, p.num_pages, p.page_log2, p.table + (int64_t)u * p.width, p.gap + u * p.most, p.late + u * p.most, j0 + threadIdx.x / (RB / 16), 256 / (RB / 16),
                  min(j0 + kMoveRows, moves));
}

// Moves of a unit: no more than rows that stay, nor than rows that leave.  given: k may ask for fewer than the budget
static int64_t most_moves(int64_t rows, int64_t budget, bool given) { return std::max<int64_t>(1, std::min(budget, given ? rows / 2 : std::min(rows / 2, rows - std::min(budget, rows)))); }
size_t paged_evict_workspace_bytes(int64_t units, int64_t rows, int64_t budget) {
    return (size_t)(((units * sizeof(int32_t) + 15) / 16 * 16) + units * ((most_moves(rows, budget, true) + 3) / 4 * 4) * (sizeof(int32_t) + sizeof(Late)));
}

template <int RB>
static int launch_evict_t(const Evict& p, int units, hipStream_t st) {
    {
        KernelTimer tm(ZIPVL_K_PAGED_EVICT, st);
        if (p.room <= 1024) hipLaunchKernelGGL((evict_select_kernel<4, 4, RB>), dim3(units), dim3(256), 0, st, p);
        else if (p.room <= 4096) hipLaunchKernelGGL((evict_select_kernel<16, 4, RB>), dim3(units), dim3(1024), 0, st, p);
        else if (p.room <= 36 * 1024) hipLaunchKernelGGL((evict_select_kernel<16, 36, RB>), dim3(units), dim3(1024), 0, st, p);
        else hipLaunchKernelGGL((evict_sweep_kernel<RB>), dim3(units), dim3(1024), 0, st, p);
        const int rc = check_launch("paged_evict");
        if (rc || p.here) return rc;
    }
    KernelTimer tm(ZIPVL_K_PAGED_MOVE, st);
    hipLaunchKernelGGL((evict_move_kernel<RB>), dim3((unsigned)((p.most + kMoveRows - 1) / kMoveRows), units), dim3(256), 0, st, p);
    return check_launch("paged_evict rows");
}

int launch_paged_evict(const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const zipvl_dims& d, const int32_t* len, const int32_t* k,
                       const float* weight, const int32_t* tokens, int32_t budget, int32_t sinks, int32_t recent, int32_t* len_out, float* weight_out,
                       int32_t* tokens_out, void* ws, hipStream_t st)
{
    const int units = d.B * d.Hkv, room = table_pages * pages.page;
    const int64_t most = (most_moves(room, budget, k != nullptr) + 3) / 4 * 4;
    char* const lists = (char*)ws + ((size_t)units * sizeof(int32_t) + 15) / 16 * 16;
    const Evict p = {len, k, weight, tokens, budget, sinks, recent, room, len_out, weight_out, tokens_out,
                     (int32_t*)ws, (int32_t*)(lists + units * most * sizeof(Late)), (Late*)lists, most, most <= kMovesHere,
                     (char*)pages.K, (char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table, table_pages};
    const int rb = d.d * (d.dtype == ZIPVL_BF16 ? 2 : 4);
    return rb == 128 ? launch_evict_t<128>(p, units, st) : rb == 256 ? launch_evict_t<256>(p, units, st) : launch_evict_t<512>(p, units, st);
}

}  // namespace zipvl
