// Rows leave a paged cache by the attention weight that they have got.
//
// Keys are stored rotated, so the order of a unit's rows means nothing to attention: what stays need not move up.  With k rows to stay, a row below k that
// stays is where it is; the i-th row at or behind k that stays goes to the i-th row below k that leaves.  No row is both read and written, as few move as
// can, and all of them at once.
//   select   a workgroup a unit: the k-th largest key by a radix descent (protected rows above all others, then by weight), ties to the lower row, weights
//            and tokens in their new places, and the list of moves
//   move     K and V of the rows on the lists
// Bounded by the latency of a few sweeps over a unit's weights, then by the bytes that move.
#include <algorithm>

#include "launch.h"
#include "wavepart.h"

namespace zipvl {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;
constexpr int kDigit = 11, kDigits = 1 << kDigit;            // a key of 32 bits goes in digits of 11, 11 and 10

struct Late { int row, token; float weight; int unused; };   // a row at or behind k that stays
struct Evict {
    const int32_t* len; const int32_t* k;
    const float* weight; const int32_t* tokens;
    int budget, sinks, recent, room;
    int32_t* len_out; float* weight_out; int32_t* tokens_out;
    int32_t *count, *gap; Late* late; int64_t most;          // moves of a unit; rows that leave below k; `most` of both a unit
};

struct EvictShared {
    uint32_t hist[kDigits];
    int sums[kEvictWaves][4];
    uint32_t digit;
    int above, newest;
};

// Order of a weight: its bits; what has the sign bit set or is no number counts as 0.
__device__ __forceinline__ uint32_t weight_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return b > 0x7F800000u ? 0u : b;
}

// Ranks of the threads' flags over the workgroup, in thread order, for up to four kinds at once; `base` moves on by the totals.
template <int KINDS>
__device__ __forceinline__ void ranks(const bool (&flag)[KINDS], int (&rank)[KINDS], int (&base)[KINDS], EvictShared& sh) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint64_t bits[KINDS];
#pragma unroll
    for (int x = 0; x < KINDS; ++x) bits[x] = __ballot(flag[x]);
    __syncthreads();
    if (lane == 0)
#pragma unroll
        for (int x = 0; x < KINDS; ++x) sh.sums[w][x] = __popcll(bits[x]);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < KINDS; ++x) {
        int before = base[x], all = 0;
        for (int y = 0; y < kEvictWaves; ++y) {
            const int v = sh.sums[y][x];
            if (y < w) before += v;
            all += v;
        }
        rank[x] = before + __popcll(bits[x] & ((1ull << lane) - 1));
        base[x] += all;
    }
}

__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(Evict p) {
    __shared__ EvictShared sh;
    const int u = blockIdx.x, tid = threadIdx.x;
    const int len = max(0, min(p.len[u], p.room));
    int k = min(len, p.budget);
    if (p.k) k = max(0, min(k, p.k[u]));
    const float* weight = p.weight + (int64_t)u * p.room;
    const int32_t* tokens = p.tokens ? p.tokens + (int64_t)u * p.room : nullptr;
    float* weight_out = p.weight_out + (int64_t)u * p.room;
    int32_t* tokens_out = p.tokens ? p.tokens_out + (int64_t)u * p.room : nullptr;

    // the newest token: rows without one (negative) are new and follow each other behind it
    int newest = -1;
    if (tokens) {
        if (tid == 0) sh.newest = -1;
        __syncthreads();
        for (int r = tid; r < len; r += kEvictThreads) newest = max(newest, tokens[r]);
        atomicMax(&sh.newest, newest);
        __syncthreads();
        newest = sh.newest;
    }
    int fresh = 0;                                           // new rows
    if (tokens)
        for (int r0 = 0; r0 < len; r0 += kEvictThreads) {
            const int r = r0 + tid;
            const bool flag[1] = {r < len && tokens[r] < 0};
            int rank[1], base[1] = {fresh};
            ranks(flag, rank, base, sh);
            fresh = base[0];
        }
    const int last = tokens ? newest + fresh : len - 1;

    // f(row, there, key, token) for every row, in order, by all threads
    auto sweep = [&](auto&& f) {
        int fresh_before = 0;
        for (int r0 = 0; r0 < len; r0 += kEvictThreads) {
            const int r = r0 + tid;
            const bool there = r < len;
            int token = r;
            if (tokens) {
                token = there ? tokens[r] : 0;
                const bool flag[1] = {token < 0};
                int rank[1], base[1] = {fresh_before};
                ranks(flag, rank, base, sh);
                if (token < 0) token = newest + 1 + rank[0];
                fresh_before = base[0];
            }
            const float x = there ? weight[r] : 0.f;
            const bool sure = token < p.sinks || token > last - p.recent;
            f(r, there, x, weight_key(x) | (sure ? 0x80000000u : 0u), token);
        }
    };
    // the k-th largest key, and how many rows have a larger one
    uint32_t prefix = 0, mask = 0;
    int above = 0;
    if (k > 0 && k < len)
        for (int shift : {32 - kDigit, 32 - 2 * kDigit, 0}) {
            const uint32_t digits = shift ? kDigits : 1u << (32 - 2 * kDigit);
            for (int x = tid; x < kDigits; x += kEvictThreads) sh.hist[x] = 0;
            __syncthreads();
            sweep([&](int, bool there, float, uint32_t key, int) {
                if (there && (key & mask) == prefix) atomicAdd(&sh.hist[key >> shift & (digits - 1)], 1u);
            });
            __syncthreads();
            if (tid < 64) {                                  // from the top, 64 at a time
                int before = above;
                for (int x = (int)digits - 64; x >= 0; x -= 64) {
                    const int mine = sh.hist[x + 63 - tid], upto = before + wave_scan(mine);
                    if (upto - mine < k && k <= upto) {
                        sh.digit = x + 63 - tid;
                        sh.above = upto - mine;
                    }
                    before = __builtin_amdgcn_readlane(upto, 63);
                    if (before >= k) break;
                }
            }
            __syncthreads();
            prefix |= sh.digit << shift;
            mask |= (digits - 1) << shift;
            above = sh.above;
            __syncthreads();
        }
    const int ties = k - above;                              // of the rows with that key, the first ones
    int base[3] = {0, 0, 0};
    int32_t* gap = p.gap + u * p.most;
    Late* late = p.late + u * p.most;
    sweep([&](int r, bool there, float x, uint32_t key, int token) {
        const bool tie[1] = {there && k < len && key == prefix};
        int tied[1], tie_base[1] = {base[0]};
        ranks(tie, tied, tie_base, sh);
        base[0] = tie_base[0];
        const bool stays = there && (k == len || (k > 0 && (key > prefix || (tie[0] && tied[0] < ties))));
        const bool flag[2] = {there && r < k && !stays, r >= k && stays};
        int rank[2], move_base[2] = {base[1], base[2]};
        ranks(flag, rank, move_base, sh);
        base[1] = move_base[0];
        base[2] = move_base[1];
        if (!there) return;
        if (flag[0] && rank[0] < p.most) gap[rank[0]] = r;
        if (flag[1] && rank[1] < p.most) late[rank[1]] = {r, token, x, 0};
        if (r >= k || stays) {
            weight_out[r] = r < k ? x : 0.f;
            if (tokens) tokens_out[r] = r < k ? token : -1;
        }
    });
    __syncthreads();
    const int moves = (int)min((int64_t)min(base[1], base[2]), p.most);
    for (int j = tid; j < moves; j += kEvictThreads) {
        const int r = gap[j];
        const Late from = late[j];
        weight_out[r] = from.weight;
        if (tokens) tokens_out[r] = from.token;
    }
    if (tid == 0) {
        p.count[u] = moves;
        p.len_out[u] = k;
    }
}

constexpr int kMoveRows = 32;                                // a workgroup
template <int RB>
__global__ __launch_bounds__(256) void evict_move_kernel(char* K, char* V, int num_pages, int page_log2, const int32_t* table, int width,
                                                         const int32_t* count, const int32_t* gap, const Late* late, int64_t most) {
    constexpr int kLanes = RB / 16;
    const int u = blockIdx.y, moves = count[u], c = threadIdx.x % kLanes;
    const int j0 = blockIdx.x * kMoveRows;
    if (j0 >= moves) return;
    table += (int64_t)u * width;
    const int page = (1 << page_log2) - 1;
    for (int j = j0 + threadIdx.x / kLanes; j < min(j0 + kMoveRows, moves); j += 256 / kLanes) {
        const int to = gap[u * most + j], from = late[u * most + j].row;
        const int pt = table[to >> page_log2], pf = table[from >> page_log2];
        if ((unsigned)pt >= (unsigned)num_pages || (unsigned)pf >= (unsigned)num_pages) continue;
        const int64_t x = (((int64_t)pt << page_log2) + (to & page)) * RB + c * 16, y = (((int64_t)pf << page_log2) + (from & page)) * RB + c * 16;
        const uintx4 kk = load16(K + y), vv = load16(V + y);
        store16(K + x, kk);
        store16(V + x, vv);
    }
}

static int64_t most_moves(int64_t rows, int64_t budget) { return std::max<int64_t>(1, std::min(budget, rows / 2)); }
size_t paged_evict_workspace_bytes(int64_t units, int64_t rows, int64_t budget) {
    return (size_t)(((units * sizeof(int32_t) + 15) / 16 * 16) + units * ((most_moves(rows, budget) + 3) / 4 * 4) * (sizeof(int32_t) + sizeof(Late)));
}

int launch_paged_evict(const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const zipvl_dims& d, const int32_t* len, const int32_t* k,
                       const float* weight, const int32_t* tokens, int32_t budget, int32_t sinks, int32_t recent, int32_t* len_out, float* weight_out,
                       int32_t* tokens_out, void* ws, hipStream_t st)
{
    const int units = d.B * d.Hkv, room = table_pages * pages.page;
    const int64_t most = (most_moves(room, budget) + 3) / 4 * 4;
    char* const lists = (char*)ws + ((size_t)units * sizeof(int32_t) + 15) / 16 * 16;
    const Evict p = {len, k, weight, tokens, budget, sinks, recent, room, len_out, weight_out, tokens_out,
                     (int32_t*)ws, (int32_t*)(lists + units * most * sizeof(Late)), (Late*)lists, most};
    {
        KernelTimer tm(ZIPVL_K_PAGED_EVICT, st);
        hipLaunchKernelGGL(evict_select_kernel, dim3(units), dim3(kEvictThreads), 0, st, p);
        const int rc = check_launch("paged_evict");
        if (rc) return rc;
    }
    const dim3 grid((unsigned)((most_moves(room, budget) + kMoveRows - 1) / kMoveRows), units);
    KernelTimer tm(ZIPVL_K_PAGED_MOVE, st);
    const int rb = d.d * (d.dtype == ZIPVL_BF16 ? 2 : 4);
#define ZIPVL_MOVE(RB)                                                                                                                                  \
    hipLaunchKernelGGL((evict_move_kernel<RB>), grid, dim3(256), 0, st, (char*)pages.K, (char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table, \
                       table_pages, p.count, p.gap, p.late, most)
    if (rb == 128) ZIPVL_MOVE(128);
    else if (rb == 256) ZIPVL_MOVE(256);
    else ZIPVL_MOVE(512);
#undef ZIPVL_MOVE
    return check_launch("paged_evict rows");
}

}  // namespace zipvl
