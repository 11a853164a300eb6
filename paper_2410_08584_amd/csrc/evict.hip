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
#include <atomic>

#include "launch.h"
#include "wavepart.h"

namespace zipvl {

constexpr int kDigit = 11, kDigits = 1 << kDigit;            // a key of 32 bits goes in digits of 11, 11 and 10
// Moves of a unit up to which the first kernel does them.  256 units of bf16, d = 128, us, here and by a second launch: 16 moves 11, 13; 128 15, 18; 256 20, 23; eight units: 128 10.5, 12.5; 256 10.7, 11.1;
// 1000 15.7, 12.5.
constexpr int kMovesHere = 256;

struct Late { int row, token; float weight; int unused; };   // a row at or behind k that stays; token and weight: of evict_sweep_kernel, whose second look at them would be another sweep
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

// Moves j = first, first + step, ... below `end` of a unit, RB / 16 threads each; move(j): to which row, from which.
template <int RB, typename F>
__device__ __forceinline__ void move_rows(char* K, char* V, int num_pages, int page_log2, const int32_t* table, int first, int step, int end, F&& move) {
    const int c = threadIdx.x % (RB / 16) * 16, page = (1 << page_log2) - 1;
#pragma unroll 4
    for (int j = first; j < end; j += step) {
        const int2 m = move(j);
        const int to = m.x, from = m.y;
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
    __attribute__((aligned(16))) uint32_t hist[kDigits + 256];
    int sums[WAVES];
    uint32_t digit, key;
    int above, equal, found_above, found_equal, newest;
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
// By one wave, between two barriers: all waves took three and four times as long.
template <int WAVES>
__device__ __forceinline__ void crossing_digit(EvictShared<WAVES>& sh, int digits, int above, int k) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x, per = digits / 64, top = digits - per * lane;      // lane l has the digits from `top` down
        int sum = 0;
#pragma unroll
        for (int x = 0; x < kDigits / 64; x += 4)
            if (x < per) {
                // lanes stand 128 bytes apart: each begins at another sixteen, or they would meet in the same banks
                const uintx4 four = *reinterpret_cast<const uintx4*>(sh.hist + top - per + ((x + 4 * lane) & (per - 1)));
                sum += four[0] + four[1] + four[2] + four[3];
            }
        const int upto = above + wave_scan(sum);
        const int at = __builtin_ctzll(__ballot(upto >= k) | 1ull << 63);                // the lane with the digit
        const int from = digits - per * at, before = __builtin_amdgcn_readlane(upto - sum, at);
        const int n = lane < per ? (int)sh.hist[from - 1 - lane] : 0, till = before + wave_scan(n);
        if (till - n < k && k <= till) {
            sh.digit = from - 1 - lane;
            sh.above = till - n;
            sh.equal = n;
        }
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

// evict_sweep_kernel, behind the list of moves: the moved rows' weights and tokens, and where moves are done here, their K and V.
template <int RB>
__device__ __forceinline__ void finish_unit(const Evict& p, const EvictUnit& x, int u, int moves, int threads) {
    __syncthreads();
#pragma unroll 4
    for (int j = threadIdx.x; j < moves; j += threads) {
        const int r = x.gap[j];
        const Late from = x.late[j];
        x.weight_out[r] = from.weight;
        if (x.tokens) x.tokens_out[r] = from.token;
    }
    if (p.here) move_rows<RB>(p.K, p.V, p.num_pages, p.page_log2, p.table + (int64_t)u * p.width, threadIdx.x / (RB / 16), threads / (RB / 16), moves, [&](int j) { return int2{x.gap[j], x.late[j].row}; });
    if (threadIdx.x == 0) {
        p.count[u] = moves;
        p.len_out[u] = x.k;
    }
}

// Units whose keys fit LDS.  A round is four rows a thread, which follow each other; their weights and tokens stay in registers, their keys in LDS.  Ranks in the order of rows are
// sums over the threads before in the wave, and over the counts of (round, wave) before, which stand in LDS.  One CU has a unit, and it is bound by the instructions of
// its sweeps and some twenty barriers.  4 units of 18432 rows, 7200 to stay, this kernel alone: 27 us (41 with keys in registers, a row a thread and round, ranks by ballots; 30 with the
// weights and tokens read a second time); 256 units of 2064 rows with 16 to leave: 10 us (12, with the k-th key's digit found by lanes that meet in LDS banks).
constexpr int kRoundsMost = 9;                               // of 4096 rows: 147 KB of keys
constexpr int kFewKeys = 256;                                // that have the first digits of the k-th are looked at one by one, instead of two more digits
template <int WAVES, int ROUNDS, int RB>
__global__ __launch_bounds__(64 * WAVES) void evict_select_kernel(Evict p) {
    constexpr int kThreads = 64 * WAVES;
    extern __shared__ __attribute__((aligned(16))) uint32_t keys[];
    __shared__ EvictShared<WAVES> sh;
    __shared__ int cells[ROUNDS * WAVES + 1];
    int* const gaps = reinterpret_cast<int*>(keys);          // the rows that others move to, when the keys are done with
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = scalar(tid >> 6);
    auto first_row = [&](int c) { return (c * kThreads + tid) * 4; };
    uintx4 weight[ROUNDS], token[ROUNDS];                    // all asked for at once, with the length
    {
        const uint32_t* const from = reinterpret_cast<const uint32_t*>(p.weight) + (int64_t)u * p.room;
        const uint32_t* const tokens = reinterpret_cast<const uint32_t*>(p.tokens) + (int64_t)u * p.room;
#pragma unroll
        for (int c = 0; c < ROUNDS; ++c) {
            weight[c] = uintx4{0, 0, 0, 0};
            token[c] = uintx4{(uint32_t)first_row(c), (uint32_t)first_row(c) + 1, (uint32_t)first_row(c) + 2, (uint32_t)first_row(c) + 3};
            if (first_row(c) < p.room) {                     // a multiple of four
                if (p.tokens) token[c] = load16(tokens + first_row(c));
                weight[c] = load16(from + first_row(c));
            }
        }
    }
    for (int y = tid; y < kDigits; y += kThreads) sh.hist[y] = 0;
    if (tid == 0) sh.newest = -1;
    const EvictUnit x = evict_unit(p, u);
    const int len = scalar(x.len), k = scalar(x.k), rounds = (len + 4 * kThreads - 1) / (4 * kThreads);
    auto held = [&](int c) -> uintx4& { return *reinterpret_cast<uintx4*>(keys + first_row(c)); };
    // f(round) of rounds with rows
    auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < ROUNDS; ++c)
            if (c < rounds) f(c);
    };
    // cells -> what all cells before hold; the total.  By one wave.
    auto scan_cells = [&]() {
        __syncthreads();
        if (tid < 64) {
            constexpr int kPer = (ROUNDS * WAVES + 63) / 64;
            int v[kPer], sum = 0;
#pragma unroll
            for (int y = 0; y < kPer; ++y) {
                const int cell = lane * kPer + y;
                sum += v[y] = cell < rounds * WAVES ? cells[cell] : 0;
            }
            const int upto = wave_scan(sum);
            int before = upto - sum;
#pragma unroll
            for (int y = 0; y < kPer; ++y) {
                const int cell = lane * kPer + y;
                if (cell < rounds * WAVES) cells[cell] = before;
                before += v[y];
            }
            if (lane == 63) cells[ROUNDS * WAVES] = upto;
        }
        __syncthreads();
        return cells[ROUNDS * WAVES];
    };
    // a thread's count of a round -> what the threads before in the wave have; the wave's to its cell
    auto in_wave = [&](int count) { return wave_scan(count) - count; };
    auto to_cell = [&](int c, int count) {
        const int upto = wave_scan(count);
        if (lane == 63) cells[c * WAVES + w] = upto;
    };
    // One more of a digit, in lanes where there is one.  Those that have the first lane's go at once: thousands of equal weights would queue for one number.
    auto count = [&](uint32_t digit, bool there) {
        const uint64_t lanes = __ballot(there);
        if (!lanes) return;
        const int leader = __builtin_ctzll(lanes);
        const uint32_t common = __builtin_amdgcn_readlane(digit, leader);
        const uint64_t same = __ballot(there && digit == common);
        if (lane == leader) atomicAdd(&sh.hist[common], (uint32_t)__popcll(same));
        if (there && digit != common) atomicAdd(&sh.hist[digit], 1u);
    };
    int last = len - 1;
    __syncthreads();
    if (x.tokens) {
        // the newest token: rows without one (negative) are new and follow each other behind it
        auto fresh_of = [&](int c) {                         // new rows of four, as bits
            int f = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) f |= ((int)token[c][e] < 0 && first_row(c) + e < len) << e;
            return f;
        };
        int newest = -1;
        each([&](int c) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (first_row(c) + e < len) newest = max(newest, (int)token[c][e]);
            to_cell(c, __popc(fresh_of(c)));
        });
        newest = wave_reduce(newest, -1, [](int a, int b) { return max(a, b); });
        if (lane == 0) atomicMax(&sh.newest, newest);
        last = scan_cells() + sh.newest;
        newest = sh.newest;
        each([&](int c) {
            const int fresh = fresh_of(c);
            if (__any(fresh)) {
                int number = newest + 1 + cells[c * WAVES + w] + in_wave(__popc(fresh));
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (fresh >> e & 1) token[c][e] = number++;
            }
        });
    }
    // keys, and the histogram of their first digit
    const int recent_from = last - p.recent;
    each([&](int c) {
        const int r = first_row(c);
        uintx4 key;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            key[e] = weight_key(__uint_as_float(weight[c][e]));
            if ((int)token[c][e] < p.sinks || (int)token[c][e] > recent_from) key[e] |= 0x80000000u;
            if (r + e >= len) key[e] = 0;
            count(key[e] >> (32 - kDigit), r + e < len);
        }
        held(c) = key;
    });
    // the k-th largest key, how many rows have a larger one and how many have it
    uint32_t prefix = 0;
    int above = 0, equal = 0;
    const bool all = k == len, some = k > 0 && k < len;
    if (some) {
        uint32_t mask = 0;
        for (int shift : {32 - kDigit, 32 - 2 * kDigit, 0}) {
            const uint32_t digits = shift ? kDigits : 1u << (32 - 2 * kDigit);
            if (mask && equal <= kFewKeys) {
                // Few rows have the first digits of the k-th key: each looks how many of the others are larger, and how many as large.
                if (tid == 0) sh.digit = 0;
                __syncthreads();
                each([&](int c) {
                    const uintx4 key = held(c);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if ((key[e] & mask) == prefix && first_row(c) + e < len) sh.hist[atomicAdd(&sh.digit, 1u) & (kDigits - 1)] = key[e];
                });
                __syncthreads();
                constexpr int kParts = kThreads / kFewKeys;  // threads to a key, next to each other
                const uint32_t mine = sh.hist[tid / kParts];
                int larger = 0, as_large = 0;
                if (tid / kParts < equal) {
                    for (int y = tid % kParts * 4; y < equal; y += 4 * kParts) {
                        const uintx4 others = *reinterpret_cast<const uintx4*>(sh.hist + y);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            larger += y + e < equal && others[e] > mine;
                            as_large += y + e < equal && others[e] == mine;
                        }
                    }
#pragma unroll
                    for (int part = 1; part < kParts; part *= 2) {
                        larger += __shfl_xor(larger, part);
                        as_large += __shfl_xor(as_large, part);
                    }
                    if (above + larger < k && k <= above + larger + as_large) {      // all that are as large write the same
                        sh.key = mine;
                        sh.found_above = above + larger;
                        sh.found_equal = as_large;
                    }
                }
                __syncthreads();
                prefix = sh.key;
                above = sh.found_above;
                equal = sh.found_equal;
                break;
            }
            if (mask) {
                for (int y = tid; y < kDigits; y += kThreads) sh.hist[y] = 0;
                __syncthreads();
                each([&](int c) {
                    const uintx4 key = held(c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) count(key[e] >> shift & (digits - 1), (key[e] & mask) == prefix && first_row(c) + e < len);
                });
            }
            crossing_digit<WAVES>(sh, (int)digits, above, k);
            prefix |= sh.digit << shift;
            mask |= (digits - 1) << shift;
            above = sh.above;
            equal = sh.equal;
            __syncthreads();
        }
    } else __syncthreads();
    const int ties = k - above;                              // of the rows with that key, the first ones stay
    const bool count_ties = some && ties < equal;
    auto tied_of = [&](const uintx4& key) {
        int t = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) t |= (key[e] == prefix) << e;
        return t;                                            // rows behind the length among them, behind all others
    };
    if (count_ties) {
        each([&](int c) { to_cell(c, __popc(tied_of(held(c)))); });
        scan_cells();
    }
    // Rows that stay, as bits; moves: rows below k that leave, rows from k on that stay, both kinds counted in one number.
    auto first = [](int n) { return (1 << max(0, min(n, 4))) - 1; };        // of four rows, those with n left
    uint64_t in_all = 0;                                     // four bits a round
    static_assert(ROUNDS <= 16, "");
    each([&](int c) {
        const int r = first_row(c);
        const uintx4 key = held(c);
        int in = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) in |= (all || (some && key[e] >= prefix)) << e;
        if (count_ties) {
            const int tied = tied_of(key);
            if (__any(tied)) {
                int rank = cells[c * WAVES + w] + in_wave(__popc(tied));
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (tied >> e & 1 && rank++ >= ties) in &= ~(1 << e);
            }
        }
        in_all |= (uint64_t)(in & first(len - r)) << 4 * c;
    });
    auto in_of = [&](int c) { return (int)(in_all >> 4 * c) & 15; };
    __syncthreads();                                         // cells and keys have been read
    each([&](int c) {
        const int in = in_of(c), low = first(k - first_row(c));
        to_cell(c, __popc(low & ~in) | __popc(in & ~low) << 16);
    });
    static_assert(ROUNDS * kThreads * 4 < 1 << 17, "at most half of the rows are of either kind: 16 bits each");
    const int total = scan_cells();
    const int moves = (int)min<int64_t>(min(total & 0xFFFF, (int)((uint32_t)total >> 16)), p.most);
    const bool copied = x.weight_out != x.weight || x.tokens_out != x.tokens;         // else old rows that stay where they are stand there already
    // The rows that others move to, and those that move; a moved row's weight and token have to wait for the first.
    each([&](int c) {
        if (c * kThreads * 4 + 256 * w >= k) return;         // of the wave
        const int leave = first(k - first_row(c)) & ~in_of(c);
        int rank = (cells[c * WAVES + w] + in_wave(__popc(leave))) & 0xFFFF;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (leave >> e & 1) gaps[rank++] = first_row(c) + e;
    });
    __syncthreads();
    each([&](int c) {
        const int r = first_row(c), in = in_of(c), low = first(k - r), there = first(len - r), come = in & ~low;
        if (__any(come)) {
            int rank = (int)((uint32_t)cells[c * WAVES + w] >> 16) + in_wave(__popc(come));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (come >> e & 1 && rank < moves) {
                    const int to = gaps[rank];
                    x.weight_out[to] = __uint_as_float(weight[c][e]);
                    if (x.tokens) x.tokens_out[to] = (int)token[c][e];
                    gaps[moves + rank++] = r + e;
                }
        }
        const int put = (in & low) | (there & ~low);         // rows that are written down; in place, weights that stay and old tokens could be left, but most rounds have some new ones
        if (!copied && !x.tokens && put == (in & low)) return;
        uintx4 v = weight[c], t = token[c];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(low >> e & 1)) {
                v[e] = 0;
                t[e] = -1;
            }
        if (put == 15) {
            store16(reinterpret_cast<uint32_t*>(x.weight_out) + r, v);
            if (x.tokens) store16(reinterpret_cast<uint32_t*>(x.tokens_out) + r, t);
        } else if (put) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (put >> e & 1) {
                    x.weight_out[r + e] = __uint_as_float(v[e]);
                    if (x.tokens) x.tokens_out[r + e] = (int)t[e];
                }
        }
    });
    __syncthreads();
    if (p.here) move_rows<RB>(p.K, p.V, p.num_pages, p.page_log2, p.table + (int64_t)u * p.width, tid / (RB / 16), kThreads / (RB / 16), moves, [&](int j) { return int2{gaps[j], gaps[moves + j]}; });
    else
        for (int j = tid; j < moves; j += kThreads) {
            x.gap[j] = gaps[j];
            x.late[j].row = gaps[moves + j];
        }
    if (tid == 0) {
        p.count[u] = moves;
        p.len_out[u] = k;
    }
}

// Units of any length, whose keys do not fit LDS: the same, in sweeps over the rows, 1024 at a time.  4 units of 36 928 rows, 8192 to stay, with the moves 176 us (36 864 in the form before: 52), of
// 131 072, 16 384 to stay, 593.
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
    const int32_t* gap = p.gap + u * p.most;
    const Late* late = p.late + u * p.most;
    move_rows<RB>(p.K, p.V, p.num_pages, p.page_log2, p.table + (int64_t)u * p.width, j0 + threadIdx.x / (RB / 16), 256 / (RB / 16), min(j0 + kMoveRows, moves),
                  [&](int j) { return int2{gap[j], late[j].row}; });
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
        // By the tables' width, which the host knows: 256 units of 2064 rows, 16 to leave, take 9 us where tables hold 2112 rows, 19 at 4096 (a second launch moves), 35 at 36 864, 31 behind.
        // Four waves for short units, of which a CU then has several: 3200 units of 500 rows 25 us, 79 with 16 waves; 256 units as long
        if (p.room <= 1024) hipLaunchKernelGGL((evict_select_kernel<4, 1, RB>), dim3(units), dim3(256), 1024 * 4, st, p);
        else if (p.room <= 4096) hipLaunchKernelGGL((evict_select_kernel<16, 1, RB>), dim3(units), dim3(1024), 4096 * 4, st, p);
        else if (p.room <= kRoundsMost * 4096) {
            const bool five = p.room <= 5 * 4096;
            auto kernel = five ? &evict_select_kernel<16, 5, RB> : &evict_select_kernel<16, kRoundsMost, RB>;
            static std::atomic<uint64_t> set[2];             // more than 64 KB of LDS has to be asked for, on every device
            int dev = 0;
            if (hipGetDevice(&dev) != hipSuccess) return set_error(ZIPVL_EHIP, "paged_evict: no current device");
            if (dev > 63 || !(set[five].load(std::memory_order_relaxed) >> dev & 1)) {
                const int most = (five ? 5 : kRoundsMost) * 4096 * 4;
                if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, most) != hipSuccess) return set_error(ZIPVL_EHIP, "paged_evict: %d bytes of LDS are refused", most);
                if (dev <= 63) set[five].fetch_or(1ull << dev, std::memory_order_relaxed);
            }
            hipLaunchKernelGGL(kernel, dim3(units), dim3(1024), (p.room + 4095) / 4096 * 4096 * 4, st, p);
        } else hipLaunchKernelGGL((evict_sweep_kernel<RB>), dim3(units), dim3(1024), 0, st, p);
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
