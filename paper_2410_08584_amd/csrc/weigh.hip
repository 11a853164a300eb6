// The attention weight that cached rows get from new queries: weight[u, r] = before[u, r] + sum over heads and tokens of exp(scale q.k - lse).
//
// Keys stay, queries come: a wave has 32 keys in registers, S = K Q^T on matrix tiles gives a lane one query and 16 keys, whose exponentials it
// adds up over all queries; the 32 lanes meet once, at the end.  No sum crosses workgroups, so no order of arrival changes a result.
// Few queries (a decode step): the read of K.  Many: products, and exponentials at a quarter of the vector rate.
#include "launch.h"
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
};

template <typename T, int D>
struct WeighCfg {
    static constexpr int RB = D * (int)sizeof(T), QT = sizeof(T) == 2 ? 64 : 32;        // queries a tile
    static constexpr int TILE = QT * RB, NL = TILE / 4096, RPL = 1024 / RB, CH = D / Elem<T>::kPerChunk;
};

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void paged_weigh_kernel(Weigh p) {
    using C = WeighCfg<T, D>;
    __shared__ __attribute__((aligned(16))) char tile[2 * C::TILE];
    const int u = blockIdx.y, k0 = blockIdx.x * 128, room = p.width << p.page_log2;
    const int len = scalar(max(0, min(p.len[u], room)));
    if (k0 >= len) return;
    const int tid = threadIdx.x, w = scalar(tid >> 6), lane = tid & 63, i = lane & 31, h = lane >> 5;
    const int b = divided(u, p.Hkv, p.inv_Hkv), g = u - b * p.Hkv;
    const int cnt = p.cnt ? scalar(max(0, min(p.cnt[u], p.n))) : p.n, rows = cnt * p.G, first = len - cnt;     // token i stands in row first + i
    const int key0 = k0 + 32 * w, key = min(key0 + i, len - 1);
    const int entry = p.table[(int64_t)u * p.width + (key >> p.page_log2)];
    const bool there = (unsigned)entry < (unsigned)p.num_pages;
    uintx4 kf[C::CH];
    {
        const char* row = p.K + (((int64_t)(there ? entry : 0) << p.page_log2) + (key & ((1 << p.page_log2) - 1))) * C::RB;
#pragma unroll
        for (int cc = 0; cc < C::CH; ++cc) kf[cc] = load16(row + (2 * cc + h) * 16);
    }
    float sum[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[r] = 0.f;
    // row r: token r / G, head r % G; the first token that sees a key of the workgroup
    const int r_first = max(0, k0 - first) * p.G, t0 = r_first / C::QT, t1 = (rows + C::QT - 1) / C::QT;
    auto request = [&](int t, int buf) {
#pragma unroll
        for (int q = 0; q < C::NL; ++q) {
            const int at = (q * 4 + w) * C::RPL + lane / (C::RB / 16), r = min(t * C::QT + at, rows - 1), token = divided(r, p.G, p.inv_G);
            const T* row = reinterpret_cast<const T*>(p.Q) + b * p.q[0] + (g * p.G + r - token * p.G) * p.q[1] + token * p.q[2];
            load_kib_to_lds_at(reinterpret_cast<const char*>(row) + swz_chunk(lane % (C::RB / 16), k_row_swizzle<C::RB>(at)),
                               lds_address(tile) + buf * C::TILE + (q * 4 + w) * 1024);
        }
    };
    if (t0 < t1) request(t0, 0);
    for (int t = t0, buf = 0; t < t1; ++t, buf ^= 1) {
        float lse[C::QT / 32];
        int last[C::QT / 32];
#pragma unroll
        for (int x = 0; x < C::QT / 32; ++x) {
            const int r = t * C::QT + 32 * x + i, rr = min(r, rows - 1), token = divided(rr, p.G, p.inv_G);
            lse[x] = p.lse[((int64_t)b * p.Hq + g * p.G + rr - token * p.G) * p.lse_pitch + token];
            if (lse[x] == -INFINITY) lse[x] = INFINITY;      // a query that sees nothing
            last[x] = r < rows ? first + token : -1;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < t1) request(t + 1, buf ^ 1);
        const bool whole = first + divided(t * C::QT, p.G, p.inv_G) >= key0 + 31 && (t + 1) * C::QT <= rows;       // every query sees every key of the wave
#pragma unroll
        for (int x = 0; x < C::QT / 32; ++x) {
            floatx16 s = {0};
#pragma unroll
            for (int cc = 0; cc < C::CH; ++cc) {
                const uintx4 qf = *reinterpret_cast<const uintx4*>(tile + buf * C::TILE + (32 * x + i) * C::RB + swz_chunk(2 * cc + h, k_row_swizzle<C::RB>(32 * x + i)));
                s = mma_frag<T>(kf[cc], qf, s);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float e = fast_exp2(fmaf(s[r], p.scale, -lse[x]) * kLog2e);
                if (!whole && key0 + acc_row(r, h) > last[x]) e = 0.f;
                sum[r] += e;
            }
        }
    }
    // over the 32 lanes of a half; lane r of it keeps key acc_row(r, h)
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        float v = sum[r];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) v += __shfl_xor(v, off);
        if ((lane & 15) == r) mine = v;
    }
    const int at = acc_row(lane & 15, h);
    const bool key_there = __shfl((int)there, at) != 0;
    if (i < 16 && key0 + at < len) {
        const int64_t x = (int64_t)u * room + key0 + at;
        p.weight[x] = (p.before ? p.before[x] : 0.f) + (key_there ? mine : 0.f);
    }
}

int launch_paged_weigh(const void* Q, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* len, const int32_t* k,
                       const float* lse, int64_t lse_pitch, const zipvl_dims& d, float scale, const float* before, float* weight, hipStream_t st)
{
    const int G = d.Hq / d.Hkv;
    const Weigh p = {(const char*)pages.K, pages.num_pages, __builtin_ctz(pages.page), table, table_pages, len, k, (const char*)Q,
                     {d.q_strides[0], d.q_strides[1], d.q_strides[2]}, lse, lse_pitch, before, weight, d.Hq, d.Hkv, G, d.n, inverse(d.Hkv), inverse(G), scale};
    const dim3 grid((unsigned)(((int64_t)table_pages * pages.page + 127) / 128), d.B * d.Hkv);
    KernelTimer tm(ZIPVL_K_PAGED_WEIGH, st);
    if (d.dtype == ZIPVL_BF16) {
        if (d.d == 128) hipLaunchKernelGGL((paged_weigh_kernel<__bf16, 128>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((paged_weigh_kernel<__bf16, 64>), grid, dim3(256), 0, st, p);
    } else {
        if (d.d == 128) hipLaunchKernelGGL((paged_weigh_kernel<float, 128>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((paged_weigh_kernel<float, 64>), grid, dim3(256), 0, st, p);
    }
    return check_launch("paged_weigh");
}

}  // namespace zipvl
