// Decode attention over pages, with prefixes that several batch elements share (Eq. (5); Algorithm 2).
#include "launch.h"
#include "rowops.h"

namespace zipvl {

struct PagedRead {
    const char *K, *V;
    int num_pages, page_log2;
    const int32_t* table; int width; const int32_t* len;
    const int32_t* prefix_table; int prefix_width; const int32_t* prefix_len;
    const int32_t* group_begin; int groups;
};

// The simplest form: a workgroup for every query head, which goes through the rows of the prefix and then its own, 16 lanes a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_head_kernel(const T* __restrict__ q, PagedRead p, int B, int Hq, int Hkv, float c, T* __restrict__ o) {
    constexpr int EPL = D / 16;
    __shared__ float red[16][D + 2];
    __shared__ int found;
    const int b = blockIdx.x / Hq, h = blockIdx.x - b * Hq, g = h / (Hq / Hkv);
    const int sub = threadIdx.x & 15, rg = threadIdx.x >> 4;
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    for (int x = threadIdx.x; x < p.groups; x += 256)
        if (p.group_begin[x] <= b && b < p.group_begin[x + 1]) found = x;
    __syncthreads();
    float qv[EPL], ov[EPL], m = -INFINITY, l = 0.f;
    RowChunk<T, EPL>::load(q + (int64_t)blockIdx.x * D + sub * EPL, qv);
#pragma unroll
    for (int e = 0; e < EPL; ++e) { qv[e] *= c; ov[e] = 0.f; }
    auto part = [&](const int32_t* table, int width, int length) {
        length = max(0, min(length, width << p.page_log2));
        for (int r0 = 0; r0 < length; r0 += 16) {
            const int r = min(r0 + rg, length - 1), page = table[r >> p.page_log2];
            const bool valid = r0 + rg < length && (unsigned)page < (unsigned)p.num_pages;
            const int64_t at = valid ? (((int64_t)page << p.page_log2) + (r & ((1 << p.page_log2) - 1))) * D : 0;
            float kf[EPL], vf[EPL];
            RowChunk<T, EPL>::load((const T*)p.K + at + sub * EPL, kf);
            RowChunk<T, EPL>::load((const T*)p.V + at + sub * EPL, vf);
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) s += qv[e] * kf[e];
            s += __shfl_xor(s, 1); s += __shfl_xor(s, 2); s += __shfl_xor(s, 4); s += __shfl_xor(s, 8);
            if (valid) {
                const float mn = fmaxf(m, s), a = fast_exp2(m - mn), w = fast_exp2(s - mn);
                l = l * a + w;
#pragma unroll
                for (int e = 0; e < EPL; ++e) ov[e] = ov[e] * a + w * vf[e];
                m = mn;
            }
        }
    };
    if (found >= 0) part(p.prefix_table + (int64_t)(found * Hkv + g) * p.prefix_width, p.prefix_width, p.prefix_len[found * Hkv + g]);
    part(p.table + (int64_t)(b * Hkv + g) * p.width, p.width, p.len[b * Hkv + g]);
#pragma unroll
    for (int e = 0; e < EPL; ++e) red[rg][sub * EPL + e] = ov[e];
    if (sub == 0) { red[rg][D] = m; red[rg][D + 1] = l; }
    __syncthreads();
    if (threadIdx.x < D) {
        float M = -INFINITY, sum = 0.f, acc = 0.f;
        for (int x = 0; x < 16; ++x) M = fmaxf(M, red[x][D]);
        for (int x = 0; x < 16; ++x) {
            const float a = M > -INFINITY ? fast_exp2(red[x][D] - M) : 0.f;
            sum += a * red[x][D + 1];
            acc += a * red[x][threadIdx.x];
        }
        o[(int64_t)blockIdx.x * D + threadIdx.x] = (T)(sum > 0.f ? acc / sum : 0.f);
    }
}

size_t decode_paged_workspace_bytes(const zipvl_dims& d, int own, int prefix) { return 16; }

int launch_decode_attn_paged(const void* q, const zipvl_pages& pages, const int32_t* table, int32_t table_pages, const int32_t* len,
                             const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_len, const int32_t* group_begin,
                             int32_t groups, const zipvl_dims& d, float scale, void* o, void* ws, hipStream_t st)
{
    const PagedRead p = {(const char*)pages.K, (const char*)pages.V, pages.num_pages, __builtin_ctz(pages.page), table, table_pages, len,
                         prefix_table, prefix_pages, prefix_len, group_begin, groups};
    KernelTimer tm(ZIPVL_K_PAGED_PARTIAL, st);
#define ZIPVL_PAGED(T, D) \
    hipLaunchKernelGGL((paged_head_kernel<T, D>), dim3(d.B * d.Hq), dim3(256), 0, st, (const T*)q, p, d.B, d.Hq, d.Hkv, scale * kLog2e, (T*)o)
    if (d.dtype == ZIPVL_BF16) { if (d.d == 128) ZIPVL_PAGED(__bf16, 128); else ZIPVL_PAGED(__bf16, 64); }
    else { if (d.d == 128) ZIPVL_PAGED(float, 128); else ZIPVL_PAGED(float, 64); }
#undef ZIPVL_PAGED
    return check_launch("decode_attn_paged");
}

}  // namespace zipvl
