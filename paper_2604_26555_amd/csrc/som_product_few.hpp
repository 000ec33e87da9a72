// Products of few rows a node (single rows of a serving loop and small batches): what counts is that the matrices are read once, at the memory's rate.
#pragma once

#include "som_product_narrow.hpp"

namespace som {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[s], c, 0, 0, 0);
    return c;
}

// Sixteen results of up to R blocks of sixteen rows of a group: eight wavefronts share the contraction, 256 bytes of every row at a time (four
// chunks of four lanes for each of sixteen rows), straight from memory in the matrix pipe's order, and their sums meet in LDS.  A longer group's
// rows go to several workgroups, which follow one another and take the matrix from the cache again: however uneven the groups are, none
// holds the others up (10,000 rows 2048 -> 1024 bf16 all on one of 1000 nodes: 674 us, spread over them 1087, and 2586 and 1182 with one
// workgroup for all of a group's rows).  Rows and results behind the last are copies of it and are not stored.
template <class T, int R>
__global__ void __launch_bounds__(512) product_few_kernel(ProductArgs<T> a, unsigned xtiles)
{
    typedef typename Fragment<T>::type Frag;
    typedef Frag Any __attribute__((aligned(sizeof(T))));
    constexpr int E = 16 / sizeof(T), kStep = 256 / sizeof(T);
    __shared__ f32x4 sums[8][R][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 15, c = lane >> 4;
    int which, first, end;
    const int e = find_group<512>(a.offsets, a.K, a.rows, [](unsigned n) { return (n + 16 * R - 1) / (16 * R); }, blockIdx.x / xtiles, which);
    if (e < 0) return;
    group_rows(a.offsets, e, a.rows, first, end);
    const int n0 = (int)(blockIdx.x % xtiles) * 16, r0 = first + 16 * R * which, depth = a.din, whole = depth / kStep;
    const T* A = a.Q + ((int64_t)e * a.dout + (n0 + l < a.dout ? n0 + l : a.dout - 1)) * depth;
    const T* X[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = r0 + 16 * r + l < end ? r0 + 16 * r + l : end - 1;
        X[r] = a.P + (int64_t)row * a.ldp;
    }
    f32x4 acc[R] = {};
#pragma unroll 2
    for (int s = wave; s < whole; s += 8) {
        Frag w[4], x[R][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = *reinterpret_cast<const Any*>(A + s * kStep + (4 * u + c) * E);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int u = 0; u < 4; ++u) x[r][u] = *reinterpret_cast<const Any*>(X[r] + s * kStep + (4 * u + c) * E);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r] = mfma16(w[u], x[r][u], acc[r]);
    }
    if (whole * kStep < depth && wave == whole % 8) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const Frag w = row_chunk(A, 16 * whole + 4 * u + c, depth, true);
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r] = mfma16(w, row_chunk(X[r], 16 * whole + 4 * u + c, depth, true), acc[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) sums[wave][r][lane] = acc[r];
    __syncthreads();
    // a lane of the pipe has row l, results 4 c .. + 3
    for (int i = threadIdx.x; i < 256 * R; i += 512) {
        const int n = n0 + (i & 15), m = i >> 4, r = m >> 4, from = (i & 15) >> 2, j = i & 3;
        const int64_t row = r0 + m;
        if (n >= a.dout || row >= end) continue;
        float x[1] = {0.0f};
#pragma unroll
        for (int w = 0; w < 8; ++w) x[0] += sums[w][r][16 * from + (m & 15)][j];
        if (a.bias) x[0] += (float)a.bias[(int64_t)e * a.dout + n];
        if (a.pre) a.pre[row * a.ldpre + n] = (T)x[0];
        activate<T>(x, a.act);
        if (a.residual) x[0] += (float)a.residual[row * a.ldr + n];
        a.out[row * a.ldo + n] = (T)x[0];
    }
}

// Where the matrices' bytes decide: up to 64 rows of one node (4096 -> 4096 bf16: 1 row 31 us by tiles of 64 and 11 like this, 64 rows 34 and 23),
// and up to 10 of several on average, of 512 bytes and more (2048 -> 1536 bf16 on 64 nodes: 4 rows each 96 and 88 us, but 32 each 101 and
// 203, as every sixteen results bring all rows).  A workgroup reads sixteen rows of a matrix: where that is little and there are many
// workgroups, their starts count.  Of 226 products drawn with up to 10 rows a node, time against that of tiles, geometric means:
//   rows of      512 to 1024 bytes: 0.95 up to 2048 workgroups, 1.33 from there to 4096, 1.36 beyond;   1024 to 2200: 0.87, 0.83, 1.07
//               2200 to 4096: 0.66, 0.84, 0.98;   4096 to 20,000: 0.42, 0.85, 0.93
// so 3000 workgroups, or any number of them for rows of 2500 bytes: 1.5 % above the better of the two on average (2048 and 4096: 2.2 %; 6000
// and 2500: 1.9 %; 3000 and 1024: 2.0 %).
template <class T>
static bool product_few(const ProductArgs<T>& a)
{
    const int64_t groups = a.offsets ? (a.K < a.rows ? a.K : a.rows) : 1, bytes = a.din * (int64_t)sizeof(T), all = groups * ((a.dout + 15) / 16);
    return a.rows <= (a.K > 1 ? 10 : 64) * groups && bytes >= 512 && (all <= 3000 || bytes >= 2500) && all < 1 << 22;
}

template <class T>
static int product_few_launch(som_ctx* ctx, const ProductArgs<T>& a, const char* what)
{
    const unsigned xtiles = (unsigned)((a.dout + 15) / 16);
    const int rows = a.K > 1 || a.rows <= 16 ? 16 : a.rows <= 32 ? 32 : 64;               // of a workgroup
    auto kern = rows == 16 ? product_few_kernel<T, 1> : rows == 32 ? product_few_kernel<T, 2> : product_few_kernel<T, 4>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(most_tiles(a.rows, a.K, a.offsets, rows) * xtiles)), dim3(512), 0, ctx->stream, a, xtiles);
    return check_hip(ctx, hipGetLastError(), what);
}

} // namespace som
