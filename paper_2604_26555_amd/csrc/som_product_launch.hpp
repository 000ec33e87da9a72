// Launches of the products with the nodes' matrices: which kernels a call takes, runs, workspaces.
#pragma once

#include "som_product_few.hpp"

namespace som {

static bool sixteen(const void* p) { return (uintptr_t)p % 16 == 0; }

// Every row of every matrix starts at a multiple of sixteen bytes and holds whole chunks of them.
template <class T>
static bool product_aligned(const ProductArgs<T>& a)
{
    constexpr int E = 16 / sizeof(T);
    return a.din % E == 0 && a.dout % E == 0 && a.ldp % E == 0 && a.ldq % E == 0 && a.ldo % E == 0 && a.ldr % E == 0 && a.ldpre % E == 0 && sixteen(a.P) &&
           sixteen(a.Q) && sixteen(a.out) && sixteen(a.bias) && sixteen(a.residual) && sixteen(a.pre);
}

constexpr int64_t kTilesWide = 1 << 20;        // workgroups in a row of the grid (a multiple of eight: they go round the dies)

template <class T, Form F, int B, bool ALIGNED>
static int product_tile_launch(som_ctx* ctx, const ProductArgs<T>& a, const char* what)
{
    static bool attr_set_dev[kMaxDevices] = {};
    bool& attr_set = attr_set_dev[ctx->device];
    auto kern = product_tile_kernel<T, F, B, ALIGNED>;
    if (!attr_set) {
        if (int rc = check_hip(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, Tile<B>::LDS),
                               "raising the dynamic LDS limit"))
            return rc;
        attr_set = true;
    }
    const int64_t xtiles = ((F == kRowsTimesA ? a.dout : a.din) + B - 1) / B, high = F == kOuterSums ? (a.dout + B - 1) / B : 1, each = high * xtiles;
    const int64_t items = F == kOuterSums ? most_runs(a.rows, a.K, a.run) : most_tiles(a.rows, a.K, a.offsets, B);
    const int64_t groups = F != kOuterSums ? ((items * xtiles + 7) / 8 + 2) * 8 : each < 16 ? items * each : (each + 7) / 8 * 8 * items;
    // (a grid's dimension holds fewer than 2^32 work-items; the workgroups behind the last find no tile)
    const int64_t wide = groups < kTilesWide ? groups : kTilesWide, rows_of_grid = (groups + wide - 1) / wide;
    if (groups >= (int64_t)1 << 31) return fail(ctx, SOM_EINVAL, "%s: more than 2^31 tiles; call with fewer rows or nodes", what);
    hipLaunchKernelGGL(kern, dim3((unsigned)wide, (unsigned)rows_of_grid), dim3(Tile<B>::THREADS), Tile<B>::LDS, ctx->stream, a, (unsigned)xtiles);
    return check_hip(ctx, hipGetLastError(), what);
}

// Which tiles a call takes: the estimated time of each size in microseconds, from timed steps of 128 bytes of the contraction.
//   A workgroup alone on its unit takes 1.1, 0.65 and 0.47 us a step (16-bit; 256, 128 and 64 rows), as many as fit (Tile<B>::MOST) 1.6, 1.35
//   (two) and 1.0 (four; 0.74 where the caches hold all operands); float32 goes by its products alone: 7.3 and 2.05 us each, and for 64
//   rows 0.55 for one and 0.49 each for four.  Beside its steps a tile takes some 9, 6 and 4 us (float32 5).  Small tiles fill the chip
//   where there are few and waste less of narrow matrices, large ones read less: 65536 rows 2048 -> 1536 on 64 nodes 540, 633 and 954 us,
//   256 rows 4096 -> 4096 on one 80, 46 and 35, 250,013 rows 37 -> 24 in float32 on 437 nodes 148, 98 and 55.  Of 2447 products and gradients
//   drawn between 64 and 4096 wide, the size that this picks takes 1.7 % longer than the best one on average, and 108 take over 15 % longer.
template <class T, Form F>
static double tile_time(const som_ctx* ctx, const ProductArgs<T>& a, int B)
{
    const double rows = a.rows, groups = a.K < rows ? a.K : rows, across = ((F == kRowsTimesA ? a.dout : a.din) + B - 1) / B;
    const double cut = rows / a.run + (a.offsets ? 0.5 * a.K : 0.5), runs = F != kOuterSums ? 1.0 : cut > a.K ? cut : a.K;
    const double tall = a.offsets ? rows / B + 0.5 * groups : (a.rows + B - 1) / B;
    const double tiles = across * (F == kOuterSums ? runs * ((a.dout + B - 1) / B) : tall > groups ? tall : groups);
    const double depth = F == kRowsTimesA ? a.din : F == kRowsTimesAt ? a.dout : rows / runs;
    const double steps = 1.0 + depth * sizeof(T) / 128.0, more = B == 256 ? 9.0 : B == 128 ? 6.0 : sizeof(T) == 4 ? 5.0 : 4.0;
    const double most = B == 256 ? Tile<256>::MOST : B == 128 ? Tile<128>::MOST : Tile<64>::MOST;
    auto step = [&](double o) {                         // o workgroups on a unit
        if (sizeof(T) == 4) return B == 256 ? 7.3 : B == 128 ? 2.05 * o : 0.08 + 0.47 * o;
        return B == 256 ? 1.1 + 0.5 * o * o : B == 128 ? 0.65 + 0.7 * (o - 1.0) : 0.47 + 0.06 * (o - 1.0) * (o - 1.0);
    };
    const double rounds = tiles / (ctx->units * most), whole = (double)(int64_t)rounds, rest = (rounds - whole) * most;
    return whole * (steps * step(most) + more) + (rest > 0.0 ? steps * step(B == 256 ? rest : rest < 1.0 ? 1.0 : rest) + more : 0.0);
}

template <class T, Form F>
static double best_tile_time(const som_ctx* ctx, const ProductArgs<T>& a)
{
    const double t256 = tile_time<T, F>(ctx, a, 256), t128 = tile_time<T, F>(ctx, a, 128), t64 = tile_time<T, F>(ctx, a, 64);
    return t256 < t128 ? (t256 < t64 ? t256 : t64) : t128 < t64 ? t128 : t64;
}

template <class T, Form F>
static int product_launch(som_ctx* ctx, const ProductArgs<T>& a, const char* what)
{
    const double t256 = tile_time<T, F>(ctx, a, 256), t128 = tile_time<T, F>(ctx, a, 128), t64 = tile_time<T, F>(ctx, a, 64);
    const bool aligned = product_aligned(a);
    if (t256 <= t128 && t256 <= t64) return aligned ? product_tile_launch<T, F, 256, true>(ctx, a, what) : product_tile_launch<T, F, 256, false>(ctx, a, what);
    if (t128 <= t64) return aligned ? product_tile_launch<T, F, 128, true>(ctx, a, what) : product_tile_launch<T, F, 128, false>(ctx, a, what);
    return aligned ? product_tile_launch<T, F, 64, true>(ctx, a, what) : product_tile_launch<T, F, 64, false>(ctx, a, what);
}

template <class T>
int product_typed(som_ctx* ctx, const NodeProduct& p)
{
    ProductArgs<T> a{};
    a.P = (const T*)p.X;
    a.ldp = p.ldx;
    a.Q = (const T*)p.A;
    a.offsets = p.offsets;
    a.rows = (int)p.rows;
    a.K = p.K;
    a.din = p.din;
    a.dout = p.dout;
    a.bias = (const T*)p.bias;
    a.residual = (const T*)p.residual;
    a.ldr = p.residual ? p.ldr : 0;
    a.pre = (T*)p.pre;
    a.ldpre = p.pre ? p.ldpre : 0;
    a.out = (T*)p.out;
    a.ldo = p.ldo;
    a.act = p.act;
    if (product_narrow<T>(p.dout, p.din)) return product_narrow_launch<T, false>(ctx, a, "product launch");
    if (product_few(a)) return product_few_launch(ctx, a, "product launch");
    // The last rows of one node, where they would start another round of tiles: as few rows of their own (64 are the most that one workgroup
    // of that kernel takes), in about the time that the matrix takes to come at 4 TB/s (4099 x 4096 x 4096 f16: 177 us in tiles, 141 with three
    // rows apart; 64 rows of 4096 -> 4096 take 23 us there).
    const int last = a.rows % 256;
    if (!a.offsets && a.rows > 256 && last > 0 && last <= 64) {
        ProductArgs<T> whole = a, rest = a;
        whole.rows = a.rows - last;
        rest.rows = last;
        rest.P = a.P + whole.rows * a.ldp;
        rest.out = a.out + whole.rows * a.ldo;
        if (a.residual) rest.residual = a.residual + whole.rows * a.ldr;
        if (a.pre) rest.pre = a.pre + whole.rows * a.ldpre;
        const double apart = 6.0 + (double)a.dout * a.din * sizeof(T) / 4e6;
        if (product_few(rest) && best_tile_time<T, kRowsTimesA>(ctx, whole) + apart < best_tile_time<T, kRowsTimesA>(ctx, a)) {
            if (int rc = product_launch<T, kRowsTimesA>(ctx, whole, "product launch")) return rc;
            return product_few_launch(ctx, rest, "product launch");
        }
    }
    return product_launch<T, kRowsTimesA>(ctx, a, "product launch");
}

// Kernel, lanes of a row and columns of a workgroup for the slopes and biases of `dout` columns.
template <class T>
static auto slope_kernel_for(int32_t dout, int& lanes, int& columns)
{
    constexpr int N = Piece<T>::N;
    lanes = dout < N ? row_lanes(dout, 8) : row_lanes((dout + N - 1) / N, 64);
    columns = lanes * (dout < N ? 1 : N);
    if (dout < N) return lanes == 1 ? slope_kernel<T, 1, 1> : lanes == 2 ? slope_kernel<T, 1, 2> : lanes == 4 ? slope_kernel<T, 1, 4> : slope_kernel<T, 1, 8>;
    return lanes == 1   ? slope_kernel<T, N, 1>
           : lanes == 2 ? slope_kernel<T, N, 2>
           : lanes == 4 ? slope_kernel<T, N, 4>
           : lanes == 8 ? slope_kernel<T, N, 8>
           : lanes == 16 ? slope_kernel<T, N, 16>
           : lanes == 32 ? slope_kernel<T, N, 32>
                         : slope_kernel<T, N, 64>;
}

template <class T>
static int runs_join(som_ctx* ctx, const int32_t* offsets, int32_t K, int64_t rows, int run, const float* parts, int64_t count, T* out)
{
    const int64_t longer = rows / ((int64_t)run + 1), y = longer < K ? longer : K;        // groups with more than one run, at most
    if (y == 0) return SOM_OK;
    // few values: by many lanes where a group can have many runs (one node's 1024 runs of 1536: 52 us by 256 lanes, 14 by 1024; 437 nodes'
    // of 888, next to none of which has more than one: 7 and 18)
    if (count <= 16384 && K > 8) {
        hipLaunchKernelGGL((runs_join_kernel<T, 4>), dim3((unsigned)((count + 63) / 64), (unsigned)y), dim3(256), 0, ctx->stream, offsets, K, (int)rows,
                           run, parts, count, out);
    } else if (count <= 16384) {
        hipLaunchKernelGGL((runs_join_kernel<T, 16>), dim3((unsigned)((count + 63) / 64), (unsigned)y), dim3(1024), 0, ctx->stream, offsets, K, (int)rows,
                           run, parts, count, out);
    } else {
        const int64_t blocks = (count + 255) / 256, share = 16 * ctx->units / y + 1;       // (most of the y find no group)
        hipLaunchKernelGGL((runs_join_kernel<T, 1>), dim3((unsigned)(blocks < share ? blocks : share), (unsigned)y), dim3(256), 0, ctx->stream, offsets, K,
                           (int)rows, run, parts, count, out);
    }
    return check_hip(ctx, hipGetLastError(), "product gradient join launch");
}

template <class T>
int product_grad_typed(som_ctx* ctx, const NodeProductGrad& p)
{
    ProductArgs<T> a{};
    a.offsets = p.offsets;
    a.rows = (int)p.rows;
    a.K = p.K;
    a.din = p.din;
    a.dout = p.dout;
    // What applies the slopes: narrow kernels as they read dY; else a pass that stores dz (and sums the biases).
    const bool sloped = p.act != SOM_ACT_NONE && p.rows > 0, narrow_rows = product_narrow<T>(p.din, p.dout);
    const bool narrow_both = narrow_rows && p.dout <= kNarrow;
    const bool stored = sloped && !narrow_both && (p.dA || p.dbias || !narrow_rows);
    int lanes, columns;
    auto slopes = slope_kernel_for<T>(p.dout, lanes, columns);
    const int64_t blocks = (p.dout + columns - 1) / columns;
    a.run = narrow_both ? narrow_run(ctx, p.rows, gradient_narrow_most<T>(p.dout, p.din))
                        : run_rows(ctx, p.rows, p.K, (int64_t)((p.dout + 255) / 256) * ((p.din + 255) / 256), 512);
    const int bias_run = narrow_both ? a.run : 4096 / lanes;               // (else four rows at a time and lane, four times)
    // workspace: dz, the runs' sums of the matrices, those of the biases
    auto pieces = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    const size_t dz_bytes = stored ? pieces((size_t)p.rows * p.dout * sizeof(T)) : 0;
    const size_t sum_bytes = p.dA && p.rows > a.run ? pieces((size_t)run_slots(p.rows, a.run) * p.dout * p.din * sizeof(float)) : 0;
    const size_t bias_bytes = p.dbias && p.rows > bias_run ? (size_t)run_slots(p.rows, bias_run) * p.dout * sizeof(float) : 0;
    if (dz_bytes + sum_bytes + bias_bytes)
        if (int rc = models_workspace(ctx, dz_bytes + sum_bytes + bias_bytes)) return rc;
    T* dz = (T*)ctx->models_blob;
    a.parts = (float*)((char*)ctx->models_blob + dz_bytes);
    float* bias_parts = (float*)((char*)a.parts + sum_bytes);
    if (narrow_both && (p.dA || p.dbias || p.rows > 0)) {
        GradientArgs<T> g{(const T*)p.dY, p.lddy, (const T*)p.X, p.ldx, (const T*)p.A, (const T*)p.pre, p.ldpre, p.offsets, (int)p.rows, p.K, p.din, p.dout,
                          p.act, a.run, (T*)p.dX, p.lddx, (T*)p.dA, (T*)p.dbias, a.parts, bias_parts};
        if (int rc = gradient_narrow_launch(ctx, g)) return rc;
    }
    if (!narrow_both && (stored || p.dbias)) {
        const int64_t runs = most_runs(p.rows, p.K, bias_run), y = runs < 32768 ? runs : 32768;
        hipLaunchKernelGGL(slopes, dim3((unsigned)blocks, (unsigned)y, (unsigned)((runs + y - 1) / y)), dim3(256), 0, ctx->stream, (const T*)p.dY, p.lddy,
                           (const T*)p.pre, p.ldpre, p.offsets, p.K, (int)p.rows, p.dout, p.act, stored ? dz : nullptr, (T*)p.dbias, bias_run, bias_parts);
        if (int rc = check_hip(ctx, hipGetLastError(), "product gradient slope launch")) return rc;
    }
    a.P = stored ? dz : (const T*)p.dY;
    a.ldp = stored ? p.dout : p.lddy;
    a.act = stored ? SOM_ACT_NONE : p.act;
    if (a.act != SOM_ACT_NONE) {                        // (else no kernel below reads pre, and how it lies is of no account)
        a.pre = (T*)p.pre;
        a.ldpre = p.ldpre;
    }
    if (!narrow_both && p.dX && p.rows > 0) {
        a.Q = (const T*)p.A;
        a.out = (T*)p.dX;
        a.ldo = p.lddx;
        int rc = SOM_OK;
        if constexpr (sizeof(T) == 2) {
            if (narrow_rows) rc = product_narrow_launch<T, true>(ctx, a, "product gradient (rows) launch");
        }
        if (!narrow_rows) rc = product_launch<T, kRowsTimesAt>(ctx, a, "product gradient (rows) launch");     // (narrow floats: done above)
        if (rc) return rc;
    }
    a.Q = (const T*)p.X;
    a.ldq = p.ldx;
    a.out = (T*)p.dA;
    a.ldo = p.din;
    if (!narrow_both && p.dA)
        if (int rc = product_launch<T, kOuterSums>(ctx, a, "product gradient (matrices) launch")) return rc;
    if (bias_bytes)
        if (int rc = runs_join(ctx, p.offsets, p.K, p.rows, bias_run, bias_parts, p.dout, (T*)p.dbias)) return rc;
    if (sum_bytes) return runs_join(ctx, p.offsets, p.K, p.rows, a.run, a.parts, (int64_t)p.dout * p.din, (T*)p.dA);
    return SOM_OK;
}

} // namespace som
