// Products of narrow rows: up to 64 results and 256 bytes of the contraction (64 floats, 128 16-bit values), as the local models of a table
// have them.  What bounds them is memory; a node's matrix stays in a wavefront's registers, rows pass through LDS that is the wavefront's own, and
// there is no barrier on the way.
#pragma once

#include "som_product_tile.hpp"

namespace som {

constexpr int kNarrow = 64;               // results at most
constexpr int kNarrowBytes = 256;         // of the contraction at most

// Chunk c of a row of `depth` values, zeros behind its end.  A chunk that the row's end cuts is read as the row's last sixteen bytes, the values that
// the chunk before has zeroed; a row shorter than a chunk value by value.
template <class T>
__device__ __forceinline__ typename Fragment<T>::type row_chunk(const T* __restrict__ row, int c, int depth, bool there)
{
    constexpr int E = 16 / sizeof(T);
    typedef typename Fragment<T>::type Frag;
    typedef Frag any __attribute__((aligned(sizeof(T))));
    const int at = c * E;
    Frag f = {};
    if (!there || at >= depth) return f;
    if (depth < E) {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (j < depth) f[j] = row[j];
        return f;
    }
    const int again = at + E > depth ? at + E - depth : 0;
    f = *reinterpret_cast<const any*>(row + at - again);
    if (again) {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (j < again) f[j] = (T)0.0f;
    }
    return f;
}

// Rows of a group times its matrix (AT: dz = P slopes(pre) times the matrix's transpose): a workgroup takes up to `chunk` rows of a group, each of
// its four wavefronts every fourth block of 32, on its own.  V: blocks of 32 results, S: steps of 32 bytes of the contraction.  Rows come
// and go in the order of memory, sixteen bytes a lane, through LDS that is the wavefront's own; the next block's are asked for ahead.  (Straight
// from memory in the matrix pipe's order, 32 bytes of each of 32 rows at a time, 200,000 rows 64 -> 64 bf16 took 41 us, 21 like this.)
template <class T, bool AT, int V, int S>
__global__ void __launch_bounds__(256) product_narrow_kernel(ProductArgs<T> a, int chunk)
{
    typedef typename Fragment<T>::type Frag;
    typedef Frag Any __attribute__((aligned(sizeof(T))));
    constexpr int E = 16 / sizeof(T), kRow = 2 * S + 1, kOut = 32 * V + 4;      // LDS rows in chunks (odd) and floats: sixteen lanes meet all banks
    constexpr int kBytes = 32 * (kRow * 16 > kOut * 4 ? kRow * 16 : kOut * 4);
    __shared__ __align__(16) char lds[4][kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    int which, lo, end;
    const int e = find_group<256>(a.offsets, a.K, a.rows, [chunk](unsigned n) { return (n + chunk - 1) / chunk; }, blockIdx.x, which);
    if (e < 0) return;
    group_rows(a.offsets, e, a.rows, lo, end);
    lo += which * chunk;
    end = end - lo > chunk ? lo + chunk : end;
    const int Nn = AT ? a.din : a.dout, depth = AT ? a.dout : a.din;
    const T* A = a.Q + (int64_t)e * a.dout * a.din;
    char* mine = lds[wave];
    // chunk number lane + 64 i of a block's, in the order of memory: its row, its place in the row and in LDS
    const int chunks = (depth + E - 1) / E;
    int row_of[S], from[S], again[S], in_p[S], in_z[AT ? S : 1];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int c = lane + 64 * i;
        row_of[i] = c / chunks;
        const int at = (c - row_of[i] * chunks) * E;
        again[i] = depth >= E && at + E > depth ? at + E - depth : 0;
        from[i] = at - again[i];
        in_p[i] = row_of[i] * (int)a.ldp + from[i];          // (32 rows of at most 2^21 values)
        if (AT) in_z[i] = row_of[i] * (int)a.ldpre + from[i];
    }
    Frag next[S], zs[AT ? S : 1];
    auto fetch = [&](int b) __attribute__((always_inline)) {
        const int64_t row0 = lo + 32 * (int64_t)b;
        const int left = end - lo - 32 * b;
        const T *p = a.P + row0 * a.ldp, *z = AT ? a.pre + row0 * a.ldpre : nullptr;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            next[i] = Frag{};
            if constexpr (AT) zs[i] = Frag{};
            if (row_of[i] >= 32 || row_of[i] >= left) continue;
            if (depth >= E) {
                next[i] = *reinterpret_cast<const Any*>(p + in_p[i]);
                if constexpr (AT)
                    if (a.act) zs[i] = *reinterpret_cast<const Any*>(z + in_z[i]);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (j < depth) next[i][j] = p[in_p[i] + j];
                    if constexpr (AT)
                        if (a.act && j < depth) zs[i][j] = z[in_z[i] + j];
                }
            }
        }
    };
    fetch(wave);                                      // (on their way while the matrix comes)
    Frag q[V][S];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int n = 32 * v + (lane & 31);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if constexpr (AT) {
#pragma unroll
                for (int j = 0; j < E; ++j) {                       // (where the chunks hold the values of dz)
                    const int at = (2 * s + h) * E, again = depth >= E && at + E > depth ? at + E - depth : 0, k = at - again + j;
                    q[v][s][j] = n < Nn && at < depth && j >= again && k < depth ? A[(int64_t)k * a.din + n] : (T)0.0f;
                }
            } else {
                q[v][s] = row_chunk(A + (int64_t)n * a.din, 2 * s + h, depth, n < Nn);
            }
        }
    }
    for (int b = wave; lo + 32 * b < end; b += 4) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            Frag x = next[i];
            if constexpr (AT) {
                if (a.act) {
                    Piece<T> g = __builtin_bit_cast(Piece<T>, x);
                    slopes<T, E>(g, __builtin_bit_cast(Piece<T>, zs[i]), a.act);
                    x = __builtin_bit_cast(Frag, g);
                }
            }
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = j < again[i] ? (T)0.0f : x[j];
            if (row_of[i] < 32) *reinterpret_cast<Frag*>(mine + (row_of[i] * kRow + (from[i] + again[i]) / E) * 16) = x;
        }
        wave_in_order();
        fetch(b + 4);
        f32x16 acc[V] = {};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            Frag p = {};
            if (2 * s + h < chunks) p = *reinterpret_cast<const Frag*>(mine + ((lane & 31) * kRow + 2 * s + h) * 16);
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = mfma(q[v][s], p, acc[v]);
        }
        // a lane has its row's results, four consecutive ones at a time; they go out in the order of memory
        float* turned = reinterpret_cast<float*>(mine);
        wave_in_order();
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(turned + (lane & 31) * kOut + 32 * v + 8 * g + 4 * h) =
                    make_float4(acc[v][4 * g], acc[v][4 * g + 1], acc[v][4 * g + 2], acc[v][4 * g + 3]);
        wave_in_order();
        constexpr int G = E;                              // results of a lane at a time
        const int groups = (Nn + G - 1) / G;
#pragma unroll 1
        for (int i = lane; i < 32 * groups; i += 64) {
            const int r = i / groups, n0 = (i - r * groups) * G, n = Nn >= G && n0 + G > Nn ? Nn - G : n0, some = Nn < G ? Nn : G;
            const int64_t row = lo + 32 * (int64_t)b + r;
            if (row >= end) break;
            float x[G];
#pragma unroll
            for (int j = 0; j < G; ++j) x[j] = turned[r * kOut + n + j];
            typedef Piece<T, G> Some;
            auto load = [&](Some& y, const T* p) __attribute__((always_inline)) {
                if (some == G) y.load(p);
                else
#pragma unroll
                    for (int j = 0; j < G; ++j) y.e[j] = j < some ? p[j] : (T)0.0f;
            };
            auto store = [&](const Some& y, T* p) __attribute__((always_inline)) {
                if (some == G) y.store(p);
                else
#pragma unroll
                    for (int j = 0; j < G; ++j)
                        if (j < some) p[j] = y.e[j];
            };
            Some y, z;
            if (!AT) {
                if (a.bias) {
                    load(y, a.bias + (int64_t)e * a.dout + n);
#pragma unroll
                    for (int j = 0; j < G; ++j) x[j] += (float)y.e[j];
                }
                if (a.pre) {
#pragma unroll
                    for (int j = 0; j < G; ++j) z.e[j] = (T)x[j];
                    store(z, a.pre + row * a.ldpre + n);
                }
                activate<T>(x, a.act);
                if (a.residual) {
                    load(y, a.residual + row * a.ldr + n);
#pragma unroll
                    for (int j = 0; j < G; ++j) x[j] += (float)y.e[j];
                }
            }
#pragma unroll
            for (int j = 0; j < G; ++j) y.e[j] = (T)x[j];
            store(y, a.out + row * a.ldo + n);
        }
        wave_in_order();
    }
}

// Sums over a run of a group's rows of float32: dA (out not null) and dbias (likewise) at once, slopes applied on the way.  Four wavefronts take
// every fourth block of eight rows; U and V: blocks of 32 results and features.
template <int U, int V>
__global__ void __launch_bounds__(256) sums_narrow_kernel(ProductArgs<float> a, float* __restrict__ dbias, float* __restrict__ bias_parts)
{
    constexpr int kAhead = 4;             // blocks of rows that are on their way together
    __shared__ float sums[4][V * 16][64];
    __shared__ float bias_sums[4][U * 32];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, l = lane & 31;
    int which, first, end;
    const int run = a.run;
    const int e = find_group<256>(a.offsets, a.K, a.rows, [run](unsigned n) { return runs_of(n, run); }, blockIdx.x, which);
    if (e < 0) return;
    group_rows(a.offsets, e, a.rows, first, end);
    const int lo = first, group = end - first;
    first += which * run;
    end = end - first > run ? first + run : end;
    f32x16 acc[U][V] = {};
    float bias[U] = {};
    int in_p[4], in_z[4], in_q[4];                    // a lane's rows of a block of eight (at most 2^21 values each)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        in_p[s] = (4 * h + s) * (int)a.ldp + l;
        in_z[s] = (4 * h + s) * (int)a.ldpre + l;
        in_q[s] = (4 * h + s) * (int)a.ldq + l;
    }
    for (int b0 = wave; first + 8 * b0 < end; b0 += 4 * kAhead) {
        f32x4 p[kAhead][U], z[kAhead][U], q[kAhead][V];
#pragma unroll
        for (int w = 0; w < kAhead; ++w) {
            const int64_t row0 = first + 8 * (int64_t)(b0 + 4 * w);
            const int left = end - first - 8 * (b0 + 4 * w);
            const float *P = a.P + row0 * a.ldp, *Z = a.pre + row0 * a.ldpre, *Q = a.Q + row0 * a.ldq;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bool there = 4 * h + s < left;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool ours = there && 32 * u + l < a.dout;
                    p[w][u][s] = ours ? P[in_p[s] + 32 * u] : 0.0f;
                    if (a.act) z[w][u][s] = ours ? Z[in_z[s] + 32 * u] : 0.0f;
                }
#pragma unroll
                for (int v = 0; v < V; ++v) q[w][v][s] = a.out && there && 32 * v + l < a.din ? Q[in_q[s] + 32 * v] : 0.0f;
            }
        }
#pragma unroll
        for (int w = 0; w < kAhead; ++w) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (a.act) {
                    Piece<float> g = __builtin_bit_cast(Piece<float>, p[w][u]);
                    slopes<float, 4>(g, __builtin_bit_cast(Piece<float>, z[w][u]), a.act);
                    p[w][u] = __builtin_bit_cast(f32x4, g);
                }
                bias[u] += (p[w][u][0] + p[w][u][1]) + (p[w][u][2] + p[w][u][3]);
#pragma unroll
                for (int v = 0; v < V; ++v) acc[u][v] = mfma(q[w][v], p[w][u], acc[u][v]);
            }
        }
    }
    const int64_t slot = group > run ? run_slot(first, lo, run) : -1, count = (int64_t)a.dout * a.din;
    float* out = slot < 0 ? a.out + e * count : a.parts + slot * count;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int r = 0; r < 16; ++r) sums[wave][v * 16 + r][lane] = acc[u][v][r];
        bias[u] += __shfl_xor(bias[u], 32);
        if (h == 0) bias_sums[wave][32 * u + l] = bias[u];
        __syncthreads();
        for (int i = threadIdx.x; a.out && i < V * 1024; i += 256) {
            const int t = i & 63, r = (i >> 6) & 15, c = i >> 6;
            const int m = 32 * u + (t & 31), n = 32 * (i >> 10) + (r & 3) + 8 * (r >> 2) + 4 * (t >> 5);
            if (m < a.dout && n < a.din) out[(int64_t)m * a.din + n] = (sums[0][c][t] + sums[1][c][t]) + (sums[2][c][t] + sums[3][c][t]);
        }
        __syncthreads();
    }
    if (dbias && (int)threadIdx.x < a.dout) {
        const int m = threadIdx.x;
        float* to = slot < 0 ? dbias + (int64_t)e * a.dout : bias_parts + slot * a.dout;
        to[m] = (bias_sums[0][m] + bias_sums[1][m]) + (bias_sums[2][m] + bias_sums[3][m]);
    }
}

// Tiles of `bm` rows that the groups can have together.
static int64_t most_tiles(int64_t rows, int32_t K, const int32_t* offsets, int bm)
{
    const int64_t full = (rows + bm - 1) / bm;
    return offsets ? full + (K < rows ? K : rows) : full;
}

// Runs of `run` rows that the groups can have together.
static int64_t most_runs(int64_t rows, int32_t K, int run) { return rows / run + K; }

// Rows a run of a sum over rows when a group alone gives `tiles` workgroups: one run a group where the groups fill the chip (longer ones
// only for a group of four times its share), shorter ones where they do not.
static int run_rows(const som_ctx* ctx, int64_t rows, int32_t K, int64_t tiles, int least)
{
    const int64_t share = (rows + K - 1) / K, runs = ctx->units / (K * tiles > ctx->units ? ctx->units : K * tiles);
    int64_t run = runs > 1 ? (share + runs - 1) / runs : K > 1 ? 4 * share : rows;
    if (runs <= 1 && run < 2048) run = 2048;
    if (run < least) run = least;
    if (run * 32000 < rows) run = rows / 32000 + 1;             // (a grid's third dimension)
    return (int)((run + 63) / 64 * 64 < 0x7fffffc0 ? (run + 63) / 64 * 64 : 0x7fffffc0);
}

// Rows of a run of narrow sums: runs that fill the chip twice, or a group's rows at once where the groups do (but no more than twice its share).
static int narrow_run(const som_ctx* ctx, int64_t rows, int32_t K)
{
    const int64_t share = (rows + K - 1) / K, runs = 2 * (int64_t)ctx->units / K, run = runs > 1 ? (share + runs - 1) / runs : 2 * share;
    const int64_t at_least = run < 256 ? 256 : run;
    return (int)(at_least < 0x7fffffc0 ? at_least : 0x7fffffc0);
}

template <class T, bool AT>
static int product_narrow_launch(som_ctx* ctx, const ProductArgs<T>& a, const char* what)
{
    const int Nn = AT ? a.din : a.dout, steps = (int)(((AT ? a.dout : a.din) * sizeof(T) + 31) / 32);
    auto kern = Nn <= 32 ? (steps <= 2   ? product_narrow_kernel<T, AT, 1, 2>
                            : steps <= 4 ? product_narrow_kernel<T, AT, 1, 4>
                                         : product_narrow_kernel<T, AT, 1, 8>)
                         : (steps <= 2   ? product_narrow_kernel<T, AT, 2, 2>
                            : steps <= 4 ? product_narrow_kernel<T, AT, 2, 4>
                                         : product_narrow_kernel<T, AT, 2, 8>);
    // Rows of a workgroup: long enough that the matrix and the search for it don't count, short enough to fill the chip four times (500,000
    // rows 64 -> 32 bf16 on 100 nodes: 512 rows 23 us, 1024 rows 29)
    int64_t chunk = (a.rows / (ctx->units * 4) + 127) / 128 * 128;
    chunk = chunk < 128 ? 128 : chunk > 1024 ? 1024 : chunk;
    hipLaunchKernelGGL(kern, dim3((unsigned)most_tiles(a.rows, a.K, a.offsets, (int)chunk)), dim3(256), 0, ctx->stream, a, (int)chunk);
    return check_hip(ctx, hipGetLastError(), what);
}

template <class T>
static bool product_narrow(int32_t results, int32_t depth)
{
    return results <= kNarrow && depth * (int64_t)sizeof(T) <= kNarrowBytes;
}

} // namespace som
