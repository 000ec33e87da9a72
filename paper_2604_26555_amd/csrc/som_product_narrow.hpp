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

// Rows of a group times its matrix (AT: dz = P slopes(pre) times the matrix's transpose, for 65 to 128 16-bit values of dz): a workgroup takes up to `chunk` rows of a group, each of
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

// Step j of a contraction over 32 rows in LDS, `stride` bytes apart, as the matrix pipe takes them: columns c0 .. + 31, eight rows (floats) or
// sixteen at a time.
template <class T>
__device__ __forceinline__ typename Fragment<T>::type columns(const char* rows, int stride, int c0, int j, int lane)
{
    union {
        typename Fragment<T>::type v;
        s16x4 s[2];
    } f;
    if constexpr (sizeof(T) == 4) {
        const char* p = rows + (8 * j + 4 * (lane >> 5)) * stride + (c0 + (lane & 31)) * 4;
#pragma unroll
        for (int s = 0; s < 4; ++s) f.v[s] = *reinterpret_cast<const float*>(p + s * stride);
    } else {
        typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
        const int row = 16 * j + 8 * (lane >> 5) + ((lane & 15) >> 2), col = c0 + (lane & 16) + 4 * (lane & 3);
        const char* p = rows + row * stride + col * 2;
        f.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)p);
        f.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)(p + 4 * stride));
    }
    return f.v;
}

// Chunks of 32 rows of `values` values in the order of memory, chunk number lane + 64 i: what a lane brings.  COLUMN: as if a row had 1, 2, 4 or 8
// of them, so that a lane's chunks all lie in the same columns; the lanes of chunks that a row does not have bring nothing.
template <class T, int S, bool COLUMN = false>
struct Block {
    static constexpr int E = 16 / sizeof(T), kRow = 2 * S + 1;       // LDS rows in chunks, an odd number of them
    typedef typename Fragment<T>::type Frag;
    typedef Frag Any __attribute__((aligned(sizeof(T))));
    int values, chunks, row[S], from[S];
    bool again[S];                                   // a row's last chunk where it is not whole: the row's last sixteen bytes
    __device__ __forceinline__ void init(int n, int lane)
    {
        values = n;
        chunks = (n + E - 1) / E;
        if (COLUMN) chunks = chunks <= 2 ? chunks : chunks <= 4 ? 4 : 8;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int c = lane + 64 * i;
            row[i] = c / chunks;
            const int at = (c - row[i] * chunks) * E;
            if (COLUMN && at >= n) row[i] = 32;
            again[i] = n >= E && at + E > n;
            from[i] = again[i] ? n - E : at;
        }
    }
    // those of the rows before `left`, zeros for the others
    __device__ __forceinline__ Frag load(int i, const T* base, int64_t ld, int left) const
    {
        Frag x = {};
        if (row[i] >= 32 || row[i] >= left) return x;
        const T* p = base + row[i] * (int)ld + from[i];             // (32 rows of at most 2^21 values)
        if (values >= E) return *reinterpret_cast<const Any*>(p);
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (j < values) x[j] = p[j];
        return x;
    }
    __device__ __forceinline__ void store(int i, char* lds, Frag x) const
    {
        if (row[i] >= 32) return;
        char* to = lds + row[i] * kRow * 16 + from[i] * (int)sizeof(T);
        if (again[i]) *reinterpret_cast<Any*>(to) = x;
        else *reinterpret_cast<Frag*>(to) = x;
    }
};

template <class T>
struct GradientArgs {
    const T* dY;
    int64_t lddy;
    const T* X;                // null where dA is
    int64_t ldx;
    const T* A;
    const T* pre;
    int64_t ldpre;
    const int32_t* offsets;
    int rows;
    int32_t K, din, dout;
    int act, run;
    T* dX;                     // each of them or null
    int64_t lddx;
    T *dA, *dbias;
    float *parts, *bias_parts; // sums of groups with more than one run
};

// The whole gradient where rows are narrow both ways (64 values each at most): dY, pre and X are read once.  A workgroup takes a run of a group's rows,
// each of its four wavefronts every fourth block of 32, which pass through LDS of its own: dz by rows for dX, dz and X by columns for dA, whose
// sums stay in registers until the wavefronts add theirs up in order.  U and V: blocks of 32 results and features.  The matrix lies in LDS as
// well: in registers it leaves one wavefront a SIMD instead of two (250,013 rows 37 -> 24 in float32 on 437 nodes 109 us, 81 like this).
// Slopes, rows and sums in passes of their own took 86 us there (floor of the bytes 26), 71 for 200,000 rows 64 -> 64 bf16 on 16 nodes (now
// 44, floor 22), 88 for 250,000 rows 37 -> 24 bf16 on 437 (now 53, floor 13).  What is left is the matrix pipe's float32 rate on blocks of
// 32 that are half empty, and a run's start and end.
template <class T, int U, int V>
struct Gradient {
    static constexpr int S = U * sizeof(T), SX = V * sizeof(T), kOut = 32 * V + 4;
    static constexpr int kRows = 32 * Block<T, S>::kRow * 16, kRowsX = 32 * Block<T, SX>::kRow * 16, kTurned = 32 * kOut * 4;
    static constexpr int kWave = kRows + (kRowsX > kTurned ? kRowsX : kTurned), kMatrix = V * S * 1024, LDS = 4 * kWave + kMatrix;
    static constexpr int STATIC_LDS = 4 * U * 32 * 4 + 64;                 // sums of the biases and of the search
    static constexpr int MOST = 2 * (LDS + STATIC_LDS) <= 160 * 1024 ? 2 : 1;      // workgroups that a unit holds, as far as runs reckon with them
};
template <class T, int U, int V>
__global__ void __launch_bounds__(256) gradient_narrow_kernel(GradientArgs<T> a)
{
    typedef Gradient<T, U, V> G;
    typedef typename Fragment<T>::type Frag;
    constexpr int E = 16 / sizeof(T), S = G::S, SX = G::SX, kOut = G::kOut, kSteps = sizeof(T);     // (32 rows, eight floats or sixteen 16-bit values a step)
    constexpr bool kExact = sizeof(T) == 2;          // biases add up what dz was before it was rounded: a lane's chunks lie in the same columns
    static_assert(G::LDS >= 4 * V * 4096 && sizeof(float) * 4 * U * 32 + 4 * sizeof(uint2) + 2 * sizeof(int) <= G::STATIC_LDS);
    extern __shared__ __align__(16) char narrow_lds[];
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
    char *rows = narrow_lds + wave * G::kWave, *rows_x = rows + G::kRows;
    float* turned = reinterpret_cast<float*>(rows_x);
    Block<T, S, kExact> P;
    Block<T, SX> Q;
    P.init(a.dout, lane);
    Q.init(a.din, lane);
    Frag next[S], zs[S], xs[SX];
    auto fetch = [&](int b) __attribute__((always_inline)) {
        const int64_t row0 = first + 32 * (int64_t)b;
        const int left = end - first - 32 * b;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            next[i] = P.load(i, a.dY + row0 * a.lddy, a.lddy, left);
            zs[i] = Frag{};
            if (a.act) zs[i] = P.load(i, a.pre + row0 * a.ldpre, a.ldpre, left);
        }
        if (a.dA)
#pragma unroll
            for (int i = 0; i < SX; ++i) xs[i] = Q.load(i, a.X + row0 * a.ldx, a.ldx, left);
    };
    fetch(wave);                                      // (on their way while the matrix comes)
    char* matrix = narrow_lds + 4 * G::kWave;         // as the matrix pipe takes it, block v and step s: 64 chunks
    if (a.dX) {
        for (int i = wave; i < V * S; i += 4) {
            const int n = i / S * 32 + l, k0 = (2 * (i % S) + h) * E;
            Frag x = {};
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (n < a.din && k0 + j < a.dout) x[j] = a.A[((int64_t)e * a.dout + k0 + j) * a.din + n];
            *reinterpret_cast<Frag*>(matrix + (i * 64 + lane) * 16) = x;
        }
    }
    // what lies behind dz's columns meets zeros of the matrix, and has to be a number
    for (int i = lane; i < G::kRows / 16; i += 64) reinterpret_cast<v4i*>(rows)[i] = v4i{};
    __syncthreads();
    f32x16 acc[U][V] = {};
    float bias[U] = {}, exact[E] = {};
    for (int b = wave; first + 32 * b < end; b += 4) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            Frag x = next[i];
            if (a.act) {
                float dz[E];
                slopes<T, E>(dz, __builtin_bit_cast(Piece<T>, x), __builtin_bit_cast(Piece<T>, zs[i]), a.act);
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    x[j] = (T)dz[j];
                    if (kExact) exact[j] += dz[j];
                }
            } else if (kExact) {
#pragma unroll
                for (int j = 0; j < E; ++j) exact[j] += (float)x[j];
            }
            P.store(i, rows, x);
        }
        if (a.dA)
#pragma unroll
            for (int i = 0; i < SX; ++i) Q.store(i, rows_x, xs[i]);
        wave_in_order();
        fetch(b + 4);
        if (a.dA || (a.dbias && !kExact)) {
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                Frag p[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    p[u] = columns<T>(rows, Block<T, S>::kRow * 16, 32 * u, j, lane);
                    if (kExact) continue;
#pragma unroll
                    for (int i = 0; i < E; ++i) bias[u] += (float)p[u][i];
                }
                if (!a.dA) continue;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Frag x = columns<T>(rows_x, Block<T, SX>::kRow * 16, 32 * v, j, lane);
#pragma unroll
                    for (int u = 0; u < U; ++u) acc[u][v] = mfma(x, p[u], acc[u][v]);
                }
            }
        }
        wave_in_order();
        if (!a.dX) continue;
        f32x16 out[V] = {};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const Frag p = *reinterpret_cast<const Frag*>(rows + (l * Block<T, S>::kRow + 2 * s + h) * 16);
#pragma unroll
            for (int v = 0; v < V; ++v) out[v] = mfma(*reinterpret_cast<const Frag*>(matrix + ((v * S + s) * 64 + lane) * 16), p, out[v]);
        }
        // a lane has its row's results, four consecutive ones at a time; they go out in the order of memory
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(turned + l * kOut + 32 * v + 8 * g + 4 * h) =
                    make_float4(out[v][4 * g], out[v][4 * g + 1], out[v][4 * g + 2], out[v][4 * g + 3]);
        wave_in_order();
#pragma unroll
        for (int i = 0; i < SX; ++i) {
            const int64_t row = first + 32 * (int64_t)b + Q.row[i];
            if (Q.row[i] >= 32 || row >= end) continue;
            Piece<T> y;
#pragma unroll
            for (int j = 0; j < E; ++j) y.e[j] = (T)turned[Q.row[i] * kOut + Q.from[i] + j];
            T* to = a.dX + row * a.lddx + Q.from[i];
            if (a.din >= E) {
                y.store(to);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (j < a.din) to[j] = y.e[j];
            }
        }
        wave_in_order();
    }
    if (!a.dA && !a.dbias) return;
    const int64_t slot = group > run ? run_slot(first, lo, run) : -1, count = (int64_t)a.dout * a.din;
    float* sums = reinterpret_cast<float*>(narrow_lds);                // of a wavefront: V 1024
    if (kExact) {
        // the lanes of a chunk's columns add theirs up; a column of two chunks takes the one that it begins or goes on in
#pragma unroll
        for (int j = 0; j < E; ++j)
            for (int o = P.chunks; o < 64; o <<= 1) exact[j] += __shfl_xor(exact[j], o);
        if (lane < P.chunks && P.row[0] == 0)
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (P.from[0] + j >= lane * E && P.from[0] + j < a.dout) bias_sums[wave][P.from[0] + j] = exact[j];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        __syncthreads();                                               // (no one reads what lies there any more)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int r = 0; r < 16; ++r) sums[(wave * V * 16 + v * 16 + r) * 64 + lane] = acc[u][v][r];
        bias[u] += __shfl_xor(bias[u], 32);
        if (!kExact && h == 0) bias_sums[wave][32 * u + l] = bias[u];
        __syncthreads();
        for (int i = threadIdx.x; a.dA && i < V * 1024; i += 256) {
            const int t = i & 63, r = (i >> 6) & 15;
            const int m = 32 * u + (t & 31), n = 32 * (i >> 10) + (r & 3) + 8 * (r >> 2) + 4 * (t >> 5);
            if (m >= a.dout || n >= a.din) continue;
            const float x = (sums[i] + sums[V * 1024 + i]) + (sums[2 * V * 1024 + i] + sums[3 * V * 1024 + i]);
            if (slot < 0) a.dA[e * count + (int64_t)m * a.din + n] = (T)x;
            else a.parts[slot * count + (int64_t)m * a.din + n] = x;
        }
    }
    if (a.dbias && (int)threadIdx.x < a.dout) {
        const int m = threadIdx.x;
        const float x = (bias_sums[0][m] + bias_sums[1][m]) + (bias_sums[2][m] + bias_sums[3][m]);
        if (slot < 0) a.dbias[(int64_t)e * a.dout + m] = (T)x;
        else a.bias_parts[slot * a.dout + m] = x;
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

// Rows a run of a sum over rows when a group alone gives `tiles` workgroups: one run a group where the groups fill the chip (several only for
// a group of half the rows that a unit takes in all, or four times its share), shorter ones where they do not.
static int run_rows(const som_ctx* ctx, int64_t rows, int32_t K, int64_t tiles, int least)
{
    const int64_t share = (rows + K - 1) / K, runs = ctx->units / (K * tiles > ctx->units ? ctx->units : K * tiles);
    const int64_t half = K * tiles / (2 * ctx->units);
    int64_t run = runs > 1 ? (share + runs - 1) / runs : K > 1 ? (half > 4 ? half : 4) * share : rows;
    if (runs <= 1 && run < 2048) run = 2048;
    if (run < least) run = least;
    return (int)((run + 63) / 64 * 64 < 0x7fffffc0 ? (run + 63) / 64 * 64 : 0x7fffffc0);
}

// Rows of a run of narrow gradients, `most` workgroups a unit: 512, or 1024 where a unit holds one, fewer where those don't fill the chip once,
// more where the runs' sums would become many, and whole rounds of the four wavefronts' blocks of 32 (200,000 rows 64 -> 64 bf16 on 16
// nodes: 391 rows, some more workgroups than fit, 65 us, 446 rows 45, 512 rows 43; 500,000 rows 64 -> 32 on 100 nodes: 512 rows 63, 1000
// rows 74; float32 64 -> 64, one a unit: 100,000 rows 76 us with 256, 60 with 512, 200,000 rows 109 with 512, 88 with 896).
static int narrow_run(const som_ctx* ctx, int64_t rows, int most)
{
    const int64_t once = rows / (ctx->units * most * 15 / 16), many = rows / (ctx->units * 16), longest = 1024 / most;
    const int64_t run = once < 256 ? 256 : once > longest ? longest : once;
    return (int)(((run > many ? run : many) + 127) / 128 * 128);
}

template <class T, bool AT>
static int product_narrow_launch(som_ctx* ctx, const ProductArgs<T>& a, const char* what)
{
    const int Nn = AT ? a.din : a.dout, steps = (int)(((AT ? a.dout : a.din) * sizeof(T) + 31) / 32);
    auto kern = Nn <= 32 ? product_narrow_kernel<T, AT, 1, 8> : product_narrow_kernel<T, AT, 2, 8>;
    if constexpr (!AT) {
        if (steps <= 2) kern = Nn <= 32 ? product_narrow_kernel<T, AT, 1, 2> : product_narrow_kernel<T, AT, 2, 2>;
        else if (steps <= 4) kern = Nn <= 32 ? product_narrow_kernel<T, AT, 1, 4> : product_narrow_kernel<T, AT, 2, 4>;
    }
    // Rows of a workgroup: long enough that the matrix and the search for it don't count, short enough to fill the chip four times (500,000
    // rows 64 -> 32 bf16 on 100 nodes: 512 rows 23 us, 1024 rows 29)
    int64_t chunk = (a.rows / (ctx->units * 4) + 127) / 128 * 128;
    chunk = chunk < 128 ? 128 : chunk > 1024 ? 1024 : chunk;
    hipLaunchKernelGGL(kern, dim3((unsigned)most_tiles(a.rows, a.K, a.offsets, (int)chunk)), dim3(256), 0, ctx->stream, a, (int)chunk);
    return check_hip(ctx, hipGetLastError(), what);
}

template <class T, int U, int V>
static int gradient_narrow_as(som_ctx* ctx, const GradientArgs<T>& a)
{
    static bool attr_set_dev[kMaxDevices] = {};
    bool& attr_set = attr_set_dev[ctx->device];
    constexpr int lds = Gradient<T, U, V>::LDS;
    auto kern = gradient_narrow_kernel<T, U, V>;
    if (!attr_set) {
        if (int rc = check_hip(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds),
                               "raising the dynamic LDS limit"))
            return rc;
        attr_set = true;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)most_runs(a.rows, a.K, a.run)), dim3(256), lds, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "product gradient (narrow) launch");
}

template <class T>
static int gradient_narrow_launch(som_ctx* ctx, const GradientArgs<T>& a)
{
    if (a.dout <= 32) return a.din <= 32 ? gradient_narrow_as<T, 1, 1>(ctx, a) : gradient_narrow_as<T, 1, 2>(ctx, a);
    return a.din <= 32 ? gradient_narrow_as<T, 2, 1>(ctx, a) : gradient_narrow_as<T, 2, 2>(ctx, a);
}

// Workgroups of its kernel that a unit holds.
template <class T>
static int gradient_narrow_most(int32_t dout, int32_t din)
{
    if (dout <= 32) return din <= 32 ? Gradient<T, 1, 1>::MOST : Gradient<T, 1, 2>::MOST;
    return din <= 32 ? Gradient<T, 2, 1>::MOST : Gradient<T, 2, 2>::MOST;
}

template <class T>
static bool product_narrow(int32_t results, int32_t depth)
{
    return results <= kNarrow && depth * (int64_t)sizeof(T) <= kNarrowBytes;
}

} // namespace som
