// One matrix per node: every row of a node's group times that node's matrix, and the gradient (kernels and launches of one element type).
//
//   product    z_s = A_e x_s + c_e,  y_s = act(z_s) + r_s                                          for s in group e
//   gradient   dz_s = dy_s act'(z_s);  dx_s = A_e^T dz_s,  dA_e = sum_s dz_s x_s^T,  dc_e = sum_s dz_s
//
// Rows of group e are offsets[e] .. offsets[e + 1] - 1 (no offsets: one node, all rows).  The group's bounds are on the device,
// so a launch covers as many tiles as there can be and every workgroup looks up its own.  Products of 16-bit rows and their
// sums are taken by the matrix pipe in float32; float32 rows go through its float32 form.
#pragma once

#include "som_rows.hpp"

#include <type_traits>

namespace som {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

// What a tile of the contraction is made of: C[m][n] = sum_k P[m][k] Q[n][k].
enum Form {
    kRowsTimesA,        // m: rows of X, n: results, k: features
    kRowsTimesAt,       // m: rows of dz, n: features, k: results
    kOuterSums          // m: results, n: features, k: rows of the group
};

template <class T>
struct ProductArgs {
    const T* P;                // X, dz, dz
    int64_t ldp;
    const T* Q;                // A, A, X
    int64_t ldq;               // X only
    const int32_t* offsets;    // null: one node
    int rows;
    int32_t K, din, dout;
    const T* bias;
    const T* residual;
    int64_t ldr;
    T* pre;
    int64_t ldpre;
    T* out;                    // Y, dX, dA
    int64_t ldo;
    int act;
    // Sums over rows (kOuterSums): a group's rows are taken in runs of `run`, every run's sum by another workgroup; with more than one run
    // a group, the sums go to `parts` in float32 (run_slot) and are added up in order afterwards
    int run;
    float* parts;
};

// Where a factor has reached its limit the product with z is formed from the limit, so that infinities give what the function
// tends to.
//   float32 rows: the error function's complement keeps the small values of the left tail to their last places;
//   16-bit rows: exponentials through the base-2 instruction, reciprocals to one unit, and the error function's complement as the falling
//   exponential times a polynomial of t = 1 / (1 + 0.4296 |z| / sqrt 2), fitted to erfc(y) exp(y^2) / 2 for the least weighted error over all
//   of 0 <= y <= 21: some 2^-14.5 of the result in the left tail, and 4.6e-7 of |z| elsewhere.  A result is rounded by 2^-11 or 2^-8 of itself.
// Results below 1e-36 in the far left, where the exponentials leave float32's range, become zeros.
template <bool EXACT>
struct Math {
    static __device__ __forceinline__ float exponential(float x) { return EXACT ? expf(x) : __builtin_amdgcn_exp2f(1.44269504f * x); }
    static __device__ __forceinline__ float reciprocal(float x) { return EXACT ? 1.0f / x : __builtin_amdgcn_rcpf(x); }
    // (1 + erf(z / sqrt 2)) / 2 for |z| <= 30; bell = exp(-z^2 / 2)
    static __device__ __forceinline__ float gauss(float z, float bell)
    {
        if (EXACT) return 0.5f * erfcf(-0.70710678f * z);
        const float t = __builtin_amdgcn_rcpf(fmaf(0.4296f * 0.70710678f, fabsf(z), 1.0f));
        const float p = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.0745519949f, 0.19671153f), 0.00396633652f), 0.134738969f), 0.117778317f), 0.121356536f);
        const float tail = bell * t * p;
        return z > 0.0f ? 1.0f - tail : tail;
    }
    // (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2
    static __device__ __forceinline__ float gate(float z)
    {
        return reciprocal(1.0f + exponential(-1.59576912f * z * fmaf(0.044715f, z * z, 1.0f)));
    }

    static __device__ __forceinline__ float activate(float z, int act)
    {
        switch (act) {
        case SOM_ACT_RELU: return z < 0.0f ? 0.0f : z;                   // (a NaN stays one)
        case SOM_ACT_SILU: return z < -110.0f ? 0.0f : z * reciprocal(1.0f + exponential(-z));
        case SOM_ACT_GELU: return z < -30.0f ? 0.0f : z > 30.0f ? z : z * gauss(z, EXACT ? 0.0f : exponential(-0.5f * z * z));
        case SOM_ACT_GELU_TANH: return z < -30.0f ? 0.0f : z > 30.0f ? z : z * gate(z);
        }
        return z;
    }

    static __device__ __forceinline__ float slope(float z, int act)
    {
        switch (act) {
        case SOM_ACT_RELU: return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
        case SOM_ACT_SILU: {
            if (fabsf(z) > 110.0f) return z > 0.0f ? 1.0f : 0.0f;
            const float g = reciprocal(1.0f + exponential(-z));
            return g * fmaf(z, 1.0f - g, 1.0f);
        }
        case SOM_ACT_GELU: {
            if (fabsf(z) > 30.0f) return z > 0.0f ? 1.0f : 0.0f;
            const float bell = exponential(-0.5f * z * z);
            return fmaf(0.39894228f * z, bell, gauss(z, bell));
        }
        case SOM_ACT_GELU_TANH: {
            if (fabsf(z) > 30.0f) return z > 0.0f ? 1.0f : 0.0f;
            const float g = gate(z);
            return g * fmaf(z * (1.0f - g) * 1.59576912f, fmaf(0.134145f, z * z, 1.0f), 1.0f);
        }
        }
        return 1.0f;
    }
};

template <class T, int N>
__device__ __forceinline__ void activate(float (&x)[N], int act)
{
    auto all = [&](int which) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = Math<sizeof(T) == 4>::activate(x[j], which);
    };
    if (act == SOM_ACT_SILU) all(SOM_ACT_SILU);
    else if (act == SOM_ACT_GELU) all(SOM_ACT_GELU);
    else if (act == SOM_ACT_GELU_TANH) all(SOM_ACT_GELU_TANH);
    else if (act == SOM_ACT_RELU) all(SOM_ACT_RELU);
}

// Rows [lo, hi) of group e, inside [0, rows) whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t* __restrict__ offsets, int e, int rows, int& lo, int& hi)
{
    if (!offsets) {
        lo = 0;
        hi = rows;
        return;
    }
    lo = offsets[e];
    hi = offsets[e + 1];
    lo = lo < 0 ? 0 : lo > rows ? rows : lo;
    hi = hi < lo ? lo : hi > rows ? rows : hi;
}

// Where a workgroup finds its work among the groups: a group of n rows has items_of(n) items of two kinds (x and y), and the items are counted in
// the groups' order.  pick(total, kind) names the item by the totals, its number among
// those of its kind, and leaves kind as it is, below zero, for none.  Called by a whole workgroup: the item's
// group and which of the group's items it is, or -1.  One pass over the offsets, a stretch of groups a lane, and two barriers.
struct Item {
    int kind, group, which;
};
template <int THREADS, class Items, class Pick>
__device__ __forceinline__ Item find_item(const int32_t* __restrict__ offsets, int K, int rows, Items items_of, Pick pick)
{
    __shared__ uint2 sums[THREADS / 64];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (K + THREADS - 1) / THREADS, k0 = tid * per, k1 = k0 + per < K ? k0 + per : K;
    uint2 mine = make_uint2(0u, 0u);
    for (int k = k0; k < k1; ++k) {
        int lo, hi;
        group_rows(offsets, k, rows, lo, hi);
        const uint2 n = items_of((unsigned)(hi - lo));
        mine.x += n.x;
        mine.y += n.y;
    }
    uint2 incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned x = __shfl_up(incl.x, o), y = __shfl_up(incl.y, o);
        if (lane >= o) {
            incl.x += x;
            incl.y += y;
        }
    }
    if (lane == 63) sums[wave] = incl;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    uint2 before = make_uint2(0u, 0u), total = make_uint2(0u, 0u);
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) {
            before.x += sums[w].x;
            before.y += sums[w].y;
        }
        total.x += sums[w].x;
        total.y += sums[w].y;
    }
    int kind = -1;
    const unsigned number = pick(total, kind);
    if (kind >= 0) {
        const unsigned count = kind ? mine.y : mine.x;
        unsigned at = kind ? before.y + incl.y - mine.y : before.x + incl.x - mine.x;
        if (number >= at && number - at < count) {
            for (int k = k0; k < k1; ++k) {
                int lo, hi;
                group_rows(offsets, k, rows, lo, hi);
                const uint2 n = items_of((unsigned)(hi - lo));
                const unsigned here = kind ? n.y : n.x;
                if (number - at < here) {
                    found[0] = k;
                    found[1] = (int)(number - at);
                    break;
                }
                at += here;
            }
        }
    }
    __syncthreads();
    return {kind, kind < 0 ? -1 : __builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[1])};
}

// The same for items of one kind, by number.
template <int THREADS, class Items>
__device__ __forceinline__ int find_group(const int32_t* __restrict__ offsets, int K, int rows, Items items_of, unsigned number, int& which)
{
    const Item it = find_item<THREADS>(
        offsets, K, rows, [&](unsigned n) { return make_uint2(items_of(n), 0u); },
        [&](uint2, int& kind) {
            kind = 0;
            return number;
        });
    which = it.which;
    return it.group;
}

// Runs of `run` rows that a group of n rows has, and which part a run's sum goes to when there are more than one: the run starts at
// `first` of a group that starts at lo.  (No other run has the same: runs behind a group's first one that start within the same `run`
// rows would be of one group, and so would two first ones of groups with more than `run` rows.)
__device__ __forceinline__ unsigned runs_of(unsigned n, unsigned run) { return n <= run ? 1u : (n - 1) / run + 1u; }
__device__ __forceinline__ int64_t run_slot(int first, int lo, int run) { return 2 * (int64_t)(first / run) + (first == lo); }
static int64_t run_slots(int64_t rows, int run) { return 2 * (rows / run + 1); }

// Sixteen bytes of 32 rows (lane l: row l % 32, chunk 2 j + l / 32) times sixteen of 32 columns: a step of 32 bytes of the contraction.
template <class T>
struct Fragment;
template <>
struct Fragment<__bf16> {
    typedef bf16x8 type;
};
template <>
struct Fragment<_Float16> {
    typedef f16x8 type;
};
template <>
struct Fragment<float> {
    typedef f32x4 type;
};
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(f32x4 a, f32x4 b, f32x16 c)
{
#pragma unroll
    for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[s], b[s], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const lds_char*)p; }

// 64 lanes' sixteen bytes from `offset` behind a buffer's base to LDS at `lds`, in lane order; offsets beyond the buffer's length
// bring zeros.  (Waited for by vmcnt, in the order of issue.)
__device__ __forceinline__ void buffer_to_lds(uint32_t lds, uint32_t offset, v4i buffer)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(buffer) : "memory", "m0");
}

__device__ __forceinline__ v4i buffer_of(const void* base, uint32_t bytes)
{
    const uint64_t a = (uint64_t)base;
    v4i r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff);
    r[2] = __builtin_amdgcn_readfirstlane((int)bytes);
    r[3] = 0x00020000;
    return r;
}

constexpr uint32_t kNowhere = 0x80000000u;     // an offset behind every buffer

// One operand of a tile: R rows (or, TR, columns) of the product by 128 bytes of the contraction, 128 R bytes of LDS a stage, which
// holds sixteen-byte chunks.
//   plain: memory holds R rows of `depth` values; an LDS row is 128 bytes, whose chunks are exchanged so that sixteen lanes that read one
//          chunk of sixteen rows meet all 64 banks
//   TR:    memory holds `depth` rows of R values, and so does LDS.  Of 16-bit values the transposing read of a half wavefront takes 64
//          bytes of four rows, of floats a wavefront reads 128 bytes of two rows four apart: what is read at once is moved apart
// ALIGNED: memory goes straight to LDS (every row starts at a multiple of sixteen bytes and holds whole chunks of them); else through
// registers, chunks at a row's end value by value.
template <class T, int R, int WAVES, bool TR>
struct Operand {
    static constexpr int E = 16 / sizeof(T), BK = 128 / sizeof(T);
    static constexpr int kBytes = R * 128, kLoads = kBytes / 1024 / WAVES;            // a wavefront's instructions of 64 chunks a stage
    static constexpr int kChunks = TR ? R / E : 8, kRowsAtOnce = 64 / kChunks;        // LDS rows that an instruction fills
    const T* base;             // the tile's first value
    int depth;                 // of the contraction
    int rows;                  // rows (TR: values in a row) that exist, counted from base
    int64_t ld;                // values
    bool brief;                // a row of the matrix has fewer values than a chunk
    int chunk, row;            // the LDS chunk and row that this lane fills first
    uint32_t offset[kLoads];   // ALIGNED: in bytes from a stage's first row

    // the place of chunk c in LDS row r
    static __device__ __forceinline__ int exchanged(int c, int r)
    {
        if (!TR) return c ^ ((r >> 1) & 7);
        if (sizeof(T) == 4) return c ^ ((r & 4) << 1);
        return R >= 128 ? c ^ ((r & 3) << 2) : c ^ ((r & 2) << 1);
    }
    __device__ __forceinline__ void init(const T* b, int d, int exist, int64_t stride, int values, int wave, int lane)
    {
        static_assert(kLoads >= 1 && kBytes % (1024 * WAVES) == 0 && 64 % kChunks == 0);
        base = b;
        depth = d;
        brief = values < E;
        rows = exist < R ? exist : R;
        ld = stride;
        chunk = lane % kChunks;
        row = wave * kLoads * kRowsAtOnce + lane / kChunks;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int from = exchanged(chunk, row + q * kRowsAtOnce) * E;
            offset[q] = (uint32_t)(row + q * kRowsAtOnce) * (uint32_t)(ld * sizeof(T)) + from * (uint32_t)sizeof(T);
            if (TR && from >= rows) offset[q] = kNowhere;
        }
    }
    // The stage that starts at k0 of the contraction, an instruction at a time; stages behind the end bring zeros and read nothing.
    __device__ __forceinline__ v4i stage(int k0) const
    {
        const int left = depth - k0, have = left < BK ? left : BK;
        const uint32_t bytes = (TR ? (uint32_t)(have - 1) * (uint32_t)ld + rows : (uint32_t)(rows - 1) * (uint32_t)ld + left) * (uint32_t)sizeof(T);
        return buffer_of(TR ? base + k0 * ld : base + k0, left > 0 ? bytes : 0u);
    }
    __device__ __forceinline__ void one(int q, uint32_t lds, v4i buffer, int k0, int wave) const
    {
        // a plain row's end is not the buffer's: chunks behind it (depth is a multiple of E) are sent nowhere
        const bool past = !TR && exchanged(chunk, row + q * kRowsAtOnce) * E >= depth - k0;
        buffer_to_lds(lds + (uint32_t)(wave * kLoads + q) * 1024, past ? kNowhere : offset[q], buffer);
    }
    // values of this lane's chunk that exist (E at most: all of it)
    __device__ __forceinline__ int left(int q, int k0) const
    {
        const int r = row + q * kRowsAtOnce, from = exchanged(chunk, r) * E;
        const int n = TR ? (k0 + r < depth ? rows - from : 0) : (r < rows ? depth - k0 - from : 0);
        return n < E ? n : E;
    }
    // A chunk at a row's end is read as the row's last sixteen bytes and moved down by `store`, which is where it is waited for.
    __device__ __forceinline__ v4i load(int q, int k0) const
    {
        typedef int any4 __attribute__((ext_vector_type(4), aligned(2)));
        const int r = row + q * kRowsAtOnce, from = exchanged(chunk, r) * E, n = left(q, k0);
        const T* p = TR ? base + (k0 + r) * ld + from : base + r * ld + k0 + from;
        v4i x = {};
        if (brief) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (j >= n) continue;
                if constexpr (sizeof(T) == 4) x[j] = __builtin_bit_cast(int, p[j]);
                else x[j / 2] |= (int)__builtin_bit_cast(uint16_t, p[j]) << (j % 2 * 16);
            }
        } else if (n > 0) {
            x = *reinterpret_cast<const any4*>(p - (E - n));
        }
        return x;
    }
    __device__ __forceinline__ void store(int q, int k0, char* stage, v4i x, int wave, int lane) const
    {
        const int n = left(q, k0);
        if (n < E && !brief) {
            const int s = 8 * (int)sizeof(T) * (E - n);                      // 16 .. 112 bits, more for a chunk of which nothing exists
            const uint64_t lo = (uint32_t)x[0] | (uint64_t)(uint32_t)x[1] << 32, hi = (uint32_t)x[2] | (uint64_t)(uint32_t)x[3] << 32;
            const uint64_t lo2 = n <= 0 ? 0u : s < 64 ? lo >> s | hi << (64 - s) : hi >> (s - 64), hi2 = n <= 0 || s >= 64 ? 0u : hi >> s;
            x[0] = (int)lo2;
            x[1] = (int)(lo2 >> 32);
            x[2] = (int)hi2;
            x[3] = (int)(hi2 >> 32);
        }
        *reinterpret_cast<v4i*>(stage + (wave * kLoads + q) * 1024 + lane * 16) = x;
    }
};

// 32 rows by step j of a stage as the matrix pipe takes them: lane l holds row l % 32, the values of chunk 2 j + l / 32.
template <class T, int R, bool TR>
__device__ __forceinline__ typename Fragment<T>::type fragment(const char* stage, int r0, int j, int lane)
{
    typedef Operand<T, R, 1, TR> Op;
    typedef typename Fragment<T>::type type;
    if constexpr (!TR) {
        const int r = r0 + (lane & 31), c = Op::exchanged(2 * j + (lane >> 5), r);
        return *reinterpret_cast<const type*>(stage + r * 128 + c * 16);
    } else if constexpr (sizeof(T) == 4) {
        type f;
        const int col = r0 + (lane & 31), row = 8 * j + 4 * (lane >> 5);
        const char* p = stage + row * (4 * R) + Op::exchanged(col >> 2, row) * 16 + (col & 3) * 4;
#pragma unroll
        for (int s = 0; s < 4; ++s) f[s] = *reinterpret_cast<const float*>(p + s * (4 * R));
        return f;
    } else {
        // Sixteen lanes exchange a block of four rows and sixteen columns: lane 4 j + q brings columns 4 q .. + 3 of row j, lane i gets
        // column i of all four.
        typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
        union {
            type v;
            s16x4 s[2];
        } f;
        const int row = 16 * j + 8 * (lane >> 5) + ((lane & 15) >> 2), col = r0 + (lane & 16) + 4 * (lane & 3);
        const char* p = stage + row * (2 * R) + Op::exchanged(col >> 3, row) * 16 + (col & 7) * 2;
        f.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)p);
        f.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)(p + 4 * (2 * R)));
        return f.v;
    }
}

// This wavefront's reads of the stage before (and DIRECT: its loads to LDS) are done, then everyone's are.
template <bool DIRECT>
__device__ __forceinline__ void stage_ready()
{
    if (DIRECT) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Tile number `tile` of `rows` rows of `wide` tiles, taken in bands of up to eight columns: a die's 32 workgroups work on some four rows and
// eight columns at a time, whose operands its cache holds (8192 x 8192 x 8192 in rows of 32 tiles 970 us, in bands 908).
__device__ __forceinline__ unsigned banded(unsigned tile, unsigned rows, unsigned wide, unsigned& x)
{
    const unsigned bands = (wide + 7) / 8, w = (wide + bands - 1) / bands, band = tile / (rows * w), rest = tile - band * rows * w;
    const unsigned mine = wide - band * w < w ? wide - band * w : w;
    x = band * w + rest % mine;
    return rest / mine;
}

// Square tiles of B rows and columns in wavefronts of WM x WN: eight wavefronts for 256, four for 128 and 64.  MOST: workgroups that a unit's 160 KB of
// LDS hold, one, two and four of them (the search's sums in front of the stages take 1 KB, as the stages begin at a multiple of it).
template <int B>
struct Tile {
    static constexpr int UNIT_LDS = 160 * 1024, SEARCH_LDS = 1024;
    static constexpr int WM = B == 256 ? 128 : B / 2, WN = B == 256 ? 64 : B / 2, WAVES = (B / WM) * (B / WN), THREADS = 64 * WAVES, LDS = 2 * 2 * B * 128,
                         MOST = UNIT_LDS / (LDS + SEARCH_LDS);
};

template <class T, Form F, int B, bool ALIGNED>
__global__ void __launch_bounds__(Tile<B>::THREADS) product_tile_kernel(ProductArgs<T> a, unsigned xtiles)
{
    constexpr int BM = B, BN = B, WM = Tile<B>::WM, WN = Tile<B>::WN, WAVES = Tile<B>::WAVES, THREADS = Tile<B>::THREADS;
    constexpr bool TP = F == kOuterSums, TQ = F != kRowsTimesA;
    typedef Operand<T, BM, WAVES, TP> OpP;
    typedef Operand<T, BN, WAVES, TQ> OpQ;
    constexpr int kStage = OpP::kBytes + OpQ::kBytes, BK = OpP::BK;
    extern __shared__ __align__(1024) char tile_lds[];
    typedef typename Fragment<T>::type Frag;
    static_assert(Tile<B>::MOST >= 1 && sizeof(uint2) * WAVES + 2 * sizeof(int) <= Tile<B>::SEARCH_LDS);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    const int Nn = F == kRowsTimesA ? a.dout : a.din;
    int e, first, end, m0 = 0;
    unsigned x;
    // The chip's eight dies take workgroups in turn; each gets a run of tiles that share operands in its cache.
    const unsigned block = blockIdx.x + blockIdx.y * gridDim.x, xcd = block % 8, turn = block / 8;
    float* part = nullptr;
    if (F == kOuterSums) {
        const unsigned run = a.run;
        // Runs differ in length, so every die takes its share of each run's tiles (a run of groups for each die, as below: 726 us
        // for 65536 rows, 2048 -> 1536, on 64 uneven nodes, 535 us like this)
        const unsigned ytiles = (a.dout + BM - 1) / BM, each = ytiles * xtiles, share = (each + 7) / 8;
        const unsigned item = each < 16 ? block / each : turn / share, tile = each < 16 ? block % each : xcd * share + turn % share;
        // Groups of more than twice the usual number of rows (kind 0) come first, so that none is the last to start.
        const unsigned usual = 2u * ((unsigned)a.rows / (unsigned)a.K + 1u);
        const Item it = find_item<THREADS>(
            a.offsets, a.K, a.rows,
            [run, usual](unsigned n) {
                const unsigned runs = runs_of(n, run);
                return n > usual ? make_uint2(runs, 0u) : make_uint2(0u, runs);
            },
            [item](uint2 total, int& kind) {
                kind = item < total.x ? 0 : 1;
                return kind ? item - total.x : item;
            });
        e = it.group;
        const int which = it.which;
        if (e < 0 || tile >= each) return;
        m0 = banded(tile, ytiles, xtiles, x) * BM;
        group_rows(a.offsets, e, a.rows, first, end);
        if (end - first > (int)run) {
            const int lo = first;
            first += which * run;
            end = end - first > (int)run ? first + (int)run : end;
            part = a.parts + run_slot(first, lo, run) * ((int64_t)a.dout * a.din);
        }
    } else {
        // One node: whole tiles (kind 0) first, its last ones (kind 1), which take less time, when those run out (4099 x 4096 x 4096: 213 us in
        // order, 178 like this).  Several: all of a group's tiles together, so that its matrix comes once (65536 rows 2048 -> 1536 on 64
        // uneven nodes, matrices of 6 MB: 530 us with the last tiles last, 509 in order).
        const bool apart = a.K == 1;
        const Item it = find_item<THREADS>(
            a.offsets, a.K, a.rows, [apart](unsigned n) { return make_uint2(apart ? n / BM : (n + BM - 1) / BM, apart && n % BM ? 1u : 0u); },
            [&](uint2 total, int& kind) __attribute__((always_inline)) {
                const unsigned whole = total.x * xtiles, run = (whole + 7) / 8, at = xcd * run;
                const unsigned mine = at < whole ? (whole - at < run ? whole - at : run) : 0u;
                const unsigned rest = total.y * xtiles, last = (rest + 7) / 8, tile = (7 - xcd) * last + turn - mine;
                kind = turn < mine ? 0 : turn - mine < last && tile < rest ? 1 : -1;
                if (kind < 0) return 0u;
                return banded(kind ? tile : at + turn, kind ? total.y : total.x, xtiles, x);
            });
        if (it.group < 0) return;
        e = it.group;
        group_rows(a.offsets, e, a.rows, first, end);
        first = it.kind == 0 ? first + it.which * BM : end - (end - first) % BM;
    }
    e = __builtin_amdgcn_readfirstlane(e);
    first = __builtin_amdgcn_readfirstlane(first);
    end = __builtin_amdgcn_readfirstlane(end);
    const int n0 = __builtin_amdgcn_readfirstlane(x) * BN;
    OpP P;
    OpQ Q;
    const int depth = F == kRowsTimesA ? a.din : F == kRowsTimesAt ? a.dout : end - first;
    if (F == kOuterSums) {
        P.init(a.P + (int64_t)first * a.ldp + m0, depth, a.dout - m0, a.ldp, a.dout, wave, lane);
        Q.init(a.Q + (int64_t)first * a.ldq + n0, depth, a.din - n0, a.ldq, a.din, wave, lane);
    } else {
        P.init(a.P + (int64_t)first * a.ldp, depth, end - first, a.ldp, depth, wave, lane);
        const T* A = a.Q + (int64_t)e * a.dout * a.din;
        Q.init(F == kRowsTimesA ? A + (int64_t)n0 * a.din : A + n0, depth, Nn - n0, a.din, a.din, wave, lane);
    }
    f32x16 acc[WM / 32][WN / 32] = {};
    const int steps = (depth + BK - 1) / BK;
    const uint32_t lds = lds_address(tile_lds);
    // blocks of 32 rows that this wavefront has; the columns' ends are left to zeros and to the stores
    const int have = ((F == kOuterSums ? a.dout - m0 : end - first) - wm + 31) / 32;
    constexpr int U = WM / 32, V = WN / 32, kLoads = OpP::kLoads + OpQ::kLoads;
    Frag p[2][U], q[2][V];
    v4i held[ALIGNED ? 1 : kLoads];                 // a stage on its way through registers
    // instruction number n of a stage
    auto fetch = [&](int i, int n, v4i bp, v4i bq) __attribute__((always_inline)) {
        const uint32_t to = lds + (i & 1) * kStage;
        if (n < OpP::kLoads) P.one(n, to, bp, i * BK, wave);
        else Q.one(n - OpP::kLoads, to + OpP::kBytes, bq, i * BK, wave);
    };
    auto load = [&](int i, int n) __attribute__((always_inline)) { held[n] = n < OpP::kLoads ? P.load(n, i * BK) : Q.load(n - OpP::kLoads, i * BK); };
    auto store = [&](int i, int n) __attribute__((always_inline)) {
        char* to = tile_lds + (i & 1) * kStage;
        if (n < OpP::kLoads) P.store(n, i * BK, to, held[n], wave, lane);
        else Q.store(n - OpP::kLoads, i * BK, to + OpP::kBytes, held[n], wave, lane);
    };
    auto fetch_all = [&](int i) __attribute__((always_inline)) {
        if constexpr (ALIGNED) {
            const v4i bp = P.stage(i * BK), bq = Q.stage(i * BK);
#pragma unroll
            for (int n = 0; n < kLoads; ++n) fetch(i, n, bp, bq);
        } else {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) store(i, n);
#pragma unroll
            for (int n = 0; n < kLoads; ++n) load(i + 1, n);
        }
    };
    // fragment number f of a step: the columns', then the rows'
    auto read = [&](int i, int j, int to, int f) __attribute__((always_inline)) {
        const char* stage = tile_lds + (i & 1) * kStage;
        if (f < V) q[to][f] = fragment<T, BN, TQ>(stage + OpP::kBytes, wn + 32 * f, j, lane);
        else p[to][f - V] = fragment<T, BM, TP>(stage, wm + 32 * (f - V), j, lane);
    };
    // The contraction for H blocks of rows.  The pipe takes 32 cycles for a product, and beside each goes a share of the other work: the
    // next step's fragments, and behind the barrier the stage after the next.  (The scheduler would gather the reads in front of
    // their use: it is kept out.)  The last fragments of a stage are in registers when the barrier comes, so that its buffer is free and
    // everyone's arrival hides behind products that need nothing.
    auto contract = [&](auto blocks) __attribute__((always_inline)) {
        constexpr int H = decltype(blocks)::value, kReads = H + V, kSlots = H * V;
#pragma unroll
        for (int f = 0; f < kReads; ++f) read(0, 0, 0, f);
        for (int i = 0; i < steps; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool last = j == 3;
                v4i bp = {}, bq = {};
                if (last) {
                    stage_ready<ALIGNED>();
                    if (ALIGNED) {
                        bp = P.stage((i + 2) * BK);
                        bq = Q.stage((i + 2) * BK);
                    }
                }
#pragma unroll
                for (int t = 0; t < kSlots; ++t) {
                    acc[t / V][t % V] = mfma(q[j & 1][t % V], p[j & 1][t / V], acc[t / V][t % V]);
#pragma unroll
                    for (int f = t * kReads / kSlots; f < (t + 1) * kReads / kSlots; ++f) read(last ? i + 1 : i, last ? 0 : j + 1, (j + 1) & 1, f);
                    if (last) {
#pragma unroll
                        for (int n = t * kLoads / kSlots; n < (t + 1) * kLoads / kSlots; ++n) {
                            if constexpr (ALIGNED) {
                                fetch(i + 2, n, bp, bq);
                            } else {
                                store(i + 2, n);
                                load(i + 3, n);
                            }
                        }
                    }
                    if (ALIGNED) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };
    if (steps > 0) {
        if constexpr (!ALIGNED) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) load(0, n);
        }
        fetch_all(0);
        if (ALIGNED) stage_ready<ALIGNED>();
        fetch_all(1);
        if (!ALIGNED) stage_ready<ALIGNED>();
        // a group's last tile leaves out the blocks of rows that it does not have
        if (have >= U) {
            contract(std::integral_constant<int, U>{});
        } else if (have <= 0) {
            for (int i = 0; i < steps; ++i) {
                stage_ready<ALIGNED>();
                fetch_all(i + 2);
            }
        } else if constexpr (U > 1) {
            if (have == 1) contract(std::integral_constant<int, 1>{});
            if constexpr (U == 4) {
                if (have == 2) contract(std::integral_constant<int, 2>{});
                if (have == 3) contract(std::integral_constant<int, 3>{});
            }
        }
    }
    // Results go out by rows: a wavefront's 32 x WN values change from the pipe's layout (lane: row, four columns at a time) to eight
    // columns a lane through LDS rows of WN + 4 floats, which keep sixteen lanes on sixteen places both ways.
    constexpr int kRow = WN + 4, kLanes = WN / 8, kAtOnce = 64 / kLanes;
    static_assert(WAVES * 32 * kRow * 4 <= 2 * kStage);
    stage_ready<ALIGNED>();                         // no one reads the stages any more, or writes to them
    float* turned = reinterpret_cast<float*>(tile_lds) + wave * 32 * kRow;
    const int n = n0 + wn + lane % kLanes * 8;
    // eight values of a row, or what is left of it
    typedef Piece<T, 8> Eight;
    constexpr bool kWhole = ALIGNED && sizeof(T) == 2;
    const int left = Nn - n;
    auto load8 = [&](Eight& x, const T* from) __attribute__((always_inline)) {
        if (kWhole || left >= 8) x.load(from);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) x.e[j] = j < left ? from[j] : (T)0.0f;
    };
    auto store8 = [&](const Eight& x, T* to) __attribute__((always_inline)) {
        if (kWhole || left >= 8) x.store(to);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) to[j] = x.e[j];
    };
    Eight c;
    if (F == kRowsTimesA && a.bias && left > 0) load8(c, a.bias + (int64_t)e * a.dout + n);
    const int rows_end = F == kOuterSums ? a.dout : end;
#pragma unroll 1
    for (int u = 0; u < WM / 32; ++u) {
        if (u >= have) break;
        const int64_t row0 = (int64_t)(F == kOuterSums ? m0 : first) + wm + 32 * u;
#pragma unroll
        for (int w = 0; w < WM / 32; ++w) {
            if (w != u) continue;
#pragma unroll
            for (int v = 0; v < WN / 32; ++v)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 x = make_float4(acc[w][v][4 * g], acc[w][v][4 * g + 1], acc[w][v][4 * g + 2], acc[w][v][4 * g + 3]);
                    *reinterpret_cast<float4*>(turned + (lane & 31) * kRow + 32 * v + 8 * g + 4 * (lane >> 5)) = x;
                }
        }
        wave_in_order();
#pragma unroll 1
        for (int r = lane / kLanes; r < 32; r += kAtOnce) {
            const int64_t row = row0 + r;
            if (row >= rows_end || left <= 0) continue;
            float x[8];
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(turned + r * kRow + lane % kLanes * 8);
            *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(turned + r * kRow + lane % kLanes * 8 + 4);
            Eight y, z, d;
            if (F == kRowsTimesA) {
                if (a.residual) load8(d, a.residual + row * a.ldr + n);
                if (a.bias)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] += (float)c.e[j];
                if (a.pre) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) z.e[j] = (T)x[j];
                    store8(z, a.pre + row * a.ldpre + n);
                }
                activate<T>(x, a.act);
                if (a.residual)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] += (float)d.e[j];
            }
            if (F == kOuterSums && part) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (kWhole || j < left) part[row * a.din + n + j] = x[j];
                continue;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y.e[j] = (T)x[j];
            T* out = F == kOuterSums ? a.out + ((int64_t)e * a.dout + row) * a.din : a.out + row * a.ldo;
            store8(y, out + n);
        }
        wave_in_order();
    }
}

// dz = g act'(z) in float32
template <class T, int N>
__device__ __forceinline__ void slopes(float (&dz)[N], const Piece<T, N>& g, const Piece<T, N>& z, int act)
{
    typedef Math<sizeof(T) == 4> M;
    auto all = [&](int which) {
#pragma unroll
        for (int j = 0; j < N; ++j) dz[j] = (float)g.e[j] * M::slope((float)z.e[j], which);
    };
    if (act == SOM_ACT_SILU) all(SOM_ACT_SILU);
    else if (act == SOM_ACT_GELU) all(SOM_ACT_GELU);
    else if (act == SOM_ACT_GELU_TANH) all(SOM_ACT_GELU_TANH);
    else all(SOM_ACT_RELU);
}

// g *= act'(z), rounded to the matrix pipe's operand
template <class T, int N>
__device__ __forceinline__ void slopes(Piece<T, N>& g, const Piece<T, N>& z, int act)
{
    float dz[N];
    slopes<T, N>(dz, g, z, act);
#pragma unroll
    for (int j = 0; j < N; ++j) g.e[j] = (T)dz[j];
}

// dz = dy act'(z), dense (where there is an activation: dz not null), and its column sums over a run of a group's rows (dbias not null),
// of the values before they are rounded: LANES lanes of N columns share a row.
template <class T, int N, int LANES>
__global__ void __launch_bounds__(256) slope_kernel(const T* __restrict__ dY, int64_t lddy, const T* __restrict__ pre, int64_t ldpre,
                                                    const int32_t* __restrict__ offsets, int K, int rows, int32_t dout, int act, T* __restrict__ dz,
                                                    T* __restrict__ dbias, int run, float* __restrict__ parts)
{
    constexpr int kRows = 256 / LANES;
    __shared__ float sums[kRows][LANES * N];
    int which, first, end;
    const int e = find_group<256>(offsets, K, rows, [run](unsigned n) { return runs_of(n, run); }, blockIdx.y + blockIdx.z * gridDim.y, which);
    if (e < 0) return;
    group_rows(offsets, e, rows, first, end);
    const int lo = first, group = end - first;
    first += which * run;
    end = end - first > run ? first + run : end;
    const int l = threadIdx.x % LANES, c = blockIdx.x * LANES + l;
    const bool mine = c * N < dout;
    const int64_t at = mine ? piece_at<T, N>(c, dout) : 0;
    float s[N] = {};
    if (mine) {
        for (int r0 = first + threadIdx.x / LANES; r0 < end; r0 += 4 * kRows) {
            Piece<T, N> g[4], z[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = r0 + u * kRows < end ? r0 + u * kRows : r0;
                g[u].load(dY + (int64_t)r * lddy + at);
                if (dz) z[u].load(pre + (int64_t)r * ldpre + at);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = r0 + u * kRows;
                if (r >= end) continue;
                float x[N];
                if (dz) {
                    slopes<T, N>(x, g[u], z[u], act);
                    Piece<T, N> d;
#pragma unroll
                    for (int j = 0; j < N; ++j) d.e[j] = (T)x[j];
                    d.store(dz + (int64_t)r * dout + at);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) x[j] = (float)g[u].e[j];
                }
#pragma unroll
                for (int j = 0; j < N; ++j) s[j] += x[j];
            }
        }
    }
    if (!dbias) return;
#pragma unroll
    for (int j = 0; j < N; ++j) sums[threadIdx.x / LANES][l * N + j] = s[j];
    __syncthreads();
    if (threadIdx.x >= LANES || !mine) return;
    Piece<T, N> out;
    float* part = group > run ? parts + run_slot(first, lo, run) * dout + at : nullptr;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float v = 0.0f;
        for (int r = 0; r < kRows; ++r) v += sums[r][l * N + j];
        if (part) part[j] = v;
        out.e[j] = (T)v;
    }
    if (!part) out.store(dbias + (int64_t)e * dout + at);
}

// The sums of groups with more than one run: `count` values a group, whose runs SHARES lanes add up between them in order.
template <class T, int SHARES>
__global__ void __launch_bounds__(SHARES == 1 ? 256 : 64 * SHARES) runs_join_kernel(const int32_t* __restrict__ offsets, int K, int rows, int run,
                                                                                    const float* __restrict__ parts, int64_t count, T* __restrict__ out)
{
    constexpr int kThreads = SHARES == 1 ? 256 : 64 * SHARES, kColumns = kThreads / SHARES;
    __shared__ float sums[SHARES][kColumns];
    int which, lo, hi;
    const int e = find_group<kThreads>(offsets, K, rows, [run](unsigned n) { return n > (unsigned)run ? 1u : 0u; }, blockIdx.y, which);
    if (e < 0) return;
    group_rows(offsets, e, rows, lo, hi);
    const int runs = (int)runs_of(hi - lo, run), l = threadIdx.x % kColumns, share = threadIdx.x / kColumns, each = (runs + SHARES - 1) / SHARES;
    const int from = share * each, to = from + each < runs ? from + each : runs;
    for (int64_t i0 = (int64_t)blockIdx.x * kColumns; i0 < count; i0 += (int64_t)gridDim.x * kColumns) {
        const int64_t i = i0 + l;
        float s = 0.0f;
        if (i < count) {
            for (int c = from; c < to; c += 8) {
                float v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = c + u < to ? parts[run_slot(lo + (c + u) * run, lo, run) * count + i] : 0.0f;
#pragma unroll
                for (int u = 0; u < 8; ++u) s += v[u];
            }
        }
        if (SHARES > 1) {
            sums[share][l] = s;
            __syncthreads();
            if (share == 0)
                for (int q = 1; q < SHARES; ++q) s += sums[q][l];
            __syncthreads();
        }
        if (share == 0 && i < count) out[(int64_t)e * count + i] = (T)s;
    }
}

} // namespace som
