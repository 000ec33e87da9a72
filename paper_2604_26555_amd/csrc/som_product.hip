// One matrix per node: every row of a node's group times that node's matrix, and the gradient.
//
//   product    z_s = A_e x_s + c_e,  y_s = act(z_s) + r_s                                          for s in group e
//   gradient   dz_s = dy_s act'(z_s);  dx_s = A_e^T dz_s,  dA_e = sum_s dz_s x_s^T,  dc_e = sum_s dz_s
//
// Rows of group e are offsets[e] .. offsets[e + 1] - 1 (no offsets: one node, all rows).  The group's bounds are on the device,
// so a launch covers as many tiles as there can be and every workgroup looks up its own.  Products of 16-bit rows and their
// sums are taken by the matrix pipe in float32; float32 rows go through its float32 form.
#include "som_rows.hpp"

#include <type_traits>

namespace som {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

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
    // a group, the sums go to `parts` in float32 (runs_slot) and are added up in order afterwards
    int run;
    float* parts;
};

// Where a factor has reached its limit the product with z is formed from the limit, so that infinities give what the function
// tends to.
//   float32 rows: the error function's complement keeps the small values of the left tail to their last places;
//   16-bit rows: exponentials through the base-2 instruction (its argument's rounding is 2^-24 of the exponent, which the falling
//   exponential outweighs), reciprocals to one unit, and the error function by Abramowitz and Stegun 7.1.26 (1.5e-7 at most): all of them
//   some 2^-20 of |z| where the result is rounded by 2^-12 or 2^-9.
template <bool EXACT>
struct Math {
    static __device__ __forceinline__ float exponential(float x) { return EXACT ? expf(x) : __builtin_amdgcn_exp2f(1.44269504f * x); }
    static __device__ __forceinline__ float reciprocal(float x) { return EXACT ? 1.0f / x : __builtin_amdgcn_rcpf(x); }
    // (1 + erf(z / sqrt 2)) / 2 for |z| <= 30; bell = exp(-z^2 / 2)
    static __device__ __forceinline__ float gauss(float z, float bell)
    {
        if (EXACT) return 0.5f * erfcf(-0.70710678f * z);
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
        const float tail = 0.5f * bell * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
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

template <class T>
__device__ __forceinline__ float activate(float z, int act)
{
    return Math<sizeof(T) == 4>::activate(z, act);
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

// Sum over a workgroup.
template <int THREADS>
__device__ __forceinline__ uint2 sum_all(uint2 v)
{
    __shared__ uint2 sums[THREADS / 64];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        v.x += __shfl_xor(v.x, o);
        v.y += __shfl_xor(v.y, o);
    }
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
    __syncthreads();
    uint2 all = make_uint2(0u, 0u);
    for (int w = 0; w < THREADS / 64; ++w) {
        all.x += sums[w].x;
        all.y += sums[w].y;
    }
    return all;
}

// The group that has the item number `item` when the groups' items are counted in order (items_of(rows): how many a group of so many
// rows has), and which of its items that is.  Called by a whole workgroup; -1 when there are fewer.
template <int THREADS, class Items>
__device__ __forceinline__ int find_group(const int32_t* __restrict__ offsets, int K, int rows, Items items_of, unsigned item, int& which)
{
    __shared__ unsigned sums[THREADS / 64];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) found[0] = -1;
    unsigned before = 0;
    for (int e0 = 0; e0 < K; e0 += THREADS) {
        unsigned mine = 0;
        if (e0 + tid < K) {
            int lo, hi;
            group_rows(offsets, e0 + tid, rows, lo, hi);
            mine = items_of((unsigned)(hi - lo));
        }
        unsigned incl = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned v = __shfl_up(incl, o);
            if (lane >= o) incl += v;
        }
        __syncthreads();                          // sums and found of the round before have been read
        if (lane == 63) sums[wave] = incl;
        __syncthreads();
        unsigned at = before + incl - mine;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) at += sums[w];
            before += sums[w];
        }
        if (item >= at && item < at + mine) {
            found[0] = e0 + tid;
            found[1] = (int)(item - at);
        }
        if (before > item) break;
    }
    __syncthreads();
    which = found[1];
    return found[0];
}

// Runs of `run` rows that a group of n rows has, and which part a run's sum goes to when there are more than one: the run starts at
// `first` of a group that starts at lo.  (No other run has the same: runs behind a group's first one that start within the same `run`
// rows would be of one group, and so would two first ones of groups with more than `run` rows.)
__device__ __forceinline__ unsigned runs_of(unsigned n, unsigned run) { return n <= run ? 1u : (n - 1) / run + 1u; }
__device__ __forceinline__ int64_t run_slot(int first, int lo, int run) { return 2 * (int64_t)(first / run) + (first == lo); }
static int64_t run_slots(int64_t rows, int run) { return 2 * (rows / run + 1); }

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

template <class T>
struct Half8;
template <>
struct Half8<__bf16> {
    typedef bf16x8 type;
};
template <>
struct Half8<_Float16> {
    typedef f16x8 type;
};

// Tiles of 64 x 64 in four wavefronts of 32 x 32, operands through LDS a value at a time: any shape, stride and alignment.
template <class T, Form F>
__global__ void __launch_bounds__(256) product_any_kernel(ProductArgs<T> a)
{
    constexpr int BM = 64, BN = 64, BK = 32, PAD = sizeof(T) == 2 ? 8 : 1;
    __shared__ __align__(16) T P[BM][BK + PAD], Q[BN][BK + PAD];
    const int M = F == kOuterSums ? a.dout : 0, Nn = F == kRowsTimesA ? a.dout : a.din;
    int e, first, end, m0 = 0, which;
    float* part = nullptr;
    if (F == kOuterSums) {
        const int run = a.run;
        e = find_group<256>(a.offsets, a.K, a.rows, [run](unsigned n) { return runs_of(n, run); }, blockIdx.z, which);
        if (e < 0) return;
        m0 = blockIdx.y * BM;
        group_rows(a.offsets, e, a.rows, first, end);
        if (end - first > run) {
            const int lo = first;
            first += which * run;
            end = end - first > run ? first + run : end;
            part = a.parts + run_slot(first, lo, run) * ((int64_t)a.dout * a.din);
        }
    } else {
        e = find_group<256>(a.offsets, a.K, a.rows, [](unsigned n) { return (n + BM - 1) / BM; }, blockIdx.y + blockIdx.z * gridDim.y, which);
        if (e < 0) return;
        group_rows(a.offsets, e, a.rows, first, end);
        first += which * BM;
    }
    const int n0 = blockIdx.x * BN;
    const T* A = F == kOuterSums ? nullptr : a.Q + (int64_t)e * a.dout * a.din;
    const int depth = F == kRowsTimesA ? a.din : F == kRowsTimesAt ? a.dout : end - first;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
    f32x16 acc = {};
    for (int k0 = 0; k0 < depth; k0 += BK) {
        __syncthreads();
        for (int i = threadIdx.x; i < BM * BK; i += 256) {
            if (F == kOuterSums) {                                   // consecutive lanes take consecutive m
                const int m = i % BM, k = i / BM;
                P[m][k] = m0 + m < M && k0 + k < depth ? a.P[(int64_t)(first + k0 + k) * a.ldp + m0 + m] : (T)0.0f;
            } else {
                const int k = i % BK, m = i / BK;
                P[m][k] = first + m < end && k0 + k < depth ? a.P[(int64_t)(first + m) * a.ldp + k0 + k] : (T)0.0f;
            }
        }
        for (int i = threadIdx.x; i < BN * BK; i += 256) {
            if (F == kRowsTimesA) {
                const int k = i % BK, n = i / BK;
                Q[n][k] = n0 + n < Nn && k0 + k < depth ? A[(int64_t)(n0 + n) * a.din + k0 + k] : (T)0.0f;
            } else {
                const int n = i % BN, k = i / BN;
                const T* row = F == kRowsTimesAt ? A + (int64_t)(k0 + k) * a.din : a.Q + (int64_t)(first + k0 + k) * a.ldq;
                Q[n][k] = n0 + n < Nn && k0 + k < depth ? row[n0 + n] : (T)0.0f;
            }
        }
        __syncthreads();
        if constexpr (sizeof(T) == 2) {
            typedef typename Half8<T>::type half8;
#pragma unroll
            for (int q = 0; q < BK; q += 16) {
                const half8 p = *reinterpret_cast<const half8*>(&P[wm + (lane & 31)][q + 8 * (lane >> 5)]);
                const half8 r = *reinterpret_cast<const half8*>(&Q[wn + (lane & 31)][q + 8 * (lane >> 5)]);
                acc = mfma(p, r, acc);
            }
        } else {
#pragma unroll
            for (int q = 0; q < BK; q += 2)
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(P[wm + (lane & 31)][q + (lane >> 5)], Q[wn + (lane & 31)][q + (lane >> 5)], acc, 0, 0, 0);
        }
    }
    const int n = n0 + wn + (lane & 31);
    if (n >= Nn) return;
    const float c = F == kRowsTimesA && a.bias ? (float)a.bias[(int64_t)e * a.dout + n] : 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int m = wm + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5);
        float z = acc[r];
        if (F == kOuterSums) {
            if (m0 + m < M) {
                if (part) part[(int64_t)(m0 + m) * a.din + n] = z;
                else a.out[((int64_t)e * a.dout + m0 + m) * a.din + n] = (T)z;
            }
            continue;
        }
        const int64_t s = (int64_t)first + m;
        if (s >= end) continue;
        if (F == kRowsTimesA) {
            z += c;
            if (a.pre) a.pre[s * a.ldpre + n] = (T)z;
            z = activate<T>(z, a.act);
            if (a.residual) z += (float)a.residual[s * a.ldr + n];
        }
        a.out[s * a.ldo + n] = (T)z;
    }
}

// ---------------------------------------------------------------------------------------------------------------- wide tiles
// 16-bit rows whose addresses, widths and leading dimensions are multiples of sixteen bytes.

typedef int v4i __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

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

// One operand of a tile: R rows (or, TR, columns) of the product by BK of the contraction, 2 R BK bytes of LDS a stage.
//   plain: memory holds R rows of `depth` values; LDS rows of 2 BK bytes, whose sixteen-byte chunks are exchanged so that sixteen lanes
//          that read one chunk of sixteen rows meet all 64 banks
//   TR:    memory holds `depth` rows of R values; LDS rows of 2 R bytes, 64-byte pieces exchanged by row & 3: the transposing read
//          of a half wavefront takes such a piece of four rows
template <class T, int R, int BK, int WAVES, bool TR>
struct Operand {
    static constexpr int kBytes = R * BK * 2, kLoads = kBytes / 1024 / WAVES;  // instructions of a wavefront a stage
    static constexpr int kChunks = TR ? R / 8 : BK / 8, kRowsAtOnce = 64 / kChunks;  // LDS rows that an instruction fills
    const T* base;             // the tile's first value
    int depth;                 // of the contraction
    uint32_t rows;             // plain: rows that exist, counted from base
    uint32_t width;            // TR: values that exist in a row, counted from base
    uint32_t ld;               // bytes
    uint32_t offset[kLoads];
    int chunk;                 // plain: which chunk this lane brings

    // the place of chunk c in LDS row r
    static __device__ __forceinline__ int exchanged(int c, int r)
    {
        return TR ? c ^ ((r & 3) << 2) : BK == 64 ? c ^ ((r >> 1) & 7) : c ^ ((r >> 2) & 3);
    }
    __device__ __forceinline__ void init(const T* b, int d, int exist, int64_t stride, int wave, int lane)
    {
        static_assert(kLoads >= 1 && kBytes % (1024 * WAVES) == 0);
        static_assert(TR || kRowsAtOnce % 16 == 0 || (BK == 64 && kRowsAtOnce == 8));
        base = b;
        depth = d;
        rows = width = (uint32_t)(exist < R ? exist : R);
        ld = (uint32_t)(stride * 2);
        const int c = lane % kChunks, r0 = wave * kLoads * kRowsAtOnce + lane / kChunks;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int r = r0 + q * kRowsAtOnce, from = exchanged(c, r) * 8;
            if (TR) offset[q] = (uint32_t)from < width ? (uint32_t)r * ld + from * 2 : kNowhere;
            else offset[q] = (uint32_t)r * ld + from * 2;
        }
        chunk = c;
    }
    // The stage that starts at k0 of the contraction, an instruction at a time; stages behind the end bring zeros and read nothing.
    __device__ __forceinline__ v4i stage(int k0) const
    {
        const int left = depth - k0, have = left < BK ? left : BK;
        const uint32_t bytes = TR ? (uint32_t)(have - 1) * ld + width * 2 : (rows - 1) * ld + (uint32_t)left * 2;
        return buffer_of(TR ? (const char*)base + (uint64_t)(uint32_t)k0 * ld : (const char*)(base + k0), left > 0 ? bytes : 0u);
    }
    __device__ __forceinline__ void one(int q, uint32_t lds, v4i buffer, int k0, int wave, int lane) const
    {
        // a plain row's end is not the buffer's: chunks behind it (depth is a multiple of eight) are sent nowhere
        const bool past = !TR && exchanged(chunk, wave * kLoads * kRowsAtOnce + lane / kChunks + q * kRowsAtOnce) * 8 >= depth - k0;
        buffer_to_lds(lds + (uint32_t)(wave * kLoads + q) * 1024, past ? kNowhere : offset[q], buffer);
    }
};

// 32 rows by 16 of the contraction as the matrix pipe takes them: lane l holds row l % 32, values 8 (l / 32) .. + 7.
template <class T, int R, int BK, bool TR>
__device__ __forceinline__ typename Half8<T>::type fragment(const char* stage, int r0, int k, int lane)
{
    typedef Operand<T, R, BK, 1, TR> Op;
    union {
        typename Half8<T>::type v;
        s16x4 s[2];
    } f;
    if constexpr (!TR) {
        const int r = r0 + (lane & 31), c = Op::exchanged(k / 8 + (lane >> 5), r);
        f.v = *reinterpret_cast<const typename Half8<T>::type*>(stage + r * (2 * BK) + c * 16);
    } else {
        // Sixteen lanes exchange a block of four rows and sixteen columns: lane 4 j + q brings columns 4 q .. + 3 of row j, lane i gets
        // column i of all four.
        typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
        const int row = k + 8 * (lane >> 5) + ((lane & 15) >> 2), col = r0 + (lane & 16) + 4 * (lane & 3);
        const char* p = stage + row * (2 * R) + Op::exchanged(col >> 3, row) * 16 + (col & 7) * 2;
        f.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)p);
        f.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)(p + 4 * (2 * R)));
    }
    return f.v;
}

template <int N>
__device__ __forceinline__ void stage_ready()
{
    // this wavefront's loads up to N outstanding ones and its reads of the stage before are done; then everyone's are
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
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

template <class T, Form F, int BM, int BN, int BK, int WM, int WN>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64) product_tile_kernel(ProductArgs<T> a, unsigned xtiles)
{
    constexpr int WAVES = (BM / WM) * (BN / WN), THREADS = WAVES * 64;
    constexpr bool TP = F == kOuterSums, TQ = F != kRowsTimesA;
    typedef Operand<T, BM, BK, WAVES, TP> OpP;
    typedef Operand<T, BN, BK, WAVES, TQ> OpQ;
    constexpr int kStage = OpP::kBytes + OpQ::kBytes;
    extern __shared__ __align__(1024) char tile_lds[];
    typedef typename Half8<T>::type half8;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    const int Nn = F == kRowsTimesA ? a.dout : a.din;
    int e, first, end, m0 = 0;
    unsigned x;
    // The chip's eight dies take workgroups in turn; each gets a run of tiles that share operands in its cache.
    const unsigned xcd = blockIdx.x % 8, turn = blockIdx.x / 8;
    float* part = nullptr;
    if (F == kOuterSums) {
        const unsigned run = a.run;
        // Runs differ in length, so every die takes its share of each run's tiles (a run of groups for each die, as below: 726 us
        // for 65536 rows, 2048 -> 1536, on 64 uneven nodes, .. us like this)
        const unsigned ytiles = (a.dout + BM - 1) / BM, each = ytiles * xtiles, share = (each + 7) / 8;
        const unsigned item = each < 16 ? blockIdx.x / each : turn / share, tile = each < 16 ? blockIdx.x % each : xcd * share + turn % share;
        int which;
        e = find_group<THREADS>(a.offsets, a.K, a.rows, [run](unsigned n) { return runs_of(n, run); }, item, which);
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
        // whole tiles first, the groups' last ones, which take less time, when those run out
        uint2 rows_of_tiles = make_uint2(0u, 0u);
        for (int k = threadIdx.x; k < a.K; k += THREADS) {
            group_rows(a.offsets, k, a.rows, first, end);
            rows_of_tiles.x += (unsigned)(end - first) / BM;
            rows_of_tiles.y += (unsigned)(end - first) % BM ? 1u : 0u;
        }
        rows_of_tiles = sum_all<THREADS>(rows_of_tiles);
        const unsigned whole = rows_of_tiles.x * xtiles, run = (whole + 7) / 8, at = xcd * run;
        const unsigned mine = at < whole ? (whole - at < run ? whole - at : run) : 0u;
        int which;
        if (turn < mine) {
            const unsigned row = banded(at + turn, rows_of_tiles.x, xtiles, x);
            e = find_group<THREADS>(a.offsets, a.K, a.rows, [](unsigned n) { return n / BM; }, row, which);
            group_rows(a.offsets, e, a.rows, first, end);
            first += which * BM;
        } else {
            const unsigned rest = rows_of_tiles.y * xtiles, last = (rest + 7) / 8, tile = (7 - xcd) * last + turn - mine;
            if (turn - mine >= last || tile >= rest) return;
            const unsigned row = banded(tile, rows_of_tiles.y, xtiles, x);
            e = find_group<THREADS>(a.offsets, a.K, a.rows, [](unsigned n) { return n % BM ? 1u : 0u; }, row, which);
            group_rows(a.offsets, e, a.rows, first, end);
            first = end - (end - first) % BM;
        }
    }
    e = __builtin_amdgcn_readfirstlane(e);
    first = __builtin_amdgcn_readfirstlane(first);
    end = __builtin_amdgcn_readfirstlane(end);
    const int n0 = __builtin_amdgcn_readfirstlane(x) * BN;
    OpP P;
    OpQ Q;
    const int depth = F == kRowsTimesA ? a.din : F == kRowsTimesAt ? a.dout : end - first;
    if (F == kOuterSums) {
        P.init(a.P + (int64_t)first * a.ldp + m0, depth, a.dout - m0, a.ldp, wave, lane);
        Q.init(a.Q + (int64_t)first * a.ldq + n0, depth, a.din - n0, a.ldq, wave, lane);
    } else {
        P.init(a.P + (int64_t)first * a.ldp, depth, end - first, a.ldp, wave, lane);
        const T* A = a.Q + (int64_t)e * a.dout * a.din;
        Q.init(F == kRowsTimesA ? A + (int64_t)n0 * a.din : A + n0, depth, Nn - n0, a.din, wave, lane);
    }
    f32x16 acc[WM / 32][WN / 32] = {};
    const int steps = (depth + BK - 1) / BK;
    const uint32_t lds = lds_address(tile_lds);
    // blocks of 32 rows that this wavefront has; the columns' ends are left to zeros and to the stores
    const int have = ((F == kOuterSums ? a.dout - m0 : end - first) - wm + 31) / 32;
    constexpr int U = WM / 32, V = WN / 32, kLoads = OpP::kLoads + OpQ::kLoads;
    half8 p[2][U], q[2][V];
    // instruction number n of a stage
    auto fetch = [&](int i, int n, v4i bp, v4i bq) {
        const uint32_t to = lds + (i & 1) * kStage;
        if (n < OpP::kLoads) P.one(n, to, bp, i * BK, wave, lane);
        else Q.one(n - OpP::kLoads, to + OpP::kBytes, bq, i * BK, wave, lane);
    };
    auto fetch_all = [&](int i) {
        const v4i bp = P.stage(i * BK), bq = Q.stage(i * BK);
#pragma unroll
        for (int n = 0; n < kLoads; ++n) fetch(i, n, bp, bq);
    };
    // fragment number f of sixteen of the contraction: the columns', then the rows'
    auto read = [&](int i, int k, int to, int f) {
        const char* stage = tile_lds + (i & 1) * kStage;
        if (f < V) q[to][f] = fragment<T, BN, BK, TQ>(stage + OpP::kBytes, wn + 32 * f, k, lane);
        else p[to][f - V] = fragment<T, BM, BK, TP>(stage, wm + 32 * (f - V), k, lane);
    };
    // The contraction for H blocks of rows.  The pipe takes 32 cycles for a product, and beside each goes a share of the other work: the
    // next sixteen's fragments, and behind the barrier the stage after the next.  (The scheduler would gather the reads in front of
    // their use: it is kept out.)  The last fragments of a stage are in registers when the barrier comes, so that its buffer is free and
    // everyone's arrival hides behind products that need nothing.
    auto contract = [&](auto blocks) {
        constexpr int H = decltype(blocks)::value, kReads = H + V, kSlots = H * V;
#pragma unroll
        for (int f = 0; f < kReads; ++f) read(0, 0, 0, f);
        for (int i = 0; i < steps; ++i) {
#pragma unroll
            for (int j = 0; j < BK / 16; ++j) {
                const bool last = j == BK / 16 - 1;
                v4i bp = {}, bq = {};
                if (last) {
                    stage_ready<0>();
                    bp = P.stage((i + 2) * BK);
                    bq = Q.stage((i + 2) * BK);
                }
#pragma unroll
                for (int t = 0; t < kSlots; ++t) {
                    acc[t / V][t % V] = mfma(q[j & 1][t % V], p[j & 1][t / V], acc[t / V][t % V]);
#pragma unroll
                    for (int f = t * kReads / kSlots; f < (t + 1) * kReads / kSlots; ++f) read(last ? i + 1 : i, last ? 0 : 16 * (j + 1), (j + 1) & 1, f);
                    if (last) {
#pragma unroll
                        for (int n = t * kLoads / kSlots; n < (t + 1) * kLoads / kSlots; ++n) fetch(i + 2, n, bp, bq);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };
    if (steps > 0) {
        fetch_all(0);
        stage_ready<0>();
        fetch_all(1);
        // a group's last tile leaves out the blocks of rows that it does not have
        if (have >= U) {
            contract(std::integral_constant<int, U>{});
        } else if (have >= 2 && U > 2) {
            if (have == 2) contract(std::integral_constant<int, (U > 2 ? 2 : 1)>{});
            else contract(std::integral_constant<int, (U > 3 ? 3 : 1)>{});
        } else if (have == 1) {
            contract(std::integral_constant<int, 1>{});
        } else {
            for (int i = 0; i < steps; ++i) {
                stage_ready<0>();
                fetch_all(i + 2);
            }
        }
    }
    // Results go out by rows: a wavefront's 32 x WN values change from the pipe's layout (lane: row, four columns at a time) to eight
    // columns a lane through LDS rows of WN + 4 floats, which keep sixteen lanes on sixteen places both ways.
    constexpr int kRow = WN + 4, kLanes = WN / 8, kAtOnce = 64 / kLanes;
    static_assert(WAVES * 32 * kRow * 4 <= 2 * kStage);
    stage_ready<0>();                               // no one reads the stages any more, or writes to them
    float* turned = reinterpret_cast<float*>(tile_lds) + wave * 32 * kRow;
    const int n = n0 + wn + lane % kLanes * 8;
    Piece<T> c;
    if (F == kRowsTimesA && a.bias && n < Nn) c.load(a.bias + (int64_t)e * a.dout + n);
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
#pragma unroll 1
        for (int r = lane / kLanes; r < 32; r += kAtOnce) {
            const int64_t row = row0 + r;
            if (row >= rows_end || n >= Nn) continue;
            float x[8];
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(turned + r * kRow + lane % kLanes * 8);
            *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(turned + r * kRow + lane % kLanes * 8 + 4);
            Piece<T> y, z, d;
            if (F == kRowsTimesA) {
                if (a.residual) d.load(a.residual + row * a.ldr + n);
                if (a.bias)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] += (float)c.e[j];
                if (a.pre) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) z.e[j] = (T)x[j];
                    z.store(a.pre + row * a.ldpre + n);
                }
                if (a.act == SOM_ACT_SILU) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = activate<T>(x[j], SOM_ACT_SILU);
                } else if (a.act == SOM_ACT_GELU) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = activate<T>(x[j], SOM_ACT_GELU);
                } else if (a.act == SOM_ACT_GELU_TANH) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = activate<T>(x[j], SOM_ACT_GELU_TANH);
                } else if (a.act == SOM_ACT_RELU) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = activate<T>(x[j], SOM_ACT_RELU);
                }
                if (a.residual)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] += (float)d.e[j];
            }
            if (F == kOuterSums && part) {
                *reinterpret_cast<float4*>(part + row * a.din + n) = *reinterpret_cast<const float4*>(x);
                *reinterpret_cast<float4*>(part + row * a.din + n + 4) = *reinterpret_cast<const float4*>(x + 4);
                continue;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y.e[j] = (T)x[j];
            T* out = F == kOuterSums ? a.out + ((int64_t)e * a.dout + row) * a.din : a.out + row * a.ldo;
            y.store(out + n);
        }
    }
}

// dz = dy act'(z), dense (where there is an activation: dz not null), and its column sums over a run of a group's rows (dbias not null):
// LANES lanes of N columns share a row.
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
        for (int r = first + threadIdx.x / LANES; r < end; r += kRows) {
            Piece<T, N> g;
            g.load(dY + (int64_t)r * lddy + at);
            if (dz) {
                Piece<T, N> z;
                z.load(pre + (int64_t)r * ldpre + at);
#pragma unroll
                for (int j = 0; j < N; ++j) g.e[j] = (T)((float)g.e[j] * Math<sizeof(T) == 4>::slope((float)z.e[j], act));
                g.store(dz + (int64_t)r * dout + at);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) s[j] += (float)g.e[j];
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

// The sums of groups with more than one run, run after run: `count` values a group.
template <class T>
__global__ void __launch_bounds__(256) runs_join_kernel(const int32_t* __restrict__ offsets, int K, int rows, int run, const float* __restrict__ parts,
                                                        int64_t count, T* __restrict__ out)
{
    int which, lo, hi;
    const int e = find_group<256>(offsets, K, rows, [run](unsigned n) { return n > (unsigned)run ? 1u : 0u; }, blockIdx.y, which);
    if (e < 0) return;
    group_rows(offsets, e, rows, lo, hi);
    const int runs = (int)runs_of(hi - lo, run);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        float s = parts[run_slot(lo, lo, run) * count + i];
        for (int c = 1; c < runs; ++c) s += parts[run_slot(lo + c * run, lo, run) * count + i];
        out[(int64_t)e * count + i] = (T)s;
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

static bool sixteen(const void* p) { return (uintptr_t)p % 16 == 0; }

// What the wide tiles ask of a call: every row of every matrix starts at a multiple of sixteen bytes and has whole chunks of them.
template <class T>
static bool product_wide(const ProductArgs<T>& a)
{
    const bool few = ((a.dout + 255) / 256 * (int64_t)((a.din + 255) / 256 + 1)) * (a.rows / 256 + a.K + 2) < 1 << 22;       // fewer than 2^32 work-items
    return few && sizeof(T) == 2 && a.din % 8 == 0 && a.dout % 8 == 0 && a.ldp % 8 == 0 && a.ldq % 8 == 0 && a.ldo % 8 == 0 && a.ldr % 8 == 0 &&
           a.ldpre % 8 == 0 && sixteen(a.P) && sixteen(a.Q) && sixteen(a.out) && sixteen(a.bias) && sixteen(a.residual) && sixteen(a.pre);
}

template <class T, Form F, int BM, int BN, int BK, int WM, int WN>
static int product_tile_launch(som_ctx* ctx, const ProductArgs<T>& a, const char* what)
{
    constexpr int lds = 2 * (BM + BN) * BK * 2;
    static bool attr_set_dev[kMaxDevices] = {};
    bool& attr_set = attr_set_dev[ctx->device];
    auto kern = product_tile_kernel<T, F, BM, BN, BK, WM, WN>;
    if (!attr_set) {
        if (int rc = check_hip(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds),
                               "raising the dynamic LDS limit"))
            return rc;
        attr_set = true;
    }
    const int64_t xtiles = ((F == kRowsTimesA ? a.dout : a.din) + BN - 1) / BN;
    const int64_t ytiles = F == kOuterSums ? most_runs(a.rows, a.K, a.run) * ((a.dout + BM - 1) / BM) : most_tiles(a.rows, a.K, a.offsets, BM);
    const int64_t each = (a.dout + BM - 1) / BM * xtiles;              // tiles of a run
    const int64_t groups = F != kOuterSums ? ((xtiles * ytiles + 7) / 8 + 2) * 8 : each < 16 ? xtiles * ytiles : (each + 7) / 8 * 8 * (ytiles * xtiles / each);
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3((BM / WM) * (BN / WN) * 64), lds, ctx->stream, a, (unsigned)xtiles);
    return check_hip(ctx, hipGetLastError(), what);
}

template <class T, Form F>
static int product_launch(som_ctx* ctx, const ProductArgs<T>& a, const char* what)
{
    if constexpr (sizeof(T) == 2) {
        if (product_wide(a)) return product_tile_launch<T, F, 256, 256, 64, 128, 64>(ctx, a, what);
    }
    const unsigned nx = (unsigned)(((F == kRowsTimesA ? a.dout : a.din) + 63) / 64);
    dim3 grid;
    if (F == kOuterSums) {
        grid = dim3(nx, (unsigned)((a.dout + 63) / 64), (unsigned)most_runs(a.rows, a.K, a.run));
    } else {
        const int64_t tiles = most_tiles(a.rows, a.K, a.offsets, 64);
        const int64_t y = tiles < 32768 ? tiles : 32768;
        grid = dim3(nx, (unsigned)y, (unsigned)((tiles + y - 1) / y));
    }
    hipLaunchKernelGGL((product_any_kernel<T, F>), grid, dim3(256), 0, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), what);
}

template <class T>
static int product_typed(som_ctx* ctx, const NodeProduct& p)
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
    a.ldr = p.ldr;
    a.pre = (T*)p.pre;
    a.ldpre = p.ldpre;
    a.out = (T*)p.out;
    a.ldo = p.ldo;
    a.act = p.act;
    return product_launch<T, kRowsTimesA>(ctx, a, "product launch");
}

// Kernel and columns of a workgroup for the slopes and biases of `dout` columns.
template <class T>
static auto slope_kernel_for(int32_t dout, int& columns)
{
    constexpr int N = Piece<T>::N;
    const int lanes = dout < N ? row_lanes(dout, 8) : row_lanes((dout + N - 1) / N, 64);
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
    const int64_t longer = rows / (run + 1), y = longer < K ? longer : K, blocks = (count + 1023) / 1024;        // groups with more than one run, at most
    if (y == 0) return SOM_OK;
    hipLaunchKernelGGL(runs_join_kernel<T>, dim3((unsigned)(blocks < 4096 ? blocks : 4096), (unsigned)y), dim3(256), 0, ctx->stream, offsets, K, (int)rows,
                       run, parts, count, out);
    return check_hip(ctx, hipGetLastError(), "product gradient join launch");
}

template <class T>
static int product_grad_typed(som_ctx* ctx, const NodeProductGrad& p)
{
    const bool sloped = p.act != SOM_ACT_NONE && p.rows > 0;
    ProductArgs<T> a{};
    a.offsets = p.offsets;
    a.rows = (int)p.rows;
    a.K = p.K;
    a.din = p.din;
    a.dout = p.dout;
    // workspace: dz, then the runs' sums (of the biases, then of the matrices)
    int columns;
    auto slopes = slope_kernel_for<T>(p.dout, columns);
    const int64_t blocks = (p.dout + columns - 1) / columns;
    int bias_run = run_rows(ctx, p.rows, p.K, blocks, 64);
    if (bias_run > 256) bias_run = p.rows / 256 + p.K < 1 << 30 ? 256 : bias_run;
    a.run = run_rows(ctx, p.rows, p.K, (int64_t)((p.dout + 255) / 256) * ((p.din + 255) / 256), 512);
    const size_t dz_bytes = sloped ? ((size_t)p.rows * p.dout * sizeof(T) + 255) / 256 * 256 : 0;
    const size_t bias_parts = p.dbias && p.rows > bias_run ? (size_t)run_slots(p.rows, bias_run) * p.dout : 0;
    const size_t sum_parts = p.dA && p.rows > a.run ? (size_t)run_slots(p.rows, a.run) * p.dout * p.din : 0;
    if (dz_bytes + bias_parts + sum_parts)
        if (int rc = models_workspace(ctx, dz_bytes + (bias_parts > sum_parts ? bias_parts : sum_parts) * sizeof(float))) return rc;
    T* dz = (T*)ctx->models_blob;
    float* parts = (float*)((char*)ctx->models_blob + dz_bytes);
    if (sloped || p.dbias) {
        const int64_t runs = most_runs(p.rows, p.K, bias_run), y = runs < 32768 ? runs : 32768;
        hipLaunchKernelGGL(slopes, dim3((unsigned)blocks, (unsigned)y, (unsigned)((runs + y - 1) / y)), dim3(256), 0, ctx->stream, (const T*)p.dY, p.lddy,
                           (const T*)p.pre, p.ldpre, p.offsets, p.K, (int)p.rows, p.dout, p.act, sloped ? dz : nullptr, (T*)p.dbias, bias_run, parts);
        if (int rc = check_hip(ctx, hipGetLastError(), "product gradient slope launch")) return rc;
        if (bias_parts)
            if (int rc = runs_join(ctx, p.offsets, p.K, p.rows, bias_run, parts, p.dout, (T*)p.dbias)) return rc;
    }
    a.P = sloped ? dz : (const T*)p.dY;
    a.ldp = sloped ? p.dout : p.lddy;
    if (p.dX && p.rows > 0) {
        a.Q = (const T*)p.A;
        a.out = (T*)p.dX;
        a.ldo = p.lddx;
        if (int rc = product_launch<T, kRowsTimesAt>(ctx, a, "product gradient (rows) launch")) return rc;
    }
    if (p.dA) {
        a.Q = (const T*)p.X;
        a.ldq = p.ldx;
        a.out = (T*)p.dA;
        a.ldo = p.din;
        a.parts = parts;
        if (int rc = product_launch<T, kOuterSums>(ctx, a, "product gradient (matrices) launch")) return rc;
        if (sum_parts) return runs_join(ctx, p.offsets, p.K, p.rows, a.run, parts, (int64_t)p.dout * p.din, (T*)p.dA);
    }
    return SOM_OK;
}

int node_product_run(som_ctx* ctx, int type, const NodeProduct& p)
{
    if (p.rows == 0) return SOM_OK;
    if (type == SOM_ROWS_FLOAT) return product_typed<float>(ctx, p);
    if (type == SOM_ROWS_BFLOAT) return product_typed<__bf16>(ctx, p);
    return product_typed<_Float16>(ctx, p);
}

int node_product_grad_run(som_ctx* ctx, int type, const NodeProductGrad& p)
{
    if (type == SOM_ROWS_FLOAT) return product_grad_typed<float>(ctx, p);
    if (type == SOM_ROWS_BFLOAT) return product_grad_typed<__bf16>(ctx, p);
    return product_grad_typed<_Float16>(ctx, p);
}

} // namespace som
