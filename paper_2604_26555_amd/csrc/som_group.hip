// Rows sorted by node and back: the way of a table's rows to one local model per node.
//
//   group         places of the (row, node) pairs p = t k + j in the nodes' order, pairs of a node in the order of p:
//                 slot_p = offsets_{node_p} + #{p' < p: node_p' = node_p},  order_{slot_p} = p
//   dispatch      Y_{slot(t,j)} = w_tj X_t
//   combine       out_t = sum_j w_tj Y_{slot(t,j)}                                  (float32, j ascending)
//   combine_grad  dY_{slot(t,j)} = w_tj dout_t,  dw_tj = <dout_t, Y_{slot(t,j)}>    (float32)
//
// Pairs without a node (node outside 0..K-1) have slot -1 and take part in nothing; the sort keeps them as node K, behind
// all others, which gives every entry of `order` a writer.
#include "som_rows.hpp"

namespace som {

constexpr int kGroupBlocks = 1024;        // wavefronts that share the pairs
constexpr int kGroupWords = 32768 + 64;   // counters of a workgroup in LDS (131 KB)
constexpr int64_t kGroupSmall = 16384;    // pairs that one workgroup sorts, in one launch
constexpr int kGroupStarts = 2048;        // nodes whose starts every workgroup of the scatter sums up by itself

__device__ __forceinline__ int pair_node(const int32_t* __restrict__ node, int64_t p, int K)
{
    const int b = node[p];
    return b >= 0 && b < K ? b : K;
}

// Lanes of the wavefront whose value is this lane's: a ballot for every bit.
__device__ __forceinline__ uint64_t lanes_alike(int b, int bits)
{
    uint64_t m = ~0ull;
    for (int q = 0; q < bits; ++q) {
        const bool set = (b >> q) & 1;
        const uint64_t v = __ballot(set);
        m &= set ? v : ~v;
    }
    return m;
}

// The chip's eight dies take workgroups in turn; each gets a run of them, so that lines which neighbours share are written whole from one
// die's cache.  (1,000,000 rows of 50 floats to 1024 nodes: dispatch 107 us in turn, 77 in runs.)
__device__ __forceinline__ int64_t run_of_die(unsigned groups) { return (int64_t)(blockIdx.x % 8) * ((groups + 7) / 8) + blockIdx.x / 8; }

// Exclusive sums over the threads of a workgroup.
template <int THREADS>
__device__ __forceinline__ uint32_t sums_before(uint32_t mine)
{
    __shared__ uint32_t wave_sum[THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 63) wave_sum[wave] = incl;
    __syncthreads();
    uint32_t at = incl - mine;
    for (int w = 0; w < wave; ++w) at += wave_sum[w];
    return at;
}

// A wavefront's pairs [lo, hi) to their places, 64 at a time in order; place[b]: the next place of node b (LDS, this wavefront's own).
__device__ __forceinline__ void scatter_pairs(const int32_t* __restrict__ node, int64_t lo, int64_t hi, int K, volatile uint32_t* place,
                                              int32_t* __restrict__ order, int32_t* __restrict__ slot)
{
    const int lane = threadIdx.x & 63, bits = 32 - __builtin_clz((unsigned)(K + 1));
    int next = lo + lane < hi ? pair_node(node, lo + lane, K) : K + 1;
    for (int64_t p0 = lo; p0 < hi; p0 += 64) {
        const int64_t p = p0 + lane;
        const int b = next;
        next = p + 64 < hi ? pair_node(node, p + 64, K) : K + 1;
        const uint64_t alike = lanes_alike(b, bits);
        const int rank = __builtin_popcountll(alike & ((1ull << lane) - 1ull));
        if (p < hi) {
            const uint32_t at = place[b] + rank;
            __builtin_amdgcn_wave_barrier();
            if ((alike >> lane) == 1ull) place[b] = at + 1u;  // the last of its node
            if (slot) slot[p] = b < K ? (int32_t)at : -1;
            if (order) order[at] = b < K ? (int32_t)p : -1;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Few pairs: one workgroup of 16 wavefronts, `waves` of which have counters (and pairs).  What it takes is latency: a row's eight pairs and
// 128 nodes 4 us on the GPU, and 36 us with the four launches that larger calls had.
__global__ void __launch_bounds__(1024) group_small_kernel(const int32_t* __restrict__ node, int pairs, int K, int waves, int32_t* __restrict__ offsets,
                                                           int32_t* __restrict__ order, int32_t* __restrict__ slot)
{
    extern __shared__ uint32_t group_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, columns = K + 1;
    for (int i = tid; i < waves * columns; i += 1024) group_lds[i] = 0u;
    const int each = ((pairs + waves - 1) / waves + 63) / 64 * 64, lo = wave < waves ? wave * each : pairs, hi = lo + each < pairs ? lo + each : pairs;
    __syncthreads();
    for (int p = lo + lane; p < hi; p += 64) atomicAdd(&group_lds[wave * columns + pair_node(node, p, K)], 1u);
    __syncthreads();
    const int per = (columns + 1023) / 1024, k0 = tid * per, k1 = k0 + per < columns ? k0 + per : columns;
    uint32_t mine = 0u;
    for (int k = k0; k < k1; ++k)
        for (int w = 0; w < waves; ++w) mine += group_lds[w * columns + k];
    uint32_t at = sums_before<1024>(mine);
    for (int k = k0; k < k1; ++k) {
        offsets[k] = (int32_t)at;
        for (int w = 0; w < waves; ++w) {
            const uint32_t n = group_lds[w * columns + k];
            group_lds[w * columns + k] = at;
            at += n;
        }
    }
    __syncthreads();
    if (lo < hi) scatter_pairs(node, lo, hi, K, group_lds + wave * columns, order, slot);
}

__global__ void __launch_bounds__(256) group_hist_kernel(const int32_t* __restrict__ node, int64_t pairs, int K, int64_t per_block, int blocks,
                                                         unsigned groups, uint32_t* __restrict__ hist)
{
    extern __shared__ uint32_t group_lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t block = run_of_die(groups) * (blockDim.x >> 6) + wave;
    uint32_t* count = group_lds + wave * (K + 1);
    for (int k = lane; k <= K; k += 64) count[k] = 0u;
    wave_in_order();
    if (block >= blocks) return;                              // (no barrier: a wavefront works on its own)
    const int64_t lo = block * per_block, hi = lo + per_block < pairs ? lo + per_block : pairs;
    for (int64_t p = lo + lane; p < hi; p += 256) {
        int b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) b[u] = p + 64 * u < hi ? pair_node(node, p + 64 * u, K) : -1;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (b[u] >= 0) atomicAdd(&count[b[u]], 1u);
    }
    wave_in_order();
    for (int k = lane; k <= K; k += 64) hist[(size_t)block * (K + 1) + k] = count[k];
}

// hist[block][k] -> pairs of node k in the blocks before; total[k]: all of them.  16 nodes and 64 runs of blocks per workgroup; a run's
// counts are read once, all together.
__global__ void __launch_bounds__(1024) group_columns_kernel(uint32_t* __restrict__ hist, int columns, int blocks, uint32_t* __restrict__ total)
{
    constexpr int kRun = kGroupBlocks / 64;
    __shared__ uint32_t run[64][17];
    const int l = threadIdx.x & 15, seg = threadIdx.x >> 4;
    const int k = blockIdx.x * 16 + l, kc = k < columns ? k : columns - 1;
    const int per = (blocks + 63) / 64, lo = seg * per;
    uint32_t v[kRun], s = 0u;
#pragma unroll
    for (int u = 0; u < kRun; ++u) v[u] = u < per && lo + u < blocks ? hist[(size_t)(lo + u) * columns + kc] : 0u;
#pragma unroll
    for (int u = 0; u < kRun; ++u) s += v[u];
    run[seg][l] = s;
    __syncthreads();
    // sums over the runs: a wavefront takes a column of sixteen
    {
        const int column = threadIdx.x >> 6, r = threadIdx.x & 63;
        uint32_t incl = run[r][column];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(incl, o);
            if (r >= o) incl += x;
        }
        run[r][column] = incl;
    }
    __syncthreads();
    if (k >= columns) return;
    if (seg == 63) total[k] = run[63][l];
    uint32_t at = run[seg][l] - s;
#pragma unroll
    for (int u = 0; u < kRun; ++u) {
        if (u < per && lo + u < blocks) hist[(size_t)(lo + u) * columns + k] = at;
        at += v[u];
    }
}

// total[0..K] -> exclusive sums start[0..K] and offsets[0..K] (start[K] = offsets[K]: pairs that have a node)
__global__ void __launch_bounds__(1024) group_starts_kernel(const uint32_t* __restrict__ total, int K, uint32_t* __restrict__ start,
                                                            int32_t* __restrict__ offsets)
{
    const int per = (K + 1024) / 1024, k0 = threadIdx.x * per;
    uint32_t mine = 0u;
    for (int u = 0; u < per; ++u) mine += k0 + u < K ? total[k0 + u] : 0u;
    uint32_t at = sums_before<1024>(mine);
    for (int u = 0; u < per && k0 + u <= K; ++u) {
        start[k0 + u] = at;
        offsets[k0 + u] = (int32_t)at;
        at += k0 + u < K ? total[k0 + u] : 0u;
    }
}

// OWN: the starts are summed up from the totals here (K < kGroupStarts, four wavefronts), and the first workgroup stores the offsets.
template <bool OWN>
__global__ void __launch_bounds__(256) group_scatter_kernel(const int32_t* __restrict__ node, int64_t pairs, int K, int64_t per_block, int blocks,
                                                            unsigned groups, const uint32_t* __restrict__ hist, const uint32_t* __restrict__ start,
                                                            int32_t* __restrict__ offsets, int32_t* __restrict__ order, int32_t* __restrict__ slot)
{
    extern __shared__ uint32_t group_lds[];
    __shared__ uint32_t starts[OWN ? kGroupStarts : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t block = run_of_die(groups) * (blockDim.x >> 6) + wave;
    if (OWN) {
        constexpr int kPer = kGroupStarts / 256;
        uint32_t v[kPer], mine = 0u;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int k = threadIdx.x * kPer + u;
            v[u] = k < K ? start[k] : 0u;                     // (the totals)
            mine += v[u];
        }
        uint32_t at = sums_before<256>(mine);
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int k = threadIdx.x * kPer + u;
            starts[k] = at;
            if (blockIdx.x == 0 && k <= K) offsets[k] = (int32_t)at;
            at += v[u];
        }
        __syncthreads();
    }
    if (block >= blocks) return;                              // (no barrier below: a wavefront works on its own)
    uint32_t* place = group_lds + wave * (K + 1);
    for (int k = lane; k <= K; k += 64) place[k] = (OWN ? starts[k] : start[k]) + hist[(size_t)block * (K + 1) + k];
    wave_in_order();
    const int64_t lo = block * per_block, hi = lo + per_block < pairs ? lo + per_block : pairs;
    scatter_pairs(node, lo, hi, K, place, order, slot);
}

// Workgroups for `items` rows or pairs, `each` of them a workgroup at a time and `across` workgroups for each, in eights: a grid holds fewer
// than 2^32 work-items.
static dim3 row_grid(int64_t items, int each, int64_t across = 1)
{
    const int64_t groups = ((items + each - 1) / each + 7) / 8 * 8, most = (1 << 23) / across / 8 * 8;
    return dim3((unsigned)((groups < most ? groups : most) * across));
}

// A lane per piece of a row; LANES of them and `across` neighbouring workgroups share a row (with a row's parts in different corners of the grid
// 16384 rows of 2048 bf16 to four nodes: sorted 91 us, 75 like this; combined 83 and 70).
template <class T, int LANES>
__global__ void __launch_bounds__(256) dispatch_kernel(const T* __restrict__ X, int64_t rows, int D, int64_t ldx, const int32_t* __restrict__ slot, int k,
                                                       const float* __restrict__ weight, T* __restrict__ Y, int64_t places, int64_t ldy, unsigned across)
{
    constexpr int N = Piece<T>::N;
    const unsigned group = (unsigned)run_of_die(gridDim.x);
    const int c = group % across * LANES + threadIdx.x % LANES;
    if (c * N >= D) return;
    const int64_t at = piece_at<T>(c, D);
    for (int64_t t = (int64_t)(group / across) * (256 / LANES) + threadIdx.x / LANES; t < rows; t += (int64_t)(gridDim.x / across) * (256 / LANES)) {
        Piece<T> x;
        x.load(X + t * ldx + at);
        for (int j0 = 0; j0 < k; j0 += 4) {
            int s[4];
            float w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t p = t * k + (j0 + u < k ? j0 + u : j0);
                s[u] = slot[p];
                w[u] = weight ? weight[p] : 1.0f;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (j0 + u >= k || (uint64_t)(int64_t)s[u] >= (uint64_t)places) continue;
                Piece<T> y = x;
                if (weight)
#pragma unroll
                    for (int e = 0; e < N; ++e) y.e[e] = (T)((float)x.e[e] * w[u]);
                y.store(Y + (int64_t)s[u] * ldy + at);
            }
        }
    }
}

template <class T, int LANES>
__global__ void __launch_bounds__(256) combine_kernel(const T* __restrict__ Y, int64_t places, int D, int64_t ldy, const int32_t* __restrict__ slot,
                                                      int64_t rows, int k, const float* __restrict__ weight, T* __restrict__ out, int64_t ldo, unsigned across)
{
    constexpr int N = Piece<T>::N;
    const unsigned group = (unsigned)run_of_die(gridDim.x);
    const int c = group % across * LANES + threadIdx.x % LANES;
    if (c * N >= D) return;
    const int64_t at = piece_at<T>(c, D);
    for (int64_t t = (int64_t)(group / across) * (256 / LANES) + threadIdx.x / LANES; t < rows; t += (int64_t)(gridDim.x / across) * (256 / LANES)) {
        float sum[N];
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0.0f;
        for (int j0 = 0; j0 < k; j0 += 4) {
            int s[4];
            float w[4];
            Piece<T> y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t p = t * k + (j0 + u < k ? j0 + u : j0);
                s[u] = slot[p];
                w[u] = weight ? weight[p] : 1.0f;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j0 + u < k && (uint64_t)(int64_t)s[u] < (uint64_t)places) y[u].load(Y + (int64_t)s[u] * ldy + at);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (j0 + u >= k || (uint64_t)(int64_t)s[u] >= (uint64_t)places) continue;
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] = fmaf(w[u], (float)y[u].e[e], sum[e]);
            }
        }
        Piece<T> o;
#pragma unroll
        for (int e = 0; e < N; ++e) o.e[e] = (T)sum[e];
        o.store(out + t * ldo + at);
    }
}

// A group of lanes per pair.
template <class T, int LANES>
__global__ void __launch_bounds__(256) combine_grad_kernel(const T* __restrict__ dout, int64_t rows, int D, int64_t lddo, const T* __restrict__ Y,
                                                           int64_t places, int64_t ldy, const int32_t* __restrict__ slot, int k,
                                                           const float* __restrict__ weight, T* __restrict__ dY, int64_t lddy,
                                                           float* __restrict__ dweight)
{
    constexpr int N = Piece<T>::N;
    const int l = threadIdx.x % LANES;
    const int pieces = (D + N - 1) / N;
    const int64_t pairs = rows * k;
    for (int64_t p = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; p < pairs; p += (int64_t)gridDim.x * (256 / LANES)) {
        const int s = slot[p];
        float dot = 0.0f;
        if ((uint64_t)(int64_t)s < (uint64_t)places) {
            const T* g = dout + (int64_t)((uint32_t)p / (uint32_t)k) * lddo;
            const float w = weight ? weight[p] : 1.0f;
            for (int c0 = l; c0 < pieces; c0 += 4 * LANES) {
                Piece<T> x[4], y[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (c0 + q * LANES >= pieces) continue;
                    const int64_t at = piece_at<T>(c0 + q * LANES, D);
                    x[q].load(g + at);
                    if (dweight) y[q].load(Y + (int64_t)s * ldy + at);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = c0 + q * LANES;
                    if (c >= pieces) continue;
                    const int64_t at = piece_at<T>(c, D);
                    const int again = c * N - (int)at;        // leading elements that the piece before holds too
                    if (dweight)
#pragma unroll
                        for (int u = 0; u < N; ++u) dot = u >= again ? fmaf((float)x[q].e[u], (float)y[q].e[u], dot) : dot;
                    if (dY) {
                        if (weight)
#pragma unroll
                            for (int u = 0; u < N; ++u) x[q].e[u] = (T)((float)x[q].e[u] * w);
                        x[q].store(dY + (int64_t)s * lddy + at);
                    }
                }
            }
        }
        if (!dweight) continue;
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) dot += __shfl_xor(dot, o);
        if (l == 0) dweight[p] = dot;
    }
}

// Rows of fewer elements than a piece: a lane per row or pair.
template <class T>
__global__ void __launch_bounds__(256) dispatch_short_kernel(const T* __restrict__ X, int64_t rows, int D, int64_t ldx, const int32_t* __restrict__ slot,
                                                             int k, const float* __restrict__ weight, T* __restrict__ Y, int64_t places, int64_t ldy)
{
    for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < rows * k; p += (int64_t)gridDim.x * 256) {
        const int s = slot[p];
        if ((uint64_t)(int64_t)s >= (uint64_t)places) continue;
        const T* from = X + (int64_t)((uint32_t)p / (uint32_t)k) * ldx;
        for (int d = 0; d < D; ++d) Y[(int64_t)s * ldy + d] = weight ? (T)((float)from[d] * weight[p]) : from[d];
    }
}

template <class T>
__global__ void __launch_bounds__(256) combine_short_kernel(const T* __restrict__ Y, int64_t places, int D, int64_t ldy, const int32_t* __restrict__ slot,
                                                            int64_t rows, int k, const float* __restrict__ weight, T* __restrict__ out, int64_t ldo)
{
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < rows; t += (int64_t)gridDim.x * 256) {
        for (int d = 0; d < D; ++d) {
            float sum = 0.0f;
            for (int j = 0; j < k; ++j) {
                const int s = slot[t * k + j];
                if ((uint64_t)(int64_t)s >= (uint64_t)places) continue;
                sum = fmaf(weight ? weight[t * k + j] : 1.0f, (float)Y[(int64_t)s * ldy + d], sum);
            }
            out[t * ldo + d] = (T)sum;
        }
    }
}

template <class T>
__global__ void __launch_bounds__(256) combine_grad_short_kernel(const T* __restrict__ dout, int64_t rows, int D, int64_t lddo, const T* __restrict__ Y,
                                                                 int64_t places, int64_t ldy, const int32_t* __restrict__ slot, int k,
                                                                 const float* __restrict__ weight, T* __restrict__ dY, int64_t lddy,
                                                                 float* __restrict__ dweight)
{
    for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < rows * k; p += (int64_t)gridDim.x * 256) {
        const int s = slot[p];
        float dot = 0.0f;
        if ((uint64_t)(int64_t)s < (uint64_t)places) {
            const T* from = dout + (int64_t)((uint32_t)p / (uint32_t)k) * lddo;
            for (int d = 0; d < D; ++d) {
                const float g = (float)from[d];
                if (dweight) dot = fmaf(g, (float)Y[(int64_t)s * ldy + d], dot);
                if (dY) dY[(int64_t)s * lddy + d] = weight ? (T)(g * weight[p]) : from[d];
            }
        }
        if (dweight) dweight[p] = dot;
    }
}

int group_run(som_ctx* ctx, const int32_t* node, int64_t pairs, int32_t K, int32_t* offsets, int32_t* order, int32_t* slot)
{
    if (pairs == 0) return launch_fill_zero(ctx, offsets, (size_t)(K + 1) * sizeof(int32_t));
    static bool attr_set_dev[kMaxDevices] = {};
    bool& attr_set = attr_set_dev[ctx->device];
    if (!attr_set) {
        for (const void* f : {reinterpret_cast<const void*>(group_small_kernel), reinterpret_cast<const void*>(group_hist_kernel),
                              reinterpret_cast<const void*>(group_scatter_kernel<true>), reinterpret_cast<const void*>(group_scatter_kernel<false>)})
            if (int rc = check_hip(ctx, hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kGroupWords * 4),
                                   "raising the dynamic LDS limit"))
                return rc;
        attr_set = true;
    }
    const int most = kGroupWords / (K + 1);                   // wavefronts of a workgroup that have counters, one at least: K <= kGroupNodes
    if (pairs <= kGroupSmall && most >= 4) {
        const int64_t useful = (pairs + 63) / 64;
        const int waves = (int)(useful < most ? (useful < 16 ? useful : 16) : most < 16 ? most : 16);
        hipLaunchKernelGGL(group_small_kernel, dim3(1), dim3(1024), (size_t)waves * (K + 1) * sizeof(uint32_t), ctx->stream, node, (int)pairs, K, waves,
                           offsets, order, slot);
        return check_hip(ctx, hipGetLastError(), "group launch");
    }
    int64_t per_block = (pairs + kGroupBlocks - 1) / kGroupBlocks;
    per_block = per_block < 256 ? 256 : (per_block + 63) / 64 * 64;
    const int blocks = (int)((pairs + per_block - 1) / per_block);
    const int waves = most >= 4 ? 4 : most;
    const size_t words = (size_t)(K + 1) * (blocks + 2);
    if (int rc = models_workspace(ctx, words * sizeof(uint32_t))) return rc;
    uint32_t* hist = (uint32_t*)ctx->models_blob;
    uint32_t* total = hist + (size_t)(K + 1) * blocks;
    uint32_t* start = total + K + 1;
    const size_t lds = (size_t)waves * (K + 1) * sizeof(uint32_t);
    const unsigned groups = (blocks + waves - 1) / waves;
    const dim3 grid((groups + 7) / 8 * 8), wg(64 * waves);
    hipLaunchKernelGGL(group_hist_kernel, grid, wg, lds, ctx->stream, node, pairs, K, per_block, blocks, groups, hist);
    if (int rc = check_hip(ctx, hipGetLastError(), "group histogram launch")) return rc;
    hipLaunchKernelGGL(group_columns_kernel, dim3((K + 16) / 16), dim3(1024), 0, ctx->stream, hist, K + 1, blocks, total);
    if (int rc = check_hip(ctx, hipGetLastError(), "group columns launch")) return rc;
    if (K < kGroupStarts) {
        hipLaunchKernelGGL(group_scatter_kernel<true>, grid, wg, lds, ctx->stream, node, pairs, K, per_block, blocks, groups, hist, total, offsets, order,
                           slot);
        return check_hip(ctx, hipGetLastError(), "group scatter launch");
    }
    hipLaunchKernelGGL(group_starts_kernel, dim3(1), dim3(1024), 0, ctx->stream, total, K, start, offsets);
    if (int rc = check_hip(ctx, hipGetLastError(), "group starts launch")) return rc;
    hipLaunchKernelGGL(group_scatter_kernel<false>, grid, wg, lds, ctx->stream, node, pairs, K, per_block, blocks, groups, hist, start, offsets, order, slot);
    return check_hip(ctx, hipGetLastError(), "group scatter launch");
}

// f<T, LANES>(): the kernel for this many lanes a row
#define SOM_ROW_KERNELS(kernel, T)                                                                                                             \
    (lanes == 1 ? kernel<T, 1> : lanes == 2 ? kernel<T, 2> : lanes == 4 ? kernel<T, 4> : lanes == 8 ? kernel<T, 8> : lanes == 16 ? kernel<T, 16> : \
     lanes == 32 ? kernel<T, 32> : kernel<T, 64>)

template <class T>
static int dispatch_typed(som_ctx* ctx, const T* X, int64_t rows, int32_t D, int64_t ldx, const int32_t* slot, int32_t k, const float* weight, T* Y,
                          int64_t places, int64_t ldy)
{
    if (D < Piece<T>::N) {
        hipLaunchKernelGGL(dispatch_short_kernel<T>, row_grid(rows * k, 256), dim3(256), 0, ctx->stream, X, rows, D, ldx, slot, k,
                           weight, Y, places, ldy);
    } else {
        const int pieces = (D + Piece<T>::N - 1) / Piece<T>::N, lanes = row_lanes(pieces, 64);
        hipLaunchKernelGGL(SOM_ROW_KERNELS(dispatch_kernel, T), row_grid(rows, 256 / lanes, (pieces + lanes - 1) / lanes), dim3(256), 0, ctx->stream, X,
                           rows, D, ldx, slot, k, weight, Y, places, ldy, (unsigned)((pieces + lanes - 1) / lanes));
    }
    return check_hip(ctx, hipGetLastError(), "dispatch launch");
}

template <class T>
static int combine_typed(som_ctx* ctx, const T* Y, int64_t places, int32_t D, int64_t ldy, const int32_t* slot, int64_t rows, int32_t k,
                         const float* weight, T* out, int64_t ldo)
{
    if (D < Piece<T>::N) {
        hipLaunchKernelGGL(combine_short_kernel<T>, row_grid(rows, 256), dim3(256), 0, ctx->stream, Y, places, D, ldy, slot, rows, k,
                           weight, out, ldo);
    } else {
        const int pieces = (D + Piece<T>::N - 1) / Piece<T>::N, lanes = row_lanes(pieces, 64);
        hipLaunchKernelGGL(SOM_ROW_KERNELS(combine_kernel, T), row_grid(rows, 256 / lanes, (pieces + lanes - 1) / lanes), dim3(256), 0, ctx->stream, Y,
                           places, D, ldy, slot, rows, k, weight, out, ldo, (unsigned)((pieces + lanes - 1) / lanes));
    }
    return check_hip(ctx, hipGetLastError(), "combine launch");
}

template <class T>
static int combine_grad_typed(som_ctx* ctx, const T* dout, int64_t rows, int32_t D, int64_t lddo, const T* Y, int64_t places, int64_t ldy,
                              const int32_t* slot, int32_t k, const float* weight, T* dY, int64_t lddy, float* dweight)
{
    if (D < Piece<T>::N) {
        hipLaunchKernelGGL(combine_grad_short_kernel<T>, row_grid(rows * k, 256), dim3(256), 0, ctx->stream, dout, rows, D, lddo, Y,
                           places, ldy, slot, k, weight, dY, lddy, dweight);
    } else {
        const int lanes = row_lanes((D + Piece<T>::N - 1) / Piece<T>::N, 64);
        hipLaunchKernelGGL(SOM_ROW_KERNELS(combine_grad_kernel, T), row_grid(rows * k, 256 / lanes), dim3(256), 0,
                           ctx->stream, dout, rows, D, lddo, Y, places, ldy, slot, k, weight, dY, lddy, dweight);
    }
    return check_hip(ctx, hipGetLastError(), "combine gradient launch");
}

int dispatch_run(som_ctx* ctx, int type, const void* X, int64_t rows, int32_t D, int64_t ldx, const int32_t* slot, int32_t k, const float* weight,
                 void* Y, int64_t places, int64_t ldy)
{
    if (rows == 0) return SOM_OK;
    if (type == SOM_ROWS_FLOAT) return dispatch_typed(ctx, (const float*)X, rows, D, ldx, slot, k, weight, (float*)Y, places, ldy);
    if (type == SOM_ROWS_BFLOAT) return dispatch_typed(ctx, (const __bf16*)X, rows, D, ldx, slot, k, weight, (__bf16*)Y, places, ldy);
    return dispatch_typed(ctx, (const _Float16*)X, rows, D, ldx, slot, k, weight, (_Float16*)Y, places, ldy);
}

int combine_run(som_ctx* ctx, int type, const void* Y, int64_t places, int32_t D, int64_t ldy, const int32_t* slot, int64_t rows, int32_t k,
                const float* weight, void* out, int64_t ldo)
{
    if (rows == 0) return SOM_OK;
    if (type == SOM_ROWS_FLOAT) return combine_typed(ctx, (const float*)Y, places, D, ldy, slot, rows, k, weight, (float*)out, ldo);
    if (type == SOM_ROWS_BFLOAT) return combine_typed(ctx, (const __bf16*)Y, places, D, ldy, slot, rows, k, weight, (__bf16*)out, ldo);
    return combine_typed(ctx, (const _Float16*)Y, places, D, ldy, slot, rows, k, weight, (_Float16*)out, ldo);
}

int combine_grad_run(som_ctx* ctx, int type, const void* dout, int64_t rows, int32_t D, int64_t lddo, const void* Y, int64_t places, int64_t ldy,
                     const int32_t* slot, int32_t k, const float* weight, void* dY, int64_t lddy, float* dweight)
{
    if (rows == 0) return SOM_OK;
    if (type == SOM_ROWS_FLOAT)
        return combine_grad_typed(ctx, (const float*)dout, rows, D, lddo, (const float*)Y, places, ldy, slot, k, weight, (float*)dY, lddy, dweight);
    if (type == SOM_ROWS_BFLOAT)
        return combine_grad_typed(ctx, (const __bf16*)dout, rows, D, lddo, (const __bf16*)Y, places, ldy, slot, k, weight, (__bf16*)dY, lddy, dweight);
    return combine_grad_typed(ctx, (const _Float16*)dout, rows, D, lddo, (const _Float16*)Y, places, ldy, slot, k, weight, (_Float16*)dY, lddy, dweight);
}

} // namespace som
