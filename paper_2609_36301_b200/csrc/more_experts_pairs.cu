// The experts' feed-forward blocks for few (token, slot) pairs: decoding, where nearly every pair has an expert of its own and a
// call is the time to read the weights of the experts that are hit.  No list of pairs, no workspace, one launch.
//
// A cluster of CTAs serves a pair.  Each takes a slice of the hidden dimension, in both products: its rows of W1 (one contiguous
// piece of memory) give a part of every activation's sum, which the CTAs exchange through distributed shared memory (2 s floats
// each); then its columns of W2 give its columns of the output, without a second exchange.  The first rows of W2 are requested
// before the exchange, so that a call waits for memory about once.  Sums and the activation stay in 32 bits.  Bound by latency for few
// pairs (8 of h = 2048, s = 64: 8.9 us, 6.3 MB), by the weights' bytes for many (512: 391 MB in 70 us, 5.6 TB/s).  (Requesting the first
// rows of W2 already in front of the first product's sums: 4 us more for 512 pairs, 1 for 64.)
#include "more_experts.cuh"

namespace more {

namespace {

constexpr int kPThreads = 256;

__device__ __forceinline__ float ld_cluster(uint32_t addr, int rank)
{
    uint32_t remote;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote));
    return v;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ void fma8(float (&acc)[8], float x, const uint4& w)
{
    acc[0] = fmaf(x, bf16_lo(w.x), acc[0]); acc[1] = fmaf(x, bf16_hi(w.x), acc[1]);
    acc[2] = fmaf(x, bf16_lo(w.y), acc[2]); acc[3] = fmaf(x, bf16_hi(w.y), acc[3]);
    acc[4] = fmaf(x, bf16_lo(w.z), acc[4]); acc[5] = fmaf(x, bf16_hi(w.z), acc[5]);
    acc[6] = fmaf(x, bf16_lo(w.w), acc[6]); acc[7] = fmaf(x, bf16_hi(w.w), acc[7]);
}
__device__ __forceinline__ uint4 ld_stream(const __nv_bfloat16* p)      // weights: read once
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Threads as `groups` column groups of 8 times as many row groups as fit: acc = sum over this thread's rows of x[row] W[row][8 columns].
template <int kBatch, bool kTwo>                  // 16-byte loads in flight per thread, twice; kTwo: as long as there are any
struct Slice {
    const __nv_bfloat16* at;      // of this thread's first row, or nullptr
    size_t step;                  // elements between its rows
    int rows, row, stride;        // rows of the slice, its first, distance
    __device__ void load(uint4 (&w)[kBatch], int from) const
    {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            w[i] = at && row + (from + i) * stride < rows ? ld_stream(at + (size_t)(from + i) * step) : make_uint4(0, 0, 0, 0);
    }
    __device__ void add(float (&acc)[8], const uint4 (&w)[kBatch], const float* x, int from) const
    {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = row + (from + i) * stride;
            if (at && r < rows) fma8(acc, x[r], w[i]);
        }
    }
    // w: the first batch, loaded; v: with kTwo the second
    __device__ void sum(float (&acc)[8], uint4 (&w)[kBatch], uint4 (&v)[kBatch], const float* x) const
    {
        const int mine = at && row < rows ? (rows - row + stride - 1) / stride : 0;
        if constexpr (kTwo) {
            for (int i = 0; i < mine; i += 2 * kBatch) {
                add(acc, w, x, i);
                if (i + 2 * kBatch < mine) load(w, i + 2 * kBatch);
                if (i + kBatch < mine) add(acc, v, x, i + kBatch);
                if (i + 3 * kBatch < mine) load(v, i + 3 * kBatch);
            }
        } else {
            uint4 here[kBatch];
            uint4 (&next)[kBatch] = kBatch > 4 ? v : here;   // (v lives on between the sums, for which 64 registers are too few)
            for (int i = 0; i < mine; i += kBatch) {
                if (i + kBatch < mine) load(next, i + kBatch);
                add(acc, w, x, i);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) w[j] = next[j];
            }
        }
    }
    __device__ void begin(uint4 (&w)[kBatch], uint4 (&v)[kBatch]) const
    {
        load(w, 0);
        if constexpr (kTwo) load(v, kBatch);
    }
};

// red[row group][8 columns of a group] -> the sum of column c of `cols`
__device__ __forceinline__ float column_sum(const float* red, int cols, int row_groups, int c)
{
    float v[4] = {0.f, 0.f, 0.f, 0.f};                 // (four chains, so that their loads do not wait for one another)
    for (int r = 0; r < row_groups; r += 4)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i < row_groups) v[i] += red[(r + i) * cols + c];
    return (v[0] + v[1]) + (v[2] + v[3]);
}

// BATCH, PER_SM: what a CTA has in flight, and how many of them are resident.  TWO: two batches are in flight all the time, in twice the
// code: 512 pairs of h = 2048, s = 64 70 us instead of 73, 128 of h = 4096, s = 128 76.5 instead of 80.3; but 8 pairs, which run their
// code once, 9.2 instead of 8.9.
template <int BATCH, int PER_SM, bool TWO>
__global__ void __launch_bounds__(kPThreads, PER_SM)
pairs_kernel(const __nv_bfloat16* __restrict__ X, const __nv_bfloat16* __restrict__ W1, const __nv_bfloat16* __restrict__ W2,
             const int32_t* __restrict__ idx, int h, int s, int M, int k, int ranks, __nv_bfloat16* __restrict__ Y)
{
    extern __shared__ float sm[];
    float* red = sm;                                   // [256 x 8]
    float* part = red + kPThreads * 8;                 // [2 s]
    float* act = part + 2 * s;                         // [s]
    float* x = act + s;                                // [slice]
    const int tid = threadIdx.x, pair = blockIdx.x / ranks, rank = blockIdx.x % ranks;
    const int e = idx[pair];
    if ((unsigned)e >= (unsigned)M) return;            // no expert: the row stays as it is (all CTAs of the cluster agree)
    const int per = (h / 8 + ranks - 1) / ranks, v0 = min(rank * per, h / 8), vn = min(per, h / 8 - v0);   // 16-byte vectors of the slice
    const int rows = vn * 8;

    // first product: columns in passes of up to 256 groups of 8
    const __nv_bfloat16* w1 = W1 + ((size_t)e * h + v0 * 8) * 2 * s;
    const int all = s / 4;
    uint4 w[BATCH], v[BATCH];
    for (int g0 = 0; g0 < all; g0 += kPThreads) {
        const int groups = min(all - g0, kPThreads), rg = kPThreads / groups;
        const int mine = tid / groups, col = (g0 + tid % groups) * 8;
        Slice<BATCH, TWO> sl{mine < rg ? w1 + (size_t)mine * 2 * s + col : nullptr, (size_t)rg * 2 * s, rows, mine, rg};
        sl.begin(w, v);
        if (g0 == 0) {
            const __nv_bfloat16* from = X + (size_t)(pair / k) * h + v0 * 8;
            for (int i = tid; i < rows; i += kPThreads) x[i] = __bfloat162float(from[i]);
            __syncthreads();
        }
        float acc[8] = {};
        sl.sum(acc, w, v, x);
        if (mine < rg)
#pragma unroll
            for (int i = 0; i < 8; ++i) red[mine * groups * 8 + (tid % groups) * 8 + i] = acc[i];
        __syncthreads();
        for (int c = tid; c < groups * 8; c += kPThreads) part[g0 * 8 + c] = column_sum(red, groups * 8, rg, c);
        __syncthreads();
    }
    cluster_arrive();
    // second product, first rows
    const int passes = (vn + kPThreads - 1) / kPThreads;
    auto slice2 = [&](int g0) {
        const int groups = min(vn - g0, kPThreads), rg = groups > 0 ? kPThreads / groups : 0;
        const int mine = groups > 0 ? tid / groups : 0;
        return Slice<BATCH, TWO>{mine < rg ? W2 + ((size_t)e * s + mine) * h + (size_t)(v0 + g0 + tid % groups) * 8 : nullptr, (size_t)rg * h, s, mine, rg};
    };
    if (passes > 0) slice2(0).begin(w, v);
    cluster_wait();
    const uint32_t part_at = smem_u32(part);
    for (int c = tid; c < s; c += kPThreads) {
        float gq[8], uq[8], g = 0.f, u = 0.f;              // (at most 8 CTAs; all their parts requested at once)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            gq[q] = q < ranks ? ld_cluster(part_at + c * 4, q) : 0.f;
            uq[q] = q < ranks ? ld_cluster(part_at + (s + c) * 4, q) : 0.f;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            g += gq[q];
            u += uq[q];
        }
        act[c] = g * sigmoid_to_round(g) * u;
    }
    __syncthreads();
    cluster_arrive();                                  // (done with the other CTAs' parts)
    for (int p = 0; p < passes; ++p) {
        const int g0 = p * kPThreads, groups = min(vn - g0, kPThreads), rg = kPThreads / groups;
        const Slice<BATCH, TWO> sl = slice2(g0);
        if (p > 0) sl.begin(w, v);
        float acc[8] = {};
        sl.sum(acc, w, v, act);
        if (tid / groups < rg)
#pragma unroll
            for (int i = 0; i < 8; ++i) red[(tid / groups) * groups * 8 + (tid % groups) * 8 + i] = acc[i];
        __syncthreads();
        for (int c = tid * 2; c < groups * 8; c += kPThreads * 2) {
            const float lo = column_sum(red, groups * 8, rg, c), hi = column_sum(red, groups * 8, rg, c + 1);
            *reinterpret_cast<uint32_t*>(Y + (size_t)pair * h + (size_t)(v0 + g0) * 8 + c) = pack_bf16(lo, hi);
        }
        __syncthreads();
    }
    cluster_wait();
}

// Shared memory of a CTA: sums by thread, both projections' parts, the activation, a slice of x.
constexpr size_t pairs_smem(int h, int s, int ranks)
{
    return sizeof(float) * (kPThreads * 8 + 3 * (size_t)s + ((size_t)h / 8 + ranks - 1) / ranks * 8);
}

}  // namespace

int launch_experts_pairs(const ExpertsArgs& a, const DeviceCtx& ctx)
{
    const long long P = (long long)a.T * a.k;
    // CTAs per pair: as many as are resident at once, two per SM, but not fewer than 32 rows each.  (8 pairs of h = 2048, s = 64: 38 us
    // with one CTA each, 9.2 with eight; 64: 38, 16.7 with four, 21 with eight; 512: 90, 96 with two, 111 with four.)
    int ranks = 1;
    while (ranks < 8 && P * ranks * 2 <= 2LL * ctx.sm_count && a.h / (ranks * 2) >= 32) ranks *= 2;
    const size_t smem = pairs_smem(a.h, a.s, ranks);
    // More pairs than two CTAs per SM hold at once: four smaller ones (512 pairs of h = 2048, s = 64: 72 us instead of 90; for fewer
    // pairs they are slower, 8: 11.3 instead of 9.2, 128 of h = 4096, s = 128: 108 instead of 84).  TWO where a thread has batches enough
    // for it (4096 pairs of h = 256, s = 16, one each: 70 us without, 76 with; 16 of h = 4096, s = 128, eight each: 19.7 and 22).
    const bool many = P > 2LL * ctx.sm_count;
    const long long per_thread = (long long)(a.h / ranks) * (a.s / 4) / kPThreads;         // rows of W1
    auto kern = many ? (per_thread >= 32 ? pairs_kernel<4, 4, true> : pairs_kernel<4, 4, false>)
                     : (per_thread >= 128 ? pairs_kernel<8, 2, true> : pairs_kernel<8, 2, false>);
    // (always the most that any call needs: the limit belongs to the kernel, and a call of another host thread with narrower experts,
    // between this and the launch, would have the launch refused)
    constexpr size_t kMost = pairs_smem(MORE_H_MAX, MORE_S_MAX, 1);
    static_assert(kMost <= 227 * 1024, "shared memory");
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMost) != cudaSuccess) return MORE_ERR_CUDA;
    if (P * ranks > 0x7fffffffLL) return MORE_ERR_TOO_LARGE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(P * ranks));
    cfg.blockDim = dim3(kPThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = a.stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)ranks;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kern, a.X, a.W1, a.W2, a.idx, a.h, a.s, a.M, a.k, ranks, a.out_y) != cudaSuccess) return MORE_ERR_CUDA;
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

}  // namespace more
