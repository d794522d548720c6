// What joins the experts' rows back to the residual stream and makes the next block's input, in one pass over each token, and the
// way back:
//
//   y = sum_j gate_j Y[t, j],   n = w_post y / rms(y),   r' = r + scale n,   x = w_pre r' / rms(r'),   rms(v) = sqrt(mean v^2 + eps)
//
//   g = dr' + (v - rh mean(rh v)) / rms(r')          v = w_pre dx, rh = r' / rms(r')          (gradient at r', and at r)
//   dy = (u - yh mean(yh u)) / rms(y)                u = scale w_post g, yh = y / rms(y)
//   S = sum_t g yh:  dscale = w_post S,  dw_post = scale S;     dw_pre = sum_t dx rh
//
// Bound by the bytes of the rows.  A token's row is spread over a warp (up to 1024 columns) or over a CTA, eight columns per
// 16-byte load, and stays in registers between the two sums of squares, so that everything is read once and written once.  All
// sums are 32-bit; rows are rounded where they are written.  The backward's column sums stay in registers while a CTA goes
// through its tokens, whose rows come through a ring in shared memory; a second kernel adds the CTAs' parts in order, so that
// results do not depend on timing.  65536 tokens of h = 2048, the L2 cache overwritten in front of each call: forward with 8 slots 2.95 GB in
// 443 to 484 us from one GPU to another (6.1 to 6.7 TB/s), backward 1.61 GB in 291 to 312 us (5.2 to 5.5 TB/s).  Figures below that compare two
// variants are of calls one after the other, whose last writes stay in L2: the backward pass takes 290 us there.
#include "sm100_common.cuh"

namespace more {

namespace {

constexpr unsigned kAll = 0xffffffffu;
static_assert(MORE_H_MAX / 8 <= 2 * 512, "two vectors for each of 512 threads");
constexpr int kStages = 8;                       // tokens on their way to a CTA, at most
constexpr int kRingBytesPerSm = 200 * 1024;      // bytes of them per SM

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void widen(const uint4& u, float (&v)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8])
{
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) { widen(*reinterpret_cast<const uint4*>(p), v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8])
{
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// In front of the end of a CTA with a ring: where a wait gave up, copies that are still under way land before the memory is released.
__device__ __forceinline__ void settle(volatile int* abort_flag)
{
    __syncthreads();
    if (!*abort_flag) return;                        // (the same for all threads: none waits any more)
    if (threadIdx.x == 0)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
    __syncthreads();
}

// Eight values as four pairs, for the instructions that work on two at a time.
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float both(uint64_t a)
{
    float x, y;
    unpack2(a, x, y);
    return x + y;
}
template <class T>
__device__ __forceinline__ void load8(const T* p, uint64_t (&v)[4])
{
    float f[8];
    load8(p, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(f[2 * i], f[2 * i + 1]);
}
template <class T>
__device__ __forceinline__ void store8(T* p, const uint64_t (&v)[4])
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(v[i], f[2 * i], f[2 * i + 1]);
    store8(p, f);
}

// Sums of three values over a CTA of up to 16 warps, as token_sum<true>: lanes trade values, so that six exchanges do instead of 15.
__device__ __forceinline__ void token_sum3(float (&v)[3], float (*buf)[16], int warps);

// Sums of N values over the threads of a token: a warp (WIDE = false) or the CTA of up to 16 warps.  buf: N x 16 floats that no other
// sum uses until another barrier has passed; places of warps that there are not hold zeros.
template <bool WIDE, int N>
__device__ __forceinline__ void token_sum(float (&v)[N], float (*buf)[16])
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[n] += __shfl_xor_sync(kAll, v[n], o);
    if constexpr (WIDE) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) buf[n][warp] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {                        // (all threads read all parts: shorter than another five shuffles)
            const float4* q = reinterpret_cast<const float4*>(buf[n]);
            const float4 a = q[0], b = q[1], c = q[2], d = q[3];
            v[n] = (((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w))) + (((c.x + c.y) + (c.z + c.w)) + ((d.x + d.y) + (d.z + d.w)));
        }
    }
}

__device__ __forceinline__ void token_sum3(float (&v)[3], float (*buf)[16], int warps)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool up = lane & 16, up8 = lane & 8;
    float x = (up ? v[1] : v[0]) + __shfl_xor_sync(kAll, up ? v[0] : v[1], 16);
    const float y = v[2] + __shfl_xor_sync(kAll, v[2], 16);
    x = (up8 ? y : x) + __shfl_xor_sync(kAll, up8 ? x : y, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    if ((lane & 7) == 0 && lane != 24) buf[up8 ? 2 : up ? 1 : 0][warp] = x;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 3; ++n) {
        const ulonglong2* q = reinterpret_cast<const ulonglong2*>(buf[n]);
        const ulonglong2 a = q[0], b = q[1];
        uint64_t s = add2(add2(a.x, a.y), add2(b.x, b.y));
        if (warps > 8) {
            const ulonglong2 c = q[2], d = q[3];
            s = add2(s, add2(add2(c.x, c.y), add2(d.x, d.y)));
        }
        v[n] = both(s);
    }
}

struct CombineParams {
    const __nv_bfloat16* Y;       // [T k][h], nullable
    const float* gate;            // [T][k], nullable: ones
    const void* residual;         // [T][h], nullable: zeros
    const float *w_post, *scale, *w_pre;   // [h], nullable
    float eps, inv_h;
    int T, h, k;
    void* out_residual;           // nullable
    __nv_bfloat16* out_x;         // nullable
    __nv_bfloat16* out_sum;       // nullable
};

template <int NV, bool WIDE, class R>
__global__ void __launch_bounds__(WIDE ? 512 : 256) combine_kernel(const __grid_constant__ CombineParams p)
{
    __shared__ __align__(16) float sums[2][1][16];
    if (WIDE) {
        if (threadIdx.x < 32) sums[threadIdx.x >> 4][0][threadIdx.x & 15] = 0.f;
        __syncthreads();
    }
    const int lane = WIDE ? threadIdx.x : threadIdx.x & 31, width = WIDE ? blockDim.x : 32;
    const int t = (int)(WIDE ? blockIdx.x : blockIdx.x * 8 + (threadIdx.x >> 5));      // (T <= 2^31 - 1: at most 2^31 - 1)
    if (!WIDE && t >= p.T) return;
    float y[NV][8], r[NV][8];
    bool live[NV];
    size_t at[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int c = (n * width + lane) * 8;
        live[n] = c < p.h;
        at[n] = (size_t)t * p.h + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[n][i] = r[n][i] = 0.f;
        if (live[n] && p.residual) load8(static_cast<const R*>(p.residual) + at[n], r[n]);
    }
    // A CTA per token and one vector per thread: there are few tokens, and a call is a chain of waits.  What does not depend on what is
    // being waited for is requested at once: the rows whatever their gates, the weights before the sums (64 rows of 4096, 16 slots: 6.4 us
    // instead of 8.1; weights only brought to the L1 cache early: 6.8).
    constexpr bool kEager = WIDE && NV == 1;
    float w_at[3][8];                                        // kEager: w_post, scale, w_pre
    if constexpr (kEager)
        if (live[0]) {
            if (p.Y && p.w_post) load8(p.w_post + lane * 8, w_at[0]);
            if (p.Y && p.scale) load8(p.scale + lane * 8, w_at[1]);
            if (p.out_x) load8(p.w_pre + lane * 8, w_at[2]);
        }
    if (p.Y) {
        // slots whose rows are requested at once: for few tokens all 16 of a call are one wait
        constexpr int J = WIDE && NV == 1 ? 16 : NV > 2 ? 2 : 4;
        for (int j0 = 0; j0 < p.k; j0 += J) {
            uint4 u[J][NV];
            float g[J];
#pragma unroll
            for (int j = 0; j < J; ++j) g[j] = j0 + j >= p.k ? 0.f : (p.gate ? p.gate[(size_t)t * p.k + j0 + j] : 1.f);
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int n = 0; n < NV; ++n)
                    u[j][n] = (kEager ? j0 + j < p.k : g[j] != 0.f) && live[n] ? *reinterpret_cast<const uint4*>(p.Y + ((size_t)t * p.k + j0 + j) * p.h + (n * width + lane) * 8)
                                                      : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int n = 0; n < NV; ++n) {
                    if (kEager && g[j] == 0.f) continue;     // (whatever the row holds)
                    float v[8];
                    widen(u[j][n], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[n][i] = fmaf(g[j], v[i], y[n][i]);
                }
        }
    }
    if (p.out_sum)
#pragma unroll
        for (int n = 0; n < NV; ++n)
            if (live[n]) store8(p.out_sum + at[n], y[n]);
    float inv = 1.f;
    if (p.w_post) {
        float q[1] = {0.f};
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[0] = fmaf(y[n][i], y[n][i], q[0]);
        token_sum<WIDE>(q, sums[0]);
        inv = rsqrtf(fmaf(q[0], p.inv_h, p.eps));
    }
    float q[1] = {0.f};
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int c = (n * width + lane) * 8;
        if (!live[n]) continue;
        float w[8];
        if (p.w_post) {
            if constexpr (!kEager) load8(p.w_post + c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[n][i] *= inv * (kEager ? w_at[0][i] : w[i]);
        }
        if (p.scale) {
            if constexpr (!kEager) load8(p.scale + c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[n][i] *= kEager ? w_at[1][i] : w[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            r[n][i] += y[n][i];
            q[0] = fmaf(r[n][i], r[n][i], q[0]);
        }
        if (p.out_residual) store8(static_cast<R*>(p.out_residual) + at[n], r[n]);
    }
    if (!p.out_x) return;
    token_sum<WIDE>(q, sums[1]);
    inv = rsqrtf(fmaf(q[0], p.inv_h, p.eps));
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        if (!live[n]) continue;
        float w[8];
        if constexpr (!kEager) load8(p.w_pre + (n * width + lane) * 8, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[n][i] *= inv * (kEager ? w_at[2][i] : w[i]);
        store8(p.out_x + at[n], r[n]);
    }
}

// The same for many tokens of long rows: a CTA goes through every gridDim.x-th token, whose rows (the k of them are one piece of memory)
// come into a ring in shared memory while others are worked on.
template <int NV, class R>
__global__ void __launch_bounds__(512) combine_ring_kernel(const __grid_constant__ CombineParams p, int stages, int* status)
{
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(16) float sums[2][1][16];
    __shared__ uint64_t full[kStages];
    __shared__ int abort_word;
    volatile int* abort_flag = &abort_word;
    const int tid = threadIdx.x, width = blockDim.x;
    const uint32_t rows = p.Y ? (uint32_t)p.k * p.h * 2 : 0u, bytes = rows + (p.residual ? p.h * (uint32_t)sizeof(R) : 0u);
    auto request = [&](int t, int stage) {
        const uint32_t bar = smem_u32(&full[stage]), to = smem_u32(ring) + stage * bytes;
        mbar_expect_tx(bar, bytes);
        if (p.Y) bulk_load(to, p.Y + (size_t)t * p.k * p.h, rows, bar);
        if (p.residual) bulk_load(to + rows, static_cast<const R*>(p.residual) + (size_t)t * p.h, bytes - rows, bar);
    };
    if (tid < 32) sums[tid >> 4][0][tid & 15] = 0.f;
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(&full[i]), 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < stages; ++i)
            if ((long long)blockIdx.x + (long long)i * gridDim.x < p.T) request(blockIdx.x + i * gridDim.x, i);
    }
    __syncthreads();
    uint64_t w_out[NV][4], w_in[NV][4];                      // scale times w_post; w_pre
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int c = (n * width + tid) * 8;
        auto in = [&](int i) { return p.out_x && c < p.h ? p.w_pre[c + i] : 0.f; };
        auto out = [&](int i) { return c < p.h ? (p.scale ? p.scale[c + i] : 1.f) * (p.w_post ? p.w_post[c + i] : 1.f) : 0.f; };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w_out[n][i] = pack2(out(2 * i), out(2 * i + 1));
            w_in[n][i] = pack2(in(2 * i), in(2 * i + 1));
        }
    }
    // gates of the next token: lane j of every warp has slot j's
    const int lane = tid & 31;
    auto gate_of = [&](long long t) { return lane < p.k && t < p.T ? (p.gate ? p.gate[t * p.k + lane] : 1.f) : 0.f; };
    float next_gate = gate_of(blockIdx.x);
    int stage = 0, turn = 0;
    uint32_t phase = 0;
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const float gates = next_gate;
        next_gate = gate_of(t + gridDim.x);
        const bool ok = mbar_wait_warp(smem_u32(&full[stage]), phase, abort_flag, status);    // (given up: goes on, the outputs are undefined)
        const uint8_t* from = ring + stage * bytes;
        uint64_t y[NV][4], r[NV][4];
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[n][i] = r[n][i] = pack2(0.f, 0.f);
        if (p.Y && ok)
            for (int j = 0; j < p.k; ++j) {
                const float g = __shfl_sync(kAll, gates, j);
                if (g == 0.f) continue;                      // (whatever the row holds)
                const uint64_t g2 = pack2(g, g);
#pragma unroll
                for (int n = 0; n < NV; ++n) {
                    const int c = (n * width + tid) * 8;
                    if (c >= p.h) continue;
                    uint64_t v[4];
                    load8(reinterpret_cast<const __nv_bfloat16*>(from) + (size_t)j * p.h + c, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[n][i] = fma2(g2, v[i], y[n][i]);
                }
            }
        uint64_t a = pack2(0.f, 0.f);
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + tid) * 8;
            if (p.residual && ok && c < p.h) load8(reinterpret_cast<const R*>(from + rows) + c, r[n]);
#pragma unroll
            for (int i = 0; i < 4; ++i) a = fma2(y[n][i], y[n][i], a);
        }
        float inv = 1.f;
        if (p.w_post) {
            float q[1] = {both(a)};
            token_sum<true>(q, sums[turn]);
            if (!p.out_x) turn ^= 1;                         // (no other sum's barrier before the next token's)
            inv = rsqrtf(fmaf(q[0], p.inv_h, p.eps));
        } else {
            __syncthreads();
        }
        // (every thread has its part of the stage in registers)
        if (tid == 0 && ok && t + (long long)stages * gridDim.x < p.T) request((int)(t + (long long)stages * gridDim.x), stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        const uint64_t inv2 = pack2(inv, inv);
        a = pack2(0.f, 0.f);
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + tid) * 8;
            const bool live = ok && c < p.h;
            if (p.out_sum && live) store8(p.out_sum + (size_t)t * p.h + c, y[n]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r[n][i] = fma2(mul2(y[n][i], inv2), w_out[n][i], r[n][i]);
                a = fma2(r[n][i], r[n][i], a);
            }
            if (p.out_residual && live) store8(static_cast<R*>(p.out_residual) + (size_t)t * p.h + c, r[n]);
        }
        if (!p.out_x) continue;
        float q[1] = {both(a)};
        token_sum<true>(q, sums[1]);
        inv = rsqrtf(fmaf(q[0], p.inv_h, p.eps));
        const uint64_t inv_r = pack2(inv, inv);
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + tid) * 8;
            if (!ok || c >= p.h) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[n][i] = mul2(mul2(r[n][i], inv_r), w_in[n][i]);
            store8(p.out_x + (size_t)t * p.h + c, r[n]);
        }
    }
    settle(abort_flag);
}

struct CombineBackParams {
    const void* dres;             // [T][h], nullable: zeros
    const __nv_bfloat16* dx;      // [T][h], nullable: zeros
    const __nv_bfloat16* sum;     // [T][h], nullable
    const void* res;              // [T][h]; read where dx is given
    const float *w_post, *scale, *w_pre;
    float eps, inv_h;
    int T, h, stages;
    void* out_dres;               // nullable
    __nv_bfloat16* out_dsum;      // nullable
    float* parts;                 // [parts][2][h]: S, dw_pre
    int want_parts;
    int* status;
};

// A CTA goes through every gridDim.x-th token.  The rows of the next tokens are on their way into a ring in shared memory (bulk copies,
// a row each) while one is worked on: the two sums over a row that have to be known before anything can be written are chains of
// latency, which left the memory idle half of the time when rows came by loads into registers (519 us at 65536 x 2048, now 290).
template <int NV, class R, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 2 : 1) combine_back_kernel(const __grid_constant__ CombineBackParams p)
{
    let_next_begin();
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(16) float sums[2][3][16];
    __shared__ uint64_t full[kStages];
    __shared__ int abort_word;
    volatile int* abort_flag = &abort_word;
    const int tid = threadIdx.x, width = blockDim.x;
    const uint32_t wide = p.h * sizeof(R), narrow = p.h * 2;
    const uint32_t at_res = p.dres ? wide : 0, at_dx = at_res + (p.dx ? wide : 0), at_sum = at_dx + (p.dx ? narrow : 0), bytes = at_sum + (p.sum ? narrow : 0);
    auto request = [&](int t, int stage) {
        const uint32_t bar = smem_u32(&full[stage]), to = smem_u32(ring) + stage * bytes;
        const size_t row = (size_t)t * p.h;
        mbar_expect_tx(bar, bytes);
        if (p.dres) bulk_load(to, static_cast<const R*>(p.dres) + row, wide, bar);
        if (p.dx) {
            bulk_load(to + at_res, static_cast<const R*>(p.res) + row, wide, bar);
            bulk_load(to + at_dx, p.dx + row, narrow, bar);
        }
        if (p.sum) bulk_load(to + at_sum, p.sum + row, narrow, bar);
    };
    for (int i = tid; i < 2 * 3 * 16; i += width) (&sums[0][0][0])[i] = 0.f;
    if (tid == 0) {
        for (int i = 0; i < p.stages; ++i) mbar_init(smem_u32(&full[i]), 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < p.stages; ++i)
            if ((long long)blockIdx.x + (long long)i * gridDim.x < p.T) request(blockIdx.x + i * gridDim.x, i);
    }
    __syncthreads();
    uint64_t S[NV][4], P[NV][4], w_in[NV][4], w_out[NV][4];  // column sums; w_pre, and scale times w_post
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int c = (n * width + tid) * 8;
        auto in = [&](int i) { return p.dx && c < p.h ? p.w_pre[c + i] : 0.f; };
        auto out = [&](int i) { return c < p.h ? (p.scale ? p.scale[c + i] : 1.f) * (p.w_post ? p.w_post[c + i] : 1.f) : 0.f; };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            S[n][i] = P[n][i] = pack2(0.f, 0.f);
            w_in[n][i] = pack2(in(2 * i), in(2 * i + 1));
            w_out[n][i] = pack2(out(2 * i), out(2 * i + 1));
        }
    }
    const int warps = width >> 5;
    int stage = 0;
    uint32_t phase = 0;
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const bool ok = mbar_wait_warp(smem_u32(&full[stage]), phase, abort_flag, p.status);   // (given up: goes on, the outputs are undefined)
        const uint8_t* from = ring + stage * bytes;
        uint64_t g[NV][4], r[NV][4], v[NV][4], d[NV][4], y[NV][4];
        float q[3] = {0.f, 0.f, 0.f};                        // sums of r^2, r v, y^2
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + tid) * 8;
            const bool live = ok && c < p.h;
#pragma unroll
            for (int i = 0; i < 4; ++i) g[n][i] = r[n][i] = d[n][i] = y[n][i] = pack2(0.f, 0.f);
            if (live) {
                if (p.dres) load8(reinterpret_cast<const R*>(from) + c, g[n]);
                if (p.dx) {
                    load8(reinterpret_cast<const R*>(from + at_res) + c, r[n]);
                    load8(reinterpret_cast<const __nv_bfloat16*>(from + at_dx) + c, d[n]);
                }
                if (p.sum) load8(reinterpret_cast<const __nv_bfloat16*>(from + at_sum) + c, y[n]);
            }
            uint64_t a[3] = {pack2(0.f, 0.f), pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[n][i] = mul2(d[n][i], w_in[n][i]);
                a[0] = fma2(r[n][i], r[n][i], a[0]);
                a[1] = fma2(r[n][i], v[n][i], a[1]);
                a[2] = fma2(y[n][i], y[n][i], a[2]);
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) q[i] += both(a[i]);
        }
        token_sum3(q, sums[0], warps);
        // (every thread has its part of the stage in registers)
        if (tid == 0 && ok && t + (long long)p.stages * gridDim.x < p.T) request((int)(t + (long long)p.stages * gridDim.x), stage);
        if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        const float inv = rsqrtf(fmaf(q[0], p.inv_h, p.eps)), mean = q[1] * inv * p.inv_h;       // mean of rh v
        const float inv_y = p.w_post ? rsqrtf(fmaf(q[2], p.inv_h, p.eps)) : 1.f;
        const uint64_t inv2 = pack2(inv, inv), less = pack2(-mean, -mean), inv_y2 = pack2(inv_y, inv_y);
        float m[1] = {0.f};                                  // sum of yh u
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + tid) * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) {                    // (without dx: zeros)
                const uint64_t rh = mul2(r[n][i], inv2);
                P[n][i] = fma2(d[n][i], rh, P[n][i]);
                g[n][i] = fma2(inv2, fma2(rh, less, v[n][i]), g[n][i]);
            }
            if (p.out_dres && ok && c < p.h) store8(static_cast<R*>(p.out_dres) + (size_t)t * p.h + c, g[n]);
            uint64_t a = pack2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[n][i] = mul2(y[n][i], inv_y2);
                S[n][i] = fma2(g[n][i], y[n][i], S[n][i]);
                g[n][i] = mul2(g[n][i], w_out[n][i]);
                a = fma2(g[n][i], y[n][i], a);
            }
            m[0] += both(a);
        }
        if (p.out_dsum) {
            float mean_y = 0.f;
            if (p.w_post) {
                token_sum<true>(m, sums[1]);
                mean_y = m[0] * p.inv_h;
            }
            const uint64_t less_y = pack2(-mean_y, -mean_y);
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const int c = (n * width + tid) * 8;
                if (!ok || c >= p.h) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) g[n][i] = mul2(inv_y2, fma2(y[n][i], less_y, g[n][i]));
                store8(p.out_dsum + (size_t)t * p.h + c, g[n]);
            }
        }
        if (!(p.out_dsum && p.w_post)) __syncthreads();      // the next token's first sum may overwrite this one's
    }
    settle(abort_flag);
    if (!p.want_parts) return;
    float* out = p.parts + (size_t)blockIdx.x * 2 * p.h;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int c = (n * width + tid) * 8;
        if (c < p.h) {
            store8(out + c, S[n]);
            store8(out + p.h + c, P[n]);
        }
    }
}

// out = sums over the parts, in their order: 32 columns per CTA, 32 rows of threads take every 32nd part.  (No promise that the parts stay
// the same while it runs: it begins while they are being written, and a load through the read-only path could move in front of the wait.)
__global__ void __launch_bounds__(1024) combine_columns_kernel(const float* parts, int count, int h, const float* w_post, const float* scale,
                                                                float* out_dw_post, float* out_dscale, float* out_dw_pre)
{
    wait_for_previous();
    __shared__ float buf[32][33];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;        // c in [0, 2 h)
    float v = 0.f;
    if (c < 2 * h) {
        int i = ty;
        for (; i + 96 < count; i += 128) {                   // (four loads in flight; the order of the sum is fixed all the same)
            float a[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = parts[(size_t)(i + 32 * j) * 2 * h + c];
            v += (a[0] + a[1]) + (a[2] + a[3]);
        }
        for (; i < count; i += 32) v += parts[(size_t)i * 2 * h + c];
    }
    buf[ty][tx] = v;
    __syncthreads();
    if (ty != 0 || c >= 2 * h) return;
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += buf[i][tx];
    if (c < h) {
        if (out_dw_post) out_dw_post[c] = scale ? v * scale[c] : v;
        if (out_dscale) out_dscale[c] = w_post ? v * w_post[c] : v;
    } else if (out_dw_pre) {
        out_dw_pre[c - h] = v;
    }
}

// How a token's row is spread: vectors of 8 columns per thread, and threads; a warp per token (and eight tokens per CTA) or a CTA.  Up to
// eight tokens per SM, and for rows of more than 1024 columns, a CTA: 64 ... 1184 tokens of 8 slots, h = 512, 8 to 11 us against 14 to 16 with a
// warp each, h = 1024 8 to 14 against 16.  For more tokens a warp is as good (4000: h = 256 13 us against 16 with a CTA, h = 512 20.5
// against 19.5); in between a CTA would be up to 4 us better (1300 tokens of h = 512: 12 against 16).
struct Spread {
    int nv, width;
    bool wide;
};
Spread spread(int T, int h)
{
    const int vecs = h / 8;
    Spread s;
    s.wide = vecs > 128 || T <= 148 * 8;                         // (few tokens: as many loads at once as there are)
    if (!s.wide) {
        s.width = 32;
        s.nv = vecs <= 32 ? 1 : (vecs <= 64 ? 2 : 4);
        return s;
    }
    s.nv = T <= 148 * 8 && vecs <= 512 ? 1 : 2;                  // (at most 512 threads: MORE_H_MAX / 16)
    s.width = ((vecs + s.nv - 1) / s.nv + 31) / 32 * 32;
    return s;
}

// The backward pass: threads and vectors per thread, CTAs per SM (about 512 threads of them: with 768 at 85 registers values spill, and
// what the rings leave of the L1 cache makes that slow, 322 us against 290 at 65536 x 2048), CTAs.
struct BackPlan {
    int nv, width, per_sm, ctas;
};
BackPlan plan_back(int T, int h)
{
    const int vecs = h / 8;
    BackPlan b;
    b.nv = vecs <= 512 ? 1 : 2;
    b.width = ((vecs + b.nv - 1) / b.nv + 31) / 32 * 32;
    b.per_sm = 512 / b.width;
    if (b.per_sm > 8) b.per_sm = 8;
    b.ctas = T < 148 * b.per_sm ? T : 148 * b.per_sm;
    return b;
}

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// The ring: stages of `token` bytes for each of per_sm CTAs, which becomes fewer where two do not fit.  0: not even for one.
int ring_stages(size_t token, int* per_sm)
{
    while (*per_sm > 1 && kRingBytesPerSm / *per_sm < 2 * token) --*per_sm;
    const size_t n = kRingBytesPerSm / *per_sm / token;
    return n < 2 ? 0 : n > kStages ? kStages : (int)n;
}
// The limit belongs to the kernel, not to a call: always the largest ring, or a call of another host thread with shorter rows, between
// this and the launch, would have the launch refused.
template <class Kernel>
int allow_ring(Kernel kern)
{
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytesPerSm) == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}
template <int NV, class R, int THREADS>
int launch_back(CombineBackParams p, const BackPlan& b, cudaStream_t st)
{
    const size_t token = (size_t)p.h * ((p.dres ? sizeof(R) : 0) + (p.dx ? sizeof(R) + 2 : 0) + (p.sum ? 2 : 0));
    int per_sm = b.per_sm;
    p.stages = ring_stages(token, &per_sm);                          // (two of the longest rows, 96 KB each, fit)
    const size_t smem = p.stages * token;
    if (allow_ring(combine_back_kernel<NV, R, THREADS>) != MORE_OK) return MORE_ERR_CUDA;
    combine_back_kernel<NV, R, THREADS><<<b.ctas, b.width, smem, st>>>(p);
    return MORE_OK;
}
template <int NV, class R>
int launch_ring(const CombineParams& p, int* status, cudaStream_t st, bool* done)
{
    const size_t token = (size_t)p.h * ((p.Y ? 2 * (size_t)p.k : 0) + (p.residual ? sizeof(R) : 0));
    const int width = ((p.h / 8 + NV - 1) / NV + 31) / 32 * 32;
    int per_sm = 512 / width > 8 ? 8 : 512 / width;
    const int stages = ring_stages(token, &per_sm);
    *done = stages > 0;
    if (!*done) return MORE_OK;
    const int ctas = p.T < 148 * per_sm ? p.T : 148 * per_sm;
    const size_t smem = stages * token;
    if (allow_ring(combine_ring_kernel<NV, R>) != MORE_OK) return MORE_ERR_CUDA;
    combine_ring_kernel<NV, R><<<ctas, width, smem, st>>>(p, stages, status);
    return MORE_OK;
}
template <int NV, bool WIDE, class R>
void launch_forward(const CombineParams& p, int width, cudaStream_t st)
{
    combine_kernel<NV, WIDE, R><<<WIDE ? (unsigned)p.T : ((unsigned)p.T + 7) / 8, WIDE ? width : 256, 0, st>>>(p);
}

}  // namespace

}  // namespace more

using namespace more;

extern "C" {

int more_combine(const void* Y, const float* gate, const void* residual, int residual_type, const float* w_post, const float* scale,
                 const float* w_pre, float eps, int T, int h, int k, void* out_residual, void* out_x, void* out_sum, void* stream)
{
    if (residual_type != MORE_RESIDUAL_BF16 && residual_type != MORE_RESIDUAL_FP32) return MORE_ERR_MODE;
    if (T < 0 || h < 8 || h % 8 != 0 || h > MORE_H_MAX || k < 1 || k > MORE_K_MAX || !(eps >= 0.f)) return MORE_ERR_SHAPE;
    if (T == 0) return MORE_OK;
    if ((!Y && !residual) || (!out_residual && !out_x && !out_sum) || (out_x && !w_pre)) return MORE_ERR_NULL;
    if (misaligned(Y, 16) || misaligned(gate, 4) || misaligned(residual, 16) || misaligned(w_post, 16) || misaligned(scale, 16) ||
        misaligned(w_pre, 16) || misaligned(out_residual, 16) || misaligned(out_x, 16) || misaligned(out_sum, 16))
        return MORE_ERR_ALIGN;
    DeviceCtx* ctx = nullptr;
    const int found = device_ctx(&ctx);
    if (found != MORE_OK) return found;
    CombineParams p;
    p.Y = static_cast<const __nv_bfloat16*>(Y); p.gate = gate; p.residual = residual;
    p.w_post = Y ? w_post : nullptr; p.scale = Y ? scale : nullptr; p.w_pre = w_pre;      // (nothing to join: the next block's norm alone)
    p.eps = eps; p.inv_h = 1.f / (float)h; p.T = T; p.h = h; p.k = k;
    p.out_residual = out_residual; p.out_x = static_cast<__nv_bfloat16*>(out_x); p.out_sum = static_cast<__nv_bfloat16*>(out_sum);
    const Spread sp = spread(T, h);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool f32 = residual_type == MORE_RESIDUAL_FP32;
#define MORE_FORWARD(NV, WIDE) (f32 ? launch_forward<NV, WIDE, float>(p, sp.width, st) : launch_forward<NV, WIDE, __nv_bfloat16>(p, sp.width, st))
    bool done = false;
    // Through a ring where there are more than eight tokens per SM and two stages, of 2 h k bytes and the residual's, fit its 200 KB (in bf16
    // h = 2048: up to 24 slots, 4096: 11, 8192: 5); else a CTA per token.  us with and without it, 65536 tokens of 8 slots: h = 1024 233 and 281,
    // 2048 440 and 524, 4096 888 and 1282; of one slot: h = 1024 147 and 145, 4104 563 and 851, 8192 676 and 1802.  Shorter rows of few slots
    // lose with it (h = 256, one slot: 70 and 41); of many they would gain (h = 512, 8 slots: 132 and 174), as would fewer tokens of long
    // rows (1184 of h = 4096, 8 slots: 29 and 43).
    if (T > 148 * 8 && h >= 1024) {
        const int rc = h <= 4096 ? (f32 ? launch_ring<1, float>(p, ctx->status, st, &done) : launch_ring<1, __nv_bfloat16>(p, ctx->status, st, &done))
                                 : (f32 ? launch_ring<2, float>(p, ctx->status, st, &done) : launch_ring<2, __nv_bfloat16>(p, ctx->status, st, &done));
        if (rc != MORE_OK) return rc;
    }
    if (done) {
    } else if (sp.wide) sp.nv == 1 ? MORE_FORWARD(1, true) : MORE_FORWARD(2, true);
    else sp.nv == 1 ? MORE_FORWARD(1, false) : (sp.nv == 2 ? MORE_FORWARD(2, false) : MORE_FORWARD(4, false));
#undef MORE_FORWARD
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

long long more_combine_workspace(int T, int h)
{
    if (T < 0 || h < 8 || h % 8 != 0 || h > MORE_H_MAX) return MORE_ERR_SHAPE;
    return T == 0 ? 0 : (long long)plan_back(T, h).ctas * 2 * h * (long long)sizeof(float);
}

int more_combine_backward(const void* dresidual, const void* dx, const void* sum, const void* residual_out, int residual_type,
                          const float* w_post, const float* scale, const float* w_pre, float eps, int T, int h, void* out_dresidual,
                          void* out_dsum, float* out_dw_post, float* out_dscale, float* out_dw_pre, void* workspace,
                          long long workspace_bytes, void* stream)
{
    if (residual_type != MORE_RESIDUAL_BF16 && residual_type != MORE_RESIDUAL_FP32) return MORE_ERR_MODE;
    if (T < 0 || h < 8 || h % 8 != 0 || h > MORE_H_MAX || !(eps >= 0.f)) return MORE_ERR_SHAPE;
    const bool columns = out_dw_post || out_dscale || out_dw_pre;
    if (T > 0) {
        if ((!dresidual && !dx) || (dx && (!w_pre || !residual_out))) return MORE_ERR_NULL;
        if ((out_dsum && w_post && !sum) || ((out_dw_post || out_dscale) && !sum)) return MORE_ERR_NULL;
        if (columns && !workspace) return MORE_ERR_NULL;
    }
    if ((out_dw_post && !w_post) || (out_dscale && !scale) || (out_dw_pre && T > 0 && !dx)) return MORE_ERR_NULL;
    if (misaligned(dresidual, 16) || misaligned(dx, 16) || misaligned(sum, 16) || misaligned(residual_out, 16) || misaligned(w_post, 16) ||
        misaligned(scale, 16) || misaligned(w_pre, 16) || misaligned(out_dresidual, 16) || misaligned(out_dsum, 16) ||
        misaligned(out_dw_post, 4) || misaligned(out_dscale, 4) || misaligned(out_dw_pre, 4) || misaligned(workspace, 16))
        return MORE_ERR_ALIGN;
    if (T > 0 && columns && workspace_bytes < more_combine_workspace(T, h)) return MORE_ERR_TOO_LARGE;
    DeviceCtx* ctx = nullptr;
    const int rc = device_ctx(&ctx);
    if (rc != MORE_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const BackPlan plan = plan_back(T, h);
    const int parts = plan.ctas;
    if (T > 0) {
        CombineBackParams p;
        p.dres = dresidual; p.dx = static_cast<const __nv_bfloat16*>(dx); p.sum = static_cast<const __nv_bfloat16*>(sum); p.res = residual_out;
        p.w_post = w_post; p.scale = scale; p.w_pre = w_pre;
        p.eps = dx ? eps : fmaxf(eps, 1e-37f);                        // (without dx the next norm's terms have to be zeros, not 0 / 0)
        p.inv_h = 1.f / (float)h; p.T = T; p.h = h;
        p.out_dres = out_dresidual; p.out_dsum = static_cast<__nv_bfloat16*>(out_dsum);
        p.parts = static_cast<float*>(workspace); p.want_parts = columns;
        p.status = ctx->status;
        const bool f32 = residual_type == MORE_RESIDUAL_FP32;
        const int done = plan.nv == 2       ? (f32 ? launch_back<2, float, 512>(p, plan, st) : launch_back<2, __nv_bfloat16, 512>(p, plan, st))
                         : plan.width > 256 ? (f32 ? launch_back<1, float, 512>(p, plan, st) : launch_back<1, __nv_bfloat16, 512>(p, plan, st))
                                            : (f32 ? launch_back<1, float, 256>(p, plan, st) : launch_back<1, __nv_bfloat16, 256>(p, plan, st));
        if (done != MORE_OK) return done;
        count_launch(1);
        if (cudaGetLastError() != cudaSuccess) return MORE_ERR_CUDA;
    }
    if (columns) {
        if (launch_behind(combine_columns_kernel, (2 * h + 31) / 32, 1024, 0, st, static_cast<const float*>(workspace), parts, h, w_post, scale,
                          out_dw_post, out_dscale, out_dw_pre) != cudaSuccess)
            return MORE_ERR_CUDA;
        count_launch(1);
    }
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

}  // extern "C"
