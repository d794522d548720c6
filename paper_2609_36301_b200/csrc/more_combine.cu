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
// through its tokens; a second kernel adds the CTAs' parts in order, so that results do not depend on timing.
#include "more_internal.h"

namespace more {

namespace {

constexpr unsigned kAll = 0xffffffffu;
static_assert(MORE_H_MAX / 8 <= 2 * 512, "two vectors for each of 512 threads");
constexpr int kMaxParts = 148 * 4;               // CTAs of the backward pass

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

// Sums of N values over the threads of a token: a warp (WIDE = false) or the CTA.  buf: N x 32 floats that no other sum uses
// until another barrier has passed.
template <bool WIDE, int N>
__device__ __forceinline__ void token_sum(float (&v)[N], float* buf)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[n] += __shfl_xor_sync(kAll, v[n], o);
    if constexpr (WIDE) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (lane == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) buf[n * 32 + warp] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = lane < warps ? buf[n * 32 + lane] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[n] += __shfl_xor_sync(kAll, v[n], o);
        }
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
    __shared__ float sums[2][32];
    const int lane = WIDE ? threadIdx.x : threadIdx.x & 31, width = WIDE ? blockDim.x : 32;
    const int t = WIDE ? blockIdx.x : blockIdx.x * 8 + (threadIdx.x >> 5);
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
    if (p.Y) {
        constexpr int J = NV > 2 ? 2 : 4;                   // slots whose rows are requested at once
        for (int j0 = 0; j0 < p.k; j0 += J) {
            uint4 u[J][NV];
            float g[J];
#pragma unroll
            for (int j = 0; j < J; ++j) g[j] = j0 + j >= p.k ? 0.f : (p.gate ? p.gate[(size_t)t * p.k + j0 + j] : 1.f);
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int n = 0; n < NV; ++n)
                    u[j][n] = g[j] != 0.f && live[n] ? *reinterpret_cast<const uint4*>(p.Y + ((size_t)t * p.k + j0 + j) * p.h + (n * width + lane) * 8)
                                                      : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int n = 0; n < NV; ++n) {
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
            load8(p.w_post + c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[n][i] *= inv * w[i];
        }
        if (p.scale) {
            load8(p.scale + c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[n][i] *= w[i];
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
        load8(p.w_pre + (n * width + lane) * 8, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[n][i] *= inv * w[i];
        store8(p.out_x + at[n], r[n]);
    }
}

struct CombineBackParams {
    const void* dres;             // [T][h], nullable: zeros
    const __nv_bfloat16* dx;      // [T][h], nullable: zeros
    const __nv_bfloat16* sum;     // [T][h], nullable
    const void* res;              // [T][h]; read where dx is given
    const float *w_post, *scale, *w_pre;
    float eps, inv_h;
    int T, h;
    void* out_dres;               // nullable
    __nv_bfloat16* out_dsum;      // nullable
    float* parts;                 // [parts][2][h]: S, dw_pre
    int want_parts;
};

template <int NV, bool WIDE, class R>
__global__ void __launch_bounds__(WIDE ? 512 : 256) combine_back_kernel(const __grid_constant__ CombineBackParams p)
{
    __shared__ float sums[2][4][32];
    extern __shared__ float columns[];                       // !WIDE: [2][h]
    const int lane = WIDE ? threadIdx.x : threadIdx.x & 31, width = WIDE ? blockDim.x : 32;
    const int first = WIDE ? blockIdx.x : blockIdx.x * 8 + (threadIdx.x >> 5), stride = WIDE ? gridDim.x : gridDim.x * 8;
    float S[NV][8], P[NV][8];
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) S[n][i] = P[n][i] = 0.f;
    for (int t = first; t < p.T; t += stride) {
        float g[NV][8], r[NV][8], d[NV][8], y[NV][8];
        bool live[NV];
        float q[3] = {0.f, 0.f, 0.f};                        // sums of r^2, r v, y^2
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + lane) * 8;
            const size_t at = (size_t)t * p.h + c;
            live[n] = c < p.h;
#pragma unroll
            for (int i = 0; i < 8; ++i) g[n][i] = r[n][i] = d[n][i] = y[n][i] = 0.f;
            if (!live[n]) continue;
            if (p.dres) load8(static_cast<const R*>(p.dres) + at, g[n]);
            if (p.dx) {
                load8(static_cast<const R*>(p.res) + at, r[n]);
                load8(p.dx + at, d[n]);
            }
            if (p.sum) load8(p.sum + at, y[n]);
        }
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            if (!live[n]) continue;
            float w[8];
            if (p.dx) {
                load8(p.w_pre + (n * width + lane) * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[0] = fmaf(r[n][i], r[n][i], q[0]);
                    q[1] = fmaf(r[n][i], d[n][i] * w[i], q[1]);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) q[2] = fmaf(y[n][i], y[n][i], q[2]);
        }
        token_sum<WIDE>(q, sums[0][0]);
        const float inv = rsqrtf(fmaf(q[0], p.inv_h, p.eps)), mean = q[1] * inv * p.inv_h;       // mean of rh v
        const float inv_y = p.w_post ? rsqrtf(fmaf(q[2], p.inv_h, p.eps)) : 1.f;
        float m[1] = {0.f};                                  // sum of yh u
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + lane) * 8;
            if (!live[n]) continue;
            float w[8];
            if (p.dx) {
                load8(p.w_pre + c, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float rh = r[n][i] * inv;
                    P[n][i] = fmaf(d[n][i], rh, P[n][i]);
                    g[n][i] = fmaf(inv, fmaf(d[n][i], w[i], -rh * mean), g[n][i]);
                }
            }
            if (p.out_dres) store8(static_cast<R*>(p.out_dres) + (size_t)t * p.h + c, g[n]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[n][i] *= inv_y;
                S[n][i] = fmaf(g[n][i], y[n][i], S[n][i]);
            }
            if (p.scale) {
                load8(p.scale + c, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[n][i] *= w[i];
            }
            if (p.w_post) {
                load8(p.w_post + c, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    g[n][i] *= w[i];
                    m[0] = fmaf(g[n][i], y[n][i], m[0]);
                }
            }
        }
        if (p.out_dsum) {
            float mean_y = 0.f;
            if (p.w_post) {
                token_sum<WIDE>(m, sums[1][0]);
                mean_y = m[0] * p.inv_h;
            }
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                if (!live[n]) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) g[n][i] = inv_y * fmaf(-y[n][i], mean_y, g[n][i]);
                store8(p.out_dsum + (size_t)t * p.h + (n * width + lane) * 8, g[n]);
            }
        }
        if constexpr (WIDE)
            if (!(p.out_dsum && p.w_post)) __syncthreads();  // the next token's first sum may overwrite this one's
    }
    if (!p.want_parts) return;
    float* out = p.parts + (size_t)blockIdx.x * 2 * p.h;
    if constexpr (WIDE) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * width + lane) * 8;
            if (c < p.h) {
                store8(out + c, S[n]);
                store8(out + p.h + c, P[n]);
            }
        }
    } else {
        for (int w = 0; w < 8; ++w) {                        // the CTA's warps in turn
            if ((int)(threadIdx.x >> 5) == w)
#pragma unroll
                for (int n = 0; n < NV; ++n) {
                    const int c = (n * width + lane) * 8;
                    if (c >= p.h) continue;
                    float a[8], b[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) a[i] = b[i] = 0.f;
                    if (w > 0) {
                        load8(columns + c, a);
                        load8(columns + p.h + c, b);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        a[i] += S[n][i];
                        b[i] += P[n][i];
                    }
                    store8(w < 7 ? columns + c : out + c, a);
                    store8(w < 7 ? columns + p.h + c : out + p.h + c, b);
                }
            __syncthreads();
        }
    }
}

// out = sums over the parts, in their order: 32 columns per CTA, 32 rows of threads take every 32nd part.
__global__ void __launch_bounds__(1024) combine_columns_kernel(const float* __restrict__ parts, int count, int h, const float* __restrict__ w_post,
                                                                const float* __restrict__ scale, float* out_dw_post, float* out_dscale, float* out_dw_pre)
{
    __shared__ float buf[32][33];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;        // c in [0, 2 h)
    float v = 0.f;
    if (c < 2 * h)
        for (int i = ty; i < count; i += 32) v += parts[(size_t)i * 2 * h + c];
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

// How a token's row is spread: vectors of 8 columns per thread, and threads; a warp per token (and eight tokens per CTA) or a CTA.
struct Spread {
    int nv, width;
    bool wide;
};
Spread spread(int T, int h, bool backward)
{
    const int vecs = h / 8;
    Spread s;
    s.wide = vecs > (backward ? 64 : 128) || T <= 148 * 8;       // (few tokens: as many loads at once as there are)
    if (!s.wide) {
        s.width = 32;
        s.nv = vecs <= 32 ? 1 : (vecs <= 64 ? 2 : 4);
        return s;
    }
    s.nv = T <= 148 * 8 && vecs <= 512 ? 1 : 2;                  // (at most 512 threads: MORE_H_MAX / 16)

    s.width = ((vecs + s.nv - 1) / s.nv + 31) / 32 * 32;
    return s;
}

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int backward_parts(int T, int h)
{
    const long long want = spread(T, h, true).wide ? T : (T + 7) / 8;
    return (int)(want < kMaxParts ? want : kMaxParts);
}

template <int NV, bool WIDE, class R>
void launch_back(const CombineBackParams& p, int blocks, int width, cudaStream_t st)
{
    combine_back_kernel<NV, WIDE, R><<<blocks, WIDE ? width : 256, WIDE ? 0 : 2 * p.h * sizeof(float), st>>>(p);
}
template <int NV, bool WIDE, class R>
void launch_forward(const CombineParams& p, int width, cudaStream_t st)
{
    combine_kernel<NV, WIDE, R><<<WIDE ? p.T : (p.T + 7) / 8, WIDE ? width : 256, 0, st>>>(p);
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
    const int rc = device_ctx(&ctx);
    if (rc != MORE_OK) return rc;
    CombineParams p;
    p.Y = static_cast<const __nv_bfloat16*>(Y); p.gate = gate; p.residual = residual;
    p.w_post = Y ? w_post : nullptr; p.scale = Y ? scale : nullptr; p.w_pre = w_pre;      // (nothing to join: the next block's norm alone)
    p.eps = eps; p.inv_h = 1.f / (float)h; p.T = T; p.h = h; p.k = k;
    p.out_residual = out_residual; p.out_x = static_cast<__nv_bfloat16*>(out_x); p.out_sum = static_cast<__nv_bfloat16*>(out_sum);
    const Spread sp = spread(T, h, false);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool f32 = residual_type == MORE_RESIDUAL_FP32;
#define MORE_FORWARD(NV, WIDE) (f32 ? launch_forward<NV, WIDE, float>(p, sp.width, st) : launch_forward<NV, WIDE, __nv_bfloat16>(p, sp.width, st))
    if (sp.wide) sp.nv == 1 ? MORE_FORWARD(1, true) : MORE_FORWARD(2, true);
    else sp.nv == 1 ? MORE_FORWARD(1, false) : (sp.nv == 2 ? MORE_FORWARD(2, false) : MORE_FORWARD(4, false));
#undef MORE_FORWARD
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

long long more_combine_workspace(int T, int h)
{
    if (T < 0 || h < 8 || h % 8 != 0 || h > MORE_H_MAX) return MORE_ERR_SHAPE;
    return T == 0 ? 0 : (long long)backward_parts(T, h) * 2 * h * (long long)sizeof(float);
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
    const int parts = T > 0 ? backward_parts(T, h) : 0;
    if (T > 0) {
        CombineBackParams p;
        p.dres = dresidual; p.dx = static_cast<const __nv_bfloat16*>(dx); p.sum = static_cast<const __nv_bfloat16*>(sum); p.res = residual_out;
        p.w_post = w_post; p.scale = scale; p.w_pre = w_pre;
        p.eps = eps; p.inv_h = 1.f / (float)h; p.T = T; p.h = h;
        p.out_dres = out_dresidual; p.out_dsum = static_cast<__nv_bfloat16*>(out_dsum);
        p.parts = static_cast<float*>(workspace); p.want_parts = columns;
        const Spread sp = spread(T, h, true);
        const bool f32 = residual_type == MORE_RESIDUAL_FP32;
#define MORE_BACK(NV, WIDE) (f32 ? launch_back<NV, WIDE, float>(p, parts, sp.width, st) : launch_back<NV, WIDE, __nv_bfloat16>(p, parts, sp.width, st))
        if (sp.wide) sp.nv == 1 ? MORE_BACK(1, true) : MORE_BACK(2, true);
        else sp.nv == 1 ? MORE_BACK(1, false) : (sp.nv == 2 ? MORE_BACK(2, false) : MORE_BACK(4, false));
#undef MORE_BACK
        count_launch(1);
        if (cudaGetLastError() != cudaSuccess) return MORE_ERR_CUDA;
    }
    if (columns) {
        combine_columns_kernel<<<(2 * h + 31) / 32, 1024, 0, st>>>(static_cast<const float*>(workspace), parts, h, w_post, scale, out_dw_post,
                                                                  out_dscale, out_dw_pre);
        count_launch(1);
    }
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

}  // extern "C"
