// The experts' gated feed-forward blocks behind the router (the layer's expert products, "scatter2scatter, SwiGLU,
// scatter2scatter" in the paper's forward flowchart), forward and backward, over the (token, slot) pairs of a routing:
//
//   u = X[token] W1[e],  a = silu(u_gate) u_up,  Y[pair] = a W2[e]            e = expert of the pair
//   c = d[token] W2[e]^T,  dgate = <c, a>,  du = gate c (silu'(u_gate) u_up, silu(u_gate)),  dX = sum over slots of du W1[e]^T
//   dW1[e] = sum of X[token]^T du,  dW2[e] = sum of (gate a)^T d[token]
//
// Two kernels do all of it, both persistent with one CTA per SM: a TMA warp, a warp that issues the tcgen05 MMAs, eight warps
// that read the finished accumulator (two of 256 tensor-memory columns, used in turn, so that the products of the next unit run
// meanwhile).
//
//   rows_kernel<MODE>   tiles of up to 128 pairs of one expert against its weights.  The rows of a tile are anywhere in X: they
//                       come by gathering TMA loads (four rows of 128 bytes each), only as many as the tile has, and land in the
//                       swizzled layout that the MMAs read.  W1 and W2 are used as they are stored, the forward products with
//                       them as MN-major operands, the backward ones as K-major ones: nothing is transposed.
//   weights_kernel      dW of one expert: 128 x 256 outputs, contracted over the expert's pairs 64 at a time, both operands
//                       MN-major from gathered rows; rows behind the last pair are out of the tensor's bounds and read as zeros.
//
// What bounds them: with the paper's narrow experts, the bytes: each expert's weights are read once (six bytes per h s) for as
// few as 30 tokens.  So the loads of the next tiles are requested while a tile is computed, and what does not have to be kept
// is not written: the activation goes to the second product as bf16 rows in expert order (s of them against h of an output row).
#include "more_experts.cuh"

namespace more {

namespace {

constexpr int kXThreads = 320;                       // warps 0, 1: TMA, MMA; warps 2..9: epilogue
constexpr int kXRing = 200 * 1024;
constexpr int kXPitch = 80;                          // bytes of a staged row: 32 bf16, and 16 so that rows fall on other banks
constexpr int kXStage = 8 * 32 * kXPitch;            // staging of the eight epilogue warps
constexpr int kXSmem = kXRing + kXStage + 1024 /*alignment*/ + 512 /*barriers*/;
constexpr int kXMaxStages = 12;
constexpr int kTileRows = 128;
constexpr int kATile = kTileRows * 128;              // 128 rows of 64 bf16
constexpr int kBox = 64 * 128;                       // 64 rows of 64 bf16

enum { kUp = 0, kDown = 1, kBackAct = 2, kBackX = 3 };

__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int r0, int r1, int r2, int r3)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}

// Instruction descriptor of umma_idesc with the operands' majors: fp32 += bf16 x bf16, 128 rows, n columns.
__device__ __forceinline__ uint32_t idesc_of(int n, int a_mn, int b_mn)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(128 >> 4) << 24);
}

// ------------------------------------------------------------------------------------------------ tiles
// One entry per tile of up to 128 consecutive places of one expert: (expert, first place, places, 0), experts ascending.
// tiles[0].x is how many there are.  Every CTA takes 1024 experts and counts the tiles of all experts before them itself.
__global__ void __launch_bounds__(1024) tiles_kernel(const int32_t* __restrict__ offsets, int M, int P, int capacity, int4* __restrict__ tiles)
{
    __shared__ int warp_sum[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto run = [&](int e, int& lo) {                        // (whatever the offsets hold, a run stays within the places)
        lo = min(max(offsets[e], 0), P);
        return max(min(offsets[e + 1], P) - lo, 0);
    };
    int lo, before = 0;
    for (int e = tid; e < (int)blockIdx.x * 1024; e += 1024) before += (run(e, lo) + kTileRows - 1) / kTileRows;
    const int e = blockIdx.x * 1024 + tid;
    const int n = e < M ? run(e, lo) : 0;
    const int mine = (n + kTileRows - 1) / kTileRows;
    int incl = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
    }
    for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    __shared__ int warp_before[32];
    if (lane == 31) warp_sum[warp] = incl;
    if (lane == 0) warp_before[warp] = before;
    __syncthreads();
    int at = incl - mine;
    for (int w = 0; w < 32; ++w) {
        at += warp_before[w];
        if (w < warp) at += warp_sum[w];
    }
    for (int i = 0; i < mine && at + i < capacity; ++i)
        tiles[1 + at + i] = make_int4(e, lo + i * kTileRows, min(kTileRows, n - i * kTileRows), 0);
    if (e == M - 1) tiles[0].x = min(at + mine, capacity);
}

struct RowsParams {
    const int4* tiles;
    const int32_t* pairs;
    int P, k, h, s;
    int rows;                     // of A's tensor: the row that is out of its bounds
    int nb;                       // boxes of 64 weight columns per unit
    int chunks;                   // units per tile
    int ksteps;                   // of 64
    int stages;
    __nv_bfloat16* out;           // kUp: activation [P][s]; kDown: Y [P][h]
    __nv_bfloat16* hidden;        // kUp: nullable; kBackAct: read
    const float* gate;            // kBackAct
    __nv_bfloat16* du;            // kBackAct: [P][2s]
    __nv_bfloat16* ga;            // kBackAct: gate a, [P][s]
    float* dgate_part;            // kBackAct: [2 chunks][P]
    __half* dx;                   // kBackX: [P][h] scaled
    float* dx_scale;              // kBackX: [P][dx_groups], a power of two per 128 columns
    int dx_groups;
    int* status;
};

struct Control {
    uint64_t full[kXMaxStages], empty[kXMaxStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort;
};
static_assert(sizeof(Control) <= 512, "control block");

// A warp's 32 rows x 32 columns, one row per lane, to memory by way of shared memory, so that four lanes write 64 consecutive
// bytes of a row.  row_of(r): start of row r in elements or -1; col, limit: first column and how many a row has.
template <class RowOf>
__device__ __forceinline__ void store_rows32(uint32_t stage, int lane, const uint32_t (&u)[16], void* out, RowOf row_of, int col, int limit)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * kXPitch + i * 16), "r"(u[4 * i]), "r"(u[4 * i + 1]),
                     "r"(u[4 * i + 2]), "r"(u[4 * i + 3]) : "memory");
    __syncwarp();
    const int c = col + (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (lane >> 2);
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(stage + r * kXPitch + (lane & 3) * 16) : "memory");
        const long long at = row_of(r);
        if (at >= 0 && c < limit) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at + c) = v;
    }
    __syncwarp();
}

__device__ __forceinline__ void pack32(const float (&a)[16], const float (&b)[16], uint32_t (&u)[16])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i] = pack_bf16(a[2 * i], a[2 * i + 1]);
        u[8 + i] = pack_bf16(b[2 * i], b[2 * i + 1]);
    }
}

// Common start of both kernels: barriers, tensor memory.  Returns the tensor-memory base.
__device__ __forceinline__ uint32_t open_cta(Control* c, int stages, int warp)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(smem_u32(&c->full[i]), 1);
            mbar_init(smem_u32(&c->empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c->acc_full[i]), 1);
            mbar_init(smem_u32(&c->acc_empty[i]), 8);
        }
        c->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c->tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    return c->tmem;
}
__device__ __forceinline__ void close_cta(Control* c, uint32_t tmem, int warp)
{
    tc_fence_before();
    __syncthreads();
    if (c->abort && threadIdx.x == 0)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);   // loads that may still be in flight land before the memory is released
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

template <int MODE>
__global__ void __launch_bounds__(kXThreads, 1)
rows_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mw, const __grid_constant__ RowsParams p)
{
    constexpr bool kByToken = MODE == kUp || MODE == kBackAct;      // rows of A are tokens, else places in expert order
    constexpr bool kMn = MODE == kUp || MODE == kDown;              // weights as an MN-major operand
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging = ring + kXRing;
    Control* ctl = reinterpret_cast<Control*>(smem_raw + (ring - smem_u32(smem_raw)) + kXRing + kXStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = open_cta(ctl, p.stages, warp);
    volatile int* abort_flag = &ctl->abort;
    const int units = p.tiles[0].x * p.chunks;
    const uint32_t stage_bytes = kATile + p.nb * kBox;

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        bool live = true;
        int4 tile = make_int4(0, 0, 0, 0);
        int row[4] = {0, 0, 0, 0};
        auto fetch = [&](int unit) {                                // the tile of a unit and this lane's four rows of it
            if (unit >= units) return;
            tile = p.tiles[1 + unit / p.chunks];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 4 * lane + j;
                int v = -1;
                if (r < tile.z) v = kByToken ? p.pairs[tile.y + r] : tile.y + r;
                row[j] = v;
            }
        };
        fetch(blockIdx.x);
        for (int unit = blockIdx.x; unit < units && live; unit += gridDim.x) {
            const int e = tile.x, gathers = (tile.z + 3) / 4, chunk = unit % p.chunks;
            int r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)                             // a row that does not exist is out of bounds: zeros
                r[j] = row[j] < 0 || row[j] >= p.P ? p.rows : (kByToken ? (int)((unsigned)row[j] / (unsigned)p.k) : row[j]);
            fetch(unit + gridDim.x);
            for (int ks = 0; ks < p.ksteps; ++ks) {
                const uint32_t full = smem_u32(&ctl->full[stage]);
                if (!mbar_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort_flag, p.status)) { live = false; break; }
                const uint32_t at = ring + stage * stage_bytes;
                if (lane == 0) mbar_expect_tx(full, gathers * 512 + p.nb * kBox);
                __syncwarp();
                if (lane < gathers) tma_gather4(at + lane * 512, &ma, full, ks * 64, r[0], r[1], r[2], r[3]);
                if (lane < p.nb) {
                    int x, y;
                    if (MODE == kUp) {
                        const int half = p.nb / 2, b = lane < half ? lane : lane - half;
                        x = (lane < half ? 0 : p.s) + (chunk * half + b) * 64;
                        y = ks * 64;
                    } else if (kMn) {
                        x = (chunk * p.nb + lane) * 64;
                        y = ks * 64;
                    } else {
                        x = ks * 64;
                        y = (chunk * p.nb + lane) * 64;
                    }
                    tma_load_3d(at + kATile + lane * kBox, &mw, full, x, y, e);
                }
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        const uint32_t idesc = idesc_of(p.nb * 64, 0, kMn);
        const uint64_t a0 = umma_desc_sw128(ring, 16, 1024);
        const uint64_t b0 = kMn ? umma_desc_sw128(ring + kATile, kBox, 1024) : umma_desc_sw128(ring + kATile, 16, 1024);
        const uint32_t a_hi = (uint32_t)(a0 >> 32), b_hi = (uint32_t)(b0 >> 32);
        constexpr uint32_t kBStep = kMn ? 2048 >> 4 : 32 >> 4;
        int stage = 0, it = 0;
        uint32_t phase = 0;
        bool live = true;
        for (int unit = blockIdx.x; unit < units && live; unit += gridDim.x, ++it) {
            const int buf = it & 1;
            if (!mbar_wait(smem_u32(&ctl->acc_empty[buf]), ((it >> 1) & 1) ^ 1u, abort_flag, p.status)) break;
            tc_fence_after();
            for (int ks = 0; ks < p.ksteps; ++ks) {
                if (!mbar_wait(smem_u32(&ctl->full[stage]), phase, abort_flag, p.status)) { live = false; break; }
                tc_fence_after();
                const uint32_t off = (stage * stage_bytes) >> 4;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    tc_mma_bf16_ss_elect(tmem + buf * 256, (uint32_t)a0 + off + q * 2, a_hi, (uint32_t)b0 + off + q * kBStep, b_hi, idesc,
                                         ks > 0 || q > 0);
                tc_commit_elect(smem_u32(&ctl->empty[stage]));
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
            if (live) tc_commit_elect(smem_u32(&ctl->acc_full[buf]));
        }
    } else {
        const int quarter = warp & 3, side = warp >= 6;             // lane quarter of the accumulator; half of the columns
        const uint32_t stage = staging + (warp - 2) * 32 * kXPitch;
        int it = 0;
        for (int unit = blockIdx.x; unit < units; unit += gridDim.x, ++it) {
            const int4 tile = p.tiles[1 + unit / p.chunks];
            const int chunk = unit % p.chunks, buf = it & 1;
            const int r0 = quarter * 32;                            // this warp's first row of the tile
            const bool mine = r0 + lane < tile.z;
            const int place = tile.y + r0 + lane;
            int pair = -1;
            float gate = 0.f;
            if constexpr (MODE != kUp) {
                if (mine) pair = p.pairs[place];
                if (pair >= p.P) pair = -1;
                if constexpr (MODE == kBackAct)
                    if (pair >= 0) gate = p.gate[pair];
            }
            const uint32_t acc = tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16);
            if (!mbar_wait(smem_u32(&ctl->acc_full[buf]), (it >> 1) & 1, abort_flag, p.status)) break;
            tc_fence_after();
            const bool any = r0 < tile.z;                           // (a warp whose rows are all behind the tile has nothing to do)
            auto by_place = [&](int r, int width) { return r0 + r < tile.z ? (long long)(tile.y + r0 + r) * width : -1ll; };
            if constexpr (MODE == kUp) {
                const int cols = p.nb * 32, per = cols / 2;         // s columns of the unit; of this warp
                const int s0 = chunk * cols + side * per;
                for (int c = 0; c < per && any && s0 + c < p.s; c += 32) {
                    float g0[16], g1[16], u0[16], u1[16];
                    tmem_ld16(acc + side * per + c, g0);
                    tmem_ld16(acc + side * per + c + 16, g1);
                    tmem_ld16(acc + cols + side * per + c, u0);
                    tmem_ld16(acc + cols + side * per + c + 16, u1);
                    tmem_ld_wait16(g0); tmem_ld_wait16(g1); tmem_ld_wait16(u0); tmem_ld_wait16(u1);
                    uint32_t u[16];
                    if (p.hidden) {
                        pack32(g0, g1, u);
                        store_rows32(stage, lane, u, p.hidden, [&](int r) { return by_place(r, 2 * p.s); }, s0 + c, p.s);
                        pack32(u0, u1, u);
                        store_rows32(stage, lane, u, p.hidden + p.s, [&](int r) { return by_place(r, 2 * p.s); }, s0 + c, p.s);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        g0[i] = g0[i] * sigmoidf(g0[i]) * u0[i];
                        g1[i] = g1[i] * sigmoidf(g1[i]) * u1[i];
                    }
                    pack32(g0, g1, u);
                    store_rows32(stage, lane, u, p.out, [&](int r) { return by_place(r, p.s); }, s0 + c, p.s);
                }
            } else if constexpr (MODE == kDown) {
                const int per = p.nb * 32, c0 = chunk * p.nb * 64 + side * per;
                auto by_pair = [&](int r) {
                    const int q = __shfl_sync(0xffffffffu, pair, r);
                    return q >= 0 ? (long long)q * p.h : -1ll;
                };
                for (int c = 0; c < per && any && c0 + c < p.h; c += 32) {
                    float v0[16], v1[16];
                    tmem_ld16(acc + side * per + c, v0);
                    tmem_ld16(acc + side * per + c + 16, v1);
                    tmem_ld_wait16(v0); tmem_ld_wait16(v1);
                    uint32_t u[16];
                    pack32(v0, v1, u);
                    store_rows32(stage, lane, u, p.out, by_pair, c0 + c, p.h);
                }
            } else if constexpr (MODE == kBackAct) {
                const int per = p.nb * 32, s0 = chunk * p.nb * 64 + side * per;
                float dg_sum = 0.f;
                for (int c = 0; c < per && any && s0 + c < p.s; c += 32) {
                    uint32_t hg[16], hu[16];                        // both projections of this row, 32 columns
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint4 a = make_uint4(0, 0, 0, 0), b = a;
                        const int col = s0 + c + i * 8;
                        if (mine && col < p.s) {
                            const __nv_bfloat16* from = p.hidden + (long long)place * 2 * p.s + col;
                            a = *reinterpret_cast<const uint4*>(from);
                            b = *reinterpret_cast<const uint4*>(from + p.s);
                        }
                        hg[4 * i] = a.x; hg[4 * i + 1] = a.y; hg[4 * i + 2] = a.z; hg[4 * i + 3] = a.w;
                        hu[4 * i] = b.x; hu[4 * i + 1] = b.y; hu[4 * i + 2] = b.z; hu[4 * i + 3] = b.w;
                    }
                    float c0[16], c1[16];
                    tmem_ld16(acc + side * per + c, c0);
                    tmem_ld16(acc + side * per + c + 16, c1);
                    tmem_ld_wait16(c0); tmem_ld_wait16(c1);
                    uint32_t ug[16], uu[16], ua[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float r_g[2], r_u[2], r_a[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float g = j ? bf16_hi(hg[i]) : bf16_lo(hg[i]), up = j ? bf16_hi(hu[i]) : bf16_lo(hu[i]);
                            const float cc = i < 8 ? c0[2 * i + j] : c1[2 * i + j - 16];
                            const float sg = sigmoidf(g), silu = g * sg, act = silu * up, da = gate * cc;
                            dg_sum = fmaf(cc, act, dg_sum);
                            r_a[j] = gate * act;
                            r_u[j] = da * silu;
                            r_g[j] = da * up * fmaf(silu, 1.f - sg, sg);
                        }
                        ug[i] = pack_bf16(r_g[0], r_g[1]);
                        uu[i] = pack_bf16(r_u[0], r_u[1]);
                        ua[i] = pack_bf16(r_a[0], r_a[1]);
                    }
                    store_rows32(stage, lane, ug, p.du, [&](int r) { return by_place(r, 2 * p.s); }, s0 + c, p.s);
                    store_rows32(stage, lane, uu, p.du + p.s, [&](int r) { return by_place(r, 2 * p.s); }, s0 + c, p.s);
                    if (p.ga) store_rows32(stage, lane, ua, p.ga, [&](int r) { return by_place(r, p.s); }, s0 + c, p.s);
                }
                if (pair >= 0) p.dgate_part[(long long)(chunk * 2 + side) * p.P + pair] = dg_sum;
            } else {
                // The rows of the slots are added later: each 128 columns of a row are kept in fp16 behind a power of two that
                // brings their largest to [2^14, 2^15): an eighth of bf16's rounding for the same bytes.
                const int per = p.nb * 32, c0 = chunk * p.nb * 64 + side * per;
                auto by_pair = [&](int r) {
                    const int q = __shfl_sync(0xffffffffu, pair, r);
                    return q >= 0 ? (long long)q * p.h : -1ll;
                };
                for (int g = 0; g < per && any && c0 + g < p.h; g += 128) {
                    const int end = min(per, g + 128);
                    float top = 0.f;
                    for (int c = g; c < end && c0 + c < p.h; c += 32) {
                        float v0[16], v1[16];
                        tmem_ld16(acc + side * per + c, v0);
                        tmem_ld16(acc + side * per + c + 16, v1);
                        tmem_ld_wait16(v0); tmem_ld_wait16(v1);
#pragma unroll
                        for (int i = 0; i < 16; ++i) top = max3(top, fabsf(v0[i]), fabsf(v1[i]));
                    }
                    const int ex = max(15, __float_as_int(top) >> 23);
                    const float up = ex < 255 ? __int_as_float((268 - ex) << 23) : 1.f, down = ex < 255 ? __int_as_float((ex - 14) << 23) : 1.f;
                    if (pair >= 0) p.dx_scale[(long long)pair * p.dx_groups + (c0 + g) / per] = down;
                    for (int c = g; c < end && c0 + c < p.h; c += 32) {
                        float v0[16], v1[16];
                        tmem_ld16(acc + side * per + c, v0);
                        tmem_ld16(acc + side * per + c + 16, v1);
                        tmem_ld_wait16(v0); tmem_ld_wait16(v1);
                        uint32_t u[16];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const __half2 a = __floats2half2_rn(v0[2 * i] * up, v0[2 * i + 1] * up);
                            const __half2 b = __floats2half2_rn(v1[2 * i] * up, v1[2 * i + 1] * up);
                            u[i] = *reinterpret_cast<const uint32_t*>(&a);
                            u[8 + i] = *reinterpret_cast<const uint32_t*>(&b);
                        }
                        store_rows32(stage, lane, u, p.dx, by_pair, c0 + c, p.h);
                    }
                }
            }
            tc_fence_before();
            warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);
        }
    }
    close_cta(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------------------ gradients of the weights
struct WeightsParams {
    const int32_t* offsets;
    const int32_t* pairs;
    int P, T, k, M;
    int a_by_token;               // dW1: A = X by token, B = du by place; dW2: A = gate a by place, B = d by token
    int rows, cols;               // of an expert's output
    int mtiles, chunks, nb;
    int stages;
    __nv_bfloat16* out;           // [M][rows][cols]
    int* status;
};

__global__ void __launch_bounds__(kXThreads, 1)
weights_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb, const __grid_constant__ WeightsParams p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging = ring + kXRing;
    Control* ctl = reinterpret_cast<Control*>(smem_raw + (ring - smem_u32(smem_raw)) + kXRing + kXStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = open_cta(ctl, p.stages, warp);
    volatile int* abort_flag = &ctl->abort;
    const int per_expert = p.mtiles * p.chunks;
    const long long units = (long long)p.M * per_expert;
    const uint32_t stage_bytes = (2 + p.nb) * kBox;
    auto run = [&](int e, int& lo) {
        lo = min(max(p.offsets[e], 0), p.P);
        return max(min(p.offsets[e + 1], p.P) - lo, 0);
    };

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        bool live = true;
        const int g = lane & 15, side = lane >> 4;                  // rows 4 g .. 4 g + 3 of a step, every other box
        for (long long unit = blockIdx.x; unit < units && live; unit += gridDim.x) {
            const int e = (int)(unit / per_expert), rem = (int)(unit % per_expert), mt = rem / p.chunks, chunk = rem % p.chunks;
            int lo;
            const int n = run(e, lo);
            const int a_boxes = p.rows - mt * 128 > 64 ? 2 : 1;
            int pr[4];
            auto fetch = [&](int at) {
#pragma unroll
                for (int j = 0; j < 4; ++j) pr[j] = at + 4 * g + j < n ? p.pairs[lo + at + 4 * g + j] : -1;
            };
            fetch(0);
            for (int at = 0; at < n; at += 64) {
                const int gathers = (min(64, n - at) + 15) / 16 * 4;       // whole MMA steps of 16 rows
                int by_token[4], by_place[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool live = pr[j] >= 0 && pr[j] < p.P;
                    by_token[j] = live ? (int)((unsigned)pr[j] / (unsigned)p.k) : p.T;      // (out of bounds: zeros)
                    by_place[j] = live ? lo + at + 4 * g + j : p.P;
                }
                fetch(at + 64);
                const uint32_t full = smem_u32(&ctl->full[stage]);
                if (!mbar_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort_flag, p.status)) { live = false; break; }
                const uint32_t base = ring + stage * stage_bytes;
                if (lane == 0) mbar_expect_tx(full, gathers * 512 * (a_boxes + p.nb));
                __syncwarp();
                if (g < gathers) {
                    for (int b = side; b < a_boxes; b += 2) {
                        const int x = mt * 128 + b * 64;
                        if (p.a_by_token) tma_gather4(base + b * kBox + g * 512, &ma, full, x, by_token[0], by_token[1], by_token[2], by_token[3]);
                        else tma_gather4(base + b * kBox + g * 512, &ma, full, x, by_place[0], by_place[1], by_place[2], by_place[3]);
                    }
                    for (int b = side; b < p.nb; b += 2) {
                        const int x = (chunk * p.nb + b) * 64;
                        if (p.a_by_token) tma_gather4(base + (2 + b) * kBox + g * 512, &mb, full, x, by_place[0], by_place[1], by_place[2], by_place[3]);
                        else tma_gather4(base + (2 + b) * kBox + g * 512, &mb, full, x, by_token[0], by_token[1], by_token[2], by_token[3]);
                    }
                }
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        const uint32_t idesc = idesc_of(p.nb * 64, 1, 1);
        const uint64_t a0 = umma_desc_sw128(ring, kBox, 1024), b0 = umma_desc_sw128(ring + 2 * kBox, kBox, 1024);
        const uint32_t a_hi = (uint32_t)(a0 >> 32), b_hi = (uint32_t)(b0 >> 32);
        int stage = 0, it = 0;
        uint32_t phase = 0;
        bool live = true;
        for (long long unit = blockIdx.x; unit < units && live; unit += gridDim.x) {
            int lo;
            const int n = run((int)(unit / per_expert), lo);
            if (n == 0) continue;                                   // (the epilogue writes zeros without an accumulator)
            const int buf = it & 1;
            if (!mbar_wait(smem_u32(&ctl->acc_empty[buf]), ((it >> 1) & 1) ^ 1u, abort_flag, p.status)) break;
            tc_fence_after();
            for (int at = 0; at < n; at += 64) {
                const int steps = (min(64, n - at) + 15) / 16;
                if (!mbar_wait(smem_u32(&ctl->full[stage]), phase, abort_flag, p.status)) { live = false; break; }
                tc_fence_after();
                const uint32_t off = (stage * stage_bytes) >> 4;
                for (int q = 0; q < steps; ++q)
                    tc_mma_bf16_ss_elect(tmem + buf * 256, (uint32_t)a0 + off + q * 128, a_hi, (uint32_t)b0 + off + q * 128, b_hi, idesc,
                                         at > 0 || q > 0);
                tc_commit_elect(smem_u32(&ctl->empty[stage]));
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
            if (live) tc_commit_elect(smem_u32(&ctl->acc_full[buf]));
            ++it;
        }
    } else {
        const int quarter = warp & 3, side = warp >= 6;
        const uint32_t stage = staging + (warp - 2) * 32 * kXPitch;
        int it = 0;
        for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
            const int e = (int)(unit / per_expert), rem = (int)(unit % per_expert), mt = rem / p.chunks, chunk = rem % p.chunks;
            int lo;
            const int n = run(e, lo);
            const int row0 = mt * 128 + quarter * 32, per = p.nb * 32, c0 = chunk * p.nb * 64 + side * per;
            auto row_of = [&](int r) { return row0 + r < p.rows ? ((long long)e * p.rows + row0 + r) * p.cols : -1ll; };
            uint32_t u[16];
            if (n == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) u[i] = 0;
                for (int c = 0; c < per && row0 < p.rows && c0 + c < p.cols; c += 32)
                    store_rows32(stage, lane, u, p.out, row_of, c0 + c, p.cols);
                continue;
            }
            const int buf = it & 1;
            const uint32_t acc = tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16);
            if (!mbar_wait(smem_u32(&ctl->acc_full[buf]), (it >> 1) & 1, abort_flag, p.status)) break;
            tc_fence_after();
            for (int c = 0; c < per && row0 < p.rows && c0 + c < p.cols; c += 32) {
                float v0[16], v1[16];
                tmem_ld16(acc + side * per + c, v0);
                tmem_ld16(acc + side * per + c + 16, v1);
                tmem_ld_wait16(v0); tmem_ld_wait16(v1);
                pack32(v0, v1, u);
                store_rows32(stage, lane, u, p.out, row_of, c0 + c, p.cols);
            }
            tc_fence_before();
            warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);
            ++it;
        }
    }
    close_cta(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------------------ joining the slots
// dX[t] = sum over the token's slots of their rows (fp16 behind a scale per 128 columns); dgate[p] = sum of its parts.  A pair
// whose id is no expert was in no tile: it adds nothing and its gate gradient is 0.
struct JoinParams {
    const int32_t* idx;
    const __half* dx;
    const float* dx_scale;
    const float* dgate_part;
    int P, T, k, h, M, dx_groups, parts, group_cols;
    __nv_bfloat16* out_dx;
    float* out_dgate;
};
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinParams p)
{
    const int vecs = p.h / 8;
    const long long all = p.out_dx ? (long long)p.T * vecs : 0;
    const long long first = (long long)blockIdx.x * 256 + threadIdx.x, stride = (long long)gridDim.x * 256;
    for (long long i = first; i < all; i += stride) {
        const int t = (int)(i / vecs), c = (int)(i % vecs) * 8, grp = c / p.group_cols;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < p.k; ++j) {
            const long long pair = (long long)t * p.k + j;
            if ((unsigned)p.idx[pair] >= (unsigned)p.M) continue;
            const float sc = p.dx_scale[pair * p.dx_groups + grp];
            const uint4 u = *reinterpret_cast<const uint4*>(p.dx + pair * p.h + c);
            const __half2* q = reinterpret_cast<const __half2*>(&u);
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const float2 f = __half22float2(q[a]);
                v[2 * a] = fmaf(f.x, sc, v[2 * a]);
                v[2 * a + 1] = fmaf(f.y, sc, v[2 * a + 1]);
            }
        }
        *reinterpret_cast<uint4*>(p.out_dx + (long long)t * p.h + c) =
            make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
    if (!p.out_dgate) return;
    for (long long i = first; i < p.P; i += stride) {
        float sum = 0.f;
        if ((unsigned)p.idx[i] < (unsigned)p.M)
            for (int q = 0; q < p.parts; ++q) sum += p.dgate_part[(long long)q * p.P + i];
        p.out_dgate[i] = sum;
    }
}

// ------------------------------------------------------------------------------------------------ host side
size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

long long tile_capacity(int T, int M, int k)
{
    const long long P = (long long)T * k;
    return (P < M ? P : M) + P / kTileRows;
}

struct Workspace {                 // offsets of the pieces, and the total
    size_t act = 0, du = 0, ga = 0, dgate = 0, dx = 0, dx_scale = 0, total = 0;
};
int back_boxes(int s) { return s > 192 ? 4 : (s + 63) / 64; }      // boxes of s rows per unit of the activation's backward
int dx_group_cols(int h) { return h > 128 ? 128 : (h > 64 ? 64 : 32); }   // columns that share a scale: half a unit of kBackX
int row_boxes(int h) { return h > 128 ? 4 : (h > 64 ? 2 : 1); }

Workspace lay_out(int T, int h, int s, int M, int k, bool backward)
{
    const size_t P = (size_t)T * k;
    Workspace w;
    size_t at = up256(16 * (size_t)(1 + tile_capacity(T, M, k)));
    if (!backward) {
        w.act = at; at += up256(P * s * 2);
    } else {
        const int nb = back_boxes(s), chunks = (s + nb * 64 - 1) / (nb * 64), g = dx_group_cols(h);
        w.du = at; at += up256(P * s * 4);
        w.ga = at; at += up256(P * s * 2);
        w.dgate = at; at += up256(P * 4 * 2 * chunks);
        w.dx = at; at += up256(P * h * 2);
        w.dx_scale = at; at += up256(P * 4 * ((h + g - 1) / g));
    }
    w.total = at;
    return w;
}

// 2-D [rows][cols] for gathering loads: one row high.
int gather_map(const void* ptr, long long rows, int cols, CUtensorMap* out)
{
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)cols * 2};
    const uint32_t box[2] = {64, 1};
    return encode_tensor_map(ptr, 2, dims, strides, box, out);
}
// Weights [M][rows][cols], box 64 x 64 of one expert.
int weight_map(const void* ptr, int M, int rows, int cols, CUtensorMap* out)
{
    const uint64_t dims[3] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)M};
    const uint64_t strides[2] = {(uint64_t)cols * 2, (uint64_t)rows * cols * 2};
    const uint32_t box[3] = {64, 64, 1};
    return encode_tensor_map(ptr, 3, dims, strides, box, out);
}

template <class Kernel>
int allow_smem(Kernel kern)
{
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kXSmem) == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

template <int MODE>
int launch_rows(const CUtensorMap& ma, const CUtensorMap& mw, RowsParams p, long long tiles, const DeviceCtx& ctx, cudaStream_t st)
{
    if (allow_smem(rows_kernel<MODE>) != MORE_OK) return MORE_ERR_CUDA;
    p.stages = kXRing / (kATile + p.nb * kBox);
    if (p.stages > kXMaxStages) p.stages = kXMaxStages;
    p.status = ctx.status;
    const long long units = tiles * p.chunks;
    const int grid = units < ctx.sm_count ? (int)units : ctx.sm_count;
    rows_kernel<MODE><<<grid, kXThreads, kXSmem, st>>>(ma, mw, p);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

int launch_tiles(const ExpertsArgs& a, cudaStream_t st)
{
    const long long P = (long long)a.T * a.k;
    tiles_kernel<<<(a.M + 1023) / 1024, 1024, 0, st>>>(a.offsets, a.M, (int)P, (int)tile_capacity(a.T, a.M, a.k), static_cast<int4*>(a.workspace));
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

int launch_weights(const CUtensorMap& ma, const CUtensorMap& mb, WeightsParams p, const DeviceCtx& ctx, cudaStream_t st)
{
    if (allow_smem(weights_kernel) != MORE_OK) return MORE_ERR_CUDA;
    p.nb = p.cols > 128 ? 4 : (p.cols > 64 ? 2 : 1);
    p.mtiles = (p.rows + 127) / 128;
    p.chunks = (p.cols + p.nb * 64 - 1) / (p.nb * 64);
    p.stages = kXRing / ((2 + p.nb) * kBox);
    if (p.stages > kXMaxStages) p.stages = kXMaxStages;
    p.status = ctx.status;
    const long long units = (long long)p.M * p.mtiles * p.chunks;
    const int grid = units < ctx.sm_count ? (int)units : ctx.sm_count;
    weights_kernel<<<grid, kXThreads, kXSmem, st>>>(ma, mb, p);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

int launch_experts(const ExpertsArgs& a, const DeviceCtx& ctx)
{
    const long long P = (long long)a.T * a.k;
    const Workspace w = lay_out(a.T, a.h, a.s, a.M, a.k, false);
    char* base = static_cast<char*>(a.workspace);
    CUtensorMap mx, mact, m1, m2;
    int rc = gather_map(a.X, a.T, a.h, &mx);
    if (rc == MORE_OK) rc = gather_map(base + w.act, P, a.s, &mact);
    if (rc == MORE_OK) rc = weight_map(a.W1, a.M, a.h, 2 * a.s, &m1);
    if (rc == MORE_OK) rc = weight_map(a.W2, a.M, a.s, a.h, &m2);
    if (rc == MORE_OK) rc = launch_tiles(a, a.stream);
    if (rc != MORE_OK) return rc;
    RowsParams p{};
    p.tiles = static_cast<const int4*>(a.workspace);
    p.pairs = a.pairs;
    p.P = (int)P; p.k = a.k; p.h = a.h; p.s = a.s;
    const long long tiles = tile_capacity(a.T, a.M, a.k);
    p.rows = a.T;
    p.nb = a.s > 64 ? 4 : 2;
    p.chunks = (a.s + p.nb * 32 - 1) / (p.nb * 32);
    p.ksteps = (a.h + 63) / 64;
    p.out = reinterpret_cast<__nv_bfloat16*>(base + w.act);
    p.hidden = a.out_hidden;
    rc = launch_rows<kUp>(mx, m1, p, tiles, ctx, a.stream);
    if (rc != MORE_OK) return rc;
    p.rows = (int)P;
    p.nb = row_boxes(a.h);
    p.chunks = (a.h + p.nb * 64 - 1) / (p.nb * 64);
    p.ksteps = (a.s + 63) / 64;
    p.out = a.out_y;
    return launch_rows<kDown>(mact, m2, p, tiles, ctx, a.stream);
}

int launch_experts_backward(const ExpertsArgs& a, const DeviceCtx& ctx)
{
    const long long P = (long long)a.T * a.k;
    const Workspace w = lay_out(a.T, a.h, a.s, a.M, a.k, true);
    char* base = static_cast<char*>(a.workspace);
    CUtensorMap mx, md, mdu, mga, m1, m2;
    int rc = gather_map(a.X, a.T, a.h, &mx);
    if (rc == MORE_OK) rc = gather_map(a.dout, a.T, a.h, &md);
    if (rc == MORE_OK) rc = gather_map(base + w.du, P, 2 * a.s, &mdu);
    if (rc == MORE_OK) rc = gather_map(base + w.ga, P, a.s, &mga);
    if (rc == MORE_OK) rc = weight_map(a.W1, a.M, a.h, 2 * a.s, &m1);
    if (rc == MORE_OK) rc = weight_map(a.W2, a.M, a.s, a.h, &m2);
    if (rc == MORE_OK) rc = launch_tiles(a, a.stream);
    if (rc != MORE_OK) return rc;
    const long long tiles = tile_capacity(a.T, a.M, a.k);
    RowsParams p{};
    p.tiles = static_cast<const int4*>(a.workspace);
    p.pairs = a.pairs;
    p.P = (int)P; p.k = a.k; p.h = a.h; p.s = a.s;
    p.rows = a.T;
    p.nb = back_boxes(a.s);
    p.chunks = (a.s + p.nb * 64 - 1) / (p.nb * 64);
    p.ksteps = (a.h + 63) / 64;
    p.hidden = const_cast<__nv_bfloat16*>(a.hidden);
    p.gate = a.gate;
    p.du = reinterpret_cast<__nv_bfloat16*>(base + w.du);
    p.ga = a.out_dw2 ? reinterpret_cast<__nv_bfloat16*>(base + w.ga) : nullptr;
    p.dgate_part = reinterpret_cast<float*>(base + w.dgate);
    const int parts = 2 * p.chunks;
    rc = launch_rows<kBackAct>(md, m2, p, tiles, ctx, a.stream);
    if (rc != MORE_OK) return rc;
    p.dx_groups = (a.h + dx_group_cols(a.h) - 1) / dx_group_cols(a.h);
    p.dx = reinterpret_cast<__half*>(base + w.dx);
    p.dx_scale = reinterpret_cast<float*>(base + w.dx_scale);
    if (a.out_dx) {
        p.rows = (int)P;
        p.nb = row_boxes(a.h);
        p.chunks = (a.h + p.nb * 64 - 1) / (p.nb * 64);
        p.ksteps = (2 * a.s + 63) / 64;
        rc = launch_rows<kBackX>(mdu, m1, p, tiles, ctx, a.stream);
        if (rc != MORE_OK) return rc;
    }
    if (a.out_dx || a.out_dgate) {
        JoinParams j{};
        j.idx = a.idx; j.dx = p.dx; j.dx_scale = p.dx_scale; j.dgate_part = p.dgate_part;
        j.P = (int)P; j.T = a.T; j.k = a.k; j.h = a.h; j.M = a.M; j.dx_groups = p.dx_groups; j.parts = parts;
        j.group_cols = dx_group_cols(a.h);
        j.out_dx = a.out_dx; j.out_dgate = a.out_dgate;
        const long long items = a.out_dx ? (long long)a.T * (a.h / 8) : P;
        const long long blocks = (items + 255) / 256;
        join_kernel<<<(int)(blocks < 148 * 16 ? blocks : 148 * 16), 256, 0, a.stream>>>(j);
        count_launch(1);
        if (cudaGetLastError() != cudaSuccess) return MORE_ERR_CUDA;
    }
    WeightsParams q{};
    q.offsets = a.offsets; q.pairs = a.pairs; q.P = (int)P; q.T = a.T; q.k = a.k; q.M = a.M;
    if (a.out_dw1) {
        q.a_by_token = 1; q.rows = a.h; q.cols = 2 * a.s; q.out = a.out_dw1;
        rc = launch_weights(mx, mdu, q, ctx, a.stream);
        if (rc != MORE_OK) return rc;
    }
    if (a.out_dw2) {
        q.a_by_token = 0; q.rows = a.s; q.cols = a.h; q.out = a.out_dw2;
        rc = launch_weights(mga, md, q, ctx, a.stream);
    }
    return rc;
}

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int check_sizes(int T, int h, int s, int M, int k)
{
    if (T < 0 || h < 8 || s < 8 || h % 8 != 0 || s % 8 != 0 || h > MORE_H_MAX || s > MORE_S_MAX) return MORE_ERR_SHAPE;
    if (M < 1 || M > MORE_M_MAX || k < 1 || k > MORE_K_MAX || k > M) return MORE_ERR_SHAPE;
    if ((long long)T * k > 0x7fffffffLL) return MORE_ERR_TOO_LARGE;            // pairs are named by int32 positions
    return MORE_OK;
}

}  // namespace

}  // namespace more

using namespace more;

extern "C" {

long long more_experts_workspace(int T, int h, int s, int M, int k, int backward)
{
    const int rc = check_sizes(T, h, s, M, k);
    return rc == MORE_OK ? (long long)lay_out(T, h, s, M, k, backward != 0).total : rc;
}

int more_experts(const void* X, const void* W1, const void* W2, const int32_t* idx, const int32_t* offsets, const int32_t* sorted_pairs,
                 int T, int h, int s, int M, int k, void* out_y, void* out_hidden, int path, void* workspace, long long workspace_bytes,
                 void* stream)
{
    if (path != MORE_EXPERTS_AUTO && path != MORE_EXPERTS_PAIRS && path != MORE_EXPERTS_TILES) return MORE_ERR_MODE;
    int rc = check_sizes(T, h, s, M, k);
    if (rc != MORE_OK) return rc;
    if (T == 0) return MORE_OK;
    if (!X || !W1 || !W2 || !idx || !out_y) return MORE_ERR_NULL;
    const bool listed = offsets && sorted_pairs;
    if (!listed && (path == MORE_EXPERTS_TILES || out_hidden)) return MORE_ERR_NULL;
    if (path == MORE_EXPERTS_PAIRS && out_hidden) return MORE_ERR_SHAPE;
    if (misaligned(X, 16) || misaligned(W1, 16) || misaligned(W2, 16) || misaligned(idx, 4) || misaligned(offsets, 4) ||
        misaligned(sorted_pairs, 4) || misaligned(out_y, 16) || misaligned(out_hidden, 16) || misaligned(workspace, 256))
        return MORE_ERR_ALIGN;
    const bool pairwise = path == MORE_EXPERTS_PAIRS || !listed || (path == MORE_EXPERTS_AUTO && !out_hidden && more_experts_path(T, h, s, M, k) == MORE_EXPERTS_PAIRS);
    if (!pairwise) {
        if (!workspace) return MORE_ERR_NULL;
        if (workspace_bytes < more_experts_workspace(T, h, s, M, k, 0)) return MORE_ERR_TOO_LARGE;
    }
    DeviceCtx* ctx = nullptr;
    rc = device_ctx(&ctx);
    if (rc != MORE_OK) return rc;
    ExpertsArgs a{};
    a.X = static_cast<const __nv_bfloat16*>(X); a.W1 = static_cast<const __nv_bfloat16*>(W1); a.W2 = static_cast<const __nv_bfloat16*>(W2);
    a.idx = idx; a.offsets = offsets; a.pairs = sorted_pairs;
    a.T = T; a.h = h; a.s = s; a.M = M; a.k = k;
    a.out_y = static_cast<__nv_bfloat16*>(out_y); a.out_hidden = static_cast<__nv_bfloat16*>(out_hidden);
    a.workspace = workspace;
    a.stream = static_cast<cudaStream_t>(stream);
    return pairwise ? launch_experts_pairs(a, *ctx) : launch_experts(a, *ctx);
}

int more_experts_path(int T, int h, int s, int M, int k)
{
    const int rc = check_sizes(T, h, s, M, k);
    if (rc != MORE_OK) return rc;
    const long long P = (long long)T * k;
    return P <= 1024 && P <= M ? MORE_EXPERTS_PAIRS : MORE_EXPERTS_TILES;
}

int more_experts_backward(const void* X, const void* W1, const void* W2, const int32_t* idx, const int32_t* offsets,
                          const int32_t* sorted_pairs, const float* gate, const void* hidden, const void* dout, int T, int h, int s, int M,
                          int k, void* out_dx, float* out_dgate, void* out_dw1, void* out_dw2, void* workspace, long long workspace_bytes,
                          void* stream)
{
    int rc = check_sizes(T, h, s, M, k);
    if (rc != MORE_OK) return rc;
    if (T > 0 && (!X || !W1 || !W2 || !idx || !offsets || !sorted_pairs || !gate || !hidden || !dout || !workspace)) return MORE_ERR_NULL;
    if (misaligned(X, 16) || misaligned(W1, 16) || misaligned(W2, 16) || misaligned(idx, 4) || misaligned(offsets, 4) ||
        misaligned(sorted_pairs, 4) || misaligned(gate, 4) || misaligned(hidden, 16) || misaligned(dout, 16) || misaligned(out_dx, 16) ||
        misaligned(out_dgate, 4) || misaligned(out_dw1, 16) || misaligned(out_dw2, 16) || misaligned(workspace, 256))
        return MORE_ERR_ALIGN;
    if (T > 0 && workspace_bytes < more_experts_workspace(T, h, s, M, k, 1)) return MORE_ERR_TOO_LARGE;
    DeviceCtx* ctx = nullptr;
    rc = device_ctx(&ctx);
    if (rc != MORE_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        const size_t n = (size_t)M * h * s * 2;
        if (out_dw1 && cudaMemsetAsync(out_dw1, 0, 2 * n, st) != cudaSuccess) return MORE_ERR_CUDA;
        if (out_dw2 && cudaMemsetAsync(out_dw2, 0, n, st) != cudaSuccess) return MORE_ERR_CUDA;
        return MORE_OK;
    }
    ExpertsArgs a{};
    a.X = static_cast<const __nv_bfloat16*>(X); a.W1 = static_cast<const __nv_bfloat16*>(W1); a.W2 = static_cast<const __nv_bfloat16*>(W2);
    a.idx = idx; a.offsets = offsets; a.pairs = sorted_pairs;
    a.T = T; a.h = h; a.s = s; a.M = M; a.k = k;
    a.gate = gate; a.hidden = static_cast<const __nv_bfloat16*>(hidden); a.dout = static_cast<const __nv_bfloat16*>(dout);
    a.out_dx = static_cast<__nv_bfloat16*>(out_dx); a.out_dgate = out_dgate;
    a.out_dw1 = static_cast<__nv_bfloat16*>(out_dw1); a.out_dw2 = static_cast<__nv_bfloat16*>(out_dw2);
    a.workspace = workspace;
    a.stream = st;
    return launch_experts_backward(a, *ctx);
}

}  // extern "C"
