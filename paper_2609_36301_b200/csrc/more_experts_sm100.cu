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
constexpr int kGatherWarps = 4;                      // ... and, where rows are gathered, warps 10..13
constexpr int kXGatherThreads = kXThreads + kGatherWarps * 32;
constexpr int kXRing = 160 * 1024;
constexpr int kXStaging = 64 * 1024;                 // what the epilogue passes from the tensor memory's layout to memory's
constexpr int kXSmem = kXRing + kXStaging + 1024 /*alignment*/ + 1024 /*barriers*/;
constexpr int kXMaxStages = 12;
constexpr int kTileRows = 128;
constexpr int kATile = kTileRows * 128;              // 128 rows of 64 bf16
constexpr int kBox = 64 * 128;                       // 64 rows of 64 bf16

enum { kUp = 0, kDown = 1, kBackAct = 2, kBackX = 3 };

// Loads as a converged warp issues them: every lane passes the same operands and elect.sync picks the lane that issues.  (The
// instructions take their operands from uniform registers; behind a branch that one lane takes each cost ~150 clocks to issue,
// in this form a fraction of that.)
// Up to four gathers of four rows each, `step` bytes of shared memory apart, as many as `count` says.
__device__ __forceinline__ void tma_gather4x4(uint32_t dst, uint32_t step, const CUtensorMap* map, uint32_t bar, int x, int count, const int (&r)[16])
{
    asm volatile(
        "{\n\t.reg .pred pe, p0, p1, p2, p3;\n\t.reg .b32 d1, d2, d3;\n\t"
        "elect.sync _|pe, 0xffffffff;\n\t"
        "setp.gt.and.s32 p0, %5, 0, pe;\n\tsetp.gt.and.s32 p1, %5, 1, pe;\n\tsetp.gt.and.s32 p2, %5, 2, pe;\n\tsetp.gt.and.s32 p3, %5, 3, pe;\n\t"
        "add.u32 d1, %0, %1;\n\tadd.u32 d2, d1, %1;\n\tadd.u32 d3, d2, %1;\n\t"
        "@p0 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%2, {%4, %6, %7, %8, %9}], [%3];\n\t"
        "@p1 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [d1], [%2, {%4, %10, %11, %12, %13}], [%3];\n\t"
        "@p2 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [d2], [%2, {%4, %14, %15, %16, %17}], [%3];\n\t"
        "@p3 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [d3], [%2, {%4, %18, %19, %20, %21}], [%3];\n\t}"
        ::"r"(dst), "r"(step), "l"(map), "r"(bar), "r"(x), "r"(count), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
          "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tma_load_2d_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
        "@pe cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
        "@pe cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void expect_elect(uint32_t bar, uint32_t bytes)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
        "@pe mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes) : "memory");
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
    float* dgate_part;            // kBackAct: [chunks][P]
    __half* dx;                   // kBackX: [P][h] scaled
    float* dx_scale;              // kBackX: [P][dx_groups], a power of two per 128 columns
    int dx_groups;
    int* status;
};

struct Control {
    uint64_t full[kXMaxStages], empty[kXMaxStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort;
    int pair[kTileRows];
};
static_assert(sizeof(Control) <= 1024, "control block");

// Barrier of the eight epilogue warps.
__device__ __forceinline__ void epilogue_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// Staging: rows of `pitch` bytes, a power of two; the 16-byte pieces of a row are permuted by the row's number, so that neither a
// warp that writes a piece of 32 rows nor one that reads along a row meets itself on a bank.
__device__ __forceinline__ uint32_t staged(uint32_t base, int pitch, int row, int piece) { return base + row * pitch + ((piece ^ (row & 7)) << 4); }
__device__ __forceinline__ void st_piece(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 ld_piece(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// 16 fp32 of a row into staging, from piece `piece` on; 32 values as bf16.
__device__ __forceinline__ void stage_f32(uint32_t base, int pitch, int row, int piece, const float (&v)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        st_piece(staged(base, pitch, row, piece + i), __float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]),
                 __float_as_uint(v[4 * i + 3]));
}
__device__ __forceinline__ void stage_bf16(uint32_t base, int pitch, int row, int piece, const float (&v)[16])
{
#pragma unroll
    for (int i = 0; i < 2; ++i)
        st_piece(staged(base, pitch, row, piece + i), pack_bf16(v[8 * i], v[8 * i + 1]), pack_bf16(v[8 * i + 2], v[8 * i + 3]),
                 pack_bf16(v[8 * i + 4], v[8 * i + 5]), pack_bf16(v[8 * i + 6], v[8 * i + 7]));
}
// 8 fp32 of a row, two pieces.
__device__ __forceinline__ void unstage8(uint32_t base, int pitch, int row, int piece, float (&v)[8])
{
    const uint4 a = ld_piece(staged(base, pitch, row, piece)), b = ld_piece(staged(base, pitch, row, piece + 1));
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8])
{
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// Common start of both kernels: barriers, tensor memory.  Returns the tensor-memory base.
__device__ __forceinline__ uint32_t open_cta(Control* c, int stages, int producers, int warp)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(smem_u32(&c->full[i]), producers);
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

// The tiles of a CTA's units in turn, and the pair in place `r` of each: a unit's pair is requested a unit ahead, its tile two.
struct TilesAhead {
    const RowsParams& p;
    int units, r, pair, next_pair;
    int4 tile, next_tile, last_tile;
    __device__ TilesAhead(const RowsParams& q, int n, int row) : p(q), units(n), r(row), pair(-1), next_pair(-1)
    {
        tile = next_tile = last_tile = make_int4(0, 0, 0, 0);
        if ((int)blockIdx.x < units) tile = p.tiles[1 + blockIdx.x / p.chunks];
        if ((int)(blockIdx.x + gridDim.x) < units) next_tile = p.tiles[1 + (blockIdx.x + gridDim.x) / p.chunks];
        if (r < tile.z) pair = p.pairs[tile.y + r];
        ask(blockIdx.x);
    }
    __device__ void ask(int unit)
    {
        next_pair = r < next_tile.z ? p.pairs[next_tile.y + r] : -1;
        last_tile = make_int4(0, 0, 0, 0);
        const long long u = unit + 2ll * gridDim.x;
        if (u < units) last_tile = p.tiles[1 + (int)u / p.chunks];
    }
    __device__ void next(int unit)                          // after `unit`
    {
        tile = next_tile;
        pair = next_pair;
        next_tile = last_tile;
        ask(unit + gridDim.x);
    }
};

template <int MODE>
__global__ void __launch_bounds__(MODE == kUp || MODE == kBackAct ? kXGatherThreads : kXThreads, 1)
rows_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mw, const __grid_constant__ RowsParams p)
{
    constexpr bool kByToken = MODE == kUp || MODE == kBackAct;      // rows of A are tokens, else places in expert order
    constexpr bool kMn = MODE == kUp || MODE == kDown;              // weights as an MN-major operand
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, staging = ring + kXRing;
    Control* ctl = reinterpret_cast<Control*>(smem_raw + (ring - smem_u32(smem_raw)) + kXRing + kXStaging);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = open_cta(ctl, p.stages, kByToken ? 1 + kGatherWarps : 1, warp);
    volatile int* abort_flag = &ctl->abort;
    const int units = p.tiles[0].x * p.chunks;
    const uint32_t stage_bytes = kATile + p.nb * kBox;

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        bool live = true;
        int4 next = make_int4(0, 0, 0, 0);
        if ((int)blockIdx.x < units) next = p.tiles[1 + blockIdx.x / p.chunks];
        for (int unit = blockIdx.x; unit < units && live; unit += gridDim.x) {
            const int4 tile = next;
            if (unit + (int)gridDim.x < units) next = p.tiles[1 + (unit + gridDim.x) / p.chunks];
            const int chunk = unit % p.chunks, boxes = kByToken ? 0 : (tile.z + 31) / 32;
            for (int ks = 0; ks < p.ksteps; ++ks) {
                const uint32_t full = smem_u32(&ctl->full[stage]);
                if (!mbar_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort_flag, p.status)) { live = false; break; }
                const uint32_t at = ring + stage * stage_bytes;
                __syncwarp();
                expect_elect(full, boxes * 4096 + p.nb * kBox);
                for (int b = 0; b < p.nb; ++b) {
                    int x, y;
                    if (MODE == kUp) {
                        const int half = p.nb / 2;
                        x = (b < half ? 0 : p.s) + (chunk * half + (b < half ? b : b - half)) * 64;
                        y = ks * 64;
                    } else if (kMn) {
                        x = (chunk * p.nb + b) * 64;
                        y = ks * 64;
                    } else {
                        x = ks * 64;
                        y = (chunk * p.nb + b) * 64;
                    }
                    tma_load_3d_elect(at + kATile + b * kBox, &mw, full, x, y, tile.x);
                }
                for (int b = 0; b < boxes; ++b) tma_load_2d_elect(at + b * 4096, &ma, full, ks * 64, tile.y + b * 32);
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (kByToken && warp >= 10) {
        // Rows 16 i + 4 w .. + 3 of the tile for i = 0, 1, ... are warp w's: up to eight gathers a step.
        const int r0 = (warp - 10) * 4;
        int stage = 0;
        uint32_t phase = 0;
        bool live = true;
        const int r = (lane >> 2) * 16 + r0 + (lane & 3);
        TilesAhead ahead(p, units, r);
        for (int unit = blockIdx.x; unit < units && live; unit += gridDim.x) {
            const int gathers = (max(0, ahead.tile.z - r0) + 15) / 16;
            const int mine = ahead.pair < 0 || ahead.pair >= p.P ? p.rows : (int)((unsigned)ahead.pair / (unsigned)p.k);    // (no such row: out of bounds, zeros)
            int lo[16], hi[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                lo[i] = __shfl_sync(0xffffffffu, mine, i);
                hi[i] = __shfl_sync(0xffffffffu, mine, 16 + i);
            }
            ahead.next(unit);
            for (int ks = 0; ks < p.ksteps; ++ks) {
                const uint32_t full = smem_u32(&ctl->full[stage]);
                if (!mbar_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort_flag, p.status)) { live = false; break; }
                const uint32_t at = ring + stage * stage_bytes + r0 * 128;
                __syncwarp();
                expect_elect(full, gathers * 512);
                tma_gather4x4(at, 2048, &ma, full, ks * 64, gathers, lo);
                if (gathers > 4) tma_gather4x4(at + 8192, 2048, &ma, full, ks * 64, gathers - 4, hi);
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
    } else if (warp < 10) {
        // Two steps per pass: the warps that have rows copy columns of the accumulator into staging, thread by row; then all
        // eight work along rows, so that memory is read and written in whole lines and a tile of few rows occupies them all.
        const int quarter = warp & 3, side = warp >= 6;             // lane quarter of the accumulator; half of the columns
        const int r0 = quarter * 32, row = r0 + lane;               // this warp's first row of a tile, this thread's
        const int tid = threadIdx.x - 64;
        constexpr int kPitch = MODE == kUp || MODE == kBackAct ? (MODE == kUp ? 512 : 256) : 512;
        int it = 0;
        TilesAhead ahead(p, units, row);
        for (int unit = blockIdx.x; unit < units; unit += gridDim.x, ++it) {
            const int4 tile = ahead.tile;
            const int chunk = unit % p.chunks, buf = it & 1;
            const int my_pair = ahead.pair < p.P ? ahead.pair : -1;
            if constexpr (MODE != kUp)
                if (side == 0) ctl->pair[row] = my_pair;            // (read behind the first barrier below)
            ahead.next(unit);
            const uint32_t acc = tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16);
            // after a wait that gave up the loop goes on without work: no warp is left alone at a barrier
            uint4 kept[4][2];                                       // kBackAct: both projections of this thread's first items
            if constexpr (MODE == kBackAct) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = (i * 256 + tid) >> 3, col = chunk * p.nb * 64 + (tid & 7) * 8;
                    if (r < tile.z && col < p.s) {
                        const __nv_bfloat16* from = p.hidden + (long long)(tile.y + r) * 2 * p.s + col;
                        kept[i][0] = *reinterpret_cast<const uint4*>(from);
                        kept[i][1] = *reinterpret_cast<const uint4*>(from + p.s);
                    }
                }
            }
            const bool ok = mbar_wait(smem_u32(&ctl->acc_full[buf]), (it >> 1) & 1, abort_flag, p.status);
            tc_fence_after();
            const int rows = ok ? tile.z : 0;
            const bool any = r0 < rows;                             // (a warp whose rows are all behind the tile copies nothing)
            auto release = [&]() {
                tc_fence_before();
                warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);
            };
            if constexpr (MODE == kUp) {
                const int cols = p.nb * 32, passes = (min(cols, p.s - chunk * cols) + 63) / 64;
                for (int pass = 0; pass < passes; ++pass) {
                    if (any) {                                      // 64 gate columns, then the 64 others: one half of each per warp
                        float v[4][16];
#pragma unroll
                        for (int i = 0; i < 4; ++i) tmem_ld16(acc + (i >= 2 ? cols : 0) + pass * 64 + side * 32 + (i & 1) * 16, v[i]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            tmem_ld_wait16(v[i]);
                            stage_f32(staging, kPitch, row, (i >= 2 ? 16 : 0) + side * 8 + (i & 1) * 4, v[i]);
                        }
                    }
                    if (pass == passes - 1) release();
                    epilogue_sync();
                    const int s0 = chunk * cols + pass * 64 + (tid & 7) * 8;
                    for (int r = tid >> 3; r < rows; r += 32) {
                        if (s0 >= p.s) continue;
                        float g[8], u[8], a[8];
                        unstage8(staging, kPitch, r, (tid & 7) * 2, g);
                        unstage8(staging, kPitch, r, 16 + (tid & 7) * 2, u);
#pragma unroll
                        for (int i = 0; i < 8; ++i) a[i] = g[i] * sigmoidf(g[i]) * u[i];
                        const long long place = tile.y + r;
                        *reinterpret_cast<uint4*>(p.out + place * p.s + s0) = pack8(a);
                        if (p.hidden) {
                            *reinterpret_cast<uint4*>(p.hidden + place * 2 * p.s + s0) = pack8(g);
                            *reinterpret_cast<uint4*>(p.hidden + place * 2 * p.s + p.s + s0) = pack8(u);
                        }
                    }
                    epilogue_sync();
                }
            } else if constexpr (MODE == kBackAct) {
                const int width = p.nb * 64, passes = (min(width, p.s - chunk * width) + 63) / 64;
                float dg[4] = {0.f, 0.f, 0.f, 0.f};
                for (int pass = 0; pass < passes; ++pass) {
                    if (any) {
                        float v[2][16];
#pragma unroll
                        for (int i = 0; i < 2; ++i) tmem_ld16(acc + pass * 64 + side * 32 + i * 16, v[i]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            tmem_ld_wait16(v[i]);
                            stage_f32(staging, kPitch, row, side * 8 + i * 4, v[i]);
                        }
                    }
                    if (pass == passes - 1) release();
                    epilogue_sync();
                    const int s0 = chunk * width + pass * 64 + (tid & 7) * 8;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = (i * 256 + tid) >> 3;
                        if (r >= rows || s0 >= p.s) continue;
                        const long long place = tile.y + r;
                        const __nv_bfloat16* from = p.hidden + place * 2 * p.s + s0;
                        const uint4 hg = pass == 0 ? kept[i][0] : *reinterpret_cast<const uint4*>(from);
                        const uint4 hu = pass == 0 ? kept[i][1] : *reinterpret_cast<const uint4*>(from + p.s);
                        const int pair = ctl->pair[r];
                        const float gate = pair >= 0 ? p.gate[pair] : 0.f;
                        const uint32_t wg[4] = {hg.x, hg.y, hg.z, hg.w}, wu[4] = {hu.x, hu.y, hu.z, hu.w};
                        float c[8], out_g[8], out_u[8], out_a[8];
                        unstage8(staging, kPitch, r, (tid & 7) * 2, c);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float g = j & 1 ? bf16_hi(wg[j / 2]) : bf16_lo(wg[j / 2]), up = j & 1 ? bf16_hi(wu[j / 2]) : bf16_lo(wu[j / 2]);
                            const float sg = sigmoidf(g), silu = g * sg, act = silu * up, da = gate * c[j];
                            dg[i] = fmaf(c[j], act, dg[i]);
                            out_a[j] = gate * act;
                            out_u[j] = da * silu;
                            out_g[j] = da * up * fmaf(silu, 1.f - sg, sg);
                        }
                        *reinterpret_cast<uint4*>(p.du + place * 2 * p.s + s0) = pack8(out_g);
                        *reinterpret_cast<uint4*>(p.du + place * 2 * p.s + p.s + s0) = pack8(out_u);
                        if (p.ga) *reinterpret_cast<uint4*>(p.ga + place * p.s + s0) = pack8(out_a);
                    }
                    epilogue_sync();
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {                       // the eight threads of a row
                    const int r = (i * 256 + tid) >> 3;
#pragma unroll
                    for (int o = 4; o > 0; o >>= 1) dg[i] += __shfl_xor_sync(0xffffffffu, dg[i], o);
                    const int pair = r < rows ? ctl->pair[r] : -1;
                    if ((tid & 7) == 0 && pair >= 0) p.dgate_part[(long long)chunk * p.P + pair] = dg[i];
                }
                epilogue_sync();                                    // (the pairs are read)
            } else {
                const int per = p.nb * 32, c0 = chunk * p.nb * 64;
                if (any) {
                    float up = 1.f;
                    if constexpr (MODE == kBackX) {
                        // The rows of the slots are added later: each `per` (128, where h > 128) columns of a row are kept in fp16
                        // behind a power of two that brings their largest to [2^14, 2^15): an eighth of bf16's rounding for the
                        // same bytes.
                        float top = 0.f;
                        for (int c = 0; c < per && c0 + side * per + c < p.h; c += 32) {
                            float v0[16], v1[16];
                            tmem_ld16(acc + side * per + c, v0);
                            tmem_ld16(acc + side * per + c + 16, v1);
                            tmem_ld_wait16(v0); tmem_ld_wait16(v1);
#pragma unroll
                            for (int i = 0; i < 16; ++i) top = max3(top, fabsf(v0[i]), fabsf(v1[i]));
                        }
                        const int ex = max(15, __float_as_int(top) >> 23);
                        up = ex < 255 ? __int_as_float((268 - ex) << 23) : 1.f;
                        const float down = ex < 255 ? __int_as_float((ex - 14) << 23) : 1.f;
                        if (my_pair >= 0 && c0 + side * per < p.h) p.dx_scale[(long long)my_pair * p.dx_groups + c0 / per + side] = down;
                    }
                    for (int c = 0; c < per && c0 + side * per + c < p.h; c += 32) {
                        float v[2][16];
#pragma unroll
                        for (int i = 0; i < 2; ++i) tmem_ld16(acc + side * per + c + i * 16, v[i]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            tmem_ld_wait16(v[i]);
                            const int piece = (side * per + c + i * 16) / 8;
                            if constexpr (MODE == kDown) {
                                stage_bf16(staging, kPitch, row, piece, v[i]);
                            } else {
                                uint32_t w[8];
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    const __half2 q = __floats2half2_rn(v[i][2 * j] * up, v[i][2 * j + 1] * up);
                                    w[j] = *reinterpret_cast<const uint32_t*>(&q);
                                }
                                st_piece(staged(staging, kPitch, row, piece), w[0], w[1], w[2], w[3]);
                                st_piece(staged(staging, kPitch, row, piece + 1), w[4], w[5], w[6], w[7]);
                            }
                        }
                    }
                }
                release();
                epilogue_sync();
                // a warp per row: up to 512 consecutive bytes
                uint16_t* out = MODE == kDown ? reinterpret_cast<uint16_t*>(p.out) : reinterpret_cast<uint16_t*>(p.dx);
                const bool in = lane < p.nb * 8 && c0 + lane * 8 < p.h;
#pragma unroll 4
                for (int r = warp - 2; r < rows; r += 8) {
                    const int pair = ctl->pair[r];
                    const uint4 v = ld_piece(staged(staging, kPitch, r, lane));
                    if (pair >= 0 && in) *reinterpret_cast<uint4*>(out + (long long)pair * p.h + c0 + lane * 8) = v;
                }
                epilogue_sync();
            }
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

// The runs of a CTA's units in turn, the next one's bounds requested while the present one is worked on.
struct Units {
    const WeightsParams& p;
    uint32_t per_expert, units, unit;
    int e, rem;                   // of the present unit: expert, which of the expert's units
    int lo, n;                    // its run
    int next_e, next_rem, raw_lo, raw_hi;
    __device__ explicit Units(const WeightsParams& q) : p(q), per_expert(q.mtiles * q.chunks), units((uint32_t)q.M * per_expert), unit(blockIdx.x)
    {
        request();
        take();
    }
    __device__ void request()                               // (of the unit that `unit` names)
    {
        if (unit >= units) return;
        next_e = (int)(unit / per_expert);
        next_rem = (int)(unit - (uint32_t)next_e * per_expert);
        raw_lo = p.offsets[next_e];
        raw_hi = p.offsets[next_e + 1];
    }
    __device__ void take()                                  // (whatever the offsets hold, a run stays within the places)
    {
        e = next_e;
        rem = next_rem;
        lo = min(max(raw_lo, 0), p.P);
        n = max(min(raw_hi, p.P) - lo, 0);
        unit += gridDim.x;
        request();
    }
    __device__ bool more() const { return unit - gridDim.x < units; }
    __device__ void next() { take(); }
    __device__ int mtile() const { return p.chunks == 1 ? rem : rem / p.chunks; }
    __device__ int chunk() const { return p.chunks == 1 ? 0 : rem % p.chunks; }
};

__global__ void __launch_bounds__(kXGatherThreads, 1)
weights_kernel(const __grid_constant__ CUtensorMap mtoken, const __grid_constant__ CUtensorMap mplace, const __grid_constant__ CUtensorMap mplace16,
               const __grid_constant__ WeightsParams p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, staging = ring + kXRing;
    Control* ctl = reinterpret_cast<Control*>(smem_raw + (ring - smem_u32(smem_raw)) + kXRing + kXStaging);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = open_cta(ctl, p.stages, kGatherWarps, warp);
    volatile int* abort_flag = &ctl->abort;
    const uint32_t stage_bytes = (2 + p.nb) * kBox;

    if (warp >= 10) {
        // Each of these warps loads 16 of a step's 64 rows, one K-step of the MMAs, of both operands: rows by token by gathers,
        // consecutive places in one piece.  Rows behind the run's last are out of bounds, zeros: of the places, too, only then
        // row by row (what lies there belongs to another expert).
        const int part = warp - 10;
        int stage = 0;
        uint32_t phase = 0;
        bool live = true;
        Units u(p);
        while (u.more() && u.n == 0) u.next();
        int at = 0, next_pair = -1;
        auto fetch = [&]() {
            const int r = at + part * 16 + (lane & 15);
            next_pair = u.more() && r < u.n ? p.pairs[u.lo + r] : -1;
        };
        fetch();
        while (u.more() && live) {
            const int lo = u.lo, mt = u.mtile(), chunk = u.chunk(), r0 = at + part * 16, rows = min(16, u.n - r0);
            const int a_boxes = p.rows - mt * 128 > 64 ? 2 : 1;
            const bool in = next_pair >= 0 && next_pair < p.P;
            const int mine = in ? (int)((unsigned)next_pair / (unsigned)p.k) : p.T;
            const bool whole = __all_sync(0xffffffffu, in);
            int token[16], place[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                token[i] = __shfl_sync(0xffffffffu, mine, i);
                place[i] = token[i] == p.T ? p.P : lo + r0 + i;
            }
            at += 64;
            if (at >= u.n) {
                at = 0;
                do u.next(); while (u.more() && u.n == 0);
            }
            fetch();
            const uint32_t full = smem_u32(&ctl->full[stage]);
            if (!mbar_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort_flag, p.status)) { live = false; break; }
            const uint32_t base = ring + stage * stage_bytes + part * 2048;
            __syncwarp();
            expect_elect(full, rows > 0 ? 2048 * (a_boxes + p.nb) : 0);
            if (rows > 0) {
                const int a_x = mt * 128, b_x = chunk * p.nb * 64;
                const uint32_t a_at = base, b_at = base + 2 * kBox;
                const int t_boxes = p.a_by_token ? a_boxes : p.nb, p_boxes = p.a_by_token ? p.nb : a_boxes;
                const int t_x = p.a_by_token ? a_x : b_x, p_x = p.a_by_token ? b_x : a_x;
                const uint32_t t_at = p.a_by_token ? a_at : b_at, p_at = p.a_by_token ? b_at : a_at;
                for (int b = 0; b < t_boxes; ++b) tma_gather4x4(t_at + b * kBox, 512, &mtoken, full, t_x + b * 64, 4, token);
                for (int b = 0; b < p_boxes; ++b) {
                    if (whole) tma_load_2d_elect(p_at + b * kBox, &mplace16, full, p_x + b * 64, lo + r0);
                    else tma_gather4x4(p_at + b * kBox, 512, &mplace, full, p_x + b * 64, 4, place);
                }
            }
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == 1) {
        const uint32_t idesc = idesc_of(p.nb * 64, 1, 1);
        const uint64_t a0 = umma_desc_sw128(ring, kBox, 1024), b0 = umma_desc_sw128(ring + 2 * kBox, kBox, 1024);
        const uint32_t a_hi = (uint32_t)(a0 >> 32), b_hi = (uint32_t)(b0 >> 32);
        int stage = 0, it = 0;
        uint32_t phase = 0;
        bool live = true;
        for (Units u(p); u.more() && live; u.next()) {
            const int n = u.n;
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
    } else if (warp >= 2) {
        const int quarter = warp & 3, side = warp >= 6, row = quarter * 32 + lane;
        int it = 0;
        for (Units w(p); w.more(); w.next()) {
            const int mt = w.mtile(), per = p.nb * 32, c0 = w.chunk() * p.nb * 64;
            const int rows = min(128, p.rows - mt * 128);
            __nv_bfloat16* out = p.out + ((long long)w.e * p.rows + mt * 128) * p.cols + c0;
            const bool some = w.n > 0;
            bool ok = true;
            if (some) {
                const int buf = it & 1;
                const uint32_t acc = tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16);
                ok = mbar_wait(smem_u32(&ctl->acc_full[buf]), (it >> 1) & 1, abort_flag, p.status);   // (given up: goes on without work)
                tc_fence_after();
                for (int c = 0; ok && c < per && quarter * 32 < rows && c0 + side * per + c < p.cols; c += 32) {
                    float v[2][16];
#pragma unroll
                    for (int i = 0; i < 2; ++i) tmem_ld16(acc + side * per + c + i * 16, v[i]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        tmem_ld_wait16(v[i]);
                        stage_bf16(staging, 512, row, (side * per + c + i * 16) / 8, v[i]);
                    }
                }
                tc_fence_before();
                warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);
                ++it;
                epilogue_sync();
            }
            // threads along rows: as many pieces of 16 bytes as a unit is wide, a power of two
            const int pieces = p.nb * 8, piece = (threadIdx.x - 64) & (pieces - 1), step = 256 / pieces;
            if (ok && c0 + piece * 8 < p.cols)
#pragma unroll 4
                for (int r = (threadIdx.x - 64) / pieces; r < rows; r += step) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (some) v = ld_piece(staged(staging, 512, r, piece));
                    *reinterpret_cast<uint4*>(out + (long long)r * p.cols + piece * 8) = v;
                }
            if (some) epilogue_sync();
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
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

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
        w.dgate = at; at += up256(P * 4 * chunks);
        w.dx = at; at += up256(P * h * 2);
        w.dx_scale = at; at += up256(P * 4 * ((h + g - 1) / g));
    }
    w.total = at;
    return w;
}

// 2-D [rows][cols]; for gathering loads the box is one row high.
int rows_map(const void* ptr, long long rows, int cols, int high, CUtensorMap* out)
{
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)cols * 2};
    const uint32_t box[2] = {64, (uint32_t)high};
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
    rows_kernel<MODE><<<grid, MODE == kUp || MODE == kBackAct ? kXGatherThreads : kXThreads, kXSmem, st>>>(ma, mw, p);
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

int launch_weights(const CUtensorMap& mtoken, const CUtensorMap& mplace, const CUtensorMap& mplace16, WeightsParams p, const DeviceCtx& ctx, cudaStream_t st)
{
    if (allow_smem(weights_kernel) != MORE_OK) return MORE_ERR_CUDA;
    p.nb = p.cols > 128 ? 4 : (p.cols > 64 ? 2 : 1);
    p.mtiles = (p.rows + 127) / 128;
    p.chunks = (p.cols + p.nb * 64 - 1) / (p.nb * 64);
    p.stages = kXRing / ((2 + p.nb) * kBox);
    if (p.stages > kXMaxStages) p.stages = kXMaxStages;
    p.status = ctx.status;
    const long long units = (long long)p.M * p.mtiles * p.chunks;
    if (units > 0x7fffffffLL) return MORE_ERR_TOO_LARGE;
    const int grid = units < ctx.sm_count ? (int)units : ctx.sm_count;
    weights_kernel<<<grid, kXGatherThreads, kXSmem, st>>>(mtoken, mplace, mplace16, p);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

int launch_experts(const ExpertsArgs& a, const DeviceCtx& ctx)
{
    const long long P = (long long)a.T * a.k;
    const Workspace w = lay_out(a.T, a.h, a.s, a.M, a.k, false);
    char* base = static_cast<char*>(a.workspace);
    CUtensorMap mx, mact, m1, m2;
    int rc = rows_map(a.X, a.T, a.h, 1, &mx);
    if (rc == MORE_OK) rc = rows_map(base + w.act, P, a.s, 32, &mact);
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
    CUtensorMap mx, md, mdu[3], mga[2], m1, m2;             // by token; by place one row, 16 rows and 32 rows high; weights
    int rc = rows_map(a.X, a.T, a.h, 1, &mx);
    if (rc == MORE_OK) rc = rows_map(a.dout, a.T, a.h, 1, &md);
    for (int i = 0; i < 3 && rc == MORE_OK; ++i) rc = rows_map(base + w.du, P, 2 * a.s, i == 0 ? 1 : 8 << i, &mdu[i]);
    for (int i = 0; i < 2 && rc == MORE_OK; ++i) rc = rows_map(base + w.ga, P, a.s, i == 0 ? 1 : 16, &mga[i]);
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
    const int parts = p.chunks;
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
        rc = launch_rows<kBackX>(mdu[2], m1, p, tiles, ctx, a.stream);
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
        rc = launch_weights(mx, mdu[0], mdu[1], q, ctx, a.stream);
        if (rc != MORE_OK) return rc;
    }
    if (a.out_dw2) {
        q.a_by_token = 0; q.rows = a.s; q.cols = a.h; q.out = a.out_dw2;
        rc = launch_weights(md, mga[0], mga[1], q, ctx, a.stream);
    }
    return rc;
}

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
