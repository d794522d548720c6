// The experts' gated feed-forward blocks behind the router (the layer's expert products, "scatter2scatter, SwiGLU,
// scatter2scatter" in the paper's forward flowchart), forward and backward, over the (token, slot) pairs of a routing:
//
//   u = X[token] W1[e],  a = silu(u_gate) u_up,  Y[pair] = a W2[e]            e = expert of the pair
//   c = d[token] W2[e]^T,  dgate = <c, a>,  du = gate c (silu'(u_gate) u_up, silu(u_gate)),  dX = sum over slots of du W1[e]^T
//   dW1[e] = sum of X[token]^T du,  dW2[e] = sum of (gate a)^T d[token]
//
// Two kernels do all of it, both persistent with one CTA per SM: warps that load, a warp that issues the tcgen05 MMAs, and eight warps
// behind the accumulators (two of 256 tensor-memory columns, used in turn, so that the products of the next unit run meanwhile).  All
// eight read them where values are worked on (kUp, kBackAct) and in weights_kernel; where rows are only rounded (kDown, kBackX) four
// read them and four write the rows out.
//
//   rows_kernel<MODE>   tiles of up to 128 pairs of one expert against its weights.  W1 and W2 come by TMA and are used as they are
//                       stored, the forward products with them as MN-major operands, the backward ones as K-major ones: nothing
//                       is transposed.
//   weights_kernel      dW of one expert: 128 x 256 outputs, contracted over the expert's pairs 64 at a time, both operands
//                       MN-major.
//
// Rows that are anywhere in X or d come by gathering TMA loads, four rows of 128 bytes each, in the swizzled layout that the MMAs read.
// One costs the warp that issues it 100 to 200 clocks, so several warps share them.  (Asynchronous 16-byte copies by threads were
// slower: 144 us against 105 for the first product of 16384 x 8 pairs, h = 512, 4096 experts of s = 64.)
//
// What bounds them: with the paper's narrow experts, the bytes: each expert's weights are read once (six bytes per h s) for as
// few as 30 tokens.  A stage of the ring in shared memory is as long as what it holds, so that tiles of few rows have more
// weights in flight, and gradients of weights leave shared memory by TMA stores that nobody waits for.  The activation goes
// to the second product as bf16 rows in expert order (s of them against h of an output row).  Measured (DRAM bytes and time of one
// launch, cold): 16384 x 8 pairs of 4096 experts, h = 512, s = 64: kUp 560 MB in 97 us, kDown 360 MB in 72 us; 32768 x 4 of the same:
// kBackAct 363 MB in 85 us, kBackX 688 MB in 115 us, the gradients of both weights 872 MB in 193 us, where issuing loads and passing
// tiles through shared memory take as long as an SM's stores.  Few wide experts are bound by what the SMs read from L2: 32768 x 8
// pairs of 256 experts, h = 512, s = 256, kUp 160 us, of which the MMAs alone take 82 and the gathers alone 150 (about 10 clocks per
// row of 128 bytes), kDown 103 us.  Times of whole calls in these comments compare variants in calls one after the other, whose last
// writes stay in L2; with that overwritten in front of each call the long ones take 4 to 12 % more (65536 x 4 pairs of 8192 experts,
// backward: 825 us and 896 to 925).
#include "more_experts.cuh"

#include <math.h>

namespace more {

namespace {

// Warp 1 issues the MMAs, warps 2..9 are the epilogue, warp 0 and those from 10 on load: stage n is the (n mod loaders)th one's, as
// opening a stage and issuing its loads costs a warp 700 to 3000 clocks, several times what a stage may take.  In the forward gather
// two warps share a stage, and it is there sooner: 58 us instead of 62 for 3001 x 6 pairs of 504 experts, h = 1000, s = 40, 265
// instead of 279 for 32768 x 8 of 256, h = 512, s = 256, nothing lost elsewhere.  (The backward one was 20 to 50 us slower for
// 65536 x 4 of 8192, whose stages are small: every loader goes through all stages' places.  Seven loaders there, and for the weights'
// gradients: 500 us instead of 510 with five for the backward pass of 8192 x 4 pairs of 64 experts, h = 4096, s = 256.)
constexpr int kTeams = 5, kTeam = 2;                 // kUp: stages are taken by teams of two
constexpr int kBackLoaders = 7, kFewLoaders = 3;     // where rows are gathered on the way back; where none are
constexpr int threads_of(int loaders) { return (9 + loaders) * 32; }
__host__ __device__ constexpr int team_of(int mode) { return mode == 0 /* kUp */ ? kTeam : 1; }
__host__ __device__ constexpr int takers_of(int mode) { return mode == 0 ? kTeams : mode == 2 /* kBackAct */ ? kBackLoaders : kFewLoaders; }
constexpr int rows_threads(int mode) { return threads_of(takers_of(mode) * team_of(mode)); }
__device__ __forceinline__ int loader_of(int warp) { return warp == 0 ? 0 : warp - 9; }
constexpr int kTileRows = 128;
constexpr int kBox = 64 * 128;                       // 64 rows of 64 bf16
constexpr int kRowPitch = 528;                       // a staged output row: 256 16-bit values, and 16 bytes so that rows fall on other banks
constexpr int kXStaging = kTileRows * kRowPitch;     // what the epilogue passes from the tensor memory's layout to memory's
constexpr int kXRing = 153 * 1024;
constexpr int kXControl = 1536 + kTeams * kTeam * 512;
constexpr int kXSmem = kXRing + kXStaging + 1024 /*alignment*/ + kXControl;
static_assert(kXSmem <= 227 * 1024, "shared memory");
static_assert(kXStaging >= kTileRows * 128, "an operand of fewer rows than the MMA's 128 is read past its end");
constexpr int kSlots = 16;                           // stages in flight at most
// kBackAct adds up this many steps (512 columns) in the tensor memory, whose sums are truncated at every 16 columns, and those sums in
// rounding registers: the gate gradients, which leave in 32 bits, were 4.6e-6 off relative to their size at h = 4096, 4e-6 of it a
// bias towards zero, in one piece, and are as good as at h = 512, 4.7e-7, in pieces.
constexpr int kSumSteps = 8;

// Gradients of weights add up a run of pairs in pieces of this many, for the same reason: in one piece a run comes out too small by up to
// n / 16 x 2/3 x 2^-24, and 524288 pairs of one expert did by 5.2e-4 (an eighth of bf16's half step, growing with the run); in pieces
// it is 2e-5 at most, at any length.  And what waits for an accumulator waits for a piece, well inside its budget: a run of 4e8 pairs in
// one piece took longer than that.  One expert, h = 512, s = 64, 65536 pairs: the backward pass 1223 us with one piece, 1243 with eight.
constexpr int kRunPiece = 8192;
static_assert(MORE_PAIRS_MAX <= 0x7fffffff - kRunPiece, "places are counted in 32 bits");

enum { kUp = 0, kDown = 1, kBackAct = 2, kBackX = 3 };

// Loads as a converged warp issues them: every lane passes the same operands and elect.sync picks the lane that issues.  (The
// instructions take their operands from uniform registers; behind a branch that one lane takes each costs ~150 clocks to issue.)
// What passes once (weights, their gradients) leaves the L2 cache first, rows by token, which k experts read at different times, last.
__device__ __forceinline__ uint64_t passes_once()
{
    uint64_t h;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(h));
    return h;
}
__device__ __forceinline__ uint64_t comes_normally()
{
    uint64_t h;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(h));
    return h;
}
__device__ __forceinline__ uint64_t comes_again()
{
    uint64_t h;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(h));
    return h;
}
__device__ __forceinline__ void tma_load_2d_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
        "@pe cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, uint64_t hint)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
        "@pe cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(hint)
        : "memory");
}
__device__ __forceinline__ void expect_elect(uint32_t bar, uint32_t bytes)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
        "@pe mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes) : "memory");
}
// Up to four gathers of four rows each, 512 bytes of shared memory apart, as many as `count` says.
__device__ __forceinline__ void tma_gather16(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int count, int4 a, int4 b, int4 c, int4 d,
                                            uint64_t hint)
{
    asm volatile(
        "{\n\t.reg .pred pe, p0, p1, p2, p3;\n\t.reg .b32 d1, d2, d3;\n\t"
        "elect.sync _|pe, 0xffffffff;\n\t"
        "setp.gt.and.s32 p0, %4, 0, pe;\n\tsetp.gt.and.s32 p1, %4, 1, pe;\n\tsetp.gt.and.s32 p2, %4, 2, pe;\n\tsetp.gt.and.s32 p3, %4, 3, pe;\n\t"
        "add.u32 d1, %0, 512;\n\tadd.u32 d2, %0, 1024;\n\tadd.u32 d3, %0, 1536;\n\t"
        "@p0 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %5, %6, %7, %8}], [%2], %21;\n\t"
        "@p1 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint [d1], [%1, {%3, %9, %10, %11, %12}], [%2], %21;\n\t"
        "@p2 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint [d2], [%1, {%3, %13, %14, %15, %16}], [%2], %21;\n\t"
        "@p3 cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint [d3], [%1, {%3, %17, %18, %19, %20}], [%2], %21;\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(count), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w),
          "r"(c.x), "r"(c.y), "r"(c.z), "r"(c.w), "r"(d.x), "r"(d.y), "r"(d.z), "r"(d.w), "l"(hint)
        : "memory");
}
// Stores that read shared memory by themselves; a warp issues, commits and waits for its own.
__device__ __forceinline__ void tma_store_3d_elect(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2, uint64_t hint)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
        "@pe cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group.L2::cache_hint [%0, {%2, %3, %4}], [%1], %5;\n\t}"
        ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2), "l"(hint) : "memory");
}
// (every lane, so that it is the issuing one's groups that are meant, whichever that is)
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void bulk_read_done() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }   // all but the last N have read
__device__ __forceinline__ void bulk_all_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// Instruction descriptor of umma_idesc with the operands' majors: fp32 += bf16 x bf16, 128 rows, n columns.
__device__ __forceinline__ uint32_t idesc_of(int n, int a_mn, int b_mn)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(128 >> 4) << 24);
}
// A value requested ahead: what is computed from it stays behind this point (otherwise it is computed, and waited for, at once).
__device__ __forceinline__ int hold(int v)
{
    asm volatile("" : "+r"(v));
    return v;
}

struct Control {
    uint64_t full[kSlots], empty[kSlots], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort;
    int pair[kTileRows];
    float gate[kTileRows];
    int4 rows[kTeams * kTeam][kTileRows / 4];   // of each loader's tile
};
static_assert(sizeof(Control) <= kXControl && kBackLoaders <= kTeams * kTeam, "control block");
static_assert(kTeams < kSlots && kBackLoaders < kSlots && kFewLoaders < kSlots, "Ring::wait_empty");

// The ring of stages, each as long as what it holds (a multiple of 1024 bytes).  Every loader, and the warp that empties it, goes
// through the same sequence of lengths and so knows where each stage lies.
struct Ring {
    uint32_t head = 0;                    // next free byte
    uint32_t end = 0;                     // bytes of all stages so far, gaps at the ring's end included
    int n = 0;                            // stages so far
    uint32_t begun = 0;                   // lane i < 16: `end` at which the last stage of slot i began
    int empty = -1;                       // a loader: the last stage that it knows to be empty, and with it all before
    // Where the next stage of that length lies; `from`: the value of `end` in front of it.
    __device__ uint32_t place(uint32_t bytes, uint32_t* from)
    {
        const bool wraps = head + bytes > (uint32_t)kXRing;
        const uint32_t at = wraps ? 0u : head;
        *from = end;
        end += bytes + (wraps ? (uint32_t)kXRing - head : 0u);
        head = at + bytes;
        return at;
    }
    // A loader's view of the next stage: true if it is its own.  *at: where it lies; *last: the stage that has to be empty before it is
    // written, or less than 0.
    __device__ bool mine(uint32_t bytes, int loader, int loaders, int lane, uint32_t* at, int* last)
    {
        uint32_t from;
        *at = place(bytes, &from);
        const bool own = n % loaders == loader;
        if (own) {
            // Of the last 16 stages those that began more than a ring's length before this one's end have to be empty, and the
            // one whose slot this is (a slot that had none yet counts as one of long ago); they are emptied in order.
            const unsigned old = __ballot_sync(0xffffffffu, lane < kSlots && (lane >= n || lane == n % kSlots || (int)(end - (uint32_t)kXRing - begun) > 0));
            *last = n - kSlots + __popc(old) - 1;
        }
        if (lane == n % kSlots) begun = from;
        return own;
    }
    // Waits until stage `last` is empty (see mine), for a loader that is to write `stage`.  A barrier tells a phase from the one after the
    // next by nothing, and a wait for stage m is one for m's phase only if the stage before m in its slot is known to be empty and the
    // one behind m cannot be.  For `last` >= stage - 16 the latter holds, as what comes behind `stage` is not emptied before it.  For the
    // former the loader may first have to wait for stage - 16, of its own slot: of that one the stage before is known to be empty (the loader's
    // stage before this one was at most 15 back, and it waited for one at most 16 before that) and the one behind is `stage` itself.
    // (Needed where few long stages follow many short ones.  Without it stages in use were written over, and a launch over 62478 x 6
    // pairs of 16083 experts, h = 432, s = 24, gave up its waits where units of dW2 follow those of dW1.)  False: the CTA is giving up.
    __device__ bool wait_empty(int stage, int last, Control* c, volatile int* abort_flag, int* status)
    {
        if (last < 0) return true;
        if (last - kSlots > empty && !wait_for(stage - kSlots, c, abort_flag, status)) return false;
        empty = last;
        return wait_for(last, c, abort_flag, status);
    }
    __device__ static bool wait_for(int stage, Control* c, volatile int* abort_flag, int* status)
    {
        return mbar_wait_warp(smem_u32(&c->empty[stage % kSlots]), (uint32_t)(stage / kSlots) & 1u, abort_flag, status);
    }
    // The same as mine, and waits until it may be written.  (*live: false if the CTA is giving up.)
    __device__ bool open(uint32_t bytes, int loader, int loaders, Control* c, int lane, volatile int* abort_flag, int* status, uint32_t* at, bool* live)
    {
        int last;
        if (!mine(bytes, loader, loaders, lane, at, &last)) return false;
        if (!wait_empty(n, last, c, abort_flag, status)) *live = false;
        __syncwarp();
        return *live;
    }
    __device__ int slot() const { return n % kSlots; }
    __device__ uint32_t parity() const { return (uint32_t)(n / kSlots) & 1u; }
};

// ------------------------------------------------------------------------------------------------ tiles
// One entry per tile of up to 128 consecutive places of one expert: (expert, first place, places, 0), experts ascending.
// tiles[0].x is how many there are.  Every CTA takes 1024 experts and counts the tiles of all experts before them itself.
__global__ void __launch_bounds__(1024) tiles_kernel(const int32_t* __restrict__ offsets, int M, int P, int capacity, int4* __restrict__ tiles)
{
    let_next_begin();
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
    int others = warp_before[lane] + (lane < warp ? warp_sum[lane] : 0);
    for (int o = 16; o > 0; o >>= 1) others += __shfl_xor_sync(0xffffffffu, others, o);
    const int at = others + incl - mine;
    for (int i = 0; i < mine && at + i < capacity; ++i)
        tiles[1 + at + i] = make_int4(e, lo + i * kTileRows, min(kTileRows, n - i * kTileRows), 0);
    if (e == M - 1) tiles[0].x = min(at + mine, capacity);
}

// Barrier of the eight epilogue warps.
__device__ __forceinline__ void epilogue_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
// Four of them hand two buffers to the other four and back: barriers 2, 3: a buffer is full; 4, 5: it is free again.
__device__ __forceinline__ void hand_over(int barrier) { asm volatile("bar.arrive %0, 256;" ::"r"(barrier) : "memory"); }
__device__ __forceinline__ void take_over(int barrier) { asm volatile("bar.sync %0, 256;" ::"r"(barrier) : "memory"); }

__device__ __forceinline__ void st_piece(uint32_t at, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// (Not volatile: several may be in flight.  The barriers around them keep them in their place.)
__device__ __forceinline__ uint4 ld_piece(const uint8_t* at) { return *reinterpret_cast<const uint4*>(at); }
// Rows of staging (of kPrivatePitch bytes, written by this warp's threads) to memory, 16 bytes a thread, `pieces` (4 or 8) a row; dst: of
// row 0, ld: from row to row; limit: columns to write.
constexpr int kPrivatePitch = 144;                   // 64 16-bit values, and 16 bytes so that rows fall on other banks
static_assert(8 * 32 * kPrivatePitch <= kXStaging, "staging");
__device__ __forceinline__ void write_rows(const uint8_t* from, int pieces, int lane, int rows, int limit, __nv_bfloat16* dst, int ld)
{
    __syncwarp();
    const int piece = lane & (pieces - 1), first = lane / pieces, step = 32 / pieces;
    const bool in = piece * 8 < limit;
    for (int r = first; r - first < rows; r += 4 * step) {          // (four loads, then four stores)
        uint4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ld_piece(from + ((r + i * step) & 31) * kPrivatePitch + piece * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (in && r + i * step < rows) *reinterpret_cast<uint4*>(dst + (long long)(r + i * step) * ld + piece * 8) = v[i];
    }
    __syncwarp();
}
// Rows of `pitch` bytes, a power of two; the 16-byte pieces of a row are permuted by the row's number, so that neither a warp that
// writes a piece of 32 rows nor one that reads along a row meets itself on a bank (pitch 128: the layout of a TMA box).
__device__ __forceinline__ uint32_t staged(uint32_t base, int pitch, int row, int piece) { return base + row * pitch + ((piece ^ (row & 7)) << 4); }
__device__ __forceinline__ void stage_f32(uint32_t base, int pitch, int row, int piece, const float (&v)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        st_piece(staged(base, pitch, row, piece + i), make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                                                 __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])));
}
__device__ __forceinline__ void add_staged(const uint8_t* base, int pitch, int row, int piece, float (&v)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 a = *reinterpret_cast<const float4*>(base + staged(0, pitch, row, piece + i));
        v[4 * i] += a.x; v[4 * i + 1] += a.y; v[4 * i + 2] += a.z; v[4 * i + 3] += a.w;
    }
}
__device__ __forceinline__ void unstage8(const uint8_t* base, int pitch, int row, int piece, float (&v)[8])
{
    const uint4 a = ld_piece(base + staged(0, pitch, row, piece)), b = ld_piece(base + staged(0, pitch, row, piece + 1));
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
}
template <int N>
__device__ __forceinline__ uint4 pack8(const float (&v)[N], int at = 0)
{
    return make_uint4(pack_bf16(v[at], v[at + 1]), pack_bf16(v[at + 2], v[at + 3]), pack_bf16(v[at + 4], v[at + 5]), pack_bf16(v[at + 6], v[at + 7]));
}
__device__ __forceinline__ uint4 pack8_half(const float (&v)[16], int at, float scale)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 q = __floats2half2_rn(v[at + 2 * i] * scale, v[at + 2 * i + 1] * scale);
        w[i] = *reinterpret_cast<const uint32_t*>(&q);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Common start of both kernels: barriers, tensor memory.  loads: warps that share a stage; readers: those that read an accumulator.  Returns the tensor-memory base.
__device__ __forceinline__ uint32_t open_cta(Control* c, int loads, int readers, int warp)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(smem_u32(&c->full[i]), loads);
            mbar_init(smem_u32(&c->empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c->acc_full[i]), 1);
            mbar_init(smem_u32(&c->acc_empty[i]), readers);
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

// Division of 0 ... 2^31 - 1 by a small number: with 2^s >= d, m = ceil(2^(31 + s) / d) < 2^32, n / d = n m >> (31 + s) (the excess
// n (m d - 2^(31 + s)) / (d 2^(31 + s)) < 2^31 d / (d 2^(31 + s)) = 2^-s <= 1 / d is never enough to reach the next quotient).
struct Divide {
    uint32_t m;
    int shift;
    __host__ void by(int d)
    {
        int s = 0;
        while ((1 << s) < d) ++s;
        shift = 31 + s;
        m = (uint32_t)(((1ull << shift) + (unsigned)d - 1) / (unsigned)d);
    }
    __device__ int operator()(int n) const { return (int)((unsigned long long)(uint32_t)n * m >> shift); }
};

struct RowsParams {
    const int4* tiles;
    const int32_t* pairs;
    int P, h, s;
    Divide by_k;                  // pair -> token
    int rows;                     // of A's tensor: the row that is out of its bounds
    int nb;                       // boxes of 64 weight columns per unit
    int chunks;                   // units per tile
    int ksteps;                   // of 64
    int weights_once;             // most experts have a tile or two
    __nv_bfloat16* out;           // kUp: activation [P][s]; kDown: Y [P][h]
    __nv_bfloat16* hidden;        // kUp: nullable; kBackAct: read
    const float* gate;            // kBackAct
    __nv_bfloat16* du;            // kBackAct: [P][2s]
    __nv_bfloat16* ga;            // kBackAct: gate a, [P][s], nullable
    float* dgate_part;            // kBackAct: [chunks][P]
    __half* dx;                   // kBackX: [P][h] scaled
    uint8_t* dx_scale;            // kBackX: [P][dx_groups], a power of two per 32 columns, as fp32's exponent
    int dx_groups;
    int* status;
};

// The tiles of a CTA's units in turn, and the pairs in N places r, r + 32, ... of each, for a converged warp.  A warp's lanes hold the
// tiles of 32 units, the next 32 are requested when they begin; pairs are requested a unit ahead.  (What a unit is came from memory
// once per unit before, a wait of 400 to 1000 clocks for each warp: what the ring leaves of the L1 cache is next to nothing.)
template <int N>
struct TilesAhead {
    const RowsParams& p;
    int units, r, lane, index, ahead;
    int4 batch, next_batch;                                  // this lane's: expert, first place, places, chunk
    int4 coming;                                             // the unit after the present one
    int next_pair[N];
    int chunk, pair[N];
    int4 tile;
    __device__ TilesAhead(const RowsParams& q, int n, int row) : p(q), units(n), r(row), lane(threadIdx.x & 31), index(-1), ahead(0)
    {
        next_batch = request(0);
        turn();
        coming = of(0);
        ask_pairs();
        next();
    }
    __device__ int4 request(int first)                       // of units first ... first + 31 of this CTA
    {
        const long long u = blockIdx.x + (long long)(first + lane) * gridDim.x;
        if (u >= units) return make_int4(0, 0, 0, 0);
        int4 t = p.tiles[1 + (int)((unsigned)u / (unsigned)p.chunks)];
        t.w = (int)((unsigned)u % (unsigned)p.chunks);
        return t;
    }
    __device__ void turn()
    {
        batch = make_int4(hold(next_batch.x), hold(next_batch.y), hold(next_batch.z), hold(next_batch.w));
        next_batch = request(ahead + 32);
    }
    __device__ int4 of(int i) const
    {
        return make_int4(__shfl_sync(0xffffffffu, batch.x, i), __shfl_sync(0xffffffffu, batch.y, i), __shfl_sync(0xffffffffu, batch.z, i),
                         __shfl_sync(0xffffffffu, batch.w, i));
    }
    __device__ void ask_pairs()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) next_pair[i] = r + 32 * i < coming.z ? p.pairs[coming.y + r + 32 * i] : -1;
    }
    __device__ bool more() const { return (long long)blockIdx.x + (long long)index * gridDim.x < units; }
    __device__ void next()
    {
        ++index;
        tile = coming;
        chunk = coming.w;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            pair[i] = hold(next_pair[i]);
            if (pair[i] >= p.P) pair[i] = -1;
        }
        if ((++ahead & 31) == 0) turn();
        coming = of(ahead & 31);
        if constexpr (N > 0) ask_pairs();
    }
};

// Bytes of the rows of a tile, 64 columns, in a stage: gathered rows as many groups of eight as there are, others all 128 by boxes of 32.
template <bool GATHER>
__device__ __forceinline__ uint32_t row_bytes(int rows) { return GATHER ? (uint32_t)(rows + 7) / 8 * 1024 : 4u * 4096; }
// Those 128 are the rows of the tile once, or a tile of up to 64 twice, up to 32 four times: each lane quarter of the accumulator is
// read by warps of its own, which then share the columns.  How many of the four boxes differ:
__device__ __forceinline__ int unlike_boxes(int rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// Steps of 64 columns per stage, of `bytes` each.  The warp that issues the MMAs spends about 400 clocks on a stage, more than the 64
// columns of a small tile of kBackAct take to come: two of those make a stage (156 us instead of 170 for the activation's backward of
// 65536 x 4 pairs of 8192 experts, h = 512, s = 64; up to 24 KB gained no more there and cost 2 % on tiles of 128 rows; in kUp,
// whose weights weigh twice as much, it cost 2 %).
template <int MODE>
__device__ __forceinline__ int stage_steps(uint32_t bytes, int left) { return MODE == kBackAct && bytes <= 16 * 1024 && left > 1 ? 2 : 1; }

template <int MODE>
__global__ void __launch_bounds__(rows_threads(MODE), 1)
rows_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mw, const __grid_constant__ RowsParams p)
{
    constexpr bool kGather = MODE == kUp || MODE == kBackAct;       // rows of A are tokens', else places in expert order
    constexpr bool kMn = MODE == kUp || MODE == kDown;              // weights as an MN-major operand
    constexpr bool kCompute = kGather;                              // values are worked on behind the product, not only rounded
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, staging = ring + kXRing;
    uint8_t* const staging_at = smem_raw + (ring - smem_u32(smem_raw)) + kXRing;
    Control* ctl = reinterpret_cast<Control*>(staging_at + kXStaging);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    let_next_begin();
    const uint32_t tmem = open_cta(ctl, team_of(MODE), kCompute ? 8 : 4, warp);
    wait_for_previous();
    volatile int* abort_flag = &ctl->abort;
    const int units = p.tiles[0].x * p.chunks;

    if (warp == 0 || warp >= 10) {
        constexpr int kMine = takers_of(MODE), kMembers = team_of(MODE);
        const int loader = loader_of(warp) / kMembers, member = loader_of(warp) % kMembers;
        int4* rows = ctl->rows[loader_of(warp)];
        const uint64_t again = comes_again(), once = p.weights_once ? passes_once() : comes_normally();
        Ring rg;
        bool live = true;
        for (TilesAhead<kGather ? 4 : 0> u(p, units, lane); u.more() && live; u.next()) {
            const uint32_t a_bytes = row_bytes<kGather>(u.tile.z), bytes = a_bytes + p.nb * kBox;
            const int gathers = (u.tile.z + 3) / 4, unlike = unlike_boxes(u.tile.z);
            uint32_t share = 0;                                     // bytes of this warp's loads
            if constexpr (kGather) {
                for (int g = member * 4; g < gathers; g += 4 * kMembers) share += min(4, gathers - g) * 512;
                share += kMn ? p.nb / kMembers * kBox : member == 0 ? p.nb * kBox : 0;
            } else {
                share = bytes;
            }
            if constexpr (kGather) {
#pragma unroll
                for (int i = 0; i < 4; ++i)                         // (a row that does not exist is out of bounds: zeros)
                    reinterpret_cast<int*>(rows)[i * 32 + lane] = u.pair[i] < 0 ? p.rows : p.by_k(u.pair[i]);
                __syncwarp();
            }
            for (int ks = 0, steps; ks < p.ksteps && live; ks += steps, ++rg.n) {
                uint32_t at;
                steps = stage_steps<MODE>(bytes, p.ksteps - ks);
                if (!rg.open(steps * bytes, loader, kMine, ctl, lane, abort_flag, p.status, &at, &live)) continue;
                const uint32_t full = smem_u32(&ctl->full[rg.slot()]);
                at += ring;
                expect_elect(full, steps * share);
                for (int i = 0; i < steps; ++i, at += bytes) {
                    const int x_k = (ks + i) * 64;
                    if constexpr (kMn) {
                        for (int b = member; b < p.nb; b += kMembers) {
                            const int half = p.nb / 2;
                            const int x = MODE == kDown ? (u.chunk * p.nb + b) * 64 : (b < half ? 0 : p.s) + (u.chunk * half + (b < half ? b : b - half)) * 64;
                            tma_load_3d_elect(at + a_bytes + b * kBox, &mw, full, x, x_k, u.tile.x, once);
                        }
                    } else if (member == 0) {
                        tma_load_3d_elect(at + a_bytes, &mw, full, x_k, u.chunk * p.nb * 64, u.tile.x, once);
                    }
                    if constexpr (kGather) {
                        for (int g = member * 4; g < gathers; g += 4 * kMembers)
                            tma_gather16(at + g * 512, &ma, full, x_k, gathers - g, rows[g], rows[g + 1], rows[g + 2], rows[g + 3], again);
                    } else {
                        for (int b = 0; b < 4; ++b) tma_load_2d_elect(at + b * 4096, &ma, full, x_k, u.tile.y + (b & (unlike - 1)) * 32);
                    }
                }
            }
            __syncwarp();                                           // (the rows are read)
        }
    } else if (warp == 1) {
        const uint32_t idesc = idesc_of(p.nb * 64, 0, kMn);
        const uint64_t a0 = umma_desc_sw128(ring, 16, 1024), b0 = umma_desc_sw128(ring, kMn ? kBox : 16, 1024);
        const uint32_t a_hi = (uint32_t)(a0 >> 32), b_hi = (uint32_t)(b0 >> 32);
        constexpr uint32_t kBStep = kMn ? 2048 >> 4 : 32 >> 4;
        Ring rg;
        int it = 0;
        bool live = true;
        for (TilesAhead<0> u(p, units, 0); u.more() && live; u.next()) {
            const uint32_t a_bytes = row_bytes<kGather>(u.tile.z), bytes = a_bytes + p.nb * kBox;
            for (int ks = 0, steps; ks < p.ksteps; ks += steps) {
                steps = stage_steps<MODE>(bytes, p.ksteps - ks);
                const int in_block = MODE == kBackAct ? ks % kSumSteps : ks;
                const uint32_t d = tmem + (it & 1) * 256;
                if (in_block == 0) {
                    if (!mbar_wait_warp(smem_u32(&ctl->acc_empty[it & 1]), ((it >> 1) & 1) ^ 1u, abort_flag, p.status)) { live = false; break; }
                    tc_fence_after();
                }
                uint32_t from;
                const uint32_t off = rg.place(steps * bytes, &from);
                if (!mbar_wait_warp(smem_u32(&ctl->full[rg.slot()]), rg.parity(), abort_flag, p.status)) { live = false; break; }
                tc_fence_after();
                uint32_t al = (uint32_t)a0 + (off >> 4), bl = (uint32_t)b0 + ((off + a_bytes) >> 4);
                for (int i = 0; i < steps; ++i, al += bytes >> 4, bl += bytes >> 4) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        tc_mma_bf16_ss_elect(d, al + q * 2, a_hi, bl + q * kBStep, b_hi, idesc, in_block > 0 || i > 0 || q > 0);
                }
                tc_commit_elect(smem_u32(&ctl->empty[rg.slot()]));
                ++rg.n;
                if (ks + steps == p.ksteps || (MODE == kBackAct && in_block + steps == kSumSteps)) {
                    tc_commit_elect(smem_u32(&ctl->acc_full[it & 1]));
                    ++it;
                }
            }
        }
    } else if constexpr (MODE == kUp) {
        // Thread by row: a warp works on 32 rows and half of the columns, and passes what it has to write through staging of its own, so
        // that it is written along rows.
        const int quarter = warp & 3, side = warp >= 6;             // lane quarter of the accumulator; half of the columns
        const int r0 = quarter * 32;                                // this warp's first row of a tile
        const uint32_t at = (warp - 2) * 32 * kPrivatePitch;        // of this warp's staging
        const uint32_t mine = staging + at + lane * kPrivatePitch;
        int it = 0;
        for (TilesAhead<0> u(p, units, 0); u.more(); u.next(), ++it) {
            const int buf = it & 1, rows = min(32, u.tile.z - r0), place0 = u.tile.y + r0;
            const uint32_t acc = tmem + buf * 256 + ((uint32_t)r0 << 16);
            const int cols = p.nb * 32, per = cols / 2, s0 = u.chunk * cols + side * per;      // s columns of the unit; of this warp
            if (!mbar_wait_warp(smem_u32(&ctl->acc_full[buf]), (it >> 1) & 1, abort_flag, p.status)) break;
            tc_fence_after();
            if (rows > 0 && s0 < p.s) {
                const int limit = min(per, p.s - s0);
                if (p.hidden)
                    for (int half = 0; half < 2; ++half) {
                        for (int c = 0; c < limit; c += 16) {
                            float v[16];
                            tmem_ld16(acc + half * cols + side * per + c, v);
                            tmem_ld_wait16(v);
                            st_piece(mine + c * 2, pack8(v, 0));
                            st_piece(mine + c * 2 + 16, pack8(v, 8));
                        }
                        write_rows(staging_at + at, per / 8, lane, rows, limit, p.hidden + (long long)place0 * 2 * p.s + half * p.s + s0, 2 * p.s);
                    }
                for (int c = 0; c < limit; c += 16) {
                    float g[16], v[16];
                    tmem_ld16(acc + side * per + c, g);
                    tmem_ld16(acc + cols + side * per + c, v);
                    tmem_ld_wait16(g); tmem_ld_wait16(v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) g[i] = g[i] * sigmoid_to_round(g[i]) * v[i];      // (to bf16: an operand of the second product)
                    st_piece(mine + c * 2, pack8(g, 0));
                    st_piece(mine + c * 2 + 16, pack8(g, 8));
                }
                write_rows(staging_at + at, per / 8, lane, rows, limit, p.out + (long long)place0 * p.s + s0, p.s);
            }
            tc_fence_before();
            warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);
        }
    } else if constexpr (MODE == kBackAct) {
        // The warps that have rows add columns of the accumulator up in staging, thread by row; then all eight work along rows, so that
        // memory is read and written in whole lines and a tile of few rows occupies them all.
        const int quarter = warp & 3, side = warp >= 6;             // lane quarter of the accumulator; half of every 64 columns
        const int r0 = quarter * 32, row = r0 + lane;               // this warp's first row of a tile, this thread's
        const int tid = threadIdx.x - 64, blocks = (p.ksteps + kSumSteps - 1) / kSumSteps;
        int it = 0;
        for (TilesAhead<1> u(p, units, row); u.more(); u.next()) {
            const int4 tile = u.tile;
            const int first = u.chunk * p.nb * 64, passes = (min(p.nb * 64, p.s - first) + 63) / 64;      // of 64 columns, at most two
            // requested before the waits: both projections of this thread's first items, this row's gate
            uint4 kept[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (i * 256 + tid) >> 3, col = first + (tid & 7) * 8;
                if (r < tile.z && col < p.s) {
                    const __nv_bfloat16* from = p.hidden + (long long)(tile.y + r) * 2 * p.s + col;
                    kept[i][0] = *reinterpret_cast<const uint4*>(from);
                    kept[i][1] = *reinterpret_cast<const uint4*>(from + p.s);
                }
            }
            const float gate = side == 0 && u.pair[0] >= 0 ? p.gate[u.pair[0]] : 0.f;
            bool ok = true;
            for (int block = 0; block < blocks; ++block, ++it) {
                const int buf = it & 1;
                const uint32_t acc = tmem + buf * 256 + ((uint32_t)r0 << 16);
                // after a wait that gave up the loop goes on without work: no warp is left alone at a barrier
                ok &= mbar_wait_warp(smem_u32(&ctl->acc_full[buf]), (it >> 1) & 1, abort_flag, p.status);
                tc_fence_after();
                if (ok && r0 < tile.z)                              // (a warp whose rows are all behind the tile adds nothing)
                    for (int pass = 0; pass < passes; ++pass) {
                        float v[2][16];
#pragma unroll
                        for (int i = 0; i < 2; ++i) tmem_ld16(acc + pass * 64 + side * 32 + i * 16, v[i]);
                        const int at = pass * kTileRows * 256;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            tmem_ld_wait16(v[i]);
                            if (block > 0) add_staged(staging_at + at, 256, row, side * 8 + i * 4, v[i]);
                            stage_f32(staging + at, 256, row, side * 8 + i * 4, v[i]);
                        }
                    }
                tc_fence_before();
                warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);  // the accumulator may be filled again
            }
            if (side == 0) {                                        // (the last tile's have been read)
                ctl->pair[row] = u.pair[0];
                ctl->gate[row] = gate;
            }
            epilogue_sync();
            const int rows = ok ? tile.z : 0;
            float dg[4] = {0.f, 0.f, 0.f, 0.f};
            for (int pass = 0; pass < passes; ++pass) {
                const int s0 = first + pass * 64 + (tid & 7) * 8;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = (i * 256 + tid) >> 3;
                    if (r >= rows || s0 >= p.s) continue;
                    const long long place = tile.y + r;
                    const __nv_bfloat16* from = p.hidden + place * 2 * p.s + s0;
                    const uint4 hg = pass == 0 ? kept[i][0] : *reinterpret_cast<const uint4*>(from);
                    const uint4 hu = pass == 0 ? kept[i][1] : *reinterpret_cast<const uint4*>(from + p.s);
                    const float g_r = ctl->gate[r];
                    const uint32_t wg[4] = {hg.x, hg.y, hg.z, hg.w}, wu[4] = {hu.x, hu.y, hu.z, hu.w};
                    float c[8], out_g[8], out_u[8], out_a[8];
                    unstage8(staging_at + pass * kTileRows * 256, 256, r, (tid & 7) * 2, c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float g = j & 1 ? bf16_hi(wg[j / 2]) : bf16_lo(wg[j / 2]), up = j & 1 ? bf16_hi(wu[j / 2]) : bf16_lo(wu[j / 2]);
                        const float sg = sigmoidf(g), silu = g * sg, act = silu * up, da = g_r * c[j];
                        dg[i] = fmaf(c[j], act, dg[i]);
                        out_a[j] = g_r * act;
                        out_u[j] = da * silu;
                        out_g[j] = da * up * fmaf(silu, 1.f - sg, sg);
                    }
                    // (du and gate a to bf16: operands of the products behind)
                    *reinterpret_cast<uint4*>(p.du + place * 2 * p.s + s0) = pack8(out_g);
                    *reinterpret_cast<uint4*>(p.du + place * 2 * p.s + p.s + s0) = pack8(out_u);
                    if (p.ga) *reinterpret_cast<uint4*>(p.ga + place * p.s + s0) = pack8(out_a);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {                           // the eight threads of a row
                const int r = (i * 256 + tid) >> 3;
#pragma unroll
                for (int o = 4; o > 0; o >>= 1) dg[i] += __shfl_xor_sync(0xffffffffu, dg[i], o);
                const int pair = r < rows ? ctl->pair[r] : -1;
                if ((tid & 7) == 0 && pair >= 0) p.dgate_part[(long long)u.chunk * p.P + pair] = dg[i];
            }
            epilogue_sync();
        }
    } else if (warp < 6) {
        // The accumulator comes thread by row, memory is written along rows: these four warps round it into one of two buffers of 64
        // rows, the next four write buffers out.  (An SM writes about 25 bytes a clock; where the same warps did both, that time
        // came on top of the rest.)
        const int quarter = warp & 3, tid = threadIdx.x - 64;       // lane quarter of the accumulator
        int it = 0, piece = 0;
        for (TilesAhead<1> u(p, units, tid); u.more(); u.next(), ++it) {
            const int buf = it & 1, c0 = u.chunk * p.nb * 64, cols = min(p.nb * 64, p.h - c0);
            const uint32_t acc = tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16);
            // (after a wait that gave up the loop goes on without work: no warp is left alone at a barrier)
            const bool ok = mbar_wait_warp(smem_u32(&ctl->acc_full[buf]), (it >> 1) & 1, abort_flag, p.status);
            tc_fence_after();
            const int unlike = unlike_boxes(u.tile.z), copy = quarter / unlike, pieces = u.tile.z > 64 ? 2 : 1;
            for (int q = 0; q < pieces; ++q, ++piece) {
                const int b = piece & 1, first = (quarter % unlike) * 32 - q * 64;        // this warp's first row in the buffer
                if (piece >= 2) take_over(4 + b);
                if (tid >> 6 == q) ctl->pair[b * 64 + (tid & 63)] = ok ? u.pair[0] : -1;
                if (ok && first >= 0 && first < 64 && q * 64 + first < u.tile.z)
                    for (int c = copy * 32; c < cols; c += 4 / unlike * 32) {
                        float v[2][16];
                        tmem_ld16(acc + c, v[0]);
                        tmem_ld16(acc + c + 16, v[1]);
                        tmem_ld_wait16(v[0]); tmem_ld_wait16(v[1]);
                        const int at = (b * 64 + first + lane) * kRowPitch;
                        const uint32_t to = staging + at + c * 2;
                        if constexpr (MODE == kDown) {
                            st_piece(to, pack8(v[0], 0)); st_piece(to + 16, pack8(v[0], 8));
                            st_piece(to + 32, pack8(v[1], 0)); st_piece(to + 48, pack8(v[1], 8));
                        } else {
                            // The rows of the slots are added later: each 32 columns of a row are kept in fp16 behind a power of two
                            // that brings their largest to [2^14, 2^15): an eighth of bf16's rounding for 3 % more bytes.
                            // (Columns behind the row's end are zeros: there the weights are out of bounds.)
                            float top = 0.f;
#pragma unroll
                            for (int i = 0; i < 16; ++i) top = max3(top, fabsf(v[0][i]), fabsf(v[1][i]));
                            const int ex = max(15, __float_as_int(top) >> 23);
                            const float up = ex < 255 ? __int_as_float((268 - ex) << 23) : 1.f;
                            st_piece(to, pack8_half(v[0], 0, up)); st_piece(to + 16, pack8_half(v[0], 8, up));
                            st_piece(to + 32, pack8_half(v[1], 0, up)); st_piece(to + 48, pack8_half(v[1], 8, up));
                            staging_at[at + 512 + c / 32] = (uint8_t)(ex < 255 ? ex - 14 : 127);   // (behind the row)
                        }
                    }
                if (q == pieces - 1) {
                    tc_fence_before();
                    warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);
                }
                hand_over(2 + b);
            }
        }
        if (piece >= 2) take_over(4 + (piece & 1));                  // (every hand-over is taken)
        if (piece >= 1) take_over(4 + ((piece - 1) & 1));
    } else {
        // a warp per row: up to 512 consecutive bytes
        int piece = 0;
        uint16_t* out = MODE == kDown ? reinterpret_cast<uint16_t*>(p.out) : reinterpret_cast<uint16_t*>(p.dx);
        for (TilesAhead<0> u(p, units, 0); u.more(); u.next()) {
            const int c0 = u.chunk * p.nb * 64, pieces = u.tile.z > 64 ? 2 : 1;
            const bool in = lane < p.nb * 8 && c0 + lane * 8 < p.h;
            for (int q = 0; q < pieces; ++q, ++piece) {
                const int b = piece & 1, rows = min(64, u.tile.z - q * 64);
                take_over(2 + b);
                for (int r = warp - 6; r < rows; r += 16) {
                    uint4 v[4];
                    int pair[4];
                    uint8_t ex[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = b * 64 + min(r + 4 * i, 63);
                        pair[i] = r + 4 * i < rows ? ctl->pair[at] : -1;
                        v[i] = ld_piece(staging_at + at * kRowPitch + lane * 16);
                        if (MODE == kBackX) ex[i] = staging_at[at * kRowPitch + 512 + (lane & 7)];
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (pair[i] < 0) continue;
                        if (in) *reinterpret_cast<uint4*>(out + (long long)pair[i] * p.h + c0 + lane * 8) = v[i];
                        if (MODE == kBackX && lane < p.nb * 2 && c0 + lane * 32 < p.h) p.dx_scale[(long long)pair[i] * p.dx_groups + c0 / 32 + lane] = ex[i];
                    }
                }
                hand_over(4 + b);
            }
        }
    }
    close_cta(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------------------ gradients of the weights
struct WeightsSide {
    int a_by_token;               // dW1: A = X by token, B = du by place; dW2: A = gate a by place, B = d by token
    int rows, cols;               // of an expert's output: A's columns, B's columns
    int mtiles, chunks, nb, box_rows;
    // Boxes of 64 of A's columns, rows of the accumulator.  Where the output has no more than 64 rows they are loaded twice: both halves
    // of the accumulator's lanes then hold the same, and all the warps that read it share the columns.
    __device__ int boxes_of_rows(int mt) const { return rows <= 64 || rows - mt * 128 > 64 ? 2 : 1; }
    __device__ bool twice() const { return rows <= 64; }
    // staging holds two units' boxes of this output, each in its half
    __device__ bool by_halves() const { return nb * box_rows * 128 <= kXStaging / 2; }
    __nv_bfloat16* out;           // [M][rows][cols]
};
static_assert(kXStaging / 2 % 1024 == 0, "boxes begin on 1024 bytes");
struct WeightsMaps { CUtensorMap token, place, place16, out; };     // place16: 16 rows high; token, place: one, for gathers
struct WeightsParams {
    const int32_t* offsets;
    const int32_t* pairs;
    int P, T;
    Divide by_k;
    unsigned units0, units;       // units of the first output; of both
    WeightsSide side[2];
    int* status;
    // (by selects: an index would make each field a load of its own)
    __device__ WeightsSide of(int which) const
    {
        WeightsSide o;
        o.a_by_token = which ? side[1].a_by_token : side[0].a_by_token;
        o.rows = which ? side[1].rows : side[0].rows;
        o.cols = which ? side[1].cols : side[0].cols;
        o.mtiles = which ? side[1].mtiles : side[0].mtiles;
        o.chunks = which ? side[1].chunks : side[0].chunks;
        o.nb = which ? side[1].nb : side[0].nb;
        o.box_rows = which ? side[1].box_rows : side[0].box_rows;
        o.out = which ? side[1].out : side[0].out;
        return o;
    }
};

// The runs of a CTA's units in turn, for a converged warp, whose lanes hold those of 32 units; the next 32 are requested when they begin.
struct Units {
    const WeightsParams& p;
    int lane, index;
    int which, e, mt, chunk, lo, n;                          // of the present unit: output, expert, tile of rows, chunk of columns, its run
    int batch_e, batch_rem, raw_lo, raw_hi;                  // this lane's
    int next_e, next_rem, next_lo, next_hi;
    __device__ explicit Units(const WeightsParams& q) : p(q), lane(threadIdx.x & 31), index(-1)
    {
        request(0);
        next();
    }
    __device__ void request(int first)
    {
        const unsigned long long u = blockIdx.x + (unsigned long long)(first + lane) * gridDim.x;
        next_e = next_rem = next_lo = next_hi = 0;
        if (u >= p.units) return;
        const int w = u >= p.units0;
        const unsigned v = (unsigned)u - (w ? p.units0 : 0u), per_expert = (unsigned)(p.of(w).mtiles * p.of(w).chunks);
        next_e = (int)(v / per_expert);
        next_rem = (int)(v % per_expert);
        next_lo = p.offsets[next_e];
        next_hi = p.offsets[next_e + 1];
    }
    __device__ bool more() const { return blockIdx.x + (unsigned long long)index * gridDim.x < p.units; }
    __device__ void next()
    {
        const int i = ++index & 31;
        if (i == 0) {
            batch_e = hold(next_e);
            batch_rem = hold(next_rem);
            raw_lo = min(max(hold(next_lo), 0), p.P);        // (whatever the offsets hold, a run stays within the places)
            raw_hi = max(min(hold(next_hi), p.P), raw_lo);
            request(index + 32);
        }
        which = blockIdx.x + (unsigned long long)index * gridDim.x >= p.units0;
        e = __shfl_sync(0xffffffffu, batch_e, i);
        const int rem = __shfl_sync(0xffffffffu, batch_rem, i), chunks = p.of(which).chunks;
        mt = chunks == 1 ? rem : rem / chunks;
        chunk = chunks == 1 ? 0 : rem % chunks;
        lo = __shfl_sync(0xffffffffu, raw_lo, i);
        n = __shfl_sync(0xffffffffu, raw_hi, i) - lo;
    }
};

__global__ void __launch_bounds__(threads_of(kBackLoaders), 1)
weights_kernel(const __grid_constant__ WeightsMaps m0, const __grid_constant__ WeightsMaps m1, const __grid_constant__ WeightsParams all)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, staging = ring + kXRing;
    uint8_t* const staging_at = smem_raw + (ring - smem_u32(smem_raw)) + kXRing;
    Control* ctl = reinterpret_cast<Control*>(staging_at + kXStaging);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    let_next_begin();
    const uint32_t tmem = open_cta(ctl, 1, 8, warp);
    wait_for_previous();
    volatile int* abort_flag = &ctl->abort;

    if (warp == 0 || warp >= 10) {
        // A stage is up to 64 rows, as many whole MMA steps of 16 as it needs, of both operands' boxes of 64 columns: rows by token by
        // gathers, consecutive places in pieces of 16.  Rows behind the run's last are out of bounds, zeros: of the places, too,
        // only then row by row (what lies there belongs to another expert).
        // A loader issues a stage of its own when it has come to the next one, whose pairs it has just requested.  Issuing one (16
        // gathers, 4 boxes) takes it about 4700 clocks, passing a unit 750: with five they were what a unit waited for.
        const int loader = loader_of(warp);
        int4* rows = ctl->rows[loader];                             // 64 tokens, 64 places
        const uint64_t again = comes_again();
        Ring rg;
        bool live = true;
        struct Own {
            int which, first, left, mt, chunk, last, stage, pair[2]; // output, first place, rows; the stage that has to be empty, or less than 0
            uint32_t where;
        } own;
        own.left = 0;
        auto issue = [&]() {
            if (own.left == 0 || !live) return;
            const WeightsSide o = all.of(own.which);
            const WeightsMaps& m = own.which ? m1 : m0;
            const int left = own.left, steps = (left + 15) / 16, a_boxes = o.boxes_of_rows(own.mt);
            const uint32_t box = (uint32_t)steps * 2048;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = i * 32 + lane, pair = hold(own.pair[i]);
                const bool in = pair >= 0 && pair < all.P;
                reinterpret_cast<int*>(rows)[r] = in ? all.by_k(pair) : all.T;
                reinterpret_cast<int*>(rows)[64 + r] = in ? own.first + r : all.P;
            }
            if (!rg.wait_empty(own.stage, own.last, ctl, abort_flag, all.status)) {
                live = false;
                return;
            }
            __syncwarp();
            const uint32_t full = smem_u32(&ctl->full[own.stage % kSlots]);
            expect_elect(full, box * (a_boxes + o.nb));
            const uint32_t a_at = ring + own.where, b_at = a_at + a_boxes * box;
            const int a_x = own.mt * 128, b_x = own.chunk * o.nb * 64;
            const int t_boxes = o.a_by_token ? a_boxes : o.nb, p_boxes = o.a_by_token ? o.nb : a_boxes;
            const int t_x = o.a_by_token ? a_x : b_x, p_x = o.a_by_token ? b_x : a_x;
            const int t_step = o.a_by_token && o.twice() ? 0 : 64, p_step = !o.a_by_token && o.twice() ? 0 : 64;
            const uint32_t t_at = o.a_by_token ? a_at : b_at, p_at = o.a_by_token ? b_at : a_at;
            for (int q = 0; q < steps; ++q) {
                const int4 r0 = rows[4 * q], r1 = rows[4 * q + 1], r2 = rows[4 * q + 2], r3 = rows[4 * q + 3];
                for (int b = 0; b < t_boxes; ++b) tma_gather16(t_at + b * box + q * 2048, &m.token, full, t_x + b * t_step, 4, r0, r1, r2, r3, again);
                if (left >= q * 16 + 16) {
                    for (int b = 0; b < p_boxes; ++b) tma_load_2d_elect(p_at + b * box + q * 2048, &m.place16, full, p_x + b * p_step, own.first + q * 16);
                } else {
                    const int4 s0 = rows[16 + 4 * q], s1 = rows[17 + 4 * q], s2 = rows[18 + 4 * q], s3 = rows[19 + 4 * q];
                    for (int b = 0; b < p_boxes; ++b) tma_gather16(p_at + b * box + q * 2048, &m.place, full, p_x + b * p_step, 4, s0, s1, s2, s3, again);
                }
            }
            __syncwarp();                                           // (the rows are read)
        };
        for (Units u(all); u.more() && live; u.next()) {
            const int a_boxes = all.of(u.which).boxes_of_rows(u.mt), nb = all.of(u.which).nb;
            for (int at = 0; at < u.n; at += 64, ++rg.n) {
                const int left = min(64, u.n - at);
                uint32_t where;
                int last;
                if (!rg.mine((uint32_t)((left + 15) / 16) * 2048 * (a_boxes + nb), loader, kBackLoaders, lane, &where, &last)) continue;
                int pair[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) pair[i] = i * 32 + lane < left ? all.pairs[u.lo + at + i * 32 + lane] : -1;
                issue();
                own.which = u.which;
                own.first = u.lo + at;
                own.left = left;
                own.mt = u.mt;
                own.chunk = u.chunk;
                own.last = last;
                own.stage = rg.n;
                own.where = where;
                own.pair[0] = pair[0];
                own.pair[1] = pair[1];
            }
        }
        issue();
    } else if (warp == 1) {
        const uint64_t d0 = umma_desc_sw128(ring, 0, 1024);
        Ring rg;
        int it = 0;
        bool live = true;
        for (Units u(all); u.more() && live; u.next()) {
            const int n = u.n;
            if (n == 0) continue;                                   // (the epilogue writes zeros without an accumulator)
            const int a_boxes = all.of(u.which).boxes_of_rows(u.mt), nb = all.of(u.which).nb;
            const uint32_t idesc = idesc_of(nb * 64, 1, 1);
            for (int at = 0; at < n; at += 64) {
                const int buf = it & 1, in_piece = at % kRunPiece;
                if (in_piece == 0) {
                    if (!mbar_wait_warp(smem_u32(&ctl->acc_empty[buf]), ((it >> 1) & 1) ^ 1u, abort_flag, all.status)) { live = false; break; }
                    tc_fence_after();
                }
                const uint32_t steps = (min(64, n - at) + 15) / 16, box = steps * 2048;
                uint32_t from;
                const uint32_t off = rg.place(box * (a_boxes + nb), &from);
                if (!mbar_wait_warp(smem_u32(&ctl->full[rg.slot()]), rg.parity(), abort_flag, all.status)) { live = false; break; }
                tc_fence_after();
                // boxes lie `box` apart: the distance of 64 columns in both descriptors
                const uint32_t a_lo = ((uint32_t)d0 + (off >> 4)) | (box >> 4) << 16, b_lo = a_lo + (a_boxes * box >> 4), hi = (uint32_t)(d0 >> 32);
                for (uint32_t q = 0; q < steps; ++q)
                    tc_mma_bf16_ss_elect(tmem + buf * 256, a_lo + q * 128, hi, b_lo + q * 128, hi, idesc, in_piece > 0 || q > 0);
                tc_commit_elect(smem_u32(&ctl->empty[rg.slot()]));
                ++rg.n;
                if (in_piece + 64 == kRunPiece || at + 64 >= n) {
                    tc_commit_elect(smem_u32(&ctl->acc_full[buf]));
                    ++it;
                }
            }
        }
    } else {
        // bf16 boxes of 64 columns in the layout of a swizzled TMA store, which cuts off what is behind the ends, of 128 rows, or of 64
        // where no more are needed; two units' worth of them where staging holds that
        const int quarter = warp & 3, side = warp >= 6, tid = threadIdx.x - 64;
        const uint64_t once = passes_once();
        int it = 0;
        uint32_t half = 0;                                          // of staging, where units' boxes fit one; a unit after the other
        bool halves = true;                                         // the unit before kept to its half of staging
        for (Units w(all); w.more(); w.next()) {
            const WeightsSide p = all.of(w.which);
            const int copies = p.twice() ? 2 : 1, copy = p.twice() ? quarter >> 1 : 0, row0 = (p.twice() ? quarter & 1 : quarter) * 32, row = row0 + lane;
            const int box = p.box_rows * 128;
            const int mt = w.mt, per = p.nb * 32, c0 = w.chunk * p.nb * 64;
            const int rows = min(128, p.rows - mt * 128);
            if (w.n == 0) {                                         // zeros: threads along rows, 16 bytes each
                const int pieces = p.nb * 8, c = c0 + (tid & (pieces - 1)) * 8;
                __nv_bfloat16* out = p.out + ((long long)w.e * p.rows + mt * 128) * p.cols + c;
                if (c < p.cols)
                    for (int r = tid / pieces; r < rows; r += 256 / pieces)
                        *reinterpret_cast<uint4*>(out + (long long)r * p.cols) = make_uint4(0, 0, 0, 0);
                continue;
            }
            const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), to = staging + (p.by_halves() ? half : 0);
            bool ok = mbar_wait_warp(smem_u32(&ctl->acc_full[it & 1]), (it >> 1) & 1, abort_flag, all.status);   // (given up: goes on without work)
            tc_fence_after();
            // a long run: the sum so far is added to the next piece's accumulator, whose place it then has, and its own is free
            for (int left = w.n - kRunPiece; left > 0; left -= kRunPiece) {
                const int before = it++ & 1;
                ok &= mbar_wait_warp(smem_u32(&ctl->acc_full[it & 1]), (it >> 1) & 1, abort_flag, all.status);
                tc_fence_after();
                for (int c = copy * 32; ok && c < per && row0 < rows && c0 + side * per + c < p.cols; c += copies * 32)
                    for (int i = 0; i < 32; i += 16) {
                        float v[16], sum[16];
                        tmem_ld16(lanes + before * 256 + side * per + c + i, sum);
                        tmem_ld16(lanes + (it & 1) * 256 + side * per + c + i, v);
                        tmem_ld_wait16(sum); tmem_ld_wait16(v);
                        uint32_t u[2][8];
#pragma unroll
                        for (int j = 0; j < 16; ++j) u[j / 8][j % 8] = __float_as_uint(sum[j] + v[j]);
                        tmem_st8(lanes + (it & 1) * 256 + side * per + c + i, u[0]);
                        tmem_st8(lanes + (it & 1) * 256 + side * per + c + i + 8, u[1]);
                    }
                tmem_st_wait();
                tc_fence_before();
                warp_arrive(smem_u32(&ctl->acc_empty[before]), lane);
            }
            const int buf = it & 1;
            const uint32_t acc = lanes + buf * 256;
            if (warp < 6) halves && p.by_halves() ? bulk_read_done<1>() : bulk_read_done<0>();
            halves = p.by_halves();
            epilogue_sync();
            for (int c = copy * 32; ok && c < per && row0 < rows && c0 + side * per + c < p.cols; c += copies * 32) {
                float v[2][16];
#pragma unroll
                for (int i = 0; i < 2; ++i) tmem_ld16(acc + side * per + c + i * 16, v[i]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    tmem_ld_wait16(v[i]);
                    const int col = side * per + c + i * 16;
                    st_piece(staged(to + col / 64 * box, 128, row, col % 64 / 8), pack8(v[i], 0));
                    st_piece(staged(to + col / 64 * box, 128, row, col % 64 / 8 + 1), pack8(v[i], 8));
                }
            }
            tc_fence_before();
            warp_arrive(smem_u32(&ctl->acc_empty[buf]), lane);
            ++it;
            half ^= kXStaging / 2;
            fence_async_smem();
            epilogue_sync();
            // A box for each of four warps where two units' boxes fit: issuing a store takes about 200 clocks (65536 x 4 pairs of 8192
            // experts, h = 512, s = 64, with seven loaders: the backward pass 825 us instead of 853); else all of them for one (of 2048
            // experts, h = 1024, s = 128, two slots: 929 us instead of 962).
            if (warp < 6) {
                for (int b = warp - 2; ok && b < p.nb && c0 + b * 64 < p.cols && (p.by_halves() ? b == warp - 2 : warp == 2); ++b)
                    tma_store_3d_elect(w.which ? &m1.out : &m0.out, to + b * box, c0 + b * 64, mt * 128, w.e, once);
                bulk_commit();
            }
        }
        if (warp < 6) bulk_all_done();
    }
    close_cta(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------------------ joining the slots
// dX[t] = sum over the token's slots of their rows (fp16 behind a scale per 32 columns); dgate[p] = sum of its parts.  A pair
// whose id is no expert was in no tile: it adds nothing and its gate gradient is 0.
struct JoinParams {
    const int32_t* idx;
    const __half* dx;
    const uint8_t* dx_scale;
    const float* dgate_part;
    int P, T, k, h, M, dx_groups, parts;
    __nv_bfloat16* out_dx;
    float* out_dgate;
};
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinParams p)
{
    let_next_begin();
    wait_for_previous();
    const int vecs = p.h / 8, width = vecs < 256 ? vecs : 256, tokens = 256 / width;      // threads of a token, tokens of a CTA
    const int mine = threadIdx.x / width, first_vec = threadIdx.x % width;
    for (long long t = p.out_dx && mine < tokens ? (long long)blockIdx.x * tokens + mine : p.T; t < p.T; t += (long long)gridDim.x * tokens)
    for (int c = first_vec * 8; c < p.h; c += width * 8) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int j0 = 0; j0 < p.k; j0 += 4) {                // four slots' loads at a time
            uint4 u[4];
            float sc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const long long pair = t * p.k + j0 + j;
                const bool in = j0 + j < p.k && (unsigned)p.idx[pair] < (unsigned)p.M;
                sc[j] = in ? __int_as_float((int)p.dx_scale[pair * p.dx_groups + c / 32] << 23) : 0.f;
                u[j] = in ? *reinterpret_cast<const uint4*>(p.dx + pair * p.h + c) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __half2* q = reinterpret_cast<const __half2*>(&u[j]);
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const float2 f = __half22float2(q[a]);
                    v[2 * a] = fmaf(f.x, sc[j], v[2 * a]);
                    v[2 * a + 1] = fmaf(f.y, sc[j], v[2 * a + 1]);
                }
            }
        }
        *reinterpret_cast<uint4*>(p.out_dx + t * p.h + c) =
            make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
    if (!p.out_dgate) return;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < p.P; i += (long long)gridDim.x * 256) {
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
int back_boxes(int s) { return s > 64 ? 2 : 1; }                    // boxes of s rows per unit of the activation's backward: their sums fit staging
int row_boxes(int h) { return h > 128 ? 4 : (h > 64 ? 2 : 1); }

Workspace lay_out(int T, int h, int s, int M, int k, bool backward)
{
    const size_t P = (size_t)T * k;
    Workspace w;
    size_t at = up256(16 * (size_t)(1 + tile_capacity(T, M, k)));
    if (!backward) {
        w.act = at; at += up256(P * s * 2);
    } else {
        const int nb = back_boxes(s), chunks = (s + nb * 64 - 1) / (nb * 64);
        w.du = at; at += up256(P * s * 4);
        w.ga = at; at += up256(P * s * 2);
        w.dgate = at; at += up256(P * 4 * chunks);
        w.dx = at; at += up256(P * h * 2);
        w.dx_scale = at; at += up256(P * (((size_t)h + 31) / 32));
    }
    w.total = at;
    return w;
}

// 2-D [rows][cols], boxes of `high` rows x 64 columns; one row high for gathers.
int rows_map(const void* ptr, long long rows, int cols, int high, CUtensorMap* out)
{
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)cols * 2};
    const uint32_t box[2] = {64, (uint32_t)high};
    return encode_tensor_map(ptr, 2, dims, strides, box, out);
}
// Weights [M][rows][cols], boxes of `high` rows x 64 columns of one expert.
int weight_map(const void* ptr, int M, int rows, int cols, int high, CUtensorMap* out)
{
    const uint64_t dims[3] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)M};
    const uint64_t strides[2] = {(uint64_t)cols * 2, (uint64_t)rows * cols * 2};
    const uint32_t box[3] = {64, (uint32_t)high, 1};
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
    p.status = ctx.status;
    const long long units = tiles * p.chunks;
    if (units > 0x7fff0000LL) return MORE_ERR_TOO_LARGE;
    const int grid = units < ctx.sm_count ? (int)units : ctx.sm_count;
    const int threads = rows_threads(MODE);
    if (launch_behind(rows_kernel<MODE>, grid, threads, kXSmem, st, ma, mw, p) != cudaSuccess) return MORE_ERR_CUDA;
    count_launch(1);
    return MORE_OK;
}

int launch_tiles(const ExpertsArgs& a, cudaStream_t st)
{
    const long long P = (long long)a.T * a.k;
    tiles_kernel<<<(a.M + 1023) / 1024, 1024, 0, st>>>(a.offsets, a.M, (int)P, (int)tile_capacity(a.T, a.M, a.k), static_cast<int4*>(a.workspace));
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MORE_OK : MORE_ERR_CUDA;
}

// dW1, dW2 or both, in one launch: what one leaves idle at its end, the other uses.
int launch_weights(const ExpertsArgs& a, const Workspace& w, const DeviceCtx& ctx)
{
    const long long P = (long long)a.T * a.k;
    char* base = static_cast<char*>(a.workspace);
    WeightsMaps m[2] = {};
    WeightsParams p{};
    p.offsets = a.offsets; p.pairs = a.pairs; p.P = (int)P; p.T = a.T; p.by_k.by(a.k);
    p.status = ctx.status;
    long long units = 0;
    int n = 0;
    for (int i = 0; i < 2; ++i) {
        __nv_bfloat16* const out = i == 0 ? a.out_dw1 : a.out_dw2;
        if (!out) continue;
        WeightsSide& o = p.side[n];
        o.a_by_token = i == 0;
        o.rows = i == 0 ? a.h : a.s; o.cols = i == 0 ? 2 * a.s : a.h; o.out = out;
        o.box_rows = o.rows > 64 ? 128 : 64;
        o.nb = row_boxes(o.cols);
        o.mtiles = (o.rows + 127) / 128;
        o.chunks = (o.cols + o.nb * 64 - 1) / (o.nb * 64);
        const char* place = base + (i == 0 ? w.du : w.ga);
        const int width = i == 0 ? 2 * a.s : a.s;
        int rc = rows_map(i == 0 ? a.X : a.dout, a.T, a.h, 1, &m[n].token);
        if (rc == MORE_OK) rc = rows_map(place, P, width, 1, &m[n].place);
        if (rc == MORE_OK) rc = rows_map(place, P, width, 16, &m[n].place16);
        if (rc == MORE_OK) rc = weight_map(out, a.M, o.rows, o.cols, o.box_rows, &m[n].out);
        if (rc != MORE_OK) return rc;
        units += (long long)a.M * o.mtiles * o.chunks;
        if (n++ == 0) p.units0 = (unsigned)units;
        if (units > 0x7fff0000LL) return MORE_ERR_TOO_LARGE;
    }
    if (n == 0) return MORE_OK;
    p.units = (unsigned)units;
    if (allow_smem(weights_kernel) != MORE_OK) return MORE_ERR_CUDA;
    const int grid = units < ctx.sm_count ? (int)units : ctx.sm_count;
    if (launch_behind(weights_kernel, grid, threads_of(kBackLoaders), kXSmem, a.stream, m[0], m[1], p) != cudaSuccess) return MORE_ERR_CUDA;
    count_launch(1);
    return MORE_OK;
}

int launch_experts(const ExpertsArgs& a, const DeviceCtx& ctx)
{
    const long long P = (long long)a.T * a.k;
    const Workspace w = lay_out(a.T, a.h, a.s, a.M, a.k, false);
    char* base = static_cast<char*>(a.workspace);
    CUtensorMap mx, mact, m1, m2;
    int rc = rows_map(a.X, a.T, a.h, 1, &mx);
    if (rc == MORE_OK) rc = rows_map(base + w.act, P, a.s, 32, &mact);
    if (rc == MORE_OK) rc = weight_map(a.W1, a.M, a.h, 2 * a.s, 64, &m1);
    if (rc == MORE_OK) rc = weight_map(a.W2, a.M, a.s, a.h, 64, &m2);
    if (rc == MORE_OK) rc = launch_tiles(a, a.stream);
    if (rc != MORE_OK) return rc;
    RowsParams p{};
    p.tiles = static_cast<const int4*>(a.workspace);
    p.pairs = a.pairs;
    p.P = (int)P; p.h = a.h; p.s = a.s;
    const long long tiles = tile_capacity(a.T, a.M, a.k);
    p.by_k.by(a.k);
    p.rows = a.T;
    p.weights_once = P <= 2LL * kTileRows * a.M;
    p.nb = a.s > 64 ? 4 : 2;
    p.chunks = (a.s + p.nb * 32 - 1) / (p.nb * 32);
    p.ksteps = (a.h + 63) / 64;
    p.out = reinterpret_cast<__nv_bfloat16*>(base + w.act);
    p.hidden = a.out_hidden;
    rc = launch_rows<kUp>(mx, m1, p, tiles, ctx, a.stream);
    if (rc != MORE_OK) return rc;
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
    CUtensorMap md, mdu, m1, m2;
    int rc = rows_map(a.dout, a.T, a.h, 1, &md);
    if (rc == MORE_OK) rc = rows_map(base + w.du, P, 2 * a.s, 32, &mdu);
    if (rc == MORE_OK) rc = weight_map(a.W1, a.M, a.h, 2 * a.s, row_boxes(a.h) * 64, &m1);
    if (rc == MORE_OK) rc = weight_map(a.W2, a.M, a.s, a.h, back_boxes(a.s) * 64, &m2);
    if (rc == MORE_OK) rc = launch_tiles(a, a.stream);
    if (rc != MORE_OK) return rc;
    const long long tiles = tile_capacity(a.T, a.M, a.k);
    RowsParams p{};
    p.tiles = static_cast<const int4*>(a.workspace);
    p.pairs = a.pairs;
    p.P = (int)P; p.h = a.h; p.s = a.s;
    p.by_k.by(a.k);
    p.rows = a.T;
    p.weights_once = P <= 2LL * kTileRows * a.M;
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
    p.dx_groups = (a.h + 31) / 32;
    p.dx = reinterpret_cast<__half*>(base + w.dx);
    p.dx_scale = reinterpret_cast<uint8_t*>(base + w.dx_scale);
    if (a.out_dx) {
        p.weights_once = 0;                                          // (a row of W1 is read in pieces, a step apart)
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
        j.out_dx = a.out_dx; j.out_dgate = a.out_dgate;
        const long long items = a.out_dx ? (long long)a.T * (a.h / 8) : P;
        const long long blocks = (items + 255) / 256;
        if (launch_behind(join_kernel, (int)(blocks < 148 * 16 ? blocks : 148 * 16), 256, 0, a.stream, j) != cudaSuccess) return MORE_ERR_CUDA;
        count_launch(1);
    }
    return launch_weights(a, w, ctx);
}

int check_sizes(int T, int h, int s, int M, int k)
{
    if (T < 0 || h < 8 || s < 8 || h % 8 != 0 || s % 8 != 0 || h > MORE_H_MAX || s > MORE_S_MAX) return MORE_ERR_SHAPE;
    if (M < 1 || M > MORE_M_MAX || k < 1 || k > MORE_K_MAX || k > M) return MORE_ERR_SHAPE;
    if ((long long)T * k > MORE_PAIRS_MAX) return MORE_ERR_TOO_LARGE;          // places are counted in 32 bits, past a run's end by up to a piece
    return MORE_OK;
}

// Which forward path.  Pairs read their expert's weights each, 9 us behind a start (20 GB/s per CTA, 6.2 TB/s in all), 0.016 us per pair at
// least.  Tiles read those of the experts that are hit, of evenly spread ids M (1 - exp(-P / M)), 20 us behind for three kernels; a
// kernel takes the bytes' time (100 GB/s per unit, 6.2 TB/s in all) or that of its stages, 0.3 us each of the first, 0.8 of the
// second, over the SMs.  Measured on eight combinations of h, s and M from 8 to 8192 pairs (us, pairs / tiles): h = 2048, s = 64,
// M = 8192: 12 / 26 at 8 pairs, 74 / 80 at 512, 137 / 133 at 1024, 260 / 222 at 2048; h = 512, s = 64, M = 64: 14 / 20 at 128, 25 / 20
// at 512, 38 / 20 at 1024; h = 256, s = 16, M = 16384: 46 / 46 at 2048, 136 / 103 at 8192; h = 4096, s = 512, M = 16: 68 / 46 at
// 8.  The choice cost 2 % at worst in the run that it was fitted to, 7 % in the next.  (Ids that cluster hit fewer experts than evenly
// spread ones, and tiles then take less than it says.)
int cheaper_path(int T, int h, int s, int M, int k)
{
    const double P = (double)T * k, weights = 6.0 * h * s, sms = 148, most = 6.2e6;     // bytes; bytes per us
    const double hit = M * -expm1(-P / M);
    double ctas = P;                                                 // as launch_experts_pairs has them
    for (int ranks = 1; ranks < 8 && ctas * 2 <= 2 * sms && h / (ranks * 2) >= 32; ranks *= 2) ctas *= 2;
    const double pairs = 9 + P * fmax(0.016, 0.008 + weights / fmin(most, fmin(ctas, 2 * sms) * 20e3));
    const double wide = (s + 127) / 128, rate = fmin(most, hit * wide * 100e3);
    const double up = hit * fmax(weights * 2 / 3 / rate, wide * ((h + 63) / 64) * 0.3 / sms);
    const double down = hit * fmax(weights / 3 / rate, ((h + 255) / 256) * ((s + 63) / 64) * 0.8 / sms);
    const double tiles = 20 + up + down;
    return pairs <= tiles ? MORE_EXPERTS_PAIRS : MORE_EXPERTS_TILES;
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
    const bool pairwise = path == MORE_EXPERTS_PAIRS || !listed || (path == MORE_EXPERTS_AUTO && !out_hidden && cheaper_path(T, h, s, M, k) == MORE_EXPERTS_PAIRS);
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
    return rc == MORE_OK ? cheaper_path(T, h, s, M, k) : rc;
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
