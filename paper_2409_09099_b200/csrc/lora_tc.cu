// Low-rank adapters on tiles of 128 rows, on the tensor cores' own memory: operands go from global to shared memory by TMA and from there to
// tcgen05.mma, sums stay in tensor memory, and no operand passes through a thread's registers.
//
//   apply     V = s x A^T, then y_out = y_in + V B^T (backward: U = s dY B, then dX_out = dX_in + U A): 128 rows, K streamed in steps
//             of 64, then 64 columns of y at a time
//   gradient  dA = U^T X, dB = dY^T V: 128 (or 256) features x rank, rows streamed in steps of 64
//
// They stream large tensors and are bound by them: a step has 16 KB of it beside 2 to 16 KB of the small operand.  On the ordinary
// (register) tensor path the same products spent 60 to 80 % of the L1 cache's wavefronts on moving operands to registers and ran at a sixth
// to a third of the memory's rate.  V and U are kept as two bf16 planes whose sum is good to 2^-17 (a rounding to one bf16 would bring as
// much error into Y, dX and the gradients as dY's own rounding has), three where gradients are fp32, so the second and third product take each
// stage more than once: memory bounds them all the same.
// One CTA works alone (cta_group::1): with at most 64 columns of the instruction's B operand, a pair has nothing to share.
//
// The waits are bounded as in the products: on expiry the CTA records SSTE_ERR_TIMEOUT, waits for the copies and products that it has itself
// started (again with a limit: what they write is about to be another's) and leaves.
#include <cuda.h>

#include "lora.cuh"

namespace {

constexpr int TC_ROWS = 128, TC_K = 64, CHUNK = 64;        // rows of a tile; of K, of columns and of rows per step: 128 bytes of bf16
constexpr unsigned long long WAIT_LIMIT_NS = 2000000000ull, STALL_LIMIT_NS = 1000000ull, LEAVE_LIMIT_NS = 1000000ull;

// ------------------------------------------------------------------ PTX wrappers (see gemm.cu for the pair forms)

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity), "r"(1000000u)
                 : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
struct Waits {
    unsigned int *status;
    volatile int *abort;
    unsigned long long limit_ns;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const
    {
        if (mbar_try(bar, parity)) return true;
        const unsigned long long start = now_ns();
        while (true) {
            if (mbar_try(bar, parity)) return true;
            if (*abort) return false;
            if (now_ns() - start > limit_ns) {
                atomicMax(status, static_cast<unsigned int>(SSTE_ERR_TIMEOUT));
                *abort = 1;
                return false;
            }
        }
    }
    // of a CTA that leaves: for something that it has started, whatever has expired before
    __device__ __forceinline__ void leaving(uint32_t bar, uint32_t parity) const
    {
        const unsigned long long start = now_ns();
        while (!mbar_try(bar, parity) && now_ns() - start < LEAVE_LIMIT_NS) {}
    }
    // of a whole warp: lane 0 waits
    __device__ __forceinline__ bool warp(uint32_t bar, uint32_t parity) const
    {
        uint32_t ok = 1;
        if ((threadIdx.x & 31) == 0) ok = (*this)(bar, parity) ? 1u : 0u;
        return __shfl_sync(0xffffffffu, ok, 0) != 0;
    }
};
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map),
                 "r"(bar), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                 "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
template <int COLS>
__device__ __forceinline__ void tmem_alloc(uint32_t dst)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLS>
__device__ __forceinline__ void tmem_free(uint32_t addr)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(COLS) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
// 32 lanes x 16 columns
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float *r)
{
    uint32_t v[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __uint_as_float(v[i]);
}

// Shared-memory matrix descriptor: start, leading and stride byte offsets (>> 4), version 1, swizzle (2: 128 bytes, 4: 64, 6: 32).
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo, uint32_t sbo, uint32_t swizzle)
{
    return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | (static_cast<uint64_t>(lbo >> 4) << 16) | (static_cast<uint64_t>(sbo >> 4) << 32) |
           (1ull << 46) | (static_cast<uint64_t>(swizzle) << 61);
}
// fp32 sums of bf16 operands, 128 x N; a_mn, b_mn: the operand's rows run along the reduction
__host__ __device__ constexpr uint32_t instr_desc(bool a_mn, bool b_mn, int n)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | (static_cast<uint32_t>(n >> 3) << 17) |
           ((128u >> 4) << 24);
}
// a row of R bf16 values fills one swizzle span
template <int R>
constexpr uint32_t SWIZZLE_OF = R == 64 ? 2u : R == 32 ? 4u : 6u;

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
// Two values as the sum of two bf16 pairs; what the second cannot say (an infinity, a NaN, a value that rounds to infinity) the first does.
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo)
{
    hi = pack2(x, y);
    const float rx = x - __uint_as_float(hi << 16), ry = y - __uint_as_float(hi & 0xffff0000u);
    lo = pack2(fabsf(rx) < INFINITY ? rx : 0.0f, fabsf(ry) < INFINITY ? ry : 0.0f);
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 bytes to the same place in CTA `rank` of the cluster, counted on that CTA's barrier
__device__ __forceinline__ void store_async(uint32_t at, uint32_t bar, int rank, const float *v)
{
    asm volatile("{\n\t.reg .b32 to, b;\n\tmapa.shared::cluster.u32 to, %0, %2;\n\tmapa.shared::cluster.u32 b, %1, %2;\n\t"
                 "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [to], {%3, %4, %5, %6}, [b];\n\t}"
                 ::"r"(at), "r"(bar), "r"(rank), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
                 "r"(__float_as_uint(v[3]))
                 : "memory");
}
// what two bf16 pairs leave of two values, as a third
__device__ __forceinline__ uint32_t rest2(float x, float y, uint32_t hi, uint32_t lo)
{
    const float rx = x - __uint_as_float(hi << 16) - __uint_as_float(lo << 16),
                ry = y - __uint_as_float(hi & 0xffff0000u) - __uint_as_float(lo & 0xffff0000u);
    return pack2(fabsf(rx) < INFINITY ? rx : 0.0f, fabsf(ry) < INFINITY ? ry : 0.0f);
}
__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void sts16(uint32_t at, const uint4 &v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Place, in 16 bytes, of the ranks c .. c + 7 of a slot in the planes of V or U: 64 slots' planes one behind the other, each as it lies in shared
// memory (rows of R values in a swizzle of their length), so that a step's are one copy without a tensor map.
template <int R>
__device__ __forceinline__ size_t plane_unit(size_t slot, int c, int n_planes)
{
    const uint32_t at = static_cast<uint32_t>(slot % CHUNK) * (R / 8) + static_cast<uint32_t>(c / 8);
    return slot / CHUNK * (static_cast<size_t>(n_planes) * (CHUNK * R / 8)) + (at ^ ((at >> 3) & (R / 8 - 1)));
}
// A barrier of warps 0 to 3 that also says whether all of them passed true.
__device__ __forceinline__ bool all_of_four_warps(bool ok)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r)
                 : "r"(ok ? 1u : 0u)
                 : "memory");
    return r != 0;
}

// Stage and parity of a ring of N.
template <int N>
struct Ring {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void next()
    {
        if (++stage == N) { stage = 0; phase ^= 1u; }
    }
    // Of the thread that fills it: where it has come to, kept in shared memory, and the waits until each stage's last filling is there (a
    // stage without one counts as there).
    __device__ __forceinline__ void park(uint32_t at) const { asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(stage), "r"(phase) : "memory"); }
    static __device__ __forceinline__ void settle(const Waits &wait, uint32_t full, uint32_t at)
    {
        uint32_t stage, phase;
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(stage), "=r"(phase) : "r"(at) : "memory");
#pragma unroll 1
        for (uint32_t s = 0; s < N; ++s) wait.leaving(full + 8 * s, s < stage ? phase : phase ^ 1u);
    }
};

// Barriers, the tensor-memory address and the abort flag, in front of the stages (on a 1 KB boundary: swizzle).
constexpr int CTRL = 1024, CTRL_LOADS = 976, CTRL_CODES = 984, CTRL_TMEM = 1000, CTRL_ABORT = 1008;
struct Frame {
    uint32_t bars, stages;                  // shared addresses
    uint8_t *generic;
    uint32_t tmem;
    Waits wait;
};
template <int TMEM_COLS, typename F>
__device__ __forceinline__ Frame begin(uint8_t *raw, unsigned int *status, bool stall, int alloc_warp, F init)
{
    Frame f;
    f.bars = (smem_u32(raw) + 1023u) & ~1023u;
    f.stages = f.bars + CTRL;
    f.generic = raw + (f.bars - smem_u32(raw));
    volatile int *abort = reinterpret_cast<volatile int *>(f.generic + CTRL_ABORT);
    f.wait = Waits{status, abort, stall ? STALL_LIMIT_NS : WAIT_LIMIT_NS};
    if (threadIdx.x == 0) {
        init(f.bars);
        *abort = 0;
        Ring<1>().park(f.bars + CTRL_LOADS);
        Ring<1>().park(f.bars + CTRL_CODES);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (static_cast<int>(threadIdx.x >> 5) == alloc_warp) tmem_alloc<TMEM_COLS>(f.bars + CTRL_TMEM);
    tc_before();
    __syncthreads();
    tc_after();
    f.tmem = *reinterpret_cast<volatile uint32_t *>(f.generic + CTRL_TMEM);
    return f;
}
// `settle`: each thread's waits for what it has started, where a wait has expired.
template <int TMEM_COLS, typename F>
__device__ __forceinline__ void end(const Frame &f, int alloc_warp, F settle)
{
    tc_before();
    __syncthreads();
    tc_after();
    if (*f.wait.abort) {                                       // (nobody sets it any more: the same for all)
        settle();
        __syncthreads();
    }
    if (static_cast<int>(threadIdx.x >> 5) == alloc_warp) tmem_free<TMEM_COLS>(f.tmem);
}
// ------------------------------------------------------------------ projection to the rank and expansion

struct ApplyArgs {
    const float *scale;
    const int4 *tiles;
    float *v;                               // [T, r] or null
    uint16_t *planes;                       // for the gradients, or null (plane_unit); a slot is a row of a tile, whether the batch has it or not
    const float *v_in;                      // with planes: [T, r], split into v_planes
    uint16_t *v_planes;
    const uint16_t *y_in;                   // null: zeros
    uint16_t *y_out;                        // null: no expansion
    unsigned int *status;
    size_t ldy;
    int T, K, N, r, n_adapters, n_planes;
    int shares;                             // CTAs of a tile
    int stall;                              // test hook: the last step of K is not loaded
};
template <int R, int G>
struct ApplyCfg {
    // a step of 64 of K and one of 64 columns are as long: 128 rows of 128 bytes, and 64 x R weights
    static constexpr int W_STAGE = R * 128, STAGE = TC_ROWS * 128 + W_STAGE, V_BYTES = 2 * TC_ROWS * 2 * R, X_AREA = TC_ROWS * R * 4, X_BYTES = G == 4 ? 2 * X_AREA : G == 2 ? X_AREA : 0,
                         FIT = (232448 - 1024 - CTRL - V_BYTES - X_BYTES) / STAGE, NS = FIT > 10 ? 10 : FIT, THREADS = 320, TMEM = 512, SUMS = R == 64 ? 6 : R == 32 ? 12 : 16,
                         SMEM = 1024 + CTRL + V_BYTES + X_BYTES + NS * STAGE;
};

// V = s x a^T of a tile's 128 rows, then y_out = y_in + V b^T (TRANS: U, and both weights read across their rows).  Warp 8 loads the steps of K
// and behind them y_in and weights of 64 columns at a time, through one ring of stages, so that y is on its way while V is worked out.
// Warp 9 issues.  Warps 0 to 7 take V from tensor memory to the two planes that are the second product's operand, and then each four of
// them every other step of columns: a warp 32 rows, y_in added from the stage and the result put back in its place, from where a TMA
// store takes it (rows of a tile that is not full: plain stores of those that are the tile's).
// `shares` CTAs have a tile's columns between them, and all of them work out V: x comes from L2 for all but the first, while handing V on
// would take a launch, or a meeting, of its own (two launches, 8192 x 768 x 2304, rank 16: 23 us; this: 19.2, 70 % of the memory's rate; 16384 x 4096 x 11008,
// rank 64: 152 us, 86 %).  G > 1: a cluster of G CTAs shares K out and exchanges its sums through each other's shared memory, first with the
// neighbour, then (G = 4) with the other pair.
// Rows behind the tile's end are other requests' or none: every row of the results depends on its own row of x alone, and theirs are not kept.
template <int R, bool TRANS, int G>
__global__ void __launch_bounds__(ApplyCfg<R, G>::THREADS, 1)
lora_apply_tc(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
              const __grid_constant__ CUtensorMap map_in, const __grid_constant__ CUtensorMap map_out, const ApplyArgs in)
{
    using C = ApplyCfg<R, G>;
    extern __shared__ uint8_t smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int BAR_V = 2 * C::NS, BAR_EMPTIED = BAR_V + 2, BAR_READY = BAR_V + 4, BAR_X = BAR_V + 5, BAR_SUMS = BAR_V + 7, BAR_TAKEN = BAR_V + 9, BAR_LEFT = BAR_V + 11;
    const Frame f = begin<C::TMEM>(smem_raw, in.status, in.stall != 0, 9, [&](uint32_t bars) {
        for (int s = 0; s < C::NS; ++s) { mbar_init(bars + 8 * s, 1); mbar_init(bars + 8 * (C::NS + s), 4); }
        for (int b = 0; b < 2; ++b) { mbar_init(bars + 8 * (BAR_V + b), 1); mbar_init(bars + 8 * (BAR_EMPTIED + b), 8); }
        mbar_init(bars + 8 * BAR_READY, 8);
        mbar_init(bars + 8 * BAR_LEFT, 1);
        for (int b = 0; b < 2; ++b) mbar_init(bars + 8 * (BAR_X + b), 1);
        for (int b = 0; b < 2; ++b) { mbar_init(bars + 8 * (BAR_SUMS + b), 1); mbar_init(bars + 8 * (BAR_TAKEN + b), 4); }
        prefetch_map(&map_x);
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        prefetch_map(&map_in);
        prefetch_map(&map_out);
#pragma unroll
        for (int b = 0; b < G / 2; ++b) mbar_expect(bars + 8 * (BAR_X + b), C::X_AREA);
    });
    if (G > 1) cluster_sync();                                 // the other CTAs' barriers are there
    auto bar = [&](int i) { return f.bars + 8 * i; };
    const uint32_t v_at = f.stages, x_at = v_at + C::V_BYTES, stages = x_at + C::X_BYTES;
    ApplyArgs p = in;
    sste_pdl_wait(p.scale, p.tiles, p.v_in, p.y_in);
    sste_pdl_trigger();
    const int t_index = static_cast<int>(blockIdx.x) / p.shares, share = static_cast<int>(blockIdx.x) % p.shares, rank = share & (G - 1);
    const LoraTile tile = lora_tile_of(p.tiles, t_index, TC_ROWS, p.T, p.n_adapters);
    const bool active = tile.rows > 0 && tile.adapter >= 0;
    const int kb_all = (p.K + TC_K - 1) / TC_K, kb0 = kb_all / G * rank + kb_all % G * rank / G,
              kb1 = kb_all / G * (rank + 1) + kb_all % G * (rank + 1) / G, n_k = kb1 - kb0;
    // The tensor core's sums round towards zero: over 172 steps of 64 in one accumulator U was off by 6e-6 of its size.  So an accumulator gets
    // 8 steps at most.  Where that does not do for all, half of the accumulators take a round of steps while the epilogue adds the other half
    // up in registers, so that what is lost does not grow with K.  (16384 x 11008 x 4096, rank 64: all of them emptied at once 118.6 us, so 117, never 115.)
    constexpr int HALF = C::SUMS / 2;
    const bool rounds = n_k > 8 * C::SUMS;
    const int n_sums = rounds ? HALF : (n_k + 7) / 8, round_steps = 8 * (rounds ? HALF : C::SUMS);
    const int chunks = p.y_out ? (p.N + CHUNK - 1) / CHUNK : 0, each = chunks / p.shares, longer = chunks - each * p.shares,
              c0 = share * each + (share < longer ? share : longer), n_c = each + (share < longer ? 1 : 0);
    if (tile.rows > 0 && tile.adapter < 0 && p.y_out && p.y_in != p.y_out) {       // no adapter: the rows as they are
        const int n0 = c0 * CHUNK, n1 = (c0 + n_c) * CHUNK, vecs = ((n1 < p.N ? n1 : p.N) - n0) / 8, all = tile.rows * vecs;
        constexpr int AT_ONCE = 8;                             // loads in flight per thread
        for (int i0 = threadIdx.x; i0 < all; i0 += AT_ONCE * C::THREADS) {
            uint4 v[AT_ONCE];
            size_t at[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int i = i0 + k * C::THREADS;
                at[k] = (static_cast<size_t>(tile.row) + i / vecs) * p.ldy + n0 + 8 * (i % vecs);
                v[k] = p.y_in && i < all ? *reinterpret_cast<const uint4 *>(p.y_in + at[k]) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                if (i0 + k * C::THREADS < all) *reinterpret_cast<uint4 *>(p.y_out + at[k]) = v[k];
        }
    }
    if (active && warp == 8) {
        if (lane == 0) {
            Ring<C::NS> ring;
            bool go = true;
            for (int k = kb0; k < kb1; ++k, ring.next()) {
                if (p.stall && k + 1 == kb1) { go = false; break; }
                if (!(go = f.wait(bar(C::NS + ring.stage), ring.phase ^ 1u))) break;
                const uint32_t dst = stages + ring.stage * C::STAGE, full = bar(ring.stage);
                mbar_expect(full, C::STAGE);
                tma_load_2d(dst, &map_x, full, k * TC_K, tile.row);
                if (TRANS) tma_load_3d(dst + TC_ROWS * 128, &map_a, full, 0, k * TC_K, tile.adapter);
                else tma_load_3d(dst + TC_ROWS * 128, &map_a, full, k * TC_K, 0, tile.adapter);
            }
            const uint32_t bytes = (p.y_in ? TC_ROWS * 128 : 0) + C::W_STAGE;
            for (int c = c0; go && c < c0 + n_c; ++c, ring.next()) {
                if (!f.wait(bar(C::NS + ring.stage), ring.phase ^ 1u)) break;
                const uint32_t dst = stages + ring.stage * C::STAGE, full = bar(ring.stage);
                mbar_expect(full, bytes);
                if (p.y_in) tma_load_2d(dst, &map_in, full, c * CHUNK, tile.row);
                if (TRANS) tma_load_3d(dst + TC_ROWS * 128, &map_b, full, c * CHUNK, 0, tile.adapter);
                else tma_load_3d(dst + TC_ROWS * 128, &map_b, full, 0, c * CHUNK, tile.adapter);
            }
            ring.park(f.bars + CTRL_LOADS);
        }
    } else if (active && warp == 9) {
        if (lane == 0) {
            constexpr uint32_t to_v = instr_desc(false, TRANS, R), to_y = instr_desc(false, TRANS, CHUNK);
            const uint32_t v_acc = f.tmem + 2 * CHUNK;
            Ring<C::NS> ring;
            bool go = true;
            int round = 0;
            for (int k = 0, which = 0, in_round = 0; k < n_k; ++k, ++in_round, ring.next()) {
                if (in_round == round_steps) {
                    tc_commit(bar(BAR_V + (round & 1)));
                    ++round;
                    which = in_round = 0;
                    if (round > 1 && !(go = f.wait(bar(BAR_EMPTIED + (round & 1)), (round >> 1 & 1) ^ 1))) break;
                }
                if (!(go = f.wait(bar(ring.stage), ring.phase))) break;
                tc_after();
                const uint32_t a = stages + ring.stage * C::STAGE, b = a + TC_ROWS * 128, acc = v_acc + (which + (round & 1) * HALF) * R;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint64_t bd = TRANS ? smem_desc(b + 16 * j * (2 * R), 16, 8 * 2 * R, SWIZZLE_OF<R>) : smem_desc(b + 32 * j, 16, 1024, 2);
                    tc_mma(acc, smem_desc(a + 32 * j, 16, 1024, 2), bd, to_v, in_round >= n_sums || j > 0 ? 1u : 0u);
                }
                which = which + 1 == n_sums ? 0 : which + 1;
                // (four arrivals, as the four warps' that free a stage of y)
#pragma unroll
                for (int i = 0; i < 4; ++i) tc_commit(bar(C::NS + ring.stage));
            }
            if (go) tc_commit(bar(BAR_V + (round & 1)));
            if (go && n_c > 0) go = f.wait(bar(BAR_READY), 0);
            for (int c = 0; go && c < n_c; ++c, ring.next()) {
                const uint32_t buf = c & 1, use = c >> 1;
                if (!f.wait(bar(ring.stage), ring.phase) || !f.wait(bar(BAR_TAKEN + buf), (use & 1u) ^ 1u)) break;
                tc_after();
                const uint32_t w = stages + ring.stage * C::STAGE + TC_ROWS * 128;
#pragma unroll
                for (int k = 0; k < R / 16; ++k) {
                    const uint64_t bd = TRANS ? smem_desc(w + 16 * k * 128, 16, 1024, 2) : smem_desc(w + 32 * k, 16, 8 * 2 * R, SWIZZLE_OF<R>);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        tc_mma(f.tmem + CHUNK * buf, smem_desc(v_at + h * (C::V_BYTES / 2) + 32 * k, 16, 8 * 2 * R, SWIZZLE_OF<R>), bd, to_y,
                               k > 0 || h > 0 ? 1u : 0u);
                }
                tc_commit(bar(BAR_SUMS + buf));
            }
        }
    } else if (active) {
        const int half = warp >> 2, row = 32 * (warp & 3) + lane;
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
        const bool in_tile = row < tile.rows;
        const size_t slot = static_cast<size_t>(t_index) * TC_ROWS + row, t = static_cast<size_t>(tile.row) + row;
        const float scale = p.scale[tile.adapter];
        // eight values as two planes' 16 bytes
        auto split8 = [](const float *v, uint4 &hi, uint4 &lo) {
            split2(v[0], v[1], hi.x, lo.x);
            split2(v[2], v[3], hi.y, lo.y);
            split2(v[4], v[5], hi.z, lo.z);
            split2(v[6], v[7], hi.w, lo.w);
        };
        auto keep8 = [&](uint16_t *planes, int c, const float *v, const uint4 &hi, const uint4 &lo) {
            uint4 *to = reinterpret_cast<uint4 *>(planes) + plane_unit<R>(slot, c, p.n_planes);
            to[0] = hi;
            to[CHUNK * R / 8] = lo;
            if (p.n_planes == 3)
                to[2 * (CHUNK * R / 8)] =
                    make_uint4(rest2(v[0], v[1], hi.x, lo.x), rest2(v[2], v[3], hi.y, lo.y), rest2(v[4], v[5], hi.z, lo.z), rest2(v[6], v[7], hi.w, lo.w));
        };
        if (p.planes && share == p.shares - 1 && half == 1) {  // the forward's V for the gradients, while the products run
            const float *from = p.v_in + t * p.r;
#pragma unroll
            for (int c = 0; c < R; c += 8) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 x = in_tile && c < p.r ? *reinterpret_cast<const float4 *>(from + c + i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    v[i] = x.x;
                    v[i + 1] = x.y;
                    v[i + 2] = x.z;
                    v[i + 3] = x.w;
                }
                uint4 hi, lo;
                split8(v, hi, lo);
                keep8(p.v_planes, c, v, hi, lo);
            }
        }
        bool go = true;
        auto read_v = [&](uint32_t from, int n, float *v) {
            tmem_ld16(from, v);
            for (int k = 1; k < n; ++k) {
                float x[16];
                tmem_ld16(from + k * R, x);
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] += x[i];
            }
        };
        // 16 ranks at a time, the first of them warps 0 to 3, the next warps 4 to 7
        constexpr int Q = R == 64 ? 2 : 1;
        float sums[Q][16];
        for (int k = 0, round = 0; k < n_k; k += round_steps, ++round) {
            if (!(go = f.wait.warp(bar(BAR_V + (round & 1)), round >> 1 & 1))) break;
            tc_after();
            const int n = n_k - k < n_sums ? n_k - k : n_sums;              // sums that the round has
#pragma unroll
            for (int q = 0, c = 16 * half; q < Q && c < R; ++q, c += 32) {
                float v[16];
                read_v(f.tmem + 2 * CHUNK + (round & 1) * (HALF * R) + c + lanes, n, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[q][i] = round ? sums[q][i] + v[i] : v[i];
            }
            tc_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(BAR_EMPTIED + (round & 1)));
        }
#pragma unroll
        for (int b = 0; b < G / 2; ++b) {                      // (both sides add the same two numbers: they come to the same bits)
            if (!go) break;
            const uint32_t area = x_at + b * C::X_AREA;
#pragma unroll
            for (int q = 0, c = 16 * half; q < Q && c < R; ++q, c += 32)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    store_async(area + ((c + i) / 4 * TC_ROWS + row) * 16, bar(BAR_X + b), rank ^ (1 << b), sums[q] + i);
            if (!(go = f.wait.warp(bar(BAR_X + b), 0))) break;
#pragma unroll
            for (int q = 0, c = 16 * half; q < Q && c < R; ++q, c += 32)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const uint4 x = lds16(area + ((c + i) / 4 * TC_ROWS + row) * 16);
                    sums[q][i] += __uint_as_float(x.x);
                    sums[q][i + 1] += __uint_as_float(x.y);
                    sums[q][i + 2] += __uint_as_float(x.z);
                    sums[q][i + 3] += __uint_as_float(x.w);
                }
        }
        if (go) {
#pragma unroll
            for (int q = 0, c = 16 * half; q < Q && c < R; ++q, c += 32) {
                float *v = sums[q];
                // (rows that the batch does not have here, and columns that fill the rank up, are zeros whatever x holds)
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = in_tile && c + i < p.r ? scale * v[i] : 0.0f;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint4 hi, lo;
                    split8(v + 8 * e, hi, lo);
                    const int j = c / 8 + e, swz = R == 64 ? row & 7 : R == 32 ? (row >> 1) & 3 : (row >> 2) & 1;
                    const uint32_t at = v_at + row * (2 * R) + ((j ^ swz) << 4);
                    sts16(at, hi);
                    sts16(at + C::V_BYTES / 2, lo);
                    if (p.planes && share == 0) keep8(p.planes, c + 8 * e, v + 8 * e, hi, lo);
                }
                if (p.v && share == 0 && in_tile) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        if (c + i < p.r) *reinterpret_cast<float4 *>(p.v + t * p.r + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
            }
            fence_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(BAR_READY));
        }
        const int rows = tile.rows - 32 * (warp & 3);          // of this warp: all 32 or what the tile has
        uint32_t stage = (n_k + half) % C::NS, phase = (n_k + half) / C::NS & 1u, last_stage = 0;
        bool stored = false;
        for (int c = half; go && c < n_c; c += 2) {
            if (!f.wait.warp(bar(stage), phase) || !f.wait.warp(bar(BAR_SUMS + half), c >> 1 & 1u)) break;
            tc_after();
            const uint32_t box = stages + stage * C::STAGE + 32 * (warp & 3) * 128, mine = box + lane * 128;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                float s[16];
                tmem_ld16(f.tmem + CHUNK * half + 16 * h + lanes, s);
                if (h == 3) {
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(BAR_TAKEN + half));
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t at = mine + (((2 * h + e) ^ (lane & 7)) << 4);
                    const uint4 y = p.y_in ? lds16(at) : make_uint4(0, 0, 0, 0);
                    uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w[i] = pack2(__uint_as_float(w[i] << 16) + s[8 * e + 2 * i], __uint_as_float(w[i] & 0xffff0000u) + s[8 * e + 2 * i + 1]);
                    sts16(at, make_uint4(w[0], w[1], w[2], w[3]));
                }
            }
            const int col = (c0 + c) * CHUNK;
            fence_async();
            __syncwarp();
            if (rows >= 32) {
                if (lane == 0) {
                    tma_store_2d(&map_out, box, col, tile.row + 32 * (warp & 3));
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    // the store before this one has read its stage
                    asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                    if (stored) mbar_arrive(bar(C::NS + last_stage));
                }
                last_stage = stage;
                stored = true;
            } else {
                for (int i = lane; i < rows * 8; i += 32) {
                    const int r = i / 8, e = i % 8;
                    if (col + 8 * e < p.N)
                        *reinterpret_cast<uint4 *>(p.y_out + (static_cast<size_t>(tile.row) + 32 * (warp & 3) + r) * p.ldy + col + 8 * e) =
                            lds16(box + r * 128 + ((e ^ (r & 7)) << 4));
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::NS + stage));
            }
            stage += 2;
            if (stage >= C::NS) { stage -= C::NS; phase ^= 1u; }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    auto settle = [&] {
        if (active && warp == 8 && lane == 0) {
            Ring<C::NS>::settle(f.wait, bar(0), f.bars + CTRL_LOADS);
#pragma unroll
            for (int b = 0; b < G / 2; ++b) f.wait.leaving(bar(BAR_X + b), 0);
        }
        if (active && warp == 9 && lane == 0) {
            tc_commit(bar(BAR_LEFT));
            f.wait.leaving(bar(BAR_LEFT), 0);
        }
    };
    if (G > 1) cluster_sync();                                 // none leaves while another still writes to it
    end<C::TMEM>(f, 9, settle);
}

// ------------------------------------------------------------------ gradients of the weights

struct GradJob {
    const uint8_t *planes;                  // of U or V (plane_unit)
    const uint8_t *codes, *scales;          // the kept form of [T, N], or null: the tensor map's bf16
    void *out;
    int N, blocks;
    bool across;                            // out is [N, r] (dB), not [r, N] (dA)
};
struct GradArgs {
    GradJob job[2];
    const int *first_tile;
    const int4 *tiles;
    float *partial;                         // [CTA][its first sum, its last][MB][R][128]
    unsigned int *tickets, *status;         // a ticket per CTA
    int T, r, n_adapters, n_tiles;
    int stall;                              // test hook: a CTA's last step is not loaded
    int kept_ctas;                          // that restore job 0's z; the others have job 1 (0: all take both jobs' units)
};
constexpr int CONVERTERS = 8;               // warps, and one that copies the codes
constexpr int power_of_two_up(int n) { return n <= 32 ? 32 : n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512; }
// Planes of U and V that a gradient sums over: two (2^-17 of each value) for bf16 results, three (2^-25) for fp32 ones.
template <int R, bool KEPT, int PLANES>
struct GradShape {
    // features of a unit, in 128s: at a rank of 64 two planes are as long per row as 128 features, three take all of tensor memory
    static constexpr int MB = R == 64 && PLANES == 2 ? 2 : 1, COLUMNS = 128 * MB, PER_SM = R == 64 || KEPT || (R == 32 && PLANES == 3) ? 1 : 2;
};
template <int R, bool KEPT, int PLANES>
struct GradCfg {
    static constexpr int MB = GradShape<R, KEPT, PLANES>::MB, COLUMNS = GradShape<R, KEPT, PLANES>::COLUMNS,
                         Z_STAGE = MB * TC_ROWS * 128, PLANE = CHUNK * 2 * R, S_STAGE = PLANES * PLANE,
                         STAGE = Z_STAGE + S_STAGE, NS = !KEPT ? 4 : R == 64 ? 3 : 6, WARPS = 6 + (KEPT ? CONVERTERS + 1 : 0), THREADS = 32 * WARPS,
                         ACC = MB * PLANES * R, TMEM = power_of_two_up(2 * ACC);
    // The tensor core's sums round towards zero, so that terms of one sign lose more with every row: fp32 results leave it after 8 steps (512 rows:
    // 4e-7 of the sum) and are added up in registers; bf16 ones after 128 (8192 rows: 3e-5, a hundredth of a bf16 step) and are added up in
    // the scratch, where a CTA's part of a sum is that long at all.
    static constexpr int DRAIN = PLANES == 3 ? 8 : 128;
    // codes of a step on their way: rows of COLUMNS bytes; then each row's scales in the four-byte words that hold them; then what the row's
    // place in its words starts from, and whether there is a step at all
    static constexpr int WORDS = COLUMNS / 128 + 1, CODES = CHUNK * COLUMNS, SCALES = CHUNK * WORDS * 4, NC = !KEPT ? 0 : R == 64 ? 3 : 4,
                         CODE_STAGE = (CODES + SCALES + 16 + 127) / 128 * 128, SMEM = 1024 + CTRL + NS * STAGE + NC * CODE_STAGE;
};

// The work is a line of steps of 64 rows: block of features after block, in each the tiles of all adapters in their order (the table is sorted by
// adapter).  Each CTA has an equal stretch of it, whatever the sizes.  A sum (a block of features of an adapter) that reaches over the
// ends of stretches is put together from the CTAs' parts, in their order, by the CTA that arrives last; a CTA has two such parts at most, its
// first and its last.  With kept and bf16 features the CTAs are divided between the two jobs.
struct GradLine {
    uint32_t at, end;                       // this CTA's place and the end of its stretch
    uint32_t each, longer;                  // steps of a stretch; so many stretches, the first ones, have one more
    int steps, blocks, first_block, cta, ctas, cta0;
    __device__ __forceinline__ GradLine(const GradArgs &p)
    {
        const int c = static_cast<int>(blockIdx.x), n = static_cast<int>(gridDim.x);
        const bool apart = p.kept_ctas > 0, kept = c < p.kept_ctas;
        cta0 = apart && !kept ? p.kept_ctas : 0;
        cta = c - cta0;
        ctas = !apart ? n : kept ? p.kept_ctas : n - p.kept_ctas;
        first_block = apart && !kept ? p.job[0].blocks : 0;
        blocks = !apart ? p.job[0].blocks + p.job[1].blocks : kept ? p.job[0].blocks : p.job[1].blocks;
        const int tiles = p.first_tile[p.n_adapters];
        steps = tiles < 0 || tiles > p.n_tiles ? 0 : 2 * tiles;
        const uint32_t total = static_cast<uint32_t>(blocks) * static_cast<uint32_t>(steps);       // (the host has seen to 31 bits)
        // (no CTA in a sum's row of CTAs may be without a step: it would be waited for)
        if (static_cast<uint32_t>(ctas) > total) ctas = static_cast<int>(total);
        at = end = 0;
        if (cta >= ctas) return;
        each = total / ctas;
        longer = total - each * ctas;
        at = start_of(cta);
        end = start_of(cta + 1);
    }
    __device__ __forceinline__ uint32_t start_of(uint32_t c) const { return c * each + (c < longer ? c : longer); }
    __device__ __forceinline__ int cta_of(uint32_t place) const
    {
        const uint32_t n = longer * (each + 1);
        return static_cast<int>(place < n ? place / (each + 1) : longer + (place - n) / each);
    }
};
// A CTA's next part of a sum: steps s0 .. s1 - 1 (a step: half a tile) of one adapter and block.
struct GradPart {
    int adapter, block, s0, s1;
    uint32_t sum_from, sum_to;              // the sum's place on the line
    bool second;
    struct Step { int row, rows, slot; };   // rows 0: the step is left out by every role
    __device__ __forceinline__ bool next(const GradArgs &p, GradLine &line)
    {
        while (line.at < line.end) {
            const uint32_t b = line.at / line.steps, base = b * line.steps;
            s0 = static_cast<int>(line.at - base);
            adapter = p.tiles[s0 / 2].z;
            // (a table that is not the library's own: steps without an adapter are passed over)
            int from = 0, to = 0;
            if (adapter >= 0 && adapter < p.n_adapters) { from = 2 * p.first_tile[adapter]; to = 2 * p.first_tile[adapter + 1]; }
            if (from < 0 || to > line.steps || s0 < from || s0 >= to) { ++line.at; continue; }
            sum_from = base + from;
            sum_to = base + to;
            const uint32_t stop = sum_to < line.end ? sum_to : line.end;
            s1 = static_cast<int>(stop - base);
            block = line.first_block + static_cast<int>(b);
            second = block >= p.job[0].blocks;
            if (second) block -= p.job[0].blocks;
            line.at = stop;
            return true;
        }
        return false;
    }
    __device__ __forceinline__ Step step(const GradArgs &p, int s) const
    {
        if (s >= s1) return Step{0, 0, 0};
        const int half = CHUNK * (s & 1);
        const LoraTile tile = lora_tile_of(p.tiles, s / 2, TC_ROWS, p.T, p.n_adapters);
        const int rows = tile.adapter == adapter ? tile.rows - half : 0;
        return Step{tile.row + half, rows < 0 ? 0 : rows < CHUNK ? rows : CHUNK, s / 2 * TC_ROWS + half};
    }
};

// out = z^T s over the rows of an adapter: z 64 rows x 128 features (two boxes of 64), the planes of s side by side as the instruction's
// second operand, all with rows along the reduction; the sums over the planes are added in the end.  The next part's loads and products run
// while one's sums are stored.  A step's rows behind the tile's end are other requests' or none and may hold anything: they are overwritten
// with zeros before the product (s is zero there, but zero times an infinity is not).
// Measured: 8192 x (768 + 2304), rank 16, 17.2 us (7.7 at the copy rate; launch, first loads and the joining of the sums in the end are some 9);
// 16384 x (4096 + 11008), rank 64, 98 us (77 %); with X kept in 8 bits 125, a kept step taking twice a bf16 one's time: its restoring
// warps convert 64 x 256 codes in a step's time.  4064 x (1280 + 5120), rank 24, five of eight adapters in use: 18.6 us, 20.5 with fp32 results,
// 23 and 25 with X kept.  (Twice the features to a unit, with one CTA an SM, read the planes half as often: 8192 rows 20.5 us, 4064 rows
// 29.  z's first loads started before the kernel in front ends: they take the memory from it, 33.6 us became 34.3 for both.)
// Warps 0 to 3 store, 4 loads, 5 issues.  Of a kept z, warp 14 has codes and scales copied to shared memory, and warps 6 to 13 restore them from
// there into the stage.  (With the loads in the restoring warps' registers, each step's fence towards the tensor core waited for the
// loads of the steps ahead: 1.4 us a step.)
template <int R, int FMT, typename OUT>
__global__ void __launch_bounds__(GradCfg<R, FMT >= 0, sizeof(OUT) == 4 ? 3 : 2>::THREADS, GradShape<R, FMT >= 0, sizeof(OUT) == 4 ? 3 : 2>::PER_SM)
lora_grad_tc(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_codes,
             const GradArgs in)
{
    constexpr bool KEPT_X = FMT >= 0;
    constexpr int PLANES = sizeof(OUT) == 4 ? 3 : 2;
    using C = GradCfg<R, KEPT_X, PLANES>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ bool is_last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Frame f = begin<C::TMEM>(smem_raw, in.status, in.stall != 0, 5, [&](uint32_t bars) {
        // full: the bytes of a stage, and the converters where z is kept
        for (int s = 0; s < C::NS; ++s) { mbar_init(bars + 8 * s, KEPT_X && static_cast<int>(blockIdx.x) < in.kept_ctas ? 1 + CONVERTERS : 1); mbar_init(bars + 8 * (C::NS + s), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(bars + 8 * (2 * C::NS + b), 1); mbar_init(bars + 8 * (2 * C::NS + 2 + b), 4); }
        for (int s = 0; s < C::NC; ++s) { mbar_init(bars + 256 + 8 * s, 33); mbar_init(bars + 256 + 8 * (C::NC + s), CONVERTERS); }
        mbar_init(bars + 8 * (2 * C::NS + 4), 1);
        prefetch_map(&map_x);
        prefetch_map(&map_y);
    });
    const uint32_t full = f.bars, empty = f.bars + 8 * C::NS, sums = f.bars + 8 * 2 * C::NS, taken = sums + 16, left = taken + 16;
    GradArgs p = in;
    sste_pdl_wait(p.job[0].codes, p.job[0].scales, p.first_tile, p.tiles);
    sste_pdl_trigger();
    if (warp == 4) {
        if (lane == 0) {
            Ring<C::NS> ring;
            bool go = true;
            GradLine line(p);
            for (GradPart u; go && u.next(p, line);) {
                const CUtensorMap *z = u.second ? &map_y : &map_x;
                const bool kept = KEPT_X && !u.second;
                GradPart::Step next = u.step(p, u.s0);
                for (int s = u.s0; s < u.s1; ++s) {
                    const GradPart::Step now = next;
                    next = u.step(p, s + 1);
                    if (now.rows == 0) continue;
                    if (p.stall && s + 1 == u.s1 && line.at == line.end) { go = false; break; }
                    if (!f.wait(empty + 8 * ring.stage, ring.phase ^ 1u)) { go = false; break; }
                    const uint32_t dst = f.stages + ring.stage * C::STAGE, bar = full + 8 * ring.stage;
                    mbar_expect(bar, kept ? C::S_STAGE : C::STAGE);
                    if (!kept) {
#pragma unroll
                        for (int c = 0; c < 2 * C::MB; ++c) tma_load_2d(dst + c * (CHUNK * 128), z, bar, u.block * C::COLUMNS + c * CHUNK, now.row);
                    }
                    bulk_load(dst + C::Z_STAGE, (u.second ? p.job[1] : p.job[0]).planes + static_cast<size_t>(now.slot / CHUNK) * C::S_STAGE, C::S_STAGE, bar);
                    ring.next();
                }
            }
            ring.park(f.bars + CTRL_LOADS);
        }
    } else if (warp == 5) {
        constexpr uint32_t idesc = instr_desc(true, true, PLANES * R);
        Ring<C::NS> ring;
        int n = 0;
        bool go = true;
        GradLine line(p);
        for (GradPart u; go && u.next(p, line);) {
            GradPart::Step next = u.step(p, u.s0);
            for (int from = u.s0, s = u.s0; go && from < u.s1; from += C::DRAIN, ++n) {
                const uint32_t acc = f.tmem + (n & 1) * C::ACC;
                if (!(go = f.wait.warp(taken + 8 * (n & 1), ((n >> 1) & 1u) ^ 1u))) break;
                tc_after();
                uint32_t accumulate = 0;
                for (; s < u.s1 && s < from + C::DRAIN; ++s) {
                    const GradPart::Step now = next;
                    next = u.step(p, s + 1);
                    if (now.rows == 0) continue;
                    if (!f.wait.warp(full + 8 * ring.stage, ring.phase)) { go = false; break; }
                    tc_after();
                    const uint32_t z = f.stages + ring.stage * C::STAGE, b = z + C::Z_STAGE;
                    if ((!KEPT_X || u.second) && now.rows < CHUNK) {
                        // (four rows at a time; a quotient by the number of rows in this loop made a step 3 us longer)
                        for (int r = now.rows + lane / 8; r < CHUNK; r += 4)
#pragma unroll
                            for (int c = 0; c < 2 * C::MB; ++c) sts16(z + c * (CHUNK * 128) + r * 128 + lane % 8 * 16, make_uint4(0, 0, 0, 0));
                        fence_async();
                        __syncwarp();
                    }
                    if (lane == 0) {
#pragma unroll
                        for (int m = 0; m < C::MB; ++m)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                tc_mma(acc + m * PLANES * R, smem_desc(z + m * (2 * CHUNK * 128) + 16 * j * 128, CHUNK * 128, 1024, 2),
                                       smem_desc(b + 16 * j * (2 * R), C::PLANE, 8 * 2 * R, SWIZZLE_OF<R>), idesc, accumulate | (j > 0 ? 1u : 0u));
                        tc_commit(empty + 8 * ring.stage);
                    }
                    accumulate = 1u;
                    ring.next();
                }
                __syncwarp();
                if (go && lane == 0) tc_commit(sums + 8 * (n & 1));
            }
        }
    } else if (KEPT_X && warp >= 6) {
        const uint32_t code_full = f.bars + 256, code_empty = code_full + 8 * C::NC, code_stages = f.stages + C::NS * C::STAGE;
        const GradJob &job = p.job[0];
        Ring<C::NC ? C::NC : 1> codes;
        if (static_cast<int>(blockIdx.x) >= p.kept_ctas) {
        } else if (warp == 6 + CONVERTERS) {
            const size_t n_scales = (static_cast<size_t>(p.T) * job.N + 31) / 32;
            const bool wide = job.N % 16 == 0;
            bool go = true;
            auto announce = [&](uint32_t dst, uint32_t place, uint32_t rows, uint32_t bytes) {
                asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(code_full + 8 * codes.stage) : "memory");
                if (lane == 0) {
                    asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dst + C::CODES + C::SCALES), "r"(place), "r"(rows) : "memory");
                    mbar_expect(code_full + 8 * codes.stage, bytes);
                }
                codes.next();
            };
            GradLine line(p);
            for (GradPart u; go && u.next(p, line);) {
                const int n0 = u.block * C::COLUMNS;
                GradPart::Step next = u.step(p, u.s0);
                for (int s = u.s0; s < u.s1; ++s) {
                    const GradPart::Step now = next;
                    next = u.step(p, s + 1);
                    if (now.rows == 0) continue;
                    if (!f.wait.warp(code_empty + 8 * codes.stage, codes.phase ^ 1u)) { go = false; break; }
                    const uint32_t dst = code_stages + codes.stage * C::CODE_STAGE;
                    const size_t at = static_cast<size_t>(now.row) * job.N + n0;
                    if (!wide) {                               // (rows that the copy engine has no map for; what is not there: zeros)
                        constexpr int PER_ROW = C::COLUMNS / 8;
#pragma unroll 8
                        for (int i = lane; i < CHUNK * PER_ROW; i += 32) {
                            const int r = i / PER_ROW, c = i % PER_ROW * 8;
                            const bool in = r < now.rows && n0 + c < job.N;
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst + 8 * i),
                                         "l"(in ? job.codes + at + static_cast<size_t>(r) * job.N + c : job.codes), "r"(in ? 8 : 0)
                                         : "memory");
                        }
                    }
#pragma unroll
                    for (int i = lane; i < CHUNK * C::WORDS; i += 32) {
                        const int r = i / C::WORDS;
                        const size_t word = (at + static_cast<size_t>(r) * job.N) / 128 * 4 + 4 * (i % C::WORDS);
                        const int size = r >= now.rows || word >= n_scales ? 0 : n_scales - word < 4 ? static_cast<int>(n_scales - word) : 4;
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + C::CODES + 4 * i),
                                     "l"(size ? job.scales + word : job.scales), "r"(size)
                                     : "memory");
                    }
                    const uint32_t bar = code_full + 8 * codes.stage;
                    announce(dst, static_cast<uint32_t>(at) & 127u, static_cast<uint32_t>(now.rows), wide ? C::CODES : 0u);
                    if (wide && lane == 0) tma_load_2d(dst, &map_codes, bar, n0, now.row);
                }
            }
            if (go && f.wait.warp(code_empty + 8 * codes.stage, codes.phase ^ 1u)) announce(code_stages + codes.stage * C::CODE_STAGE, 0u, 0u, 0u);
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (lane == 0) codes.park(f.bars + CTRL_CODES);
        } else {
            // eight codes to a thread at a time: a row of a box is 128 bytes, its 16-byte parts swizzled with the row
            constexpr int PER_ROW = C::COLUMNS / 8, ROWS_AT_ONCE = 32 * CONVERTERS / PER_ROW, N = CHUNK / ROWS_AT_ONCE;
            const int t = static_cast<int>(threadIdx.x) - 192, part = t % PER_ROW, row0 = t / PER_ROW;
            Ring<C::NS> ring;
            while (true) {
                if (!f.wait.warp(code_full + 8 * codes.stage, codes.phase)) break;
                const uint32_t from = code_stages + codes.stage * C::CODE_STAGE;
                uint32_t place0, rows;                         // of the step's first row in its words of scales; 0 rows: the end
                asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(place0), "=r"(rows) : "r"(from + C::CODES + C::SCALES) : "memory");
                if (rows == 0 || !f.wait.warp(empty + 8 * ring.stage, ring.phase ^ 1u)) break;
                const uint32_t z = f.stages + ring.stage * C::STAGE + part / 8 * (CHUNK * 128) + row0 * 128;
                uint2 q[N];
                uint32_t e[N], w[N][4], nans = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) {                  // (all loads, then all stores: neither is moved past the other)
                    const int r = row0 + i * ROWS_AT_ONCE;
                    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(q[i].x), "=r"(q[i].y) : "r"(from + r * C::COLUMNS + 8 * part));
                    const uint32_t place = (place0 + static_cast<uint32_t>(r) * static_cast<uint32_t>(job.N)) & 127u;
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(e[i]) : "r"(from + C::CODES + 4 * C::WORDS * r + (place + 8 * part) / 32));
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    // rows behind the tile's end are other requests' or none
                    const bool there = row0 + i * ROWS_AT_ONCE < static_cast<int>(rows);
                    q[i] = there ? q[i] : make_uint2(0u, 0u);
                    e[i] = there ? e[i] : 0u;
                    lora_restore8<FMT == SSTE_CKPT_E4M3>(q[i], e[i], w[i], nans);
                }
                if (lora_has_nan<FMT == SSTE_CKPT_E4M3>(nans)) {
#pragma unroll
                    for (int i = 0; i < N; ++i) lora_put_nans<FMT == SSTE_CKPT_E4M3>(q[i], w[i]);
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sts16(z + i * (ROWS_AT_ONCE * 128) + (((part & 7) ^ ((row0 + i * ROWS_AT_ONCE) & 7)) << 4), make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]));
                fence_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(full + 8 * ring.stage);
                    mbar_arrive(code_empty + 8 * codes.stage);
                }
                ring.next();
                codes.next();
            }
        }
    } else {
        const int col_in = 32 * warp + lane;                   // of 128
        // Adapters without rows: zeros, a slice of 32 KB to a CTA at a time while the first steps are on their way.  (An adapter to a CTA, behind its sums:
        // three of eight adapters of 1280 x 5120 at a rank of 24 made a call of 20 us one of 31.)
        constexpr uint32_t SLICE = 2048;                       // in 16 bytes
        const uint32_t vecs0 = static_cast<uint32_t>(p.r / 8 * p.job[0].N) * static_cast<uint32_t>(sizeof(OUT) / 2),
                       vecs1 = static_cast<uint32_t>(p.r / 8 * p.job[1].N) * static_cast<uint32_t>(sizeof(OUT) / 2),
                       slices0 = (vecs0 + SLICE - 1) / SLICE, slices = slices0 + (vecs1 + SLICE - 1) / SLICE;
        for (uint32_t a = blockIdx.x / slices, k = blockIdx.x - a * slices; a < static_cast<uint32_t>(p.n_adapters);) {
            if (p.first_tile[a] == p.first_tile[a + 1]) {
                const bool second = k >= slices0;              // (an index into the jobs would put the arguments into local memory)
                const uint32_t n = second ? vecs1 : vecs0, from = (second ? k - slices0 : k) * SLICE, to = from + SLICE < n ? from + SLICE : n;
                uint4 *out = static_cast<uint4 *>(second ? p.job[1].out : p.job[0].out) + static_cast<size_t>(a) * n;
                for (uint32_t i = from + threadIdx.x; i < to; i += 128) out[i] = make_uint4(0, 0, 0, 0);
            }
            k += gridDim.x;
            const uint32_t more = k / slices;
            a += more;
            k -= more * slices;
        }
        int n = 0;
        GradLine line(p);
        for (GradPart u; u.next(p, line);) {
            const GradJob job = u.second ? p.job[1] : p.job[0];
            // the sum's parts, and where they are: a CTA's last one, unless its stretch begins with the sum
            const int first_cta = line.cta_of(u.sum_from), parts = line.cta_of(u.sum_to - 1) - first_cta + 1;
            const int first_slot = 2 * (line.cta0 + first_cta) + (u.sum_from > line.start_of(first_cta) ? 1 : 0), own = line.cta - first_cta;
            unsigned int *ticket = p.tickets + line.cta0 + first_cta;
            // The first of two parts (a CTA's last sum, whose other part is the next CTA's first and there long before): it does not go through the
            // scratch, this CTA adds the other to it as it puts it out.
            bool alone = false;
            if (parts == 2 && own == 0) {
                if (threadIdx.x == 0) {
                    is_last = *reinterpret_cast<volatile unsigned int *>(ticket) == 1u;
                    __threadfence();
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");
                alone = is_last;
                asm volatile("bar.sync 1, 128;" ::: "memory");
            }
            auto slot = [&](int k) { return k == 0 ? first_slot : 2 * (line.cta0 + first_cta + k); };
            // what this part comes to: a thread's ranks in registers where the accumulator is emptied more than once
            float *shared = p.partial + col_in;
            constexpr size_t PART = C::MB * R * 128;
            OUT *out = static_cast<OUT *>(job.out) + static_cast<size_t>(u.adapter) * p.r * job.N;
            auto put = [&](int m, int c, const float *v) {     // ranks c .. c + 15 of feature col_in of block m
                const int col = u.block * C::COLUMNS + 128 * m + col_in;
                if (col >= job.N) return;
                if (job.across) {
                    OUT *to = out + static_cast<size_t>(col) * p.r + c;
#pragma unroll
                    for (int i = 0; i < 16; i += 8) {
                        if (c + i >= p.r) break;
                        if constexpr (sizeof(OUT) == 2) {
                            *reinterpret_cast<uint4 *>(to + i) = make_uint4(pack2(v[i], v[i + 1]), pack2(v[i + 2], v[i + 3]),
                                                                            pack2(v[i + 4], v[i + 5]), pack2(v[i + 6], v[i + 7]));
                        } else {
                            *reinterpret_cast<float4 *>(to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                            *reinterpret_cast<float4 *>(to + i + 4) = make_float4(v[i + 4], v[i + 5], v[i + 6], v[i + 7]);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (c + i >= p.r) break;
                        OUT *to = out + static_cast<size_t>(c + i) * job.N + col;
                        if constexpr (sizeof(OUT) == 2) *to = __float2bfloat16_rn(v[i]);
                        else *to = v[i];
                    }
                }
            };
            auto leave = [&](int m, int c, const float *v) {
                if (parts == 1) {
                    put(m, c, v);
                } else if (alone) {
                    const float *from = shared + slot(1) * PART + (m * R + c) * 128;
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = __ldcg(from + i * 128);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = v[i] + x[i];
                    put(m, c, x);
                } else {
                    float *to = shared + slot(own) * PART;
#pragma unroll
                    for (int i = 0; i < 16; ++i) __stcg(to + (m * R + c + i) * 128, v[i]);
                }
            };
            auto read = [&](uint32_t acc, int m, int c, bool any, float *v) {
                float x[16];
                tmem_ld16(acc + m * PLANES * R + (PLANES - 1) * R + c, v);
#pragma unroll
                for (int h = PLANES - 2; h >= 0; --h) {        // the smallest first
                    tmem_ld16(acc + m * PLANES * R + h * R + c, x);
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] += x[i];
                }
                if (!any) {                                    // (nothing was added up)
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = 0.0f;
                }
            };
            float total[PLANES == 3 ? R : 1] = {};
            bool go = true;
            for (int from = u.s0; from < u.s1; from += C::DRAIN, ++n) {
                bool any = false;
                for (int s = from; s < u.s1 && s < from + C::DRAIN && !any; ++s) any = u.step(p, s).rows > 0;
                if (!(go = f.wait.warp(sums + 8 * (n & 1), (n >> 1) & 1u))) break;
                tc_after();
                const uint32_t acc = f.tmem + (n & 1) * C::ACC + (static_cast<uint32_t>(32 * warp) << 16);
                if constexpr (PLANES == 3) {
#pragma unroll
                    for (int c = 0; c < R; c += 16) {
                        float v[16];
                        read(acc, 0, c, any, v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) total[c + i] += v[i];
                    }
                } else {
                    // (a thread finds what it has itself left there)
                    float *so_far = shared + slot(own) * PART;
#pragma unroll 1
                    for (int m = 0; m < C::MB; ++m)
#pragma unroll 1
                        for (int c = 0; c < R; c += 16) {
                            float v[16];
                            read(acc, m, c, any, v);
                            if (from > u.s0) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) v[i] += __ldcg(so_far + (m * R + c + i) * 128);
                            }
                            if (from + C::DRAIN >= u.s1) {
                                leave(m, c, v);
                            } else {
#pragma unroll
                                for (int i = 0; i < 16; ++i) __stcg(so_far + (m * R + c + i) * 128, v[i]);
                            }
                        }
                }
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(taken + 8 * (n & 1));
            }
            if (!all_of_four_warps(go)) break;                 // (together: the barriers below are for all of them)
            if constexpr (PLANES == 3) {
#pragma unroll
                for (int c = 0; c < R; c += 16) leave(0, c, total + c);
            }
            if (parts == 1) continue;
            if (alone) {
                if (threadIdx.x == 0) *ticket = 0;             // as it was found
                continue;
            }
            __threadfence();
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (threadIdx.x == 0) is_last = atomicAdd(ticket, 1u) == static_cast<unsigned int>(parts - 1);
            asm volatile("bar.sync 1, 128;" ::: "memory");
            const bool last = is_last;
            asm volatile("bar.sync 1, 128;" ::: "memory");     // (before the next unit's)
            if (!last) continue;
            __threadfence();
            if (threadIdx.x == 0) *ticket = 0;
#pragma unroll 1
            for (int m = 0; m < C::MB; ++m)
#pragma unroll 1
                for (int c = 0; c < R; c += 16) {
                    float v[16];
                    constexpr int AT_ONCE = 6;                 // parts whose loads are on their way together
                    for (int k0 = 0; k0 < parts; k0 += AT_ONCE) {
                        float x[AT_ONCE][16];
#pragma unroll
                        for (int k = 0; k < AT_ONCE; ++k) {
                            const float *from = shared + slot(k0 + k < parts ? k0 + k : 0) * PART + (m * R + c) * 128;
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[k][i] = __ldcg(from + i * 128);
                        }
#pragma unroll
                        for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = k0 + k == 0 ? x[0][i] : k0 + k < parts ? v[i] + x[k][i] : v[i];
                    }
                    put(m, c, v);
                }
        }
    }
    __syncwarp();
    end<C::TMEM>(f, 5, [&] {
        if (warp == 4 && lane == 0) Ring<C::NS>::settle(f.wait, full, f.bars + CTRL_LOADS);
        if (warp == 5 && lane == 0) {
            tc_commit(left);
            f.wait.leaving(left, 0);
        }
        if (KEPT_X && warp == 6 + CONVERTERS && lane == 0) Ring<C::NC ? C::NC : 1>::settle(f.wait, f.bars + 256, f.bars + CTRL_CODES);
    });
}

// ------------------------------------------------------------------ host

int g_stall = 0;                            // test hook, see sste_debug_lora_stall

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

// bf16 tensor of two or three dimensions, innermost first; strides in elements.
bool make_map(const sste_ctx *ctx, CUtensorMap *map, const void *base, int rank, uint64_t d0, uint64_t d1, uint64_t d2, uint64_t s1, uint64_t s2,
              uint32_t b0, uint32_t b1)
{
    const cuuint64_t dims[3] = {d0, d1, d2}, strides[2] = {2 * s1, 2 * s2};
    const cuuint32_t box[3] = {b0, b1, 1}, estr[3] = {1, 1, 1};
    const CUtensorMapSwizzle swz = b0 == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : b0 == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
    return reinterpret_cast<EncodeTiledFn>(ctx->cu_tensor_map_encode)(
               map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, static_cast<cuuint32_t>(rank), const_cast<void *>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, swz, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The codes of a kept X [T, I], rows of bytes; without them any valid map.
bool make_codes_map(const sste_ctx *ctx, CUtensorMap *map, const LoraTcCall &c, uint32_t columns, bool there)
{
    if (!there) return make_map(ctx, map, c.x, 2, c.l->O, c.p->T, 1, c.ldx, 1, CHUNK, CHUNK);
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(c.l->I), static_cast<cuuint64_t>(c.p->T)}, strides[1] = {static_cast<cuuint64_t>(c.l->I)};
    const cuuint32_t box[2] = {columns, CHUNK}, estr[2] = {1, 1};
    return reinterpret_cast<EncodeTiledFn>(ctx->cu_tensor_map_encode)(
               map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(c.X_codes), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// CTAs of a gradient kernel: one or two an SM, each with a stretch of four steps or more.
int grad_ctas(int I, int O, int R, int n_tiles, bool f32, bool kept)
{
    const int columns = R == 64 && !f32 ? 256 : 128, slots = (R == 64 || kept || (R == 32 && f32) ? 1 : 2) * LR_SMS;
    const long long steps = 2ll * n_tiles * ((I + columns - 1) / columns + (O + columns - 1) / columns), ctas = (steps + 3) / 4;
    // (whole numbers of CTAs to a block of one adapter leave every sum's parts in as many CTAs: taken where they nearly fill the GPU)
    const int blocks = (I + columns - 1) / columns + (O + columns - 1) / columns, whole = blocks <= slots ? slots / blocks * blocks : 0;
    return static_cast<int>(ctas < 2 ? 2 : ctas < slots ? ctas : 20 * whole >= 19 * slots ? whole : slots);
}

template <typename K>
bool big_smem(const sste_ctx *ctx, K kern, int bytes, DeviceOnce &once)
{
    return once.run(ctx->device, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess; });
}

// CTAs to a tile, about one CTA an SM, and how many of them share K.  Counted in steps of 64 of K or of y (0.3 us each); an exchange of sums costs about
// four.  Only 33 clusters of four run at a time (of two: 74), and one more waits for a whole tile's time, so of those no more are made.
// (2048 rows, K 11008, N 4096, rank 64: 40.7 us in pairs, 30.0 in fours; 1500 rows, K 1280, N 5120, rank 32: 14.1 and 25.1.)
constexpr int LR_QUADS = 32;
struct Shares { int n, group; };
Shares shares_of(int T, int n_tiles, int K, int N)
{
    const int chunks = (N + CHUNK - 1) / CHUNK, steps = (K + TC_K - 1) / TC_K;
    // (counted by rows: a tile at a request's end stores less than a full one, but is loaded like one, so this counts it as too little)
    const int full = (T + TC_ROWS - 1) / TC_ROWS, tiles = full < n_tiles ? full : n_tiles;
    int n = tiles > 0 ? LR_SMS / tiles : 1;
    n = n < 1 ? 1 : n > chunks ? chunks : n;
    // (in a cluster everyone reads its own part of K once; alone, or as one of two clusters, x and A come again from L2, at some 8 TB/s for all SMs)
    Shares best{n, 1};
    float least = steps + static_cast<float>(chunks) / n;
    for (int g = 2; g <= 4 && g <= n; g *= 2) {
        const int room = g == 4 && n_tiles > 0 ? 4 * LR_QUADS / n_tiles : n, m = (n < room ? n : room) / g * g;
        if (m == 0) continue;
        const float cost = static_cast<float>(steps) / g + static_cast<float>(chunks) / m + (g == 2 ? 4.0f : 8.0f);
        if (cost < least) { best = Shares{m, g}; least = cost; }
    }
    return best;
}

template <int R, bool TRANS, int G>
sste_status apply_launch(const sste_ctx *ctx, const LoraTcCall &c, int K, int N, const void *a, const void *b, int shares, cudaStream_t stream)
{
    using C = ApplyCfg<R, G>;
    const sste_lora *l = c.l;
    const uint64_t r = l->rank, n = l->n_adapters;
    CUtensorMap mx, ma, mb, mi, mo;
    const bool y = c.y_out != nullptr;
    if (!make_map(ctx, &mx, c.x, 2, K, c.p->T, 1, c.ldx, 1, TC_K, TC_ROWS) ||
        !(TRANS ? make_map(ctx, &ma, a, 3, r, K, n, r, r * K, R, TC_K) : make_map(ctx, &ma, a, 3, K, r, n, K, r * K, TC_K, R)) ||
        !(TRANS ? make_map(ctx, &mb, b, 3, N, r, n, N, r * N, CHUNK, R) : make_map(ctx, &mb, b, 3, r, N, n, r, r * N, R, CHUNK)) ||
        !make_map(ctx, &mi, !y ? c.x : c.y_in ? c.y_in : c.y_out, 2, y ? N : K, c.p->T, 1, y ? c.ldy : c.ldx, 1, CHUNK, TC_ROWS) ||
        !make_map(ctx, &mo, !y ? c.x : c.y_out, 2, y ? N : K, c.p->T, 1, y ? c.ldy : c.ldx, 1, CHUNK, 32))
        return SSTE_ERR_CUDA;
    const ApplyArgs args{l->scale, c.tiles, c.v_out, c.grads ? static_cast<uint16_t *>(c.planes) : nullptr, c.v_in,
                         static_cast<uint16_t *>(c.v_planes), static_cast<const uint16_t *>(c.y_in), static_cast<uint16_t *>(c.y_out),
                         ctx->status_dev, c.ldy, c.p->T, K, N, l->rank, l->n_adapters, c.gdt == SSTE_F32 ? 3 : 2, shares, g_stall == 1};
    auto *kern = lora_apply_tc<R, TRANS, G>;
    static DeviceOnce once;
    if (!big_smem(ctx, kern, C::SMEM, once)) return SSTE_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(c.p->n_tiles) * shares);
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = G;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = G > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, mx, ma, mb, mi, mo, args) == cudaSuccess ? SSTE_OK : SSTE_ERR_CUDA;
}
template <int R, bool TRANS>
sste_status apply(const sste_ctx *ctx, const LoraTcCall &c, int K, int N, const void *a, const void *b, cudaStream_t stream)
{
    const Shares s = shares_of(c.p->T, c.p->n_tiles, K, c.y_out ? N : 2 * CHUNK);
    return s.group == 4 ? apply_launch<R, TRANS, 4>(ctx, c, K, N, a, b, s.n, stream)
         : s.group == 2 ? apply_launch<R, TRANS, 2>(ctx, c, K, N, a, b, s.n, stream)
                        : apply_launch<R, TRANS, 1>(ctx, c, K, N, a, b, s.n, stream);
}

// `first` launches the kernel in front, when nothing but a launch can fail any more: a call that is refused has added nothing to dX.
template <int R, int FMT, typename OUT, typename F>
sste_status grad_launch(const sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream, F first)
{
    constexpr bool kept = FMT >= 0;
    constexpr int PLANES = sizeof(OUT) == 4 ? 3 : 2;
    using C = GradCfg<R, kept, PLANES>;
    const sste_lora *l = c.l;
    CUtensorMap x, y, codes;
    if (!make_codes_map(ctx, &codes, c, C::COLUMNS, kept && l->I % 16 == 0)) return SSTE_ERR_CUDA;
    if (!make_map(ctx, &y, c.x, 2, l->O, c.p->T, 1, c.ldx, 1, CHUNK, CHUNK) ||
        !(kept ? make_map(ctx, &x, c.x, 2, l->O, c.p->T, 1, c.ldx, 1, CHUNK, CHUNK)          // (not used)
               : make_map(ctx, &x, c.X, 2, l->I, c.p->T, 1, c.ldX, 1, CHUNK, CHUNK)))
        return SSTE_ERR_CUDA;
    GradArgs a{};
    a.job[0] = GradJob{static_cast<const uint8_t *>(c.planes), static_cast<const uint8_t *>(c.X_codes), static_cast<const uint8_t *>(c.X_scales), c.dA, l->I,
                       (l->I + C::COLUMNS - 1) / C::COLUMNS, false};
    a.job[1] = GradJob{static_cast<const uint8_t *>(c.v_planes), nullptr, nullptr, c.dB, l->O, (l->O + C::COLUMNS - 1) / C::COLUMNS, true};
    a.first_tile = c.first_tile;
    a.tiles = c.tiles;
    a.partial = c.partial;
    a.tickets = c.tickets + LR_TICKETS;
    a.status = ctx->status_dev;
    a.T = c.p->T;
    a.r = l->rank;
    a.n_adapters = l->n_adapters;
    a.n_tiles = c.p->n_tiles;
    a.stall = g_stall == 2;
    const int ctas = grad_ctas(l->I, l->O, R, c.p->n_tiles, PLANES == 3, kept);
    // a step of the kept form takes about twice a bf16 step's time
    if (kept) {
        a.kept_ctas = static_cast<int>(2.0 * a.job[0].blocks * ctas / (2.0 * a.job[0].blocks + a.job[1].blocks) + 0.5);
        a.kept_ctas = a.kept_ctas < 1 ? 1 : a.kept_ctas > ctas - 1 ? ctas - 1 : a.kept_ctas;
    }
    auto *kern = lora_grad_tc<R, FMT, OUT>;
    static DeviceOnce once;
    if (!big_smem(ctx, kern, C::SMEM, once)) return SSTE_ERR_CUDA;
    const sste_status st = first();
    if (st != SSTE_OK) return st;
    return sste_launch(kern, dim3(static_cast<unsigned>(ctas)), dim3(C::THREADS), C::SMEM, stream, x, y, codes, a) == cudaSuccess
               ? SSTE_OK : SSTE_ERR_CUDA;
}
template <int R, typename F>
sste_status grads(const sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream, F first)
{
    const bool f32 = c.gdt == SSTE_F32;
    if (!c.X_codes) return f32 ? grad_launch<R, -1, float>(ctx, c, stream, first) : grad_launch<R, -1, __nv_bfloat16>(ctx, c, stream, first);
    if (c.fmt == SSTE_CKPT_E4M3)
        return f32 ? grad_launch<R, SSTE_CKPT_E4M3, float>(ctx, c, stream, first) : grad_launch<R, SSTE_CKPT_E4M3, __nv_bfloat16>(ctx, c, stream, first);
    return f32 ? grad_launch<R, SSTE_CKPT_INT8, float>(ctx, c, stream, first) : grad_launch<R, SSTE_CKPT_INT8, __nv_bfloat16>(ctx, c, stream, first);
}

template <int R>
sste_status forward(const sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream)
{
    return apply<R, false>(ctx, c, c.l->I, c.l->O, c.l->A, c.l->B, stream);
}
template <int R>
sste_status backward(const sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream)
{
    auto first = [&] { return apply<R, true>(ctx, c, c.l->O, c.l->I, c.l->B, c.l->A, stream); };
    return c.grads ? grads<R>(ctx, c, stream, first) : first();
}

}  // namespace

bool lora_tc_grads_fit(const sste_lora *l, const sste_lora_plan *p, sste_dtype gdt)
{
    const long long columns = lora_rank_up(l->rank) == 64 && gdt != SSTE_F32 ? 256 : 128;
    return 2 * ((l->I + columns - 1) / columns + (l->O + columns - 1) / columns) * p->n_tiles <= 0x7fffffff;
}

size_t lora_tc_partial_bytes(const sste_lora *l, const sste_lora_plan *p)
{
    const int R = lora_rank_up(l->rank);
    const size_t two = static_cast<size_t>(2) * grad_ctas(l->I, l->O, R, p->n_tiles, false, false) * R * (R == 64 ? 256 : 128) * 4,
                 three = static_cast<size_t>(2) * grad_ctas(l->I, l->O, R, p->n_tiles, true, false) * R * 128 * 4;
    return two > three ? two : three;
}

sste_status lora_tc_forward(sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream)
{
    switch (lora_rank_up(c.l->rank)) {
    case 16: return forward<16>(ctx, c, stream);
    case 32: return forward<32>(ctx, c, stream);
    default: return forward<64>(ctx, c, stream);
    }
}
sste_status lora_tc_backward(sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream)
{
    switch (lora_rank_up(c.l->rank)) {
    case 16: return backward<16>(ctx, c, stream);
    case 32: return backward<32>(ctx, c, stream);
    default: return backward<64>(ctx, c, stream);
    }
}

extern "C" sste_status sste_debug_lora_stall(int kernel)
{
    if (kernel < 0 || kernel > 2) return SSTE_ERR_INVALID_ARG;
    g_stall = kernel;
    return SSTE_OK;
}
