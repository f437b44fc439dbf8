// Low-rank adapters of many requests beside a shared linear: V = s X A^T, Y += V B^T, and their gradients U = s dY B, dX += U A,
// dA = U^T X, dB = dY^T V.
//
// With a rank of 8 to 64 these products do 8 to 64 multiply-adds for each element they stream, so memory bounds them and the tensor
// cores only have to keep up.  Batches whose runs of rows are short, or that have few rows (tiles of 16 to 64 rows, a rule of the plan), come
// here: with tiles so small the tensor cores' own path would multiply mostly padding.  Larger ones go to lora_tc.cu.  Here every
// thread fetches the operands that the instruction takes from it: the order of a reduction and of the output's columns is free as long as
// both sides agree on it, so it takes 16 consecutive bytes wherever the instruction's own layout would ask for four scattered pairs.
// They come through slots of shared memory that belong to the thread (projection, gradients) or straight into registers (expansion).
// Operands whose reduction runs across rows are paired with a byte permutation of two rows that the thread itself has loaded.
//
// Measured: one token, 768 x 768, rank 8, 4 us, which is two launches; 64 requests of one token with an adapter each, 4096 x 11008, rank 16,
// 13.5 us: 34 MB take 5.2 us at the copy rate, the rest is the chain of two kernels, start, first loads and last stores of each.
#include <initializer_list>

#include "lora.cuh"

namespace {

constexpr int LR_WARPS = 8, LR_THREADS = 32 * LR_WARPS;
constexpr int LR_MAX_RANK = 64, LR_MAX_FEATURES = 1 << 24;

// 16 x 8 += 16 x 16 times 16 x 8, bf16 with fp32 sums
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
// A pair of fp32 values as the sum of two bf16 pairs, good to 2^-17 of each: V and U meet bf16 operands in a second product, and rounded to
// one bf16 they would bring as much error into Y, dX and the gradients as the rounding of dY itself has.  What the second term cannot
// say (an infinity, a NaN, a value that rounds to infinity) the first does.
struct Split { uint32_t hi, lo; };
__device__ __forceinline__ Split split2(float x, float y)
{
    Split s;
    s.hi = pack2(x, y);
    const float rx = x - __uint_as_float(s.hi << 16), ry = y - __uint_as_float(s.hi & 0xffff0000u);
    s.lo = pack2(fabsf(rx) < INFINITY ? rx : 0.0f, fabsf(ry) < INFINITY ? ry : 0.0f);
    return s;
}
// what a split leaves of the pair, as a third pair
__device__ __forceinline__ uint32_t rest2(float x, float y, const Split &s)
{
    const float rx = x - __uint_as_float(s.hi << 16) - __uint_as_float(s.lo << 16),
                ry = y - __uint_as_float(s.hi & 0xffff0000u) - __uint_as_float(s.lo & 0xffff0000u);
    return pack2(fabsf(rx) < INFINITY ? rx : 0.0f, fabsf(ry) < INFINITY ? ry : 0.0f);
}
__device__ __forceinline__ float2 unpack2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
// element `k` of two rows as a pair
__device__ __forceinline__ uint32_t pair_of(uint32_t first, uint32_t second, int k) { return __byte_perm(first, second, k & 1 ? 0x7632 : 0x5410); }

__device__ __forceinline__ uint4 ld16(const uint16_t *p, bool valid)
{
    return valid ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0, 0, 0, 0);
}

// Operands on their way: each thread copies what it will itself take, BYTES at a time, into slots of shared memory of its own, several steps
// ahead of their use.  Nobody else looks at them, so nothing is synchronised, the layout is lane by lane and free of bank conflicts, and what
// is in flight costs no registers.  (With registers alone a warp had one step in flight and waited out every load: 14 % of the
// memory's rate.)
template <int BYTES, bool STREAM>
__device__ __forceinline__ void copy_some(uint32_t to, const void *from, int size)     // `size` bytes; the rest is filled with zeros
{
    if constexpr (STREAM) asm volatile("cp.async.cg.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(BYTES), "r"(size) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(BYTES), "r"(size) : "memory");
}
template <int BYTES, bool STREAM>
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, bool valid) { copy_some<BYTES, STREAM>(to, from, valid ? BYTES : 0); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
template <int WORDS>
__device__ __forceinline__ void lds_words(uint32_t (&w)[WORDS], uint32_t at)
{
    if constexpr (WORDS == 1) {
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
    } else if constexpr (WORDS == 2) {
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
    } else {
        const uint4 v = lds16(at);
        w[0] = v.x;
        w[1] = v.y;
        w[2] = v.z;
        w[3] = v.w;
    }
}
__device__ __forceinline__ uint32_t shared_address(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// WORDS consecutive 4-byte words
template <int WORDS>
__device__ __forceinline__ void ld_words(uint32_t (&w)[WORDS], const uint16_t *p, bool valid)
{
    if constexpr (WORDS == 1) {
        w[0] = valid ? *reinterpret_cast<const uint32_t *>(p) : 0u;
    } else if constexpr (WORDS == 2) {
        const uint2 v = valid ? *reinterpret_cast<const uint2 *>(p) : make_uint2(0, 0);
        w[0] = v.x;
        w[1] = v.y;
    } else {
        const uint4 v = ld16(p, valid);
        w[0] = v.x;
        w[1] = v.y;
        w[2] = v.z;
        w[3] = v.w;
    }
}

// Slots of a shrinking block: 2 MT vectors of x, and NT 16-byte vectors' worth of weights, for each step in flight: about 160 KB of them.
// With few rows a block lives on its weights' stream, and a memory latency at 75 GB/s is 75 KB.  (Four steps in flight, 24 KB of weights: 62 blocks
// of 4096 x 16 weights took 8.5 us.)
template <int R, int MT>
struct ShrinkStages {
    static constexpr int NT = R / 8, STEP = (2 * MT + NT) * 16 * LR_THREADS, FIT = (160 << 10) / STEP, DEPTH = FIT > 12 ? 12 : FIT < 3 ? 3 : FIT;
    // the weights' loads: 16 bytes each, or (TRANS, eight rows of NT values) 2 NT bytes: the same room
    static constexpr int W_AT = DEPTH * 2 * MT * 16 * LR_THREADS, BYTES = DEPTH * STEP;
};

// One of the two projections to the rank: V = s x a^T (TRANS false: x = X, a = A) or U = s x a (TRANS: x = dY, a = B).
struct ShrinkArgs {
    const uint16_t *x;                  // [T, K]
    const uint16_t *a;                  // per adapter [r, K]; TRANS: [K, r]
    const float *scale;
    const int4 *tiles;
    float *v;                           // [T, r] or null
    uint4 *by_rank;                     // for the expansion, see below
    uint4 *by_row;                      // for the weights' gradients, or null
    const float *v_in;                  // [T, r]: written by rows as well, in the same pass over the tiles, or null
    uint4 *v_by_row;
    uint2 *rest, *v_rest;               // with fp32 gradients: what two bf16 numbers leave of the values by rows, a third
    float *partial;                     // [blocks][splits][rows][R]
    unsigned int *tickets;              // one per block of rows, zero
    size_t ldx;
    int T, K, r, n_adapters, tile_rows, splits;
};

// V and U leave the kernel split into two bf16 numbers, in the two orders in which the products behind it take them from memory to
// registers, 16 bytes to a thread: for the expansion, which reduces over the rank, `by_rank` [slot][R / 4] holds four ranks of a row (pair,
// its rest, pair, its rest); for the gradients, which reduce over the rows, `by_row` [slot / 16][R][4] holds four rows of a rank.  A slot is
// a row of a tile, whether the batch has it or not: rows that it does not have are zeros up to the end of their 16.
//
// A block takes MT * WM * 16 rows; its warps share the rows (WM) and K, and add up in shared memory.  Where the batch has too few rows to
// fill the GPU the blocks share K as well (`splits`): each leaves its sums in the scratch, and the one that arrives last
// adds them up in their order.  (Clusters of eight blocks that add up through each other's shared memory are launched
// one per 0.7 to 1.2 us: 64 of them took 46 us for a batch of 8192 rows.)
template <int R, int MT, int WM, bool TRANS>
__global__ void __launch_bounds__(LR_THREADS, 1)
lora_shrink_kernel(const ShrinkArgs in)
{
    constexpr int WK = LR_WARPS / WM, ROWS = 16 * MT * WM, NT = R / 8, PITCH = R + 4, QROW = R / 4, QUADS = ROWS * QROW;
    extern __shared__ float4 smem4[];
    float *part = reinterpret_cast<float *>(smem4);            // [WK][ROWS][PITCH], the sums in the first
    __shared__ bool is_last;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;

    ShrinkArgs p = in;
    sste_pdl_wait(p.x, p.a, p.scale, p.tiles, p.v_in);
    // (behind the wait, unlike elsewhere, and it has to stay there: a kernel that starts now finds everything that was there before this
    // one complete, and lora_expand_kernel reads what this one does not write in front of its own wait)
    sste_pdl_trigger();
    const int split = static_cast<int>(blockIdx.x) % p.splits, block = static_cast<int>(blockIdx.x) / p.splits;
    const int subs = p.tile_rows / ROWS, t_index = block / subs, in_tile = block % subs * ROWS;
    const LoraTile tile = lora_tile_of(p.tiles, t_index, p.tile_rows, p.T, p.n_adapters);
    const int rows = tile.rows - in_tile;
    if (rows <= 0 || tile.adapter < 0) return;
    const size_t row0 = static_cast<size_t>(tile.row) + in_tile;
    const uint16_t *wa = p.a + static_cast<size_t>(tile.adapter) * p.r * p.K;

    // A warp takes groups of 32 of K for MT * 16 rows.  A thread's 16 bytes are k = 8q .. 8q + 7 of the group; step s of 16 takes
    // 8q + 4s + {0, 1} for the instruction's k = 2q, 2q + 1 and the next two for 2q + 8, 2q + 9.
    {
        using S = ShrinkStages<R, MT>;
        constexpr int W_BYTES = TRANS ? 2 * NT : 16, W_LOADS = TRANS ? 8 : NT;
        const int wm = warp % WM, wk = warp / WM;
        // (The tensor core's sums round towards zero, some 2^-27 of the sum for each instruction: after eight of them they go to `total`, whose additions
        // round to nearest.  In one sum of 47, U and V were off by 9e-7, an fp32 product by 3e-7.)
        float acc[MT][NT][4] = {}, total[MT][NT][4] = {};
        int since = 0;
        auto add_up = [&]() {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        total[m][j][i] += acc[m][j][i];
                        acc[m][j][i] = 0.0f;
                    }
        };
        const int kg_all = (p.K + 31) / 32;
        const int kg_begin = static_cast<int>(static_cast<long long>(kg_all) * split / p.splits) + wk,
                  kg_end = static_cast<int>(static_cast<long long>(kg_all) * (split + 1) / p.splits);
        const uint16_t *xr = p.x + (row0 + wm * MT * 16 + g) * p.ldx + 8 * q;
        const size_t step8 = 8 * p.ldx;
        uint32_t ok = 0;                                       // rows of this thread that the batch has
#pragma unroll
        for (int m = 0; m < 2 * MT; ++m) ok |= ((wm * MT * 16 + g + 8 * m) < rows ? 1u : 0u) << m;
        const uint32_t x_slot = shared_address(smem4) + 16 * threadIdx.x, w_slot = shared_address(smem4) + S::W_AT + W_BYTES * threadIdx.x;
        auto fetch = [&](int stage, int group) {
            if (group >= kg_end) { copies_commit(); return; }  // (nobody takes it; an empty copy costs as much as a full one)
            const int k = group * 32 + 8 * q;
            const bool in = k < p.K;
#pragma unroll
            for (int m = 0; m < 2 * MT; ++m)
                copy_async<16, true>(x_slot + (stage * 2 * MT + m) * (16 * LR_THREADS), in && (ok >> m & 1) ? xr + m * step8 + group * 32 : p.x,
                                     in && (ok >> m & 1));
            const uint32_t to = w_slot + stage * W_LOADS * (W_BYTES * LR_THREADS);
            if constexpr (!TRANS) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const bool has = in && 8 * j + g < p.r;
                    copy_async<16, false>(to + j * (16 * LR_THREADS), has ? wa + static_cast<size_t>(8 * j + g) * p.K + k : wa, has);
                }
            } else {
                // column n = g of the instruction's tile j is rank NT g + j: one load of NT values per row
                const bool has = in && NT * g < p.r;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    copy_async<2 * NT, false>(to + i * (2 * NT * LR_THREADS), has ? wa + static_cast<size_t>(k + i) * p.r + NT * g : wa, has);
            }
            copies_commit();
        };
#pragma unroll
        for (int i = 0; i < S::DEPTH - 1; ++i) fetch(i, kg_begin + i * WK);
        int stage = 0;
        for (int kg = kg_begin; kg < kg_end; kg += WK) {
            copies_wait<S::DEPTH - 2>();
            uint4 x[2 * MT];
#pragma unroll
            for (int m = 0; m < 2 * MT; ++m) x[m] = lds16(x_slot + (stage * 2 * MT + m) * (16 * LR_THREADS));
            uint32_t b[2][NT][2];
            const uint32_t from = w_slot + stage * W_LOADS * (W_BYTES * LR_THREADS);
            if constexpr (!TRANS) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint4 w = lds16(from + j * (16 * LR_THREADS));
                    b[0][j][0] = w.x;
                    b[0][j][1] = w.y;
                    b[1][j][0] = w.z;
                    b[1][j][1] = w.w;
                }
            } else {
                uint32_t w[8][NT / 2];
#pragma unroll
                for (int i = 0; i < 8; ++i) lds_words(w[i], from + i * (2 * NT * LR_THREADS));
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        b[s][j][0] = pair_of(w[4 * s][j / 2], w[4 * s + 1][j / 2], j);
                        b[s][j][1] = pair_of(w[4 * s + 2][j / 2], w[4 * s + 3][j / 2], j);
                    }
            }
            // (into the slots that were taken a step ago)
            fetch(stage == 0 ? S::DEPTH - 1 : stage - 1, kg + (S::DEPTH - 1) * WK);
            stage = stage + 1 == S::DEPTH ? 0 : stage + 1;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    mma(acc[m][j], x[2 * m].x, x[2 * m + 1].x, x[2 * m].y, x[2 * m + 1].y, b[0][j][0], b[0][j][1]);
                    mma(acc[m][j], x[2 * m].z, x[2 * m + 1].z, x[2 * m].w, x[2 * m + 1].w, b[1][j][0], b[1][j][1]);
                }
            if (++since == 4) {
                add_up();
                since = 0;
            }
        }
        add_up();
        copies_wait<0>();
        __syncthreads();                                       // the slots become the sums' room
        float *mine = part + wk * ROWS * PITCH;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = (wm * MT + m) * 16 + g;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float *at = mine + (row + 8 * h) * PITCH;
                    if constexpr (!TRANS) {
                        *reinterpret_cast<float2 *>(at + 8 * j + 2 * q) = make_float2(total[m][j][2 * h], total[m][j][2 * h + 1]);
                    } else {
                        at[NT * 2 * q + j] = total[m][j][2 * h];
                        at[NT * (2 * q + 1) + j] = total[m][j][2 * h + 1];
                    }
                }
        }
    }
    __syncthreads();

    // ---- the sums over the warps, and over the blocks that share K
    auto over_warps = [&](int i) {
        const float4 *at = reinterpret_cast<const float4 *>(part + (i / QROW) * PITCH + 4 * (i % QROW));
        float4 sum = *at;
#pragma unroll
        for (int w = 1; w < WK; ++w) {
            const float4 v = at[w * (ROWS * PITCH / 4)];
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
        return sum;
    };
    float4 *shared = reinterpret_cast<float4 *>(p.partial) + static_cast<size_t>(block) * p.splits * QUADS;
    if (p.splits > 1) {
        for (int i = threadIdx.x; i < QUADS; i += LR_THREADS) shared[split * QUADS + i] = over_warps(i);
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) is_last = atomicAdd(p.tickets + block, 1u) == static_cast<unsigned int>(p.splits - 1);
        __syncthreads();
        if (!is_last) return;
        __threadfence();
        if (threadIdx.x == 0) p.tickets[block] = 0;            // as it was found
    }
    const float s = p.scale[tile.adapter];
    for (int i = threadIdx.x; i < QUADS; i += LR_THREADS) {
        const int row = i / QROW, col = 4 * (i % QROW);
        float4 sum;
        if (p.splits > 1) {
            sum = __ldcg(shared + i);
            for (int k = 1; k < p.splits; ++k) {
                const float4 v = __ldcg(shared + k * QUADS + i);
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
        } else {
            sum = over_warps(i);
        }
        // (columns that fill the rank up are zeros whatever x holds)
        sum = col < p.r ? make_float4(s * sum.x, s * sum.y, s * sum.z, s * sum.w) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p.v && row < rows && col < p.r) *reinterpret_cast<float4 *>(p.v + (row0 + row) * p.r + col) = sum;
        *reinterpret_cast<float4 *>(part + row * PITCH + col) = sum;
        const Split lo = split2(sum.x, sum.y), hi = split2(sum.z, sum.w);
        const size_t slot = static_cast<size_t>(t_index) * p.tile_rows + in_tile + row;
        p.by_rank[slot * QROW + i % QROW] = make_uint4(lo.hi, lo.lo, hi.hi, hi.lo);
    }
    if (!p.by_row) return;
    __syncthreads();
    const size_t group0 = (static_cast<size_t>(t_index) * p.tile_rows + in_tile) / 16;
    for (int i = threadIdx.x; i < ROWS / 4 * R; i += LR_THREADS) {
        const int quad = i % 4, rank = i / 4 % R, group = i / (4 * R), row = 16 * group + 4 * quad;
        const float *at = part + row * PITCH + rank;
        const Split a = split2(at[0], at[PITCH]), b = split2(at[2 * PITCH], at[3 * PITCH]);
        const size_t place = ((group0 + group) * R + rank) * 4 + quad;
        p.by_row[place] = make_uint4(a.hi, a.lo, b.hi, b.lo);
        if (p.rest) p.rest[place] = make_uint2(rest2(at[0], at[PITCH], a), rest2(at[2 * PITCH], at[3 * PITCH], b));
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = row + k < rows && rank < p.r ? p.v_in[(row0 + row + k) * p.r + rank] : 0.0f;
        const Split c = split2(v[0], v[1]), d = split2(v[2], v[3]);
        p.v_by_row[place] = make_uint4(c.hi, c.lo, d.hi, d.lo);
        if (p.rest) p.v_rest[place] = make_uint2(rest2(v[0], v[1], c), rest2(v[2], v[3], d));
    }
}

// y_out = y_in + V b^T (TRANS false: y = Y, b = B) or + U b (TRANS: y = dX, b = A).
struct ExpandArgs {
    const uint4 *by_rank;
    const uint16_t *b;                  // per adapter [N, r]; TRANS: [r, N]
    const int4 *tiles;
    const uint16_t *y_in;               // [T, N]; null: zeros
    uint16_t *y_out;
    size_t ldy;
    int T, N, r, n_adapters, shares;    // shares: blocks of a tile
};

// A warp goes over every fourth 64 columns of its block's share of a tile: weights in registers, the next columns' on their way, the tile's rows 16
// at a time with the next 16 rows of y on their way.  Column n = i of the instruction's tile j is 8i + j of the 64, so a thread's outputs are
// 16 consecutive columns of two rows.  What does not come from the kernel before (weights, y_in) is read while that still runs: with few
// rows the weights are nearly all that is read.  (A block per 256 columns, 64 rows of one token, 4096 x 11008, rank 16: 2666 blocks in
// four rounds of waiting, 13.5 us of the call's 17.7.)
constexpr int EX_WARPS = 4, EX_THREADS = 32 * EX_WARPS;
template <int R, int MT, bool TRANS>
__global__ void __launch_bounds__(EX_THREADS, R == 64 ? 2 : R == 32 ? 3 : 4)
lora_expand_kernel(const ExpandArgs in)
{
    constexpr int KS = R / 16, QROW = R / 4, PITCH = QROW + (R == 16 ? 0 : 1), ROWS = 16 * MT;
    __shared__ uint4 v[ROWS * PITCH];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;
    ExpandArgs p = in;
    const int t_index = static_cast<int>(blockIdx.x) / p.shares, share = static_cast<int>(blockIdx.x) % p.shares;
    const LoraTile tile = lora_tile_of(p.tiles, t_index, ROWS, p.T, p.n_adapters);
    const int groups = (p.N + 63) / 64, first = static_cast<int>(static_cast<long long>(groups) * share / p.shares) + warp,
              last = static_cast<int>(static_cast<long long>(groups) * (share + 1) / p.shares);
    if (tile.rows <= 0 || (tile.adapter < 0 && p.y_in == p.y_out)) {
        sste_pdl_wait();
        sste_pdl_trigger();
        return;
    }
    const size_t row0 = static_cast<size_t>(tile.row);
    if (tile.adapter < 0) {                                    // no adapter: the rows as they are
        sste_pdl_wait(p.y_in);
        sste_pdl_trigger();
        for (int n = first; n < last; n += EX_WARPS)
#pragma unroll 4
            for (int i = lane; i < tile.rows * 8; i += 32) {
                const int col = 64 * n + 8 * (i % 8);
                if (col >= p.N) continue;
                const size_t at = (row0 + i / 8) * p.ldy + col;
                *reinterpret_cast<uint4 *>(p.y_out + at) = ld16(p.y_in + at, p.y_in != nullptr);
            }
        return;
    }
    const uint16_t *wb = p.b + static_cast<size_t>(tile.adapter) * p.r * p.N;
    struct Weights { uint32_t b[KS][8][2]; };
    auto load_weights = [&](Weights &to, int group) {
        const int n0 = 64 * group;
        const bool in = group < last;
        if constexpr (!TRANS) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int n = n0 + 8 * g + j;
                const uint16_t *at = wb + static_cast<size_t>(n) * p.r;
                const bool has = in && n < p.N;
                if constexpr (R == 16) {
                    ld_words(to.b[0][j], at + 4 * q, has && 4 * q < p.r);
                } else {
#pragma unroll
                    for (int k = 0; k < KS; k += 2) {
                        const uint4 w = ld16(at + 16 * k + 8 * q, has && 16 * k + 8 * q < p.r);
                        to.b[k][j][0] = w.x;
                        to.b[k][j][1] = w.y;
                        to.b[k + 1][j][0] = w.z;
                        to.b[k + 1][j][1] = w.w;
                    }
                }
            }
        } else {
            // (rows of four words each, paired when they are used)
            const int n = n0 + 8 * g;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int r0 = R == 16 ? 4 * q : 32 * (k / 2) + 8 * q + 4 * (k % 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 w = ld16(wb + static_cast<size_t>(r0 + i) * p.N + n, in && n < p.N && r0 < p.r);
                    to.b[k][2 * i][0] = w.x;
                    to.b[k][2 * i][1] = w.y;
                    to.b[k][2 * i + 1][0] = w.z;
                    to.b[k][2 * i + 1][1] = w.w;
                }
            }
        }
    };
    struct Rows { uint4 y[2][2]; };
    auto load_y = [&](Rows &to, int group, int m) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = 16 * m + 8 * h + g, col = 64 * group + 16 * q + 8 * e;
                to.y[h][e] = ld16(p.y_in + (row0 + row) * p.ldy + col, p.y_in && group < last && row < tile.rows && col < p.N);
            }
    };
    auto step = [&](const Weights &w, const Rows &y, int group, int m) {
        float acc[8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x[4] = {y.y[h][e].x, y.y[h][e].y, y.y[h][e].z, y.y[h][e].w};
                    const float2 f = unpack2(x[j / 2]);
                    acc[j][2 * h + e] = j & 1 ? f.y : f.x;
                }
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int at = R == 16 ? q : 8 * (k / 2) + 2 * q + k % 2;
            const uint4 a = v[(16 * m + g) * PITCH + at], c = v[(16 * m + 8 + g) * PITCH + at];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t b0, b1;
                if constexpr (!TRANS) {
                    b0 = w.b[k][j][0];
                    b1 = w.b[k][j][1];
                } else {
                    const int word = j / 2;                    // of rows r0 .. r0 + 3: words 0, 1 in [2 i], words 2, 3 in [2 i + 1]
                    b0 = pair_of(w.b[k][word / 2][word % 2], w.b[k][2 + word / 2][word % 2], j);
                    b1 = pair_of(w.b[k][4 + word / 2][word % 2], w.b[k][6 + word / 2][word % 2], j);
                }
                mma(acc[j], a.x, c.x, a.z, c.z, b0, b1);
                mma(acc[j], a.y, c.y, a.w, c.w, b0, b1);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = 16 * m + 8 * h + g, col = 64 * group + 16 * q + 8 * e, i = 2 * h + e;
                if (row < tile.rows && col < p.N)
                    *reinterpret_cast<uint4 *>(p.y_out + (row0 + row) * p.ldy + col) =
                        make_uint4(pack2(acc[0][i], acc[1][i]), pack2(acc[2][i], acc[3][i]), pack2(acc[4][i], acc[5][i]), pack2(acc[6][i], acc[7][i]));
            }
    };
    Weights w0, w1;
    Rows y0, y1;
    load_weights(w0, first);
    load_y(y0, first, 0);
    load_weights(w1, first + EX_WARPS);
    sste_pdl_wait(p.by_rank);
    sste_pdl_trigger();
    for (int i = threadIdx.x; i < ROWS * QROW; i += EX_THREADS)
        v[i / QROW * PITCH + i % QROW] = p.by_rank[static_cast<size_t>(t_index) * (ROWS * QROW) + i];
    __syncthreads();
    // (two sets of weights that take turns; four spill)
    auto group_rows = [&](Weights &w, int group) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const bool more = m + 1 < MT && 16 * (m + 1) < tile.rows;
            load_y(y1, more ? group : group + EX_WARPS, more ? m + 1 : 0);
            step(w, y0, group, m);
            y0 = y1;
            if (!more) break;
        }
        load_weights(w, group + 2 * EX_WARPS);
    };
    for (int group = first; group < last; group += 2 * EX_WARPS) {
        group_rows(w0, group);
        if (group + EX_WARPS >= last) break;
        group_rows(w1, group + EX_WARPS);
    }
}

// ---------------------------------------------------------------- gradients of the weights

// One of the two sums over rows: out [r, N] = s^T z (dA: s = U, z = X), or its transpose [N, r] (dB: s = V, z = dY).
struct GradJob {
    const uint4 *by_row;
    const uint2 *rest;                  // fp32 results: the third part of each value
    const uint16_t *z;                  // [T, N] bf16, or null and the kept form
    const uint8_t *codes, *scales;
    void *out;
    size_t ldz, n_scales;
    int N;
    int blocks;                         // of columns
    bool across;                        // out is [N, r]
};
struct GradArgs {
    GradJob job[2];
    const int *first_group;
    const int4 *groups;
    float *partial;                     // [adapter][block][split][R][columns]
    unsigned int *tickets;
    int T, r, n_adapters, n_tiles, tile_rows, splits;
};

enum { Z_BF16 = 0, Z_E4M3 = 1, Z_INT8 = 2 };

// Warps of a block: WN along the columns (64 each), WM along the rank (32 each), WT along the rows.  A wide block reads `by_row`, which is twice
// as long per row as 64 columns of z at a rank of 64, fewer times.
template <int R>
struct GradShape {
    static constexpr int MW = R / 16 < 2 ? R / 16 : 2, WM = R / 16 / MW, WN = R == 64 ? 4 : 2, WT = LR_WARPS / (WN * WM), COLUMNS = 64 * WN;
    static constexpr int SLOTS = 4 + 3 * MW, DEPTH = 4;       // vectors of z and of U or V for 16 rows; steps in flight
    static constexpr size_t SLOT_BYTES = size_t(DEPTH) * SLOTS * 16 * LR_THREADS, SUM_BYTES = size_t(R) * (COLUMNS + 4) * 4;
};

// The instruction's rows are the rank (16 at a time), its columns the features, its reduction the rows of the batch: a thread takes rows
// 4q .. 4q + 3 of a group of 16 and pairs them.
template <int R, int Z, bool REST>
__device__ __forceinline__ void grad_partial(const GradArgs &p, const GradJob &job, int adapter, int n0, int m0, int worker, int workers,
                                             const float4 *smem, float (&acc)[GradShape<R>::MW][8][4])
{
    constexpr int MW = GradShape<R>::MW;
    const int lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;
    const int all = p.n_tiles * (p.tile_rows / 16), begin = p.first_group[adapter], end = p.first_group[adapter + 1];
    if (begin < 0 || end > all) return;
    const int col = n0 + 8 * g;
    const bool has = col < job.N;
    // (a table that is not the library's own is not followed out of the tensors)
    auto group_of = [&](int f) {
        int4 t = f < end ? p.groups[f] : make_int4(0, 0, 0, 0);
        if (t.x < 0 || t.y < 0 || t.y > 16 || t.x > p.T - t.y || t.z != adapter || t.w < 0 || t.w >= all) t = make_int4(0, 0, 0, 0);
        return t;
    };
    constexpr int SLOTS = GradShape<R>::SLOTS, DEPTH = GradShape<R>::DEPTH;
    const uint32_t slot = shared_address(smem) + 16 * threadIdx.x;
    auto fetch = [&](int stage, const int4 &group) {
        const uint32_t to = slot + stage * SLOTS * (16 * LR_THREADS);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = 4 * q + i < group.y && has;
            const size_t t = static_cast<size_t>(group.x) + 4 * q + i;
            if constexpr (Z == Z_BF16) {
                copy_async<16, true>(to + i * (16 * LR_THREADS), in ? job.z + t * job.ldz + col : job.z, in);
            } else {
                const size_t at = t * job.N + col;
                copy_async<8, false>(to + i * (16 * LR_THREADS), in ? job.codes + at : job.codes, in);
                // the scale's word, as far as there are scales: its byte is picked when it is taken
                const size_t word = at / 32 / 4 * 4, left = job.n_scales - word;
                copy_some<4, false>(to + i * (16 * LR_THREADS) + 8, in ? job.scales + word : job.codes, !in ? 0 : left < 4 ? static_cast<int>(left) : 4);
            }
        }
        const uint4 *s_at = job.by_row + (static_cast<size_t>(group.w) * R + 16 * m0 + g) * 4 + q;
#pragma unroll
        for (int m = 0; m < 2 * MW; ++m)
            copy_async<16, false>(to + (4 + m) * (16 * LR_THREADS), group.y ? s_at + 8 * m * 4 : job.by_row, group.y > 0);
        if constexpr (REST) {
            const uint2 *rest = job.rest + (static_cast<size_t>(group.w) * R + 16 * m0 + g) * 4 + q;
#pragma unroll
            for (int m = 0; m < 2 * MW; ++m)
                copy_async<8, false>(to + (4 + 2 * MW + m / 2) * (16 * LR_THREADS) + 8 * (m & 1), group.y ? rest + 8 * m * 4 : job.rest, group.y > 0);
        }
        copies_commit();
    };
    int4 ahead = group_of(begin + worker);
    int4 rows[DEPTH];                                          // of the stages in flight: which rows they hold
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) {
        rows[i] = ahead;
        fetch(i, ahead);
        ahead = group_of(begin + worker + (i + 1) * workers);
    }
    int stage = 0, since = 0;
    // for the rounding's sake as in the projection: fp32 results after 64 rows, bf16 ones after 8192 (3e-5 of a sum of terms of one sign)
    constexpr int EVERY = REST ? 4 : 512;
    float total[MW][8][4] = {};
    auto add_up = [&]() {
#pragma unroll
        for (int m = 0; m < MW; ++m)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    total[m][j][i] += acc[m][j][i];
                    acc[m][j][i] = 0.0f;
                }
    };
    for (int f = begin + worker; f < end; f += workers) {
        copies_wait<DEPTH - 2>();
        const uint32_t from = slot + stage * SLOTS * (16 * LR_THREADS);
        uint32_t w[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = lds16(from + i * (16 * LR_THREADS));
            if constexpr (Z == Z_BF16) {
                w[i][0] = v.x;
                w[i][1] = v.y;
                w[i][2] = v.z;
                w[i][3] = v.w;
            } else {
                // (rows that are not there: codes of 0 and a scale of 0)
                const bool in = 4 * q + i < rows[0].y && has;
                const size_t at = (static_cast<size_t>(rows[0].x) + 4 * q + i) * job.N + col;
                const uint32_t e = v.z >> (8 * (at / 32 % 4)) & 0xffu;
                uint32_t nans = 0;
                lora_restore8<Z == Z_E4M3>(make_uint2(v.x, v.y), in ? e : 0u, w[i], nans);
                if (lora_has_nan<Z == Z_E4M3>(nans)) lora_put_nans<Z == Z_E4M3>(make_uint2(v.x, v.y), w[i]);
            }
        }
        uint4 s[2 * MW];
#pragma unroll
        for (int m = 0; m < 2 * MW; ++m) s[m] = lds16(from + (4 + m) * (16 * LR_THREADS));
        uint4 rest[MW];
#pragma unroll
        for (int m = 0; m < MW; ++m) rest[m] = REST ? lds16(from + (4 + 2 * MW + m) * (16 * LR_THREADS)) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i + 1 < DEPTH - 1; ++i) rows[i] = rows[i + 1];
        rows[DEPTH - 2] = ahead;
        fetch(stage == 0 ? DEPTH - 1 : stage - 1, ahead);      // (into the slots that were taken a step ago)
        ahead = group_of(f + DEPTH * workers);
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b0 = pair_of(w[0][j / 2], w[1][j / 2], j), b1 = pair_of(w[2][j / 2], w[3][j / 2], j);
#pragma unroll
            for (int m = 0; m < MW; ++m) {
                mma(acc[m][j], s[2 * m].x, s[2 * m + 1].x, s[2 * m].z, s[2 * m + 1].z, b0, b1);
                mma(acc[m][j], s[2 * m].y, s[2 * m + 1].y, s[2 * m].w, s[2 * m + 1].w, b0, b1);
                if constexpr (REST) mma(acc[m][j], rest[m].x, rest[m].z, rest[m].y, rest[m].w, b0, b1);
            }
        }
        if (++since == EVERY) {
            add_up();
            since = 0;
        }
    }
    copies_wait<0>();
#pragma unroll
    for (int m = 0; m < MW; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] += total[m][j][i];
}

template <int R, int Z, typename OUT>
__global__ void __launch_bounds__(LR_THREADS, R == 16 ? 2 : 1)
lora_grad_kernel(const GradArgs in)
{
    using S = GradShape<R>;
    constexpr int COLUMNS = S::COLUMNS, PITCH = COLUMNS + 4;
    extern __shared__ float4 smem4[];
    float *red = reinterpret_cast<float *>(smem4);             // [R][PITCH]
    __shared__ bool is_last;
    GradArgs p = in;
    sste_pdl_wait(p.job[0].by_row, p.job[0].z, p.job[0].codes, p.job[0].scales, p.job[0].rest, p.job[1].rest, p.job[1].by_row, p.job[1].z, p.first_group, p.groups);
    sste_pdl_trigger();                                        // (behind the wait, for the expansion's sake, see lora_shrink_kernel)
    const int split = static_cast<int>(blockIdx.x) % p.splits;
    int block = static_cast<int>(blockIdx.x) / p.splits;
    const int adapter = blockIdx.y, ticket = adapter * (p.job[0].blocks + p.job[1].blocks) + block;
    const bool second = block >= p.job[0].blocks;
    if (second) block -= p.job[0].blocks;
    const GradJob job = second ? p.job[1] : p.job[0];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;
    const int wn = warp % S::WN, wm = warp / S::WN % S::WM, wt = warp / (S::WN * S::WM);

    float acc[S::MW][8][4] = {};
    const int n0 = block * COLUMNS + wn * 64, worker = split * S::WT + wt, workers = p.splits * S::WT;
    if (n0 < job.N) {
        constexpr bool REST = sizeof(OUT) == 4;
        if (Z == Z_BF16 || second) grad_partial<R, Z_BF16, REST>(p, job, adapter, n0, wm * S::MW, worker, workers, smem4, acc);
        else grad_partial<R, Z, REST>(p, job, adapter, n0, wm * S::MW, worker, workers, smem4, acc);
    }
    __syncthreads();                                           // the slots become the sums' room
#pragma unroll 1
    for (int w = 0; w < S::WT; ++w) {
        if (wt == w) {
#pragma unroll
            for (int m = 0; m < S::MW; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float *at = red + (16 * (wm * S::MW + m) + g + 8 * h) * PITCH + wn * 64 + 16 * q;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            float4 v = make_float4(acc[m][j][2 * h + e], acc[m][j + 1][2 * h + e], acc[m][j + 2][2 * h + e],
                                                   acc[m][j + 3][2 * h + e]);
                            float4 *to = reinterpret_cast<float4 *>(at + 8 * e + j);
                            if (w) {
                                const float4 o = *to;
                                v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
                            }
                            *to = v;
                        }
                }
        }
        __syncthreads();
    }
    constexpr int QUADS = R * COLUMNS / 4, QROW = COLUMNS / 4;
    if (p.splits > 1) {
        float4 *shared = reinterpret_cast<float4 *>(p.partial) + static_cast<size_t>(ticket) * p.splits * QUADS;
        for (int i = threadIdx.x; i < QUADS; i += LR_THREADS)
            shared[split * QUADS + i] = *reinterpret_cast<const float4 *>(red + (i / QROW) * PITCH + 4 * (i % QROW));
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) is_last = atomicAdd(p.tickets + ticket, 1u) == static_cast<unsigned int>(p.splits - 1);
        __syncthreads();
        if (!is_last) return;
        __threadfence();
        if (threadIdx.x == 0) p.tickets[ticket] = 0;           // as it was found
        for (int i = threadIdx.x; i < QUADS; i += LR_THREADS) {
            float4 sum = __ldcg(shared + i);
            for (int k = 1; k < p.splits; ++k) {
                const float4 v = __ldcg(shared + k * QUADS + i);
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
            *reinterpret_cast<float4 *>(red + (i / QROW) * PITCH + 4 * (i % QROW)) = sum;
        }
        __syncthreads();
    }
    OUT *out = static_cast<OUT *>(job.out) + static_cast<size_t>(adapter) * p.r * job.N;
    for (int i = threadIdx.x; i < R * COLUMNS; i += LR_THREADS) {
        const int rank = job.across ? i % R : i / COLUMNS, n = job.across ? i / R : i % COLUMNS;
        const int col = block * COLUMNS + n;
        if (rank >= p.r || col >= job.N) continue;
        const float sum = red[rank * PITCH + n];
        const size_t at = job.across ? static_cast<size_t>(col) * p.r + rank : static_cast<size_t>(rank) * job.N + col;
        if constexpr (sizeof(OUT) == 2) out[at] = __float2bfloat16_rn(sum);
        else out[at] = sum;
    }
}

// ---------------------------------------------------------------- host

// How a batch is cut up, from sizes alone.
struct Cut {
    int shrink_rows, shrink_splits;         // rows to a block, blocks that share K
    int expand_shares;                      // blocks of a tile
    int grad_blocks, grad_splits;
    size_t shrink_partial, grad_partial;    // bytes
};
int columns_of(int R) { return R == 64 ? 256 : 128; }
int shrink_splits_of(int blocks, int K, int R)
{
    // a block streams its rows' weights at about 75 GB/s; adding up through the scratch takes 2 us
    const double alone = 2.0 * K * R / 75e3;
    int best = 1;
    double least = alone;
    for (int s = 2; s <= LR_MAX_SPLITS && blocks * s <= 2 * LR_SMS && K >= s * 256; s *= 2) {
        const double cost = alone / s + 2.0 + 0.1 * s;
        if (cost < least) { best = s; least = cost; }
    }
    return best;
}
Cut cut_of(int n_tiles, int tile_rows, int T, int K, int N, int I, int O, int n_adapters, int rank)
{
    const int R = lora_rank_up(rank);
    Cut c{};
    // the most rows (a weight is read once per block of rows) with which every SM has a block
    for (c.shrink_rows = tile_rows; c.shrink_rows > 16 && static_cast<long long>(n_tiles) * (tile_rows / c.shrink_rows) < LR_SMS;) c.shrink_rows /= 2;
    const long long blocks = static_cast<long long>(n_tiles) * (tile_rows / c.shrink_rows);
    c.shrink_splits = blocks <= LR_TICKETS ? shrink_splits_of(static_cast<int>(blocks), K, R) : 1;
    c.shrink_partial = c.shrink_splits > 1 ? static_cast<size_t>(blocks) * c.shrink_splits * c.shrink_rows * R * 4 : 0;
    // four blocks an SM, each warp with 64 columns or more
    const int groups = (N + 63) / 64, most = (groups + EX_WARPS - 1) / EX_WARPS;
    c.expand_shares = n_tiles > 0 ? 4 * LR_SMS / n_tiles : 1;
    c.expand_shares = c.expand_shares < 1 ? 1 : c.expand_shares > most ? most : c.expand_shares;
    const int columns = columns_of(R);
    c.grad_blocks = (I + columns - 1) / columns + (O + columns - 1) / columns;
    const long long grads = static_cast<long long>(c.grad_blocks) * n_adapters, steps = (static_cast<long long>(T) / n_adapters + 15) / 16;
    c.grad_splits = 1;
    while (c.grad_splits < LR_MAX_SPLITS && grads <= LR_TICKETS && grads * (c.grad_splits + 1) <= 2 * LR_SMS && steps >= 16 * (c.grad_splits + 1)) ++c.grad_splits;
    c.grad_partial = c.grad_splits > 1 ? static_cast<size_t>(grads) * c.grad_splits * R * columns * 4 : 0;
    return c;
}
constexpr int TC_TILE = 128;                // tiles of so many rows go to the kernels of lora_tc.cu
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// The scratch: tickets of both kinds, V or U by rank, U and V by rows, partial sums.
struct Scratch {
    size_t by_rank, u_by_row, v_by_row, u_rest, v_rest, partial, bytes;
};
Scratch scratch_of(const sste_lora *l, const sste_lora_plan *p)
{
    const Cut f = cut_of(p->n_tiles, p->tile_rows, p->T, l->I, l->O, l->I, l->O, l->n_adapters, l->rank);
    const Cut b = cut_of(p->n_tiles, p->tile_rows, p->T, l->O, l->I, l->I, l->O, l->n_adapters, l->rank);
    const size_t one = up256(static_cast<size_t>(p->n_tiles) * p->tile_rows * lora_rank_up(l->rank) * 4);
    size_t partial = f.shrink_partial;
    for (size_t v : {b.shrink_partial, b.grad_partial}) partial = v > partial ? v : partial;
    if (p->tile_rows == TC_TILE) partial = lora_tc_partial_bytes(l, p);
    Scratch s{};
    s.by_rank = 2 * LR_TICKETS * sizeof(unsigned int);
    s.u_by_row = s.by_rank + one;
    // (for tiles of 128 rows the two are planes, up to three of them)
    const size_t half = up256(one / 2);
    s.u_rest = s.u_by_row + one;
    s.v_by_row = s.u_rest + half;
    s.v_rest = s.v_by_row + one;
    s.partial = s.v_rest + half;
    s.bytes = s.partial + up256(partial);
    return s;
}

// An SM that has shared memory and L1 cache divided otherwise for the next kernel finishes with this one first: all kernels ask for the
// largest shared memory, as the products do (one token, 768 x 768: 5.5 us when the second kernel of the call asked for little, 4.2 with all alike).
template <typename K>
bool all_shared(K kern)
{
    return cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) == cudaSuccess;
}

template <int R, int MT, int WM, bool TRANS>
sste_status shrink_launch(const sste_ctx *ctx, const ShrinkArgs &p, int n_tiles, cudaStream_t stream)
{
    constexpr int ROWS = 16 * MT * WM, WK = LR_WARPS / WM;
    constexpr size_t sums = static_cast<size_t>(WK) * ROWS * (R + 4) * sizeof(float), slots = ShrinkStages<R, MT>::BYTES,
                     smem = sums > slots ? sums : slots;
    auto *kern = lora_shrink_kernel<R, MT, WM, TRANS>;
    static DeviceOnce once;
    if (!once.run(ctx->device, [&] {
            return all_shared(kern) && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) == cudaSuccess;
        }))
        return SSTE_ERR_CUDA;
    const unsigned grid = static_cast<unsigned>(n_tiles) * (p.tile_rows / ROWS) * p.splits;
    return sste_launch(kern, dim3(grid), dim3(LR_THREADS), smem, stream, p) == cudaSuccess ? SSTE_OK : SSTE_ERR_CUDA;
}

template <int R, bool TRANS>
sste_status shrink_rows(const sste_ctx *ctx, const ShrinkArgs &p, int n_tiles, int rows, cudaStream_t stream)
{
    // shares of a block's eight warps: along the rows where it has many, else along K; a rank of 64 has sums for 32 rows a warp
    switch (rows) {
    case 16: return shrink_launch<R, 1, 1, TRANS>(ctx, p, n_tiles, stream);
    case 32: return shrink_launch<R, 2, 1, TRANS>(ctx, p, n_tiles, stream);
    case 64: return shrink_launch<R, 2, 2, TRANS>(ctx, p, n_tiles, stream);
    default: return SSTE_ERR_INVALID_ARG;
    }
}

template <int R, bool TRANS>
sste_status expand_launch(const sste_ctx *ctx, const ExpandArgs &p, int n_tiles, int tile_rows, cudaStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(n_tiles) * p.shares);
    auto launch = [&](auto kern, DeviceOnce &once) {
        if (!once.run(ctx->device, [&] { return all_shared(kern); })) return SSTE_ERR_CUDA;
        return sste_launch(kern, grid, dim3(EX_THREADS), 0, stream, p) == cudaSuccess ? SSTE_OK : SSTE_ERR_CUDA;
    };
    static DeviceOnce once[3];
    return tile_rows == 16 ? launch(lora_expand_kernel<R, 1, TRANS>, once[0]) : tile_rows == 32 ? launch(lora_expand_kernel<R, 2, TRANS>, once[1])
                                                                                                : launch(lora_expand_kernel<R, 4, TRANS>, once[2]);
}

template <int R, int Z, typename OUT>
sste_status grad_launch(const sste_ctx *ctx, const GradArgs &p, cudaStream_t stream)
{
    using S = GradShape<R>;
    constexpr size_t smem = S::SLOT_BYTES > S::SUM_BYTES ? S::SLOT_BYTES : S::SUM_BYTES;
    auto *kern = lora_grad_kernel<R, Z, OUT>;
    static DeviceOnce once;
    if (!once.run(ctx->device, [&] {
            return all_shared(kern) && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) == cudaSuccess;
        }))
        return SSTE_ERR_CUDA;
    const dim3 grid(static_cast<unsigned>(p.job[0].blocks + p.job[1].blocks) * p.splits, static_cast<unsigned>(p.n_adapters));
    return sste_launch(kern, grid, dim3(LR_THREADS), smem, stream, p) == cudaSuccess ? SSTE_OK : SSTE_ERR_CUDA;
}
template <int R>
sste_status grad_by_type(const sste_ctx *ctx, const GradArgs &p, int z, sste_dtype gdt, cudaStream_t stream)
{
    const bool f32 = gdt == SSTE_F32;
    if (z == Z_E4M3) return f32 ? grad_launch<R, Z_E4M3, float>(ctx, p, stream) : grad_launch<R, Z_E4M3, __nv_bfloat16>(ctx, p, stream);
    if (z == Z_INT8) return f32 ? grad_launch<R, Z_INT8, float>(ctx, p, stream) : grad_launch<R, Z_INT8, __nv_bfloat16>(ctx, p, stream);
    return f32 ? grad_launch<R, Z_BF16, float>(ctx, p, stream) : grad_launch<R, Z_BF16, __nv_bfloat16>(ctx, p, stream);
}

// f(the rank's tile as a type)
template <int V>
struct Rank { static constexpr int value = V; };
template <typename F>
sste_status by_rank(int rank, F f)
{
    return rank <= 16 ? f(Rank<16>()) : rank <= 32 ? f(Rank<32>()) : f(Rank<64>());
}

bool tile_rows_ok(int rows) { return rows == 16 || rows == 32 || rows == 64 || rows == 128; }

sste_status lora_ok(const sste_lora *l, const sste_lora_plan *p)
{
    if (!l || !p || !l->A || !l->B || !l->scale || (!p->table && p->n_tiles > 0)) return SSTE_ERR_INVALID_ARG;
    if (l->n_adapters < 1 || l->n_adapters > 65535 || p->n_adapters != l->n_adapters || p->T < 0 || p->n_tiles < 0 ||
        p->n_tiles > LR_MAX_TILES || !tile_rows_ok(p->tile_rows))
        return SSTE_ERR_INVALID_ARG;
    if (l->rank < 8 || l->rank > LR_MAX_RANK || l->rank % 8 || l->I < 8 || l->I % 8 || l->O < 8 || l->O % 8 || l->I > LR_MAX_FEATURES ||
        l->O > LR_MAX_FEATURES)
        return SSTE_ERR_SHAPE;
    if (!sste_aligned(l->A, 16) || !sste_aligned(l->B, 16) || !sste_aligned(l->scale, 4) || !sste_aligned(p->table, 16))
        return SSTE_ERR_ALIGN;
    return SSTE_OK;
}
// a [T, cols] bf16 tensor with rows `ld` elements apart
sste_status rows_ok(const void *t, long long ld, int cols)
{
    if (ld < cols || ld % 8) return SSTE_ERR_SHAPE;
    return sste_aligned(t, 16) ? SSTE_OK : SSTE_ERR_ALIGN;
}
const int4 *tiles_of(const sste_lora_plan *p) { return reinterpret_cast<const int4 *>(static_cast<const int *>(p->table) + lora_tiles_at(p->n_adapters)); }

}  // namespace

// ---- the plan

extern "C" size_t sste_lora_plan_ints(int T, int requests, int n_adapters, int min_tiles)
{
    if (T < 0 || requests < 0 || n_adapters < 1) return 0;
    // (a tile of 16 rows has one group; of more rows, a tile that is not full may have up to seven groups without rows)
    const size_t tiles = static_cast<size_t>(T) / 16 + static_cast<size_t>(requests);
    return 2 * lora_tiles_at(n_adapters) + 4 * (2 * tiles + 8 * static_cast<size_t>(requests) + 9 * static_cast<size_t>(min_tiles > 0 ? min_tiles : 0));
}

namespace {

// f(first row, rows, adapter) for each tile: neighbouring requests of one adapter are one run of rows
template <typename F>
void each_tile(const int *offsets, const int *adapters, int requests, int tile_rows, F f)
{
    for (int i = 0; i < requests;) {
        int j = i + 1;
        while (j < requests && adapters[j] == adapters[i]) ++j;
        for (int row = offsets[i]; row < offsets[j];) {
            const int rows = offsets[j] - row < tile_rows ? offsets[j] - row : tile_rows;
            f(row, rows, adapters[i]);
            row += rows;
        }
        i = j;
    }
}

}  // namespace

extern "C" sste_status sste_lora_plan_build(const int *offsets, const int *adapters, int requests, int T, int n_adapters, int tile_rows,
                                            int min_tiles, int *table, size_t table_ints, sste_lora_plan *plan)
{
    if (!plan || !table || requests < 0 || (requests > 0 && (!offsets || !adapters))) return SSTE_ERR_INVALID_ARG;
    if (T < 0 || n_adapters < 1 || n_adapters > 65535 || min_tiles < 0 || (tile_rows != 0 && !tile_rows_ok(tile_rows)))
        return SSTE_ERR_INVALID_ARG;
    for (int i = 0; i < requests; ++i)
        if (offsets[i] < 0 || offsets[i + 1] < offsets[i] || offsets[i + 1] > T || adapters[i] < -1 || adapters[i] >= n_adapters)
            return SSTE_ERR_INVALID_ARG;
    auto count = [&](int rows_per_tile) {
        long long n = 0;
        each_tile(offsets, adapters, requests, rows_per_tile, [&](int, int, int) { ++n; });
        return n;
    };
    // As many rows to a tile as a run of rows has on average: what a tile has too many costs room in the scratch and blocks without work.  Below
    // 1024 rows there are too few tiles of 128 for the GPU (800 rows, 768 x 2304, rank 16: 6.5 us with tiles of 32, 8.1 with 128; 1600 rows: 9.3 and
    // 8.8; 4096: 17.3 and 12.6).
    int rows = tile_rows;
    if (rows == 0) {
        long long runs = 0, covered = requests > 0 ? static_cast<long long>(offsets[requests]) - offsets[0] : 0;
        for (int i = 0; i < requests; ++i) runs += i == 0 || adapters[i] != adapters[i - 1];
        for (rows = 16; rows < 128 && covered > rows * runs;) rows *= 2;
        if (rows > 32 && covered < 1024) rows = 32;
    }
    const long long n = count(rows), n_all = n > min_tiles ? n : min_tiles;
    const size_t at = lora_tiles_at(n_adapters);
    const size_t per_tile = static_cast<size_t>(rows) / 16, ints = 2 * at + 4 * static_cast<size_t>(n_all) * (1 + per_tile);
    if (n_all > LR_MAX_TILES || table_ints < ints) return SSTE_ERR_WORKSPACE;
    // counting sort by adapter, rows without one last; the table's own head holds the counters
    for (size_t i = 0; i < ints; ++i) table[i] = 0;
    each_tile(offsets, adapters, requests, rows, [&](int, int, int a) { if (a >= 0) ++table[a + 1]; });
    for (int a = 0; a < n_adapters; ++a) table[a + 1] += table[a];
    const int with = table[n_adapters];
    int without = with;
    auto put = [&](int i, int row, int r, int a) {
        int *t = table + at + 4 * static_cast<size_t>(i);
        t[0] = row;
        t[1] = r;
        t[2] = a;
        t[3] = 0;
    };
    each_tile(offsets, adapters, requests, rows, [&](int row, int r, int a) { put(a >= 0 ? table[a]++ : without++, row, r, a); });
    for (int a = n_adapters; a > 0; --a) table[a] = table[a - 1];         // (each counter has arrived at the next one's start)
    table[0] = 0;
    for (long long i = n; i < n_all; ++i) put(static_cast<int>(i), 0, 0, -1);
    // the groups of the tiles that have an adapter, in the tiles' order
    int *first = table + at + 4 * static_cast<size_t>(n_all), *group = first + at;
    int groups = 0;
    for (int a = 0; a < n_adapters; ++a) {
        first[a] = groups;
        for (int i = table[a]; i < table[a + 1]; ++i) {
            const int *t = table + at + 4 * static_cast<size_t>(i);
            for (int r = 0; r < t[1]; r += 16, ++groups, group += 4) {
                group[0] = t[0] + r;
                group[1] = t[1] - r < 16 ? t[1] - r : 16;
                group[2] = a;
                group[3] = static_cast<int>(static_cast<size_t>(i) * per_tile) + r / 16;
            }
        }
    }
    first[n_adapters] = groups;
    plan->T = T;
    plan->n_adapters = n_adapters;
    plan->tile_rows = rows;
    plan->n_tiles = static_cast<int>(n_all);
    plan->table = nullptr;
    return SSTE_OK;
}

// ---- the calls

extern "C" size_t sste_lora_scratch_bytes(const sste_lora *l, const sste_lora_plan *p)
{
    if (!l || !p || l->rank < 1 || l->rank > LR_MAX_RANK || l->n_adapters < 1 || l->I < 1 || l->O < 1 || p->T < 0 || p->n_tiles < 0 ||
        p->n_tiles > LR_MAX_TILES || !tile_rows_ok(p->tile_rows))
        return 0;
    return scratch_of(l, p).bytes;
}

extern "C" sste_status sste_lora_fwd(sste_ctx *ctx, const sste_lora *l, const sste_lora_plan *p, const void *X, long long ldx,
                                     const void *Y_in, void *Y_out, long long ldy, float *V, void *scratch, size_t scratch_bytes,
                                     void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    sste_status st = lora_ok(l, p);
    if (st != SSTE_OK) return st;
    if (p->T == 0 || p->n_tiles == 0) return SSTE_OK;
    if (!X || !Y_out || X == Y_out) return SSTE_ERR_INVALID_ARG;
    if ((st = rows_ok(X, ldx, l->I)) != SSTE_OK || (st = rows_ok(Y_out, ldy, l->O)) != SSTE_OK) return st;
    if (!sste_aligned(Y_in, 16) || !sste_aligned(V, 16) || !sste_aligned(scratch, 256)) return SSTE_ERR_ALIGN;
    const Scratch s = scratch_of(l, p);
    if (!scratch || scratch_bytes < s.bytes) return SSTE_ERR_WORKSPACE;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    char *w = static_cast<char *>(scratch);
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (p->tile_rows == TC_TILE) {
        LoraTcCall t{};
        t.l = l;
        t.p = p;
        t.tiles = tiles_of(p);
        t.x = X;
        t.ldx = static_cast<size_t>(ldx);
        t.y_in = Y_in;
        t.y_out = Y_out;
        t.ldy = static_cast<size_t>(ldy);
        t.v_out = V;
        t.tickets = reinterpret_cast<unsigned int *>(w);
        t.planes = w + s.u_by_row;
        t.partial = reinterpret_cast<float *>(w + s.partial);
        st = lora_tc_forward(ctx, t, cs);
        if (st == SSTE_OK) sste_count_launches(1);
        return st;
    }
    const Cut c = cut_of(p->n_tiles, p->tile_rows, p->T, l->I, l->O, l->I, l->O, l->n_adapters, l->rank);
    const ShrinkArgs a{static_cast<const uint16_t *>(X), static_cast<const uint16_t *>(l->A), l->scale, tiles_of(p), V,
                       reinterpret_cast<uint4 *>(w + s.by_rank), nullptr, nullptr, nullptr, nullptr, nullptr, reinterpret_cast<float *>(w + s.partial),
                       reinterpret_cast<unsigned int *>(w), static_cast<size_t>(ldx), p->T, l->I, l->rank, l->n_adapters, p->tile_rows,
                       c.shrink_splits};
    const ExpandArgs e{a.by_rank, static_cast<const uint16_t *>(l->B), a.tiles, static_cast<const uint16_t *>(Y_in),
                       static_cast<uint16_t *>(Y_out), static_cast<size_t>(ldy), p->T, l->O, l->rank, l->n_adapters, c.expand_shares};
    st = by_rank(l->rank, [&](auto R) {
        const sste_status first = shrink_rows<decltype(R)::value, false>(ctx, a, p->n_tiles, c.shrink_rows, cs);
        return first != SSTE_OK ? first : expand_launch<decltype(R)::value, false>(ctx, e, p->n_tiles, p->tile_rows, cs);
    });
    if (st == SSTE_OK) sste_count_launches(2);
    return st;
}

extern "C" sste_status sste_lora_bwd(sste_ctx *ctx, const sste_lora *l, const sste_lora_plan *p, const void *X, long long ldx,
                                     const void *X_codes, const void *X_scales, sste_ckpt_format fmt, const void *dY, long long ldy,
                                     const float *V, const void *dX_in, void *dX_out, long long lddx, void *dA, void *dB,
                                     sste_dtype gdt, void *scratch, size_t scratch_bytes, void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    sste_status st = lora_ok(l, p);
    if (st != SSTE_OK) return st;
    const bool grads = dA || dB, kept = X_codes != nullptr;
    if (!dA != !dB || (!grads && !dX_out) || (dX_in && !dX_out)) return SSTE_ERR_INVALID_ARG;
    if (grads && gdt != SSTE_BF16 && gdt != SSTE_F32) return SSTE_ERR_DTYPE;
    const size_t elt = gdt == SSTE_F32 ? 4 : 2;
    if (grads && (!sste_aligned(dA, 16) || !sste_aligned(dB, 16))) return SSTE_ERR_ALIGN;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (p->T == 0 || p->n_tiles == 0) {                          // no rows: the sums are empty
        if (!grads) return SSTE_OK;
        sste_device_guard guard(ctx->device);
        if (!guard.ok) return SSTE_ERR_CUDA;
        const size_t n = static_cast<size_t>(l->n_adapters) * l->rank;
        SSTE_CUDA_TRY(cudaMemsetAsync(dA, 0, n * l->I * elt, cs));
        SSTE_CUDA_TRY(cudaMemsetAsync(dB, 0, n * l->O * elt, cs));
        return SSTE_OK;
    }
    if (!dY || dY == dX_out || (grads && (!V || (X && X == dX_out) || kept == (X != nullptr) || kept != (X_scales != nullptr)))) return SSTE_ERR_INVALID_ARG;
    if (grads && kept && fmt != SSTE_CKPT_E4M3 && fmt != SSTE_CKPT_INT8) return SSTE_ERR_INVALID_ARG;
    if ((st = rows_ok(dY, ldy, l->O)) != SSTE_OK || (dX_out && (st = rows_ok(dX_out, lddx, l->I)) != SSTE_OK)) return st;
    if (grads && !kept && (st = rows_ok(X, ldx, l->I)) != SSTE_OK) return st;
    if (!sste_aligned(X_codes, 16) || !sste_aligned(X_scales, 4) || !sste_aligned(dX_in, 16) || !sste_aligned(V, 16) || !sste_aligned(scratch, 256)) return SSTE_ERR_ALIGN;
    if (grads && p->tile_rows == TC_TILE && !lora_tc_grads_fit(l, p, gdt)) return SSTE_ERR_SHAPE;
    const Scratch s = scratch_of(l, p);
    if (!scratch || scratch_bytes < s.bytes) return SSTE_ERR_WORKSPACE;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    char *w = static_cast<char *>(scratch);
    if (p->tile_rows == TC_TILE) {
        LoraTcCall t{};
        t.l = l;
        t.p = p;
        t.first_tile = static_cast<const int *>(p->table);
        t.tiles = tiles_of(p);
        t.x = dY;
        t.ldx = static_cast<size_t>(ldy);
        t.y_in = dX_in;
        t.y_out = dX_out;
        t.ldy = static_cast<size_t>(lddx);
        t.grads = grads;
        t.v_in = V;
        t.X = X;
        t.ldX = static_cast<size_t>(ldx);
        t.X_codes = X_codes;
        t.X_scales = X_scales;
        t.fmt = fmt;
        t.dA = dA;
        t.dB = dB;
        t.gdt = gdt;
        t.tickets = reinterpret_cast<unsigned int *>(w);
        t.planes = w + s.u_by_row;
        t.v_planes = w + s.v_by_row;
        t.partial = reinterpret_cast<float *>(w + s.partial);
        st = lora_tc_backward(ctx, t, cs);
        if (st == SSTE_OK) sste_count_launches(1 + (grads ? 1 : 0));
        return st;
    }
    const Cut c = cut_of(p->n_tiles, p->tile_rows, p->T, l->O, l->I, l->I, l->O, l->n_adapters, l->rank);
    const int columns = columns_of(lora_rank_up(l->rank));
    uint4 *u_by_row = reinterpret_cast<uint4 *>(w + s.u_by_row), *v_by_row = reinterpret_cast<uint4 *>(w + s.v_by_row);
    uint2 *u_rest = reinterpret_cast<uint2 *>(w + s.u_rest), *v_rest = reinterpret_cast<uint2 *>(w + s.v_rest);
    const ShrinkArgs a{static_cast<const uint16_t *>(dY), static_cast<const uint16_t *>(l->B), l->scale, tiles_of(p), nullptr,
                       reinterpret_cast<uint4 *>(w + s.by_rank), grads ? u_by_row : nullptr, V, v_by_row, grads && gdt == SSTE_F32 ? u_rest : nullptr, v_rest,
                       reinterpret_cast<float *>(w + s.partial), reinterpret_cast<unsigned int *>(w), static_cast<size_t>(ldy), p->T, l->O,
                       l->rank, l->n_adapters, p->tile_rows, c.shrink_splits};
    GradArgs g{};
    g.job[0] = GradJob{u_by_row, u_rest, static_cast<const uint16_t *>(X), static_cast<const uint8_t *>(X_codes),
                       static_cast<const uint8_t *>(X_scales), dA, static_cast<size_t>(ldx), sste_ckpt_scale_bytes(static_cast<size_t>(p->T) * l->I), l->I, (l->I + columns - 1) / columns, false};
    g.job[1] = GradJob{v_by_row, v_rest, static_cast<const uint16_t *>(dY), nullptr, nullptr, dB, static_cast<size_t>(ldy), 0, l->O,
                       (l->O + columns - 1) / columns, true};
    g.first_group = reinterpret_cast<const int *>(a.tiles + p->n_tiles);
    g.groups = reinterpret_cast<const int4 *>(g.first_group + lora_tiles_at(p->n_adapters));
    g.partial = a.partial;
    g.tickets = a.tickets + LR_TICKETS;
    g.T = p->T;
    g.r = l->rank;
    g.n_adapters = l->n_adapters;
    g.n_tiles = p->n_tiles;
    g.tile_rows = p->tile_rows;
    g.splits = c.grad_splits;
    const ExpandArgs e{a.by_rank, static_cast<const uint16_t *>(l->A), a.tiles, static_cast<const uint16_t *>(dX_in),
                       static_cast<uint16_t *>(dX_out), static_cast<size_t>(lddx), p->T, l->I, l->rank, l->n_adapters, c.expand_shares};
    const int z = !kept ? Z_BF16 : fmt == SSTE_CKPT_E4M3 ? Z_E4M3 : Z_INT8;
    st = by_rank(l->rank, [&](auto R) {
        constexpr int N = decltype(R)::value;
        sste_status one = shrink_rows<N, true>(ctx, a, p->n_tiles, c.shrink_rows, cs);
        if (one == SSTE_OK && grads) one = grad_by_type<N>(ctx, g, z, gdt, cs);
        if (one == SSTE_OK && dX_out) one = expand_launch<N, true>(ctx, e, p->n_tiles, p->tile_rows, cs);
        return one;
    });
    if (st == SSTE_OK) sste_count_launches(1 + (grads ? 1 : 0) + (dX_out ? 1 : 0));
    return st;
}
