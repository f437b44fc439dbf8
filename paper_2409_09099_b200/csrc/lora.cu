// Low-rank adapters of many requests beside a shared linear: V = s X A^T, Y += V B^T, and their gradients U = s dY B, dX += U A,
// dA = U^T X, dB = dY^T V.
//
// With a rank of 8 to 64 these products do 8 to 64 multiply-adds for each element they stream, so memory bounds them and the tensor
// cores only have to keep up.  Every operand goes from memory straight to the registers that the instruction takes it from: the order
// of a reduction and of the output's columns is free as long as both sides agree on it, so each thread takes 16 consecutive bytes
// wherever the instruction's own layout would ask for four scattered pairs (`kperm` and `nperm` below), and no tile passes through
// shared memory.  Operands whose reduction runs across rows are paired with a byte permutation of two rows that the thread itself has loaded.
#include "common.cuh"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace {

constexpr int LR_WARPS = 8, LR_THREADS = 32 * LR_WARPS;
constexpr int LR_MAX_RANK = 64;

// 16 x 8 += 16 x 16 times 16 x 8, bf16 with fp32 sums
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
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
__device__ __forceinline__ float2 unpack2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
// element `k` of two rows as a pair
__device__ __forceinline__ uint32_t pair_of(uint32_t first, uint32_t second, int k) { return __byte_perm(first, second, k & 1 ? 0x7632 : 0x5410); }

__device__ __forceinline__ uint4 ld16(const uint16_t *p, bool valid)
{
    return valid ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ uint4 ld16_once(const uint16_t *p, bool valid)
{
    uint4 v = make_uint4(0, 0, 0, 0);
    if (valid)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
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

// The plan's table: the first tile of each adapter (n_adapters + 1 of them, filled up to a multiple of four), then the tiles.
__host__ __device__ inline size_t tiles_at(int n_adapters) { return (static_cast<size_t>(n_adapters) + 1 + 3) / 4 * 4; }
struct Tile { int row, rows, adapter; };
__device__ __forceinline__ Tile tile_of(const int4 *tiles, int i, int tile_rows, int T, int n_adapters)
{
    const int4 t = tiles[i];
    // a table that is not the library's own is not followed out of the tensors
    const bool ok = t.x >= 0 && t.y > 0 && t.y <= tile_rows && t.x <= T - t.y && t.z >= -1 && t.z < n_adapters;
    return Tile{t.x, ok ? t.y : 0, t.z};
}

struct ApplyArgs {
    const uint16_t *x;                  // [T, K], reduced over K
    const uint16_t *a;                  // per adapter [r, K]; TRANS: [K, r]
    const uint16_t *b;                  // per adapter [N, r]; TRANS: [r, N]
    const float *scale;
    const int4 *tiles;
    const uint16_t *y_in;               // [T, N]; null: zeros
    uint16_t *y_out;                    // null: V alone
    float *v;                           // [T, r] or null
    size_t ldx, ldy;
    int T, K, N, r, n_adapters;
};

// V = s x a^T of a tile's rows, then y_out = y_in + V b^T: the forward (x = X, y = Y), and with both weights read across their rows
// (TRANS) the backward (x = dY, y = dX, V = U).
//
// A cluster of C blocks works on a tile: block c reduces the c-th part of K, the blocks exchange their sums through each other's shared
// memory (each sums a C-th of the rows, in the blocks' order, and hands the result to all), then each writes the c-th part of N.  So a
// few rows keep many SMs busy, V takes no trip through memory, and there is one launch and no workspace.  Sums have a fixed
// order.
template <int R, int MT, int WM, bool TRANS>
__global__ void __launch_bounds__(LR_THREADS, 2)
lora_apply_kernel(const ApplyArgs in)
{
    constexpr int WK = LR_WARPS / WM, TM = 16 * MT * WM, NT = R / 8, PITCH = R + 4;
    extern __shared__ float4 smem4[];
    float *part = reinterpret_cast<float *>(smem4);            // [WK][TM][PITCH]
    float *whole = part + WK * TM * PITCH;                     // [TM][PITCH]
    cg::cluster_group cluster = cg::this_cluster();
    const int C = static_cast<int>(cluster.num_blocks()), c = static_cast<int>(cluster.block_rank());
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;

    ApplyArgs p = in;
    sste_pdl_trigger();
    sste_pdl_wait(p.x, p.a, p.b, p.scale, p.tiles, p.y_in);
    const Tile tile = tile_of(p.tiles, static_cast<int>(blockIdx.x) / C, TM, p.T, p.n_adapters);
    if (tile.rows == 0) return;                                // (of all blocks of the cluster)
    const int groups = (p.N + 63) / 64, first = static_cast<int>(static_cast<long long>(groups) * c / C),
              last = static_cast<int>(static_cast<long long>(groups) * (c + 1) / C);
    if (tile.adapter < 0) {                                    // no adapter: the rows as they are
        if (!p.y_out || p.y_in == p.y_out) return;
        const int n0 = first * 64, vecs = ((last * 64 < p.N ? last * 64 : p.N) - n0) / 8;
        for (int i = threadIdx.x; i < tile.rows * vecs; i += LR_THREADS) {
            const size_t at = static_cast<size_t>(tile.row + i / vecs) * p.ldy + n0 + 8 * (i % vecs);
            *reinterpret_cast<uint4 *>(p.y_out + at) = p.y_in ? ld16(p.y_in + at, true) : make_uint4(0, 0, 0, 0);
        }
        return;
    }
    const uint16_t *wa = p.a + static_cast<size_t>(tile.adapter) * p.r * p.K;
    const uint16_t *wb = p.b + static_cast<size_t>(tile.adapter) * p.r * p.N;

    // ---- this block's part of x a^T.  A warp takes groups of 32 of K for MT * 16 rows.  kperm: a thread's 16 bytes are k = 8q .. 8q + 7
    // of the group; step s of 16 takes 8q + 4s + {0, 1} for the instruction's k = 2q, 2q + 1 and the next two for 2q + 8, 2q + 9.
    {
        const int wm = warp % WM, wk = warp / WM;
        float acc[MT][NT][4] = {};
        const int kg_all = (p.K + 31) / 32;
        const int kg_end = static_cast<int>(static_cast<long long>(kg_all) * (c + 1) / C);
        for (int kg = static_cast<int>(static_cast<long long>(kg_all) * c / C) + wk; kg < kg_end; kg += WK) {
            const int k = kg * 32 + 8 * q;
            uint4 x0[MT], x1[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int row = (wm * MT + m) * 16 + g;
                const uint16_t *at = p.x + static_cast<size_t>(tile.row + row) * p.ldx + k;
                x0[m] = ld16_once(at, k < p.K && row < tile.rows);
                x1[m] = ld16_once(at + 8 * p.ldx, k < p.K && row + 8 < tile.rows);
            }
            uint32_t b[2][NT][2];
            if constexpr (!TRANS) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const int n = 8 * j + g;
                    const uint4 w = ld16(wa + static_cast<size_t>(n) * p.K + k, k < p.K && n < p.r);
                    b[0][j][0] = w.x;
                    b[0][j][1] = w.y;
                    b[1][j][0] = w.z;
                    b[1][j][1] = w.w;
                }
            } else {
                // column n = g of tile j is r = NT g + j: one load of NT values per row
                uint32_t w[8][NT / 2];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    ld_words(w[i], wa + static_cast<size_t>(k + i) * p.r + NT * g, k < p.K && NT * g < p.r);
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        b[s][j][0] = pair_of(w[4 * s][j / 2], w[4 * s + 1][j / 2], j);
                        b[s][j][1] = pair_of(w[4 * s + 2][j / 2], w[4 * s + 3][j / 2], j);
                    }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    mma(acc[m][j], x0[m].x, x1[m].x, x0[m].y, x1[m].y, b[0][j][0], b[0][j][1]);
                    mma(acc[m][j], x0[m].z, x1[m].z, x0[m].w, x1[m].w, b[1][j][0], b[1][j][1]);
                }
        }
        float *mine = part + wk * TM * PITCH;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = (wm * MT + m) * 16 + g;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float *at = mine + (row + 8 * h) * PITCH;
                    if constexpr (!TRANS) {
                        *reinterpret_cast<float2 *>(at + 8 * j + 2 * q) = make_float2(acc[m][j][2 * h], acc[m][j][2 * h + 1]);
                    } else {
                        at[NT * 2 * q + j] = acc[m][j][2 * h];
                        at[NT * (2 * q + 1) + j] = acc[m][j][2 * h + 1];
                    }
                }
        }
    }
    __syncthreads();

    // ---- the sums over warps, then over the cluster's blocks
    constexpr int QUADS = TM * R / 4, QROW = R / 4;
    const float s = p.scale[tile.adapter];
    const int q_begin = QUADS * c / C, q_end = QUADS * (c + 1) / C;
    if (C > 1) {
        for (int i = threadIdx.x; i < QUADS; i += LR_THREADS) {
            float4 *at = reinterpret_cast<float4 *>(part + (i / QROW) * PITCH + 4 * (i % QROW));
            float4 sum = *at;
#pragma unroll
            for (int w = 1; w < WK; ++w) {
                const float4 v = at[w * (TM * PITCH / 4)];
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
            *at = sum;
        }
        cluster.sync();
    }
    for (int i = q_begin + threadIdx.x; i < q_end; i += LR_THREADS) {
        const int row = i / QROW, col = 4 * (i % QROW);
        float *at = part + row * PITCH + col;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (C > 1) {
            for (int k = 0; k < C; ++k) {
                const float4 v = *reinterpret_cast<const float4 *>(cluster.map_shared_rank(at, k));
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
        } else {
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float4 v = *reinterpret_cast<const float4 *>(at + w * TM * PITCH);
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
        }
        // (columns that fill the rank up are zeros whatever x holds)
        sum = col < p.r ? make_float4(s * sum.x, s * sum.y, s * sum.z, s * sum.w) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p.v && row < tile.rows && col < p.r)
            *reinterpret_cast<float4 *>(p.v + static_cast<size_t>(tile.row + row) * p.r + col) = sum;
        float *to = whole + row * PITCH + col;
        for (int k = 0; k < C; ++k) *reinterpret_cast<float4 *>(cluster.map_shared_rank(to, k)) = sum;
    }
    if (C > 1) cluster.sync();
    else __syncthreads();
    if (!p.y_out) return;

    // ---- this block's part of y.  A warp takes 16 rows and groups of 64 columns.  nperm: column n = i of the instruction's tile j is
    // 8i + j of the group, so a thread's outputs are 16 consecutive columns.
    constexpr int MTILES = TM / 16, SPLIT = LR_WARPS / MTILES, KS = R / 16;
    const int m = warp % MTILES, row = m * 16 + g;
    if (m * 16 >= tile.rows) return;
    Split va[KS][4];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        const int r0 = R == 16 ? 4 * q : 32 * (k / 2) + 8 * q + 4 * (k % 2);
        const float4 v0 = *reinterpret_cast<const float4 *>(whole + row * PITCH + r0);
        const float4 v1 = *reinterpret_cast<const float4 *>(whole + (row + 8) * PITCH + r0);
        va[k][0] = split2(v0.x, v0.y);
        va[k][1] = split2(v1.x, v1.y);
        va[k][2] = split2(v0.z, v0.w);
        va[k][3] = split2(v1.z, v1.w);
    }
    const bool row_ok[2] = {row < tile.rows, row + 8 < tile.rows};
    const size_t y_at = static_cast<size_t>(tile.row + row) * p.ldy;
    for (int n_group = first + warp / MTILES; n_group < last; n_group += SPLIT) {
        const int n0 = n_group * 64, col = n0 + 16 * q;
        uint4 y[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                y[h][e] = ld16_once(p.y_in + y_at + 8 * h * p.ldy + col + 8 * e, p.y_in && row_ok[h] && col + 8 * e < p.N);
        float acc[8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t w[4] = {y[h][e].x, y[h][e].y, y[h][e].z, y[h][e].w};
                    const float2 f = unpack2(w[j / 2]);
                    acc[j][2 * h + e] = j & 1 ? f.y : f.x;
                }
        if constexpr (!TRANS) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int n = n0 + 8 * g + j;
                const uint16_t *at = wb + static_cast<size_t>(n) * p.r;
                if constexpr (R == 16) {
                    uint32_t w[2];
                    ld_words(w, at + 4 * q, n < p.N && 4 * q < p.r);
                    mma(acc[j], va[0][0].hi, va[0][1].hi, va[0][2].hi, va[0][3].hi, w[0], w[1]);
                    mma(acc[j], va[0][0].lo, va[0][1].lo, va[0][2].lo, va[0][3].lo, w[0], w[1]);
                } else {
#pragma unroll
                    for (int k = 0; k < KS; k += 2) {
                        const uint4 w = ld16(at + 16 * k + 8 * q, n < p.N && 16 * k + 8 * q < p.r);
                        mma(acc[j], va[k][0].hi, va[k][1].hi, va[k][2].hi, va[k][3].hi, w.x, w.y);
                        mma(acc[j], va[k][0].lo, va[k][1].lo, va[k][2].lo, va[k][3].lo, w.x, w.y);
                        mma(acc[j], va[k + 1][0].hi, va[k + 1][1].hi, va[k + 1][2].hi, va[k + 1][3].hi, w.z, w.w);
                        mma(acc[j], va[k + 1][0].lo, va[k + 1][1].lo, va[k + 1][2].lo, va[k + 1][3].lo, w.z, w.w);
                    }
                }
            }
        } else {
            const int n = n0 + 8 * g;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int r0 = R == 16 ? 4 * q : 32 * (k / 2) + 8 * q + 4 * (k % 2);
                uint32_t w[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) ld_words(w[i], wb + static_cast<size_t>(r0 + i) * p.N + n, n < p.N && r0 < p.r);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t b0 = pair_of(w[0][j / 2], w[1][j / 2], j), b1 = pair_of(w[2][j / 2], w[3][j / 2], j);
                    mma(acc[j], va[k][0].hi, va[k][1].hi, va[k][2].hi, va[k][3].hi, b0, b1);
                    mma(acc[j], va[k][0].lo, va[k][1].lo, va[k][2].lo, va[k][3].lo, b0, b1);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (!row_ok[h] || col + 8 * e >= p.N) continue;
                const int i = 2 * h + e;
                *reinterpret_cast<uint4 *>(p.y_out + y_at + 8 * h * p.ldy + col + 8 * e) =
                    make_uint4(pack2(acc[0][i], acc[1][i]), pack2(acc[2][i], acc[3][i]), pack2(acc[4][i], acc[5][i]),
                               pack2(acc[6][i], acc[7][i]));
            }
    }
}

// ---------------------------------------------------------------- gradients of the weights

// One of the two sums over rows: out [r, N] = s^T z (dA: s = U, z = X), or its transpose [N, r] (dB: s = V, z = dY).
struct GradJob {
    const float *s;                     // [T, r]
    const uint16_t *z;                  // [T, N] bf16, or null and the kept form
    const uint8_t *codes, *scales;
    void *out;
    size_t ldz;
    int N;
    int blocks;                         // of 128 columns
    bool across;                        // out is [N, r]
};
struct GradArgs {
    GradJob job[2];
    const int *first_tile;
    const int4 *tiles;
    int T, r, n_adapters, n_tiles, tile_rows;
};

// eight kept values (within one block) as bf16 pairs
template <bool E4M3>
__device__ __forceinline__ void restore8(uint2 q, float by, uint32_t (&out)[4])
{
    const uint32_t w[2] = {q.x, q.y};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float f[4];
        if (E4M3) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[k] >> (16 * j)),
                                                                                   __NV_E4M3)));
                f[2 * j] = v.x * by;
                f[2 * j + 1] = v.y * by;
            }
        } else {
            const uint32_t u = w[k] ^ 0x80808080u;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 | j)) - 8388736.0f) * by;
            if ((u - 0x01010101u) & ~u & 0x80808080u) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if ((u >> (8 * j) & 0xffu) == 0) f[j] = __uint_as_float(0x7fc00000u);
            }
        }
        out[2 * k] = pack2(f[0], f[1]);
        out[2 * k + 1] = pack2(f[2], f[3]);
    }
}

enum { Z_BF16 = 0, Z_E4M3 = 1, Z_INT8 = 2 };

// The instruction's rows are the rank (16 at a time), its columns the features, its reduction the tokens: a thread takes rows 4q .. 4q + 3 of
// 16 tokens.  A warp sums over every (WT * C)-th group of 16 tokens of the adapter's tiles for 64 columns and up to 32 of the rank;
// then the warps of a block and the blocks of a cluster add up in a fixed order.
template <int R, int Z>
__device__ __forceinline__ void grad_partial(const GradArgs &p, const GradJob &job, int adapter, int n0, int m0, int worker, int workers,
                                             float (&acc)[R / 16 < 2 ? R / 16 : 2][8][4])
{
    constexpr int MW = R / 16 < 2 ? R / 16 : 2;
    const int lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;
    const int per_tile = p.tile_rows / 16;
    int begin = p.first_tile[adapter], end = p.first_tile[adapter + 1];
    if (begin < 0 || end > p.n_tiles) return;
    const int col = n0 + 8 * g;
    const int steps = (end - begin) * per_tile;
    for (int f = worker; f < steps; f += workers) {
        const Tile tile = tile_of(p.tiles, begin + f / per_tile, p.tile_rows, p.T, p.n_adapters);
        const int in_tile = (f % per_tile) * 16;
        if (in_tile >= tile.rows || tile.adapter != adapter) continue;
        uint32_t w[4][4];
        float s[MW][4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = in_tile + 4 * q + i;
            const bool ok = row < tile.rows;
            const size_t t = static_cast<size_t>(tile.row + row);
            if constexpr (Z == Z_BF16) {
                const uint4 v = ld16_once(job.z + t * job.ldz + col, ok && col < job.N);
                w[i][0] = v.x;
                w[i][1] = v.y;
                w[i][2] = v.z;
                w[i][3] = v.w;
            } else {
                const size_t at = t * job.N + col;
                const bool in = ok && col < job.N;
                const uint2 v = in ? *reinterpret_cast<const uint2 *>(job.codes + at) : make_uint2(Z == Z_INT8 ? 0u : 0u, 0u);
                const float by = in ? __uint_as_float(static_cast<uint32_t>(job.scales[at / 32]) << 23) : 0.0f;
                restore8<Z == Z_E4M3>(v, by, w[i]);
            }
#pragma unroll
            for (int m = 0; m < MW; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = 16 * (m0 + m) + g + 8 * h;
                    s[m][i][h] = ok && r < p.r ? job.s[t * p.r + r] : 0.0f;
                }
        }
        Split a[MW][4];
#pragma unroll
        for (int m = 0; m < MW; ++m) {
            a[m][0] = split2(s[m][0][0], s[m][1][0]);
            a[m][1] = split2(s[m][0][1], s[m][1][1]);
            a[m][2] = split2(s[m][2][0], s[m][3][0]);
            a[m][3] = split2(s[m][2][1], s[m][3][1]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b0 = pair_of(w[0][j / 2], w[1][j / 2], j), b1 = pair_of(w[2][j / 2], w[3][j / 2], j);
#pragma unroll
            for (int m = 0; m < MW; ++m) {
                mma(acc[m][j], a[m][0].hi, a[m][1].hi, a[m][2].hi, a[m][3].hi, b0, b1);
                mma(acc[m][j], a[m][0].lo, a[m][1].lo, a[m][2].lo, a[m][3].lo, b0, b1);
            }
        }
    }
}

template <int R, int Z, typename OUT>
__global__ void __launch_bounds__(LR_THREADS, 2)
lora_grad_kernel(const GradArgs in)
{
    constexpr int MW = R / 16 < 2 ? R / 16 : 2, WM = R / 16 / MW, WN = 2, WT = LR_WARPS / (WN * WM), PITCH = 128 + 4;
    __shared__ __align__(16) float red[R * PITCH];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = static_cast<int>(cluster.num_blocks()), c = static_cast<int>(cluster.block_rank());
    GradArgs p = in;
    sste_pdl_trigger();
    sste_pdl_wait(p.job[0].s, p.job[0].z, p.job[0].codes, p.job[0].scales, p.job[1].s, p.job[1].z, p.first_tile, p.tiles);
    int block = static_cast<int>(blockIdx.x) / C;
    const bool second = block >= p.job[0].blocks;
    if (second) block -= p.job[0].blocks;
    const GradJob job = second ? p.job[1] : p.job[0];
    const int adapter = blockIdx.y;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;
    const int wn = warp % WN, wm = warp / WN % WM, wt = warp / (WN * WM);

    float acc[MW][8][4] = {};
    const int n0 = block * 128 + wn * 64, worker = c * WT + wt, workers = C * WT;
    if (n0 < job.N) {
        if (Z == Z_BF16 || second) grad_partial<R, Z_BF16>(p, job, adapter, n0, wm * MW, worker, workers, acc);
        else grad_partial<R, Z>(p, job, adapter, n0, wm * MW, worker, workers, acc);
    }
    for (int w = 0; w < WT; ++w) {
        if (wt == w) {
#pragma unroll
            for (int m = 0; m < MW; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float *at = red + (16 * (wm * MW + m) + g + 8 * h) * PITCH + wn * 64 + 16 * q;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float v = acc[m][j][2 * h + e];
                            at[8 * e + j] = w ? at[8 * e + j] + v : v;
                        }
                }
        }
        __syncthreads();
    }
    if (C > 1) cluster.sync();
    OUT *out = static_cast<OUT *>(job.out) + static_cast<size_t>(adapter) * p.r * job.N;
    const int total = 128 * R, begin = static_cast<int>(static_cast<long long>(total) * c / C),
              end = static_cast<int>(static_cast<long long>(total) * (c + 1) / C);
    for (int i = begin + threadIdx.x; i < end; i += LR_THREADS) {
        const int r = job.across ? i % R : i / 128, n = job.across ? i / R : i % 128;
        float sum = 0.0f;
        for (int k = 0; k < C; ++k) sum += *cluster.map_shared_rank(red + r * PITCH + n, k);
        const int col = block * 128 + n;
        if (r >= p.r || col >= job.N) continue;
        const size_t at = job.across ? static_cast<size_t>(col) * p.r + r : static_cast<size_t>(r) * job.N + col;
        if constexpr (sizeof(OUT) == 2) out[at] = __float2bfloat16_rn(sum);
        else out[at] = sum;
    }
    if (C > 1) cluster.sync();                                 // (nobody leaves while its sums are read)
}

// ---------------------------------------------------------------- host

template <typename... KArgs>
cudaError_t launch_cluster(void (*kern)(KArgs...), dim3 grid, int cluster, size_t smem, cudaStream_t stream, KArgs... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(LR_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <int R, int MT, int WM, bool TRANS>
sste_status apply_launch(const sste_ctx *ctx, const ApplyArgs &p, int n_tiles, cudaStream_t stream)
{
    constexpr int TM = 16 * MT * WM, WK = LR_WARPS / WM;
    constexpr size_t smem = static_cast<size_t>(WK + 1) * TM * (R + 4) * sizeof(float);
    auto *kern = lora_apply_kernel<R, MT, WM, TRANS>;
    static DeviceOnce once;
    if (!once.run(ctx->device, [&] {
            return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) == cudaSuccess;
        }))
        return SSTE_ERR_CUDA;
    // blocks to a tile: enough that two blocks an SM have work, while each still has a group of 32 of K and one of 64 of N
    int C = 1;
    while (C < 8 && static_cast<long long>(n_tiles) * C < 2 * ctx->sm_count && (p.K + 31) / 32 >= 2 * C && (p.N + 63) / 64 >= 2 * C) C *= 2;
    if (launch_cluster(kern, dim3(static_cast<unsigned>(n_tiles) * C), C, smem, stream, p) != cudaSuccess) return SSTE_ERR_CUDA;
    sste_count_launches(1);
    return SSTE_OK;
}

template <int R, bool TRANS>
sste_status apply_rows(const sste_ctx *ctx, const ApplyArgs &p, int n_tiles, int tile_rows, cudaStream_t stream)
{
    // shares of a block's eight warps: along the rows where a tile has many, else along K; a rank of 64 has sums for 32 rows a warp
    switch (tile_rows) {
    case 16: return apply_launch<R, 1, 1, TRANS>(ctx, p, n_tiles, stream);
    case 32: return apply_launch<R, 2, 1, TRANS>(ctx, p, n_tiles, stream);
    case 64: return apply_launch<R, 2, 2, TRANS>(ctx, p, n_tiles, stream);
    default: return apply_launch<R, R == 64 ? 2 : 4, R == 64 ? 4 : 2, TRANS>(ctx, p, n_tiles, stream);
    }
}

template <bool TRANS>
sste_status apply(const sste_ctx *ctx, const ApplyArgs &p, int n_tiles, int tile_rows, cudaStream_t stream)
{
    if (p.r <= 16) return apply_rows<16, TRANS>(ctx, p, n_tiles, tile_rows, stream);
    if (p.r <= 32) return apply_rows<32, TRANS>(ctx, p, n_tiles, tile_rows, stream);
    return apply_rows<64, TRANS>(ctx, p, n_tiles, tile_rows, stream);
}

bool tile_rows_ok(int rows) { return rows == 16 || rows == 32 || rows == 64 || rows == 128; }

sste_status lora_ok(const sste_lora *l, const sste_lora_plan *p)
{
    if (!l || !p || !l->A || !l->B || !l->scale || (!p->table && p->n_tiles > 0)) return SSTE_ERR_INVALID_ARG;
    if (l->n_adapters < 1 || l->n_adapters > 65535 || p->n_adapters != l->n_adapters || p->T < 0 || p->n_tiles < 0 ||
        !tile_rows_ok(p->tile_rows))
        return SSTE_ERR_INVALID_ARG;
    if (l->rank < 8 || l->rank > LR_MAX_RANK || l->rank % 8 || l->I < 8 || l->I % 8 || l->O < 8 || l->O % 8) return SSTE_ERR_SHAPE;
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
const int4 *tiles_of(const sste_lora_plan *p) { return reinterpret_cast<const int4 *>(static_cast<const int *>(p->table) + tiles_at(p->n_adapters)); }

}  // namespace

// ---- the plan

extern "C" size_t sste_lora_plan_ints(int T, int requests, int n_adapters, int min_tiles)
{
    if (T < 0 || requests < 0 || n_adapters < 1) return 0;
    const size_t tiles = static_cast<size_t>(T) / 16 + static_cast<size_t>(requests);
    return tiles_at(n_adapters) + 4 * (min_tiles > 0 && static_cast<size_t>(min_tiles) > tiles ? static_cast<size_t>(min_tiles) : tiles);
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
    // the largest tiles (a weight is read once per tile) of which eight blocks each still fill the GPU twice over
    int rows = tile_rows;
    if (rows == 0)
        for (rows = 128; rows > 16 && count(rows) * 8 < 2 * 148; rows /= 2) {}
    const long long n = count(rows), n_all = n > min_tiles ? n : min_tiles;
    const size_t at = tiles_at(n_adapters);
    if (n_all > 0x0fffffff || table_ints < at + 4 * static_cast<size_t>(n_all)) return SSTE_ERR_WORKSPACE;
    // counting sort by adapter, rows without one last; the table's own head holds the counters
    for (size_t i = 0; i < at; ++i) table[i] = 0;
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
    plan->T = T;
    plan->n_adapters = n_adapters;
    plan->tile_rows = rows;
    plan->n_tiles = static_cast<int>(n_all);
    plan->table = nullptr;
    return SSTE_OK;
}

// ---- the calls

extern "C" sste_status sste_lora_fwd(sste_ctx *ctx, const sste_lora *l, const sste_lora_plan *p, const void *X, long long ldx,
                                     const void *Y_in, void *Y_out, long long ldy, float *V, void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    sste_status st = lora_ok(l, p);
    if (st != SSTE_OK) return st;
    if (p->T == 0 || p->n_tiles == 0) return SSTE_OK;
    if (!X || !Y_out) return SSTE_ERR_INVALID_ARG;
    if ((st = rows_ok(X, ldx, l->I)) != SSTE_OK || (st = rows_ok(Y_out, ldy, l->O)) != SSTE_OK) return st;
    if (!sste_aligned(Y_in, 16) || !sste_aligned(V, 16)) return SSTE_ERR_ALIGN;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    const ApplyArgs a{static_cast<const uint16_t *>(X), static_cast<const uint16_t *>(l->A), static_cast<const uint16_t *>(l->B),
                      l->scale, tiles_of(p), static_cast<const uint16_t *>(Y_in), static_cast<uint16_t *>(Y_out), V,
                      static_cast<size_t>(ldx), static_cast<size_t>(ldy), p->T, l->I, l->O, l->rank, l->n_adapters};
    return apply<false>(ctx, a, p->n_tiles, p->tile_rows, static_cast<cudaStream_t>(stream));
}

extern "C" sste_status sste_lora_bwd_input(sste_ctx *ctx, const sste_lora *l, const sste_lora_plan *p, const void *dY, long long ldy,
                                           const void *dX_in, void *dX_out, long long ldx, float *U, void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    sste_status st = lora_ok(l, p);
    if (st != SSTE_OK) return st;
    if (p->T == 0 || p->n_tiles == 0) return SSTE_OK;
    if (!dY || (!dX_out && !U) || (dX_in && !dX_out)) return SSTE_ERR_INVALID_ARG;
    if ((st = rows_ok(dY, ldy, l->O)) != SSTE_OK || (dX_out && (st = rows_ok(dX_out, ldx, l->I)) != SSTE_OK)) return st;
    if (!sste_aligned(dX_in, 16) || !sste_aligned(U, 16)) return SSTE_ERR_ALIGN;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    const ApplyArgs a{static_cast<const uint16_t *>(dY), static_cast<const uint16_t *>(l->B), static_cast<const uint16_t *>(l->A),
                      l->scale, tiles_of(p), static_cast<const uint16_t *>(dX_in), static_cast<uint16_t *>(dX_out), U,
                      static_cast<size_t>(ldy), static_cast<size_t>(ldx), p->T, l->O, l->I, l->rank, l->n_adapters};
    return apply<true>(ctx, a, p->n_tiles, p->tile_rows, static_cast<cudaStream_t>(stream));
}

namespace {

template <int R, int Z>
sste_status grad_launch(const sste_ctx *ctx, const GradArgs &p, sste_dtype gdt, cudaStream_t stream)
{
    // blocks that share the rows: enough to fill the GPU twice over, while each of a block's warps has rows to sum
    const long long blocks = static_cast<long long>(p.job[0].blocks + p.job[1].blocks) * p.n_adapters;
    const long long steps = (static_cast<long long>(p.T) / p.n_adapters + 15) / 16;
    int C = 1;
    while (C < 8 && blocks * C < 2 * ctx->sm_count && steps >= 8 * C) C *= 2;
    const dim3 grid(static_cast<unsigned>(p.job[0].blocks + p.job[1].blocks) * C, static_cast<unsigned>(p.n_adapters));
    const cudaError_t e = gdt == SSTE_F32 ? launch_cluster(lora_grad_kernel<R, Z, float>, grid, C, 0, stream, p)
                                          : launch_cluster(lora_grad_kernel<R, Z, __nv_bfloat16>, grid, C, 0, stream, p);
    if (e != cudaSuccess) return SSTE_ERR_CUDA;
    sste_count_launches(1);
    return SSTE_OK;
}

template <int R>
sste_status grad_by_kept(const sste_ctx *ctx, const GradArgs &p, bool kept, sste_ckpt_format fmt, sste_dtype gdt, cudaStream_t stream)
{
    if (!kept) return grad_launch<R, Z_BF16>(ctx, p, gdt, stream);
    return fmt == SSTE_CKPT_E4M3 ? grad_launch<R, Z_E4M3>(ctx, p, gdt, stream) : grad_launch<R, Z_INT8>(ctx, p, gdt, stream);
}

}  // namespace

extern "C" sste_status sste_lora_bwd_weight(sste_ctx *ctx, const sste_lora *l, const sste_lora_plan *p, const void *X, long long ldx,
                                            const void *X_codes, const void *X_scales, sste_ckpt_format fmt, const void *dY,
                                            long long ldy, const float *U, const float *V, void *dA, void *dB, sste_dtype gdt,
                                            void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    sste_status st = lora_ok(l, p);
    if (st != SSTE_OK) return st;
    const bool kept = X_codes != nullptr;
    if (!dA || !dB) return SSTE_ERR_INVALID_ARG;
    if (gdt != SSTE_BF16 && gdt != SSTE_F32) return SSTE_ERR_DTYPE;
    if (kept && fmt != SSTE_CKPT_E4M3 && fmt != SSTE_CKPT_INT8) return SSTE_ERR_INVALID_ARG;
    const size_t elt = gdt == SSTE_F32 ? 4 : 2;
    if (!sste_aligned(dA, elt) || !sste_aligned(dB, elt)) return SSTE_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p->T == 0 || p->n_tiles == 0) {                          // no rows: the sums are empty
        sste_device_guard guard(ctx->device);
        if (!guard.ok) return SSTE_ERR_CUDA;
        const size_t n = static_cast<size_t>(l->n_adapters) * l->rank;
        SSTE_CUDA_TRY(cudaMemsetAsync(dA, 0, n * l->I * elt, s));
        SSTE_CUDA_TRY(cudaMemsetAsync(dB, 0, n * l->O * elt, s));
        return SSTE_OK;
    }
    if (!dY || !U || !V || kept == (X != nullptr) || kept != (X_scales != nullptr)) return SSTE_ERR_INVALID_ARG;
    if ((st = rows_ok(dY, ldy, l->O)) != SSTE_OK) return st;
    if (kept ? !sste_aligned(X_codes, 16) : (st = rows_ok(X, ldx, l->I)) != SSTE_OK) return kept ? SSTE_ERR_ALIGN : st;
    if (!sste_aligned(U, 16) || !sste_aligned(V, 16)) return SSTE_ERR_ALIGN;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    GradArgs a{};
    a.job[0] = GradJob{U, static_cast<const uint16_t *>(X), static_cast<const uint8_t *>(X_codes), static_cast<const uint8_t *>(X_scales),
                       dA, static_cast<size_t>(ldx), l->I, (l->I + 127) / 128, false};
    a.job[1] = GradJob{V, static_cast<const uint16_t *>(dY), nullptr, nullptr, dB, static_cast<size_t>(ldy), l->O, (l->O + 127) / 128,
                       true};
    a.first_tile = static_cast<const int *>(p->table);
    a.tiles = tiles_of(p);
    a.T = p->T;
    a.r = l->rank;
    a.n_adapters = l->n_adapters;
    a.n_tiles = p->n_tiles;
    a.tile_rows = p->tile_rows;
    if (l->rank <= 16) return grad_by_kept<16>(ctx, a, kept, fmt, gdt, s);
    if (l->rank <= 32) return grad_by_kept<32>(ctx, a, kept, fmt, gdt, s);
    return grad_by_kept<64>(ctx, a, kept, fmt, gdt, s);
}
