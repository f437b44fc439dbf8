// What the two translation units of the low-rank adapters share: lora.cu (the plan, the calls, the kernels for few rows of an adapter) and
// lora_tc.cu (the kernels for tiles of 128 rows).
#pragma once

#include "common.cuh"

constexpr int LR_SMS = 148;
constexpr int LR_TICKETS = 1024;            // arrival counters of a projecting kernel, and again of a gradient kernel
constexpr int LR_MAX_SPLITS = 16;
constexpr int LR_MAX_TILES = 0x00ffffff;    // of a plan (a grid's and a table's indexes stay within 31 bits)

static inline int lora_rank_up(int r) { return r <= 16 ? 16 : r <= 32 ? 32 : 64; }

// The plan's table: the first tile of each adapter (n_adapters + 1 of them, filled up to a multiple of four), the tiles (row, rows, adapter, 0);
// then the same for the groups of up to 16 rows that the tiles fall into (row, rows, adapter, the group's place in the scratch).
__host__ __device__ inline size_t lora_tiles_at(int n_adapters) { return (static_cast<size_t>(n_adapters) + 1 + 3) / 4 * 4; }
struct LoraTile { int row, rows, adapter; };
__device__ __forceinline__ LoraTile lora_tile_of(const int4 *tiles, int i, int tile_rows, int T, int n_adapters)
{
    const int4 t = tiles[i];
    // a table that is not the library's own is not followed out of the tensors
    const bool ok = t.x >= 0 && t.y > 0 && t.y <= tile_rows && t.x <= T - t.y && t.z >= -1 && t.z < n_adapters;
    return LoraTile{t.x, ok ? t.y : 0, t.z};
}

// A call on tiles of 128 rows (checked by the caller).  x [T, K] is reduced over K into the rank, y [T, N] added to: forward x = X, y = Y; backward
// x = dY, y = dX.
struct LoraTcCall {
    const sste_lora *l;
    const sste_lora_plan *p;
    const int *first_tile;
    const int4 *tiles;
    const void *x;
    size_t ldx;
    const void *y_in;
    void *y_out;                            // null: no expansion
    size_t ldy;
    float *v_out;                           // forward: V or null
    // backward with gradients of the weights
    bool grads;
    const float *v_in;
    const void *X;
    size_t ldX;
    const void *X_codes, *X_scales;
    sste_ckpt_format fmt;
    void *dA, *dB;
    sste_dtype gdt;
    // scratch: tickets, two tensors split into two bf16 planes each, partial sums
    unsigned int *tickets;
    void *planes, *v_planes;
    float *partial;
};
// whether a gradient kernel's steps (64 rows of a block of features) can be counted in 31 bits
bool lora_tc_grads_fit(const sste_lora *l, const sste_lora_plan *p, sste_dtype gdt);
size_t lora_tc_partial_bytes(const sste_lora *l, const sste_lora_plan *p);
sste_status lora_tc_forward(sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream);
sste_status lora_tc_backward(sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream);

// Eight kept values (within one block of 32) as bf16 pairs; e: the block's exponent byte (0: zeros, for rows that are not there).  In
// packed bf16 arithmetic, which is exact here: an INT8 code is (128 + its low seven bits) - (128 + its sign bit), whose bf16 patterns are
// the code's own bits behind 0x43; an E4M3 code moved to the top of bf16's exponent and mantissa is itself times 2^-120, subnormals
// included.
__device__ __forceinline__ uint32_t lora_mul2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t lora_sub2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t lora_max2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Codes that stand for NaN come out as +-480 (E4M3) or -128 (INT8), beyond every other code: `nans` collects the largest (the negative
// of the smallest) code before the scale, and lora_put_nans puts them right where lora_has_nan says that there are any.
template <bool E4M3>
__device__ __forceinline__ void lora_restore8(uint2 q, uint32_t e, uint32_t (&out)[4], uint32_t &nans)
{
    const uint32_t by = (e << 7) | (e << 23), w[2] = {q.x, q.y};       // 2^e twice
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t v;
            if (E4M3) {
                const uint32_t t = __byte_perm(w[k], 0u, j ? 0x3424 : 0x1404);          // codes in the upper bytes
                v = lora_mul2(((t >> 4) & 0x07f007f0u) | (t & 0x80008000u), 0x7b807b80u);    // 2^120
                nans = lora_max2(nans, v & 0x7fff7fffu);
            } else {
                const uint32_t t = __byte_perm(w[k], 0u, j ? 0x4342 : 0x4140);          // codes in the lower bytes
                const uint32_t low = (t & 0x007f007fu) | 0x43004300u, sign = (t & 0x00800080u) | 0x43004300u;
                v = lora_sub2(low, sign);
                nans = lora_max2(nans, v ^ 0x80008000u);
            }
            out[2 * k + j] = lora_mul2(v, by);
        }
}
template <bool E4M3>
__device__ __forceinline__ bool lora_has_nan(uint32_t nans)
{
    const float least = E4M3 ? 480.0f : 128.0f;
    return __uint_as_float(nans << 16) >= least || __uint_as_float(nans & 0xffff0000u) >= least;
}
template <bool E4M3>
__device__ __forceinline__ void lora_put_nans(uint2 q, uint32_t (&out)[4])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t code = (i < 4 ? q.x : q.y) >> (8 * (i & 3)) & 0xffu;
        if (E4M3 ? (code & 0x7fu) == 0x7fu : code == 0x80u)
            out[i / 2] = i & 1 ? (out[i / 2] & 0xffffu) | 0x7fc00000u : (out[i / 2] & 0xffff0000u) | 0x7fc0u;
    }
}
