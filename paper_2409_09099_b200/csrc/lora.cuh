// What the two translation units of the low-rank adapters share: lora.cu (the plan, the calls, the kernels for few rows of an adapter) and
// lora_tc.cu (the kernels for tiles of 128 rows).
#pragma once

#include "common.cuh"

constexpr int LR_SMS = 148;
constexpr int LR_TICKETS = 1024;            // arrival counters of a projecting kernel, and again of a gradient kernel
constexpr int LR_MAX_SPLITS = 16;

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
size_t lora_tc_partial_bytes(const sste_lora *l, const sste_lora_plan *p);
sste_status lora_tc_forward(sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream);
sste_status lora_tc_backward(sste_ctx *ctx, const LoraTcCall &c, cudaStream_t stream);

// Eight kept values (within one block of 32) as bf16 pairs.
template <bool E4M3>
__device__ __forceinline__ void lora_restore8(uint2 q, float by, uint32_t (&out)[4])
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
        const __nv_bfloat162 lo = __floats2bfloat162_rn(f[0], f[1]), hi = __floats2bfloat162_rn(f[2], f[3]);
        out[2 * k] = *reinterpret_cast<const uint32_t *>(&lo);
        out[2 * k + 1] = *reinterpret_cast<const uint32_t *>(&hi);
    }
}
