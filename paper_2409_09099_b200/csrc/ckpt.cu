// Activations kept in 8 bits between the forward and the backward pass: the kept form written beside an activation's output, restored
// for a weight gradient, and the activation's gradient straight from it.
//
// The form.  32 consecutive elements share a power of two 2^e; an element is a code q with value q 2^e.  e is the least exponent at
// which the block's largest finite magnitude does not pass the largest code (448 in E4M3, 127 in INT8), so no element saturates, and
// scaling by it is exact: q = rn(x 2^-e) has one rounding, the same bits on any machine.  A code has 4 (E4M3) or 7 (INT8) significant
// bits, so q 2^e is a bf16 number: what is restored is the kept value itself and the products read it without another rounding.
// (e >= -124 keeps that true at the lower end of bf16.)  A scale for the whole tensor, as the FP8 layers have, would need a pass for the
// maximum first and loses the small rows beside an outlier; a block of 32 needs one exchange between two lanes.
//
// All kernels here are one pass over memory and bound by it: 16 elements per thread, as 32-byte vectors of bf16 and 16-byte vectors
// of codes, two lanes to a block.  Measured, with the memory's copy rate at 6.5 TB/s: 16384 x 1280 kept in 10.8 us and restored in 10.9
// (5.9 TB/s); GELU on 16384 x 5120, 63.4 us forward (6.7) and 100 us backward with the output again (5.9: it alone also waits for arithmetic,
// an exponential and some 40 instructions an element); silu gate on 16384 x 11008, 210 us (6.9) and 279 us (6.5).  Below some 2 M
// elements the launches are the time: 1.4 us each for 512 x 256.
#include "common.cuh"

namespace {

constexpr int CK_THREADS = 256;
constexpr uint32_t CK_LOWEST = 3;          // e = -124, as e + 127

struct Vec16 { uint32_t w[8]; };           // 16 bf16 values

__device__ __forceinline__ Vec16 ld_vec(const uint16_t *p)
{
    Vec16 v;
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7])
                 : "l"(p));
    return v;
}
__device__ __forceinline__ void st_vec(uint16_t *p, const Vec16 &v)
{
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]),
                 "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7]), "l"(p)
                 : "memory");
}
// the elements i .. i + 15 of an array of n; beyond its end zeros, and nothing stored
__device__ __forceinline__ Vec16 ld_unit(const uint16_t *p, size_t i, size_t n)
{
    if (i + 16 <= n) return ld_vec(p + i);
    Vec16 v;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t lo = i + 2 * k < n ? p[i + 2 * k] : 0u, hi = i + 2 * k + 1 < n ? p[i + 2 * k + 1] : 0u;
        v.w[k] = lo | (hi << 16);
    }
    return v;
}
__device__ __forceinline__ void st_unit(uint16_t *p, size_t i, size_t n, const Vec16 &v)
{
    if (i + 16 <= n) { st_vec(p + i, v); return; }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (i + 2 * k < n) p[i + 2 * k] = static_cast<uint16_t>(v.w[k]);
        if (i + 2 * k + 1 < n) p[i + 2 * k + 1] = static_cast<uint16_t>(v.w[k] >> 16);
    }
}

__device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
__device__ __forceinline__ float power_of_two(uint32_t biased) { return __uint_as_float(biased << 23); }

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// GELU in its tanh form is h s(2z), z = sqrt(2/pi) (h + 0.044715 h^3), s the logistic function: one exponential and one reciprocal,
// and none of the cancellation that 1 + tanh(z) has for negative h.  Both are good to 2^-22, far below the rounding to bf16.
constexpr float GELU_C = 0.7978845608028654f, GELU_K = 0.044715f, LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float gelu_cdf(float h)
{
    constexpr float a = -2.0f * GELU_C * LOG2E, b = a * GELU_K;
    return rcp(1.0f + ex2(h * fmaf(b * h, h, a)));
}
__device__ __forceinline__ float logistic(float g) { return rcp(1.0f + ex2(-LOG2E * g)); }

// d GELU / dh from s = gelu_cdf(h).  Beyond 12 the logistic factor is 0 or 1 in fp32 and its own slope 0: clamped there, no h^2 overflows
// against it (a NaN passes both comparisons).
__device__ __forceinline__ float gelu_slope(float h, float s)
{
    h = h > 12.0f ? 12.0f : h < -12.0f ? -12.0f : h;
    return fmaf(h * s * (1.0f - s), fmaf(6.0f * GELU_C * GELU_K * h, h, 2.0f * GELU_C), s);
}

template <int ACT>
__device__ __forceinline__ float activate(float x, float up)
{
    if (ACT == SSTE_ACT_GELU) return x * gelu_cdf(x);
    if (ACT == SSTE_ACT_SILU_GATE) return x * logistic(x) * up;
    return x;
}

// Largest finite magnitudes that the forms hold: the largest codes at the highest exponent that a finite value can ask for, whose value
// bf16 holds (1.875 and 1.96875 times 2^127); above them is clamped.  As bf16 bits.
template <bool E4M3>
constexpr uint32_t CK_LARGEST = E4M3 ? 0x7f70u : 0x7f7cu;

__device__ __forceinline__ uint32_t max_of_halves(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

// The codes of 16 elements and, in `scale`, e + 127 of the block that this lane and its neighbour share.  All lanes of the warp call.
template <bool E4M3>
__device__ __forceinline__ uint4 encode(const Vec16 &x, uint32_t &scale)
{
    // magnitudes order like their bits; infinities and NaNs are above every finite one
    uint32_t m2 = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) m2 = max_of_halves(m2, x.w[k] & 0x7fff7fffu);
    m2 = max_of_halves(m2, __shfl_xor_sync(0xffffffffu, m2, 1));
    uint32_t m = max(m2 & 0xffffu, m2 >> 16);
    const bool special = m > CK_LARGEST<E4M3>;
    Vec16 v = x;
    uint32_t lost = 0;                                 // elements that are not finite
    if (__any_sync(0xffffffffu, special)) {
        uint32_t f = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const uint32_t h = (x.w[k / 2] >> (16 * (k & 1))) & 0xffffu, a = h & 0x7fffu;
            const bool fine = a < 0x7f80u;
            const uint32_t c = fine ? min(a, CK_LARGEST<E4M3>) : 0u;
            f = max(f, c);
            lost |= fine ? 0u : 1u << k;
            v.w[k / 2] = k & 1 ? (v.w[k / 2] & 0xffffu) | ((c | (h & 0x8000u)) << 16) : (v.w[k / 2] & 0xffff0000u) | c | (h & 0x8000u);
        }
        m = max(f, __shfl_xor_sync(0xffffffffu, f, 1));
    }
    const int e = static_cast<int>(m >> 7) - (E4M3 ? 8 : 6) + ((m & 0x7fu) > (E4M3 ? 96u : 126u) ? 1 : 0);
    scale = static_cast<uint32_t>(max(e, static_cast<int>(CK_LOWEST)));
    const float by = power_of_two(254u - scale);
    uint32_t q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 a = unpack(v.w[2 * k]), b = unpack(v.w[2 * k + 1]);
        if (E4M3) {
            q[k] = static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(a.x * by, a.y * by), __NV_SATFINITE, __NV_E4M3)) |
                   static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(b.x * by, b.y * by), __NV_SATFINITE, __NV_E4M3)) << 16;
        } else {
            // adding 1.5 * 2^23 rounds to an integer, ties to even, and leaves it in the low bits: the conversion instruction shares
            // the unit of the exponentials
            constexpr float magic = 12582912.0f;
            const uint32_t lo = __byte_perm(__float_as_uint(fmaf(a.x, by, magic)), __float_as_uint(fmaf(a.y, by, magic)), 0x0040);
            const uint32_t hi = __byte_perm(__float_as_uint(fmaf(b.x, by, magic)), __float_as_uint(fmaf(b.y, by, magic)), 0x0040);
            q[k] = __byte_perm(lo, hi, 0x5410);
        }
    }
    if (lost) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (lost >> k & 1) q[k / 4] = (q[k / 4] & ~(0xffu << (8 * (k & 3)))) | (E4M3 ? 0x7fu : 0x80u) << (8 * (k & 3));
    }
    return make_uint4(q[0], q[1], q[2], q[3]);
}

// Four codes to their values times `by`.
template <bool E4M3>
__device__ __forceinline__ void decode(uint32_t q, float by, float out[4])
{
    if (E4M3) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(q >> (16 * k)), __NV_E4M3);
            const float2 f = __half22float2(__half2(r));
            out[2 * k] = f.x * by;
            out[2 * k + 1] = f.y * by;
        }
    } else {
        const uint32_t u = q ^ 0x80808080u;            // q + 128 in each byte, 0 for the code that stands for NaN
#pragma unroll
        for (int k = 0; k < 4; ++k)
            out[k] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 | k)) - 8388736.0f) * by;
        if ((u - 0x01010101u) & ~u & 0x80808080u) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if ((u >> (8 * k) & 0xffu) == 0) out[k] = __uint_as_float(0x7fc00000u);
        }
    }
}

struct Kept {
    uint4 *codes;
    uint8_t *scales;
};
struct KeptIn {
    const uint4 *codes;
    const uint8_t *scales;
};

// ---------------------------------------------------------------- forward: y = act(x[, up]), x and up kept
template <bool E4M3, int ACT>
__global__ void __launch_bounds__(CK_THREADS)
ckpt_store_kernel(const uint16_t *x, const uint16_t *up, size_t n, size_t units, const Kept kx, const Kept ku, uint16_t *y)
{
    sste_pdl_trigger();
    sste_pdl_wait(x, up);
    const size_t stride = static_cast<size_t>(gridDim.x) * CK_THREADS;
    // (units is even and a block's two lanes are neighbours; every lane of a warp makes the same number of rounds)
    for (size_t base = static_cast<size_t>(blockIdx.x) * CK_THREADS; base < units; base += stride) {
        const size_t u = base + threadIdx.x, i = u * 16;
        const bool mine = u < units;
        Vec16 a = {}, b = {};
        if (mine) {
            a = ld_unit(x, i, n);
            if (ACT == SSTE_ACT_SILU_GATE) b = ld_unit(up, i, n);
        }
        uint32_t sa, sb = 0;
        const uint4 qa = encode<E4M3>(a, sa);
        uint4 qb = {};
        if (ACT == SSTE_ACT_SILU_GATE) qb = encode<E4M3>(b, sb);
        if (!mine) continue;
        kx.codes[u] = qa;
        if (!(u & 1)) kx.scales[u >> 1] = static_cast<uint8_t>(sa);
        if (ACT == SSTE_ACT_SILU_GATE) {
            ku.codes[u] = qb;
            if (!(u & 1)) ku.scales[u >> 1] = static_cast<uint8_t>(sb);
        }
        if (ACT != SSTE_ACT_NONE) {
            Vec16 o;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float2 p = unpack(a.w[k]), r = unpack(b.w[k]);
                o.w[k] = pack(activate<ACT>(p.x, r.x), activate<ACT>(p.y, r.y));
            }
            st_unit(y, i, n, o);
        }
    }
}

// ---------------------------------------------------------------- y = act(x~[, up~]) from the kept form
template <bool E4M3, int ACT>
__global__ void __launch_bounds__(CK_THREADS)
ckpt_load_kernel(const KeptIn kx_in, const KeptIn ku_in, size_t n, size_t units, uint16_t *y)
{
    KeptIn kx = kx_in, ku = ku_in;
    sste_pdl_trigger();
    sste_pdl_wait(kx.codes, kx.scales, ku.codes, ku.scales);
    const size_t stride = static_cast<size_t>(gridDim.x) * CK_THREADS;
    for (size_t u = static_cast<size_t>(blockIdx.x) * CK_THREADS + threadIdx.x; u < units; u += stride) {
        const size_t i = u * 16;
        if (i >= n) break;                            // the second half of the last block may be empty
        const uint4 qa = sste_ld_once(kx.codes + u);
        const float sa = power_of_two(kx.scales[u >> 1]);
        uint4 qb = {};
        float sb = 0.0f;
        if (ACT == SSTE_ACT_SILU_GATE) {
            qb = sste_ld_once(ku.codes + u);
            sb = power_of_two(ku.scales[u >> 1]);
        }
        const uint32_t wa[4] = {qa.x, qa.y, qa.z, qa.w}, wb[4] = {qb.x, qb.y, qb.z, qb.w};
        Vec16 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float a[4], b[4] = {};
            decode<E4M3>(wa[k], sa, a);
            if (ACT == SSTE_ACT_SILU_GATE) decode<E4M3>(wb[k], sb, b);
            o.w[2 * k] = pack(activate<ACT>(a[0], b[0]), activate<ACT>(a[1], b[1]));
            o.w[2 * k + 1] = pack(activate<ACT>(a[2], b[2]), activate<ACT>(a[3], b[3]));
        }
        st_unit(y, i, n, o);
    }
}

// ---------------------------------------------------------------- gradients at the kept inputs, and the activation's output again
template <bool E4M3, int ACT, bool AGAIN>
__global__ void __launch_bounds__(CK_THREADS)
ckpt_act_bwd_kernel(const uint16_t *dy, const KeptIn kx_in, const KeptIn ku_in, size_t n, size_t units, uint16_t *dx, uint16_t *dup,
                    uint16_t *y)
{
    KeptIn kx = kx_in, ku = ku_in;
    sste_pdl_trigger();
    sste_pdl_wait(dy, kx.codes, kx.scales, ku.codes, ku.scales);
    const size_t stride = static_cast<size_t>(gridDim.x) * CK_THREADS;
    for (size_t u = static_cast<size_t>(blockIdx.x) * CK_THREADS + threadIdx.x; u < units; u += stride) {
        const size_t i = u * 16;
        if (i >= n) break;
        const Vec16 g = ld_unit(dy, i, n);
        const uint4 qa = sste_ld_once(kx.codes + u);
        const float sa = power_of_two(kx.scales[u >> 1]);
        uint4 qb = {};
        float sb = 0.0f;
        if (ACT == SSTE_ACT_SILU_GATE) {
            qb = sste_ld_once(ku.codes + u);
            sb = power_of_two(ku.scales[u >> 1]);
        }
        const uint32_t wa[4] = {qa.x, qa.y, qa.z, qa.w}, wb[4] = {qb.x, qb.y, qb.z, qb.w};
        Vec16 ox, ou, oy;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float a[4], b[4] = {}, gx[4], gu[4], ya[4];
            decode<E4M3>(wa[k], sa, a);
            if (ACT == SSTE_ACT_SILU_GATE) decode<E4M3>(wb[k], sb, b);
            const float2 g0 = unpack(g.w[2 * k]), g1 = unpack(g.w[2 * k + 1]);
            const float d[4] = {g0.x, g0.y, g1.x, g1.y};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (ACT == SSTE_ACT_GELU) {
                    const float s = gelu_cdf(a[j]);
                    gx[j] = d[j] * gelu_slope(a[j], s);
                    ya[j] = a[j] * s;
                } else {
                    const float s = logistic(a[j]), t = a[j] * s;
                    gx[j] = d[j] * b[j] * (s * fmaf(a[j], 1.0f - s, 1.0f));
                    gu[j] = d[j] * t;
                    ya[j] = t * b[j];
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                ox.w[2 * k + j] = pack(gx[2 * j], gx[2 * j + 1]);
                if (ACT == SSTE_ACT_SILU_GATE) ou.w[2 * k + j] = pack(gu[2 * j], gu[2 * j + 1]);
                if (AGAIN) oy.w[2 * k + j] = pack(ya[2 * j], ya[2 * j + 1]);
            }
        }
        st_unit(dx, i, n, ox);
        if (ACT == SSTE_ACT_SILU_GATE) st_unit(dup, i, n, ou);
        if (AGAIN) st_unit(y, i, n, oy);
    }
}

size_t units_of(size_t n) { return (n + 31) / 32 * 2; }
// one round per thread: the grid's own scheduling keeps more loads in flight than a loop over resident blocks does
unsigned blocks_of(size_t units)
{
    const size_t b = (units + CK_THREADS - 1) / CK_THREADS;
    return static_cast<unsigned>(b < (size_t(1) << 30) ? b : size_t(1) << 30);
}

sste_status launched()
{
    if (cudaGetLastError() != cudaSuccess) return SSTE_ERR_CUDA;
    sste_count_launches(1);
    return SSTE_OK;
}

struct CkptArgs {
    const void *codes, *scales, *up_codes, *up_scales;
};

// What all three calls ask of their arguments.  `vectors`: bf16 arrays, null ones allowed by the caller's own rules.
sste_status ckpt_ok(sste_dtype dt, sste_ckpt_format fmt, sste_activation act, const CkptArgs &k, const void *a, const void *b,
                    const void *c, const void *d)
{
    if (fmt != SSTE_CKPT_E4M3 && fmt != SSTE_CKPT_INT8) return SSTE_ERR_INVALID_ARG;
    if (act != SSTE_ACT_NONE && act != SSTE_ACT_GELU && act != SSTE_ACT_SILU_GATE) return SSTE_ERR_INVALID_ARG;
    if (dt != SSTE_BF16) return SSTE_ERR_DTYPE;
    if (!k.codes || !k.scales) return SSTE_ERR_INVALID_ARG;
    const bool gate = act == SSTE_ACT_SILU_GATE;
    if (gate != (k.up_codes != nullptr) || gate != (k.up_scales != nullptr)) return SSTE_ERR_INVALID_ARG;
    if (!sste_aligned(k.codes, 16) || !sste_aligned(k.up_codes, 16)) return SSTE_ERR_ALIGN;
    for (const void *p : {a, b, c, d})
        if (!sste_aligned(p, 32)) return SSTE_ERR_ALIGN;
    return SSTE_OK;
}

// f(E4M3 or not as a type, activation as a type)
template <bool V>
struct Flag { static constexpr bool value = V; };
template <int V>
struct Act { static constexpr int value = V; };
template <typename F>
void by_format(sste_ckpt_format fmt, sste_activation act, F f)
{
    auto with = [&](auto e4m3) {
        if (act == SSTE_ACT_GELU) f(e4m3, Act<SSTE_ACT_GELU>());
        else if (act == SSTE_ACT_SILU_GATE) f(e4m3, Act<SSTE_ACT_SILU_GATE>());
        else f(e4m3, Act<SSTE_ACT_NONE>());
    };
    if (fmt == SSTE_CKPT_E4M3) with(Flag<true>());
    else with(Flag<false>());
}

KeptIn kept_in(const void *codes, const void *scales)
{
    return KeptIn{static_cast<const uint4 *>(codes), static_cast<const uint8_t *>(scales)};
}

}  // namespace

extern "C" size_t sste_ckpt_code_bytes(size_t n) { return (n + 31) / 32 * 32; }
extern "C" size_t sste_ckpt_scale_bytes(size_t n) { return (n + 31) / 32; }

extern "C" sste_status sste_ckpt_store(sste_ctx *ctx, const void *x, const void *up, size_t n, sste_dtype dt, sste_ckpt_format fmt,
                                       sste_activation act, void *codes, void *scales, void *up_codes, void *up_scales, void *y,
                                       void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    if (n == 0) return SSTE_OK;
    const sste_status ok = ckpt_ok(dt, fmt, act, CkptArgs{codes, scales, up_codes, up_scales}, x, up, y, nullptr);
    if (ok != SSTE_OK) return ok;
    if (!x || (act == SSTE_ACT_SILU_GATE) != (up != nullptr) || (act != SSTE_ACT_NONE) != (y != nullptr)) return SSTE_ERR_INVALID_ARG;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    const size_t units = units_of(n);
    by_format(fmt, act, [&](auto e4m3, auto a) {
        sste_launch(ckpt_store_kernel<decltype(e4m3)::value, decltype(a)::value>, dim3(blocks_of(units)), dim3(CK_THREADS), 0,
                    static_cast<cudaStream_t>(stream), static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(up), n, units,
                    Kept{static_cast<uint4 *>(codes), static_cast<uint8_t *>(scales)},
                    Kept{static_cast<uint4 *>(up_codes), static_cast<uint8_t *>(up_scales)}, static_cast<uint16_t *>(y));
    });
    return launched();
}

extern "C" sste_status sste_ckpt_load(sste_ctx *ctx, const void *codes, const void *scales, const void *up_codes,
                                      const void *up_scales, size_t n, sste_ckpt_format fmt, sste_activation act, void *y,
                                      sste_dtype ydt, void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    if (n == 0) return SSTE_OK;
    const sste_status ok = ckpt_ok(ydt, fmt, act, CkptArgs{codes, scales, up_codes, up_scales}, y, nullptr, nullptr, nullptr);
    if (ok != SSTE_OK) return ok;
    if (!y) return SSTE_ERR_INVALID_ARG;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    const size_t units = units_of(n);
    by_format(fmt, act, [&](auto e4m3, auto a) {
        sste_launch(ckpt_load_kernel<decltype(e4m3)::value, decltype(a)::value>, dim3(blocks_of(units)), dim3(CK_THREADS), 0,
                    static_cast<cudaStream_t>(stream), kept_in(codes, scales), kept_in(up_codes, up_scales), n, units,
                    static_cast<uint16_t *>(y));
    });
    return launched();
}

extern "C" sste_status sste_ckpt_act_bwd(sste_ctx *ctx, const void *dy, const void *codes, const void *scales, const void *up_codes,
                                         const void *up_scales, size_t n, sste_dtype dt, sste_ckpt_format fmt, sste_activation act,
                                         void *dx, void *dup, void *y, void *stream)
{
    if (!ctx) return SSTE_ERR_INVALID_ARG;
    if (n == 0) return SSTE_OK;
    const sste_status ok = ckpt_ok(dt, fmt, act, CkptArgs{codes, scales, up_codes, up_scales}, dy, dx, dup, y);
    if (ok != SSTE_OK) return ok;
    if (act == SSTE_ACT_NONE || !dy || !dx || (act == SSTE_ACT_SILU_GATE) != (dup != nullptr)) return SSTE_ERR_INVALID_ARG;
    sste_device_guard guard(ctx->device);
    if (!guard.ok) return SSTE_ERR_CUDA;
    const size_t units = units_of(n);
    auto launch = [&](auto kernel) {
        sste_launch(kernel, dim3(blocks_of(units)), dim3(CK_THREADS), 0, static_cast<cudaStream_t>(stream),
                    static_cast<const uint16_t *>(dy), kept_in(codes, scales), kept_in(up_codes, up_scales), n, units,
                    static_cast<uint16_t *>(dx), static_cast<uint16_t *>(dup), static_cast<uint16_t *>(y));
    };
    by_format(fmt, act, [&](auto e4m3, auto a) {
        constexpr int A = decltype(a)::value == SSTE_ACT_NONE ? SSTE_ACT_GELU : decltype(a)::value;
        if (y) launch(ckpt_act_bwd_kernel<decltype(e4m3)::value, A, true>);
        else launch(ckpt_act_bwd_kernel<decltype(e4m3)::value, A, false>);
    });
    return launched();
}
