// Root-mean-square norm with the residual's addition and an output in 8 bits with scales.
//
//   h = round(x + r)                                 (r may be absent: h = x), stored in r's type
//   y = h * rstd * w,      rstd = 1 / sqrt(mean(h^2) + eps)
//   s_k = max |y| of 128 columns / 448 as fp32 (2^-126 at least), q = e4m3(y / s_k), ties to even
//
// What the definition says in exact arithmetic is what comes out, number for number: which 8-bit number a value rounds to must not
// hang on the order of a sum, or the same row would quantize differently here and in another implementation.  For that
//   - squares are added in 64 bits, and rstd is a 64-bit number;
//   - p = h 2^k w (2^k: rstd's power of two, so that p neither overflows nor vanishes where h does not) is kept with its rounding error
//     e = fma(h 2^k, w, -p), so that the largest |p + e| of a group, and from it the scale, is exact;
//   - y / s is p c with c = rstd / (2^k s) in fp32: five roundings, so at most five last places off; only where that lies within six
//     of a border between two 8-bit numbers (12 of a million values) is it computed once more in 64 bits.
// Memory bound: every operand is read once and every result written once; a row stays in registers between its two passes.
#include "sqnn_launch.h"
#include "sqnn_fp8.cuh"

#include <cuda_bf16.h>

namespace sqnn {
namespace {

struct NormArgs {
    const void *x, *r, *w;
    void *h, *y;
    uint8_t *q;
    float *s;
    int64_t ldx, ldr, ldh, ldq, lds, ldy;
    uint64_t n;
    double eps;
    uint32_t w_bf16, y_bf16;
};

template <typename T> SQNN_DEV float to_f32(T v);
template <> SQNN_DEV float to_f32<float>(float v) { return v; }
template <> SQNN_DEV float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

SQNN_DEV void load8(const float *p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
SQNN_DEV void load8(const __nv_bfloat16 *p, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(u[j] << 16);
        v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
    }
}
SQNN_DEV void store8(float *p, const float (&v)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
SQNN_DEV uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return reinterpret_cast<const uint32_t &>(b);
}
SQNN_DEV void store8(__nv_bfloat16 *p, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// Where a thread's eight elements of a slot lie.  Sixteen threads share a group of 128 columns: with VEC each has eight in a row (16-byte
// accesses; rows on 16-byte boundaries), without it every sixteenth (neighbouring threads on neighbouring elements, any alignment).
template <bool VEC> SQNN_DEV uint64_t first_of(uint64_t unit) { return VEC ? unit * 8 : (unit >> 4) * 128 + (unit & 15); }
template <bool VEC> SQNN_DEV uint64_t step_of() { return VEC ? 1 : 16; }

// Elements past n read as zero.
template <typename T, bool VEC>
SQNN_DEV void fetch(const T *row, uint64_t i, uint64_t n, float (&v)[8])
{
    if (VEC && i + 8 <= n) {
        load8(row + i, v);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            const uint64_t at = i + j * step_of<VEC>();
            v[j] = at < n ? to_f32<T>(row[at]) : 0.0f;
        }
    }
}
SQNN_DEV void put(float *p, float v) { *p = v; }
SQNN_DEV void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
template <typename T, bool VEC>
SQNN_DEV void store(T *row, uint64_t i, uint64_t n, const float (&v)[8])
{
    if (VEC && i + 8 <= n) {
        store8(row + i, v);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            const uint64_t at = i + j * step_of<VEC>();
            if (at < n) put(row + at, v[j]);
        }
    }
}

// x + r rounded once to r's type.  An fp32 sum rounded again to bf16 could be off where it lands on a middle, so it is rounded to
// odd first (the last bit says that something was cut off); two bf16 numbers cannot get there.
template <typename XT, typename RT>
SQNN_DEV float add_rounded(float x, float r)
{
    if constexpr (sizeof(RT) == 4) {
        return x + r;
    } else if constexpr (sizeof(XT) == 2) {
        return __bfloat162float(__float2bfloat16_rn(x + r));
    } else {
        const float lo = __fadd_rd(x, r), hi = __fadd_ru(x, r);
        return __bfloat162float(__float2bfloat16_rn((__float_as_uint(lo) & 1u) ? lo : hi));
    }
}

// Largest magnitude as (p, e), both with the sign taken out of p; bit patterns order magnitudes with NaN above infinity.
SQNN_DEV void larger(uint32_t &p, float &e, uint32_t q, float f)
{
    if (q > p || (q == p && f > e)) { p = q; e = f; }
}

SQNN_DEV double exp2_double(int k) { return __longlong_as_double((long long)(1023 + k) << 52); }

// One block per row.  SLOTS slots of eight elements a thread stay in registers; SLOTS = 0: rows longer than that are read a second
// time, h where it was stored.
template <typename XT, typename RT, bool RES, uint32_t SLOTS, bool VEC>
__global__ void __launch_bounds__(512) k_rmsnorm_fp8(const NormArgs A)
{
    __shared__ double part[16];
    __shared__ double rstd_s;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, T = blockDim.x;
    const uint64_t row = blockIdx.x, n = A.n;
    wait_prior_grid();
    launch_dependents();
    const XT *x = static_cast<const XT *>(A.x) + (int64_t)row * A.ldx;
    const RT *r = static_cast<const RT *>(A.r) + (RES ? (int64_t)row * A.ldr : 0);
    RT *h = static_cast<RT *>(A.h) + (RES ? (int64_t)row * A.ldh : 0);
    constexpr uint32_t KEPT = SLOTS ? SLOTS : 1;
    const uint64_t units = (n + 127) / 128 * 16;
    float v[KEPT][8];

    double sum = 0.0;
    auto take = [&](uint64_t unit, float (&a)[8]) {
        const uint64_t i = first_of<VEC>(unit);
        fetch<XT, VEC>(x, i, n, a);
        if constexpr (RES) {
            float b[8];
            fetch<RT, VEC>(r, i, n, b);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) a[j] = add_rounded<XT, RT>(a[j], b[j]);
        }
    };
    auto squares = [&](const float (&a)[8]) {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) { const double d = a[j]; sum = fma(d, d, sum); }
    };
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (uint32_t k = 0; k < SLOTS; ++k) {
            const uint64_t unit = (uint64_t)k * T + tid;
            if (unit < units) take(unit, v[k]);
            else
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) v[k][j] = 0.0f;
        }
#pragma unroll
        for (uint32_t k = 0; k < SLOTS; ++k) {
            squares(v[k]);
            const uint64_t unit = (uint64_t)k * T + tid;
            if (RES && unit < units) store<RT, VEC>(h, first_of<VEC>(unit), n, v[k]);
        }
    } else {
        for (uint64_t unit = tid; unit < units; unit += T) {
            take(unit, v[0]);
            squares(v[0]);
            if (RES) store<RT, VEC>(h, first_of<VEC>(unit), n, v[0]);
        }
    }
#pragma unroll
    for (uint32_t d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = lane < T / 32 ? part[lane] : 0.0;
#pragma unroll
        for (uint32_t d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) rstd_s = 1.0 / sqrt(sum / (double)n + A.eps);
    }
    __syncthreads();
    const double rstd = rstd_s;
    // 2^k: rstd's power of two as far as it is an fp32 number (rstd zero, infinite or NaN: any will do)
    int k2 = (int)((__double_as_longlong(rstd) >> 52) & 0x7ff) - 1023;
    k2 = k2 < -126 ? -126 : k2 > 127 ? 127 : k2;
    const float scale_h = __uint_as_float((uint32_t)(127 + k2) << 23);
    const double rest = rstd * exp2_double(-k2);                   // rstd / 2^k, exact
    const float rest32 = (float)rest;

    auto finish = [&](uint64_t unit, const float (&a)[8]) {        // all threads of a warp, in step
        const bool in = unit < units;
        const uint64_t i = first_of<VEC>(unit);
        float w[8], p[8];
        if (in) {
            if (A.w_bf16) fetch<__nv_bfloat16, VEC>(static_cast<const __nv_bfloat16 *>(A.w), i, n, w);
            else fetch<float, VEC>(static_cast<const float *>(A.w), i, n, w);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) w[j] = 0.0f;
        }
        uint32_t top = 0;
        float top_e = 0.0f;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            const float b = a[j] * scale_h;
            p[j] = b * w[j];
            const float e = fmaf(b, w[j], -p[j]);
            larger(top, top_e, __float_as_uint(p[j]) & 0x7fffffffu, p[j] < 0.0f ? -e : e);
        }
        if (A.q) {
#pragma unroll
            for (uint32_t d = 8; d; d >>= 1) {                     // the sixteen threads of the group
                const uint32_t q = __shfl_xor_sync(0xffffffffu, top, d);
                const float f = __shfl_xor_sync(0xffffffffu, top_e, d);
                larger(top, top_e, q, f);
            }
            const double most = ((double)__uint_as_float(top) + (top < 0x7f800000u ? (double)top_e : 0.0)) * rest;
            float s = (float)(most * (1.0 / (double)FP8_MAX));
            s = s < 0x1p-126f ? 0x1p-126f : s;                     // (NaN stays)
            const float c32 = rest32 * __frcp_rn(s);
            float t[8];
            bool near = false;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                t[j] = p[j] * c32;
                near |= near_fp8_border(t[j]);
            }
            if (near) {
                const double c = rest / (double)s;
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {
                    const double d = (double)(a[j] * scale_h) * (double)w[j] * c;
                    const float f = (float)d;                      // rounded to odd: no second rounding can go wrong
                    const double back = (double)f;
                    const float cut = fabs(back) > fabs(d) ? __uint_as_float(__float_as_uint(f) - 1) : f;
                    t[j] = (double)cut != d && d == d ? __uint_as_float(__float_as_uint(cut) | 1u) : f;
                }
            }
            if (in) {
                uint8_t *q = A.q + (int64_t)row * A.ldq;
                const uint32_t q01 = to_fp8x2(t[0], t[1]), q23 = to_fp8x2(t[2], t[3]), q45 = to_fp8x2(t[4], t[5]), q67 = to_fp8x2(t[6], t[7]);
                const uint2 all = make_uint2(q01 | (q23 << 16), q45 | (q67 << 16));
                if (VEC && i + 8 <= n) {
                    *reinterpret_cast<uint2 *>(q + i) = all;
                } else {
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) {
                        const uint64_t at = i + j * step_of<VEC>();
                        if (at < n) q[at] = (uint8_t)((j < 4 ? all.x : all.y) >> (8 * (j & 3)));
                    }
                }
                if ((unit & 15) == 0) A.s[(int64_t)row * A.lds + (int64_t)(unit >> 4)] = s;
            }
        }
        if (A.y && in) {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) p[j] *= rest32;
            if (A.y_bf16) store<__nv_bfloat16, VEC>(static_cast<__nv_bfloat16 *>(A.y) + (int64_t)row * A.ldy, i, n, p);
            else store<float, VEC>(static_cast<float *>(A.y) + (int64_t)row * A.ldy, i, n, p);
        }
    };
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (uint32_t k = 0; k < SLOTS; ++k) finish((uint64_t)k * T + tid, v[k]);
    } else {
        for (uint64_t base = 0; base < units; base += T) {
            const uint64_t unit = base + tid;
            if (unit < units) {                                    // h as this thread stored it, or x
                if (RES) fetch<RT, VEC>(h, first_of<VEC>(unit), n, v[0]);
                else fetch<XT, VEC>(x, first_of<VEC>(unit), n, v[0]);
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) v[0][j] = 0.0f;
            }
            finish(unit, v[0]);
        }
    }
}

template <typename XT, typename RT, bool RES>
int launch_norm(const NormArgs &A, uint32_t batch, bool vec, cudaStream_t st)
{
    const uint64_t units = (A.n + 127) / 128 * 16;
    const uint32_t most = 512;
    const uint32_t slots = units <= most ? 1 : units <= 2 * most ? 2 : units <= 4 * most ? 4 : 0;
    const uint64_t per = slots ? (units + slots - 1) / slots : most;
    const uint32_t threads = (uint32_t)((per + 31) / 32 * 32);
#define SQNN_NORM_PICK(S) (vec ? k_rmsnorm_fp8<XT, RT, RES, S, true> : k_rmsnorm_fp8<XT, RT, RES, S, false>)
    auto k = slots == 1 ? SQNN_NORM_PICK(1) : slots == 2 ? SQNN_NORM_PICK(2) : slots == 4 ? SQNN_NORM_PICK(4) : SQNN_NORM_PICK(0);
#undef SQNN_NORM_PICK
    return launch_kernel(k, batch, threads, 0, st, A);
}

uint32_t size_of(int dtype) { return dtype == SQNN_X_BF16 ? 2 : 4; }
bool known_type(int dtype) { return dtype == SQNN_X_F32 || dtype == SQNN_X_BF16; }
bool row16(const void *p, int64_t ld, uint32_t size) { return ((uintptr_t)p & 15) == 0 && (ld * (int64_t)size) % 16 == 0; }
bool aligned_to(const void *p, uint32_t size) { return ((uintptr_t)p & (size - 1)) == 0; }

int rmsnorm_queue(uint32_t batch, uint64_t n, const void *d_x, int x_dtype, int64_t ldx, const void *d_residual, int residual_dtype,
                  int64_t ldr, void *d_h, int64_t ldh, const void *d_weight, int weight_dtype, double eps, uint8_t *d_q, int64_t ldq,
                  float *d_scale, int64_t lds, void *d_y, int y_dtype, int64_t ldy, cudaStream_t st)
{
    const int64_t cols = (int64_t)n;
    if (batch == 0 || n == 0 || !d_x || !d_weight || (!d_q && !d_y)) return SQNN_E_INVALID_ARG;
    if ((d_q != nullptr) != (d_scale != nullptr) || (d_residual != nullptr) != (d_h != nullptr)) return SQNN_E_INVALID_ARG;
    if (n > (1ull << 30)) return SQNN_E_UNSUPPORTED;
    if (batch > 0x7fffffffu) return SQNN_E_UNSUPPORTED;
    if (!known_type(x_dtype) || !known_type(weight_dtype) || !aligned_to(d_x, size_of(x_dtype)) ||
        !aligned_to(d_weight, size_of(weight_dtype)) || ldx < cols || !(eps >= 0.0))
        return SQNN_E_INVALID_ARG;
    bool vec = row16(d_x, ldx, size_of(x_dtype)) && row16(d_weight, 0, 1);
    if (d_residual) {
        const uint32_t size = size_of(residual_dtype);
        if (!known_type(residual_dtype) || ldr < cols || ldh < cols || !aligned_to(d_residual, size) || !aligned_to(d_h, size))
            return SQNN_E_INVALID_ARG;
        vec = vec && row16(d_residual, ldr, size) && row16(d_h, ldh, size);
    }
    if (d_q) {
        if (ldq < cols || lds < (cols + 127) / 128 || !aligned_to(d_scale, 4)) return SQNN_E_INVALID_ARG;
        vec = vec && ((uintptr_t)d_q & 7) == 0 && ldq % 8 == 0;
    }
    if (d_y) {
        if (!known_type(y_dtype) || ldy < cols || !aligned_to(d_y, size_of(y_dtype))) return SQNN_E_INVALID_ARG;
        vec = vec && row16(d_y, ldy, size_of(y_dtype));
    }
    const NormArgs A{d_x, d_residual, d_weight, d_h, d_y, d_q, d_scale, ldx, ldr, ldh, ldq, lds, ldy, n, eps,
                     weight_dtype == SQNN_X_BF16, y_dtype == SQNN_X_BF16};
    using b16 = __nv_bfloat16;
    if (x_dtype == SQNN_X_BF16) {
        if (!d_residual) return launch_norm<b16, b16, false>(A, batch, vec, st);
        return residual_dtype == SQNN_X_BF16 ? launch_norm<b16, b16, true>(A, batch, vec, st) : launch_norm<b16, float, true>(A, batch, vec, st);
    }
    if (!d_residual) return launch_norm<float, float, false>(A, batch, vec, st);
    return residual_dtype == SQNN_X_BF16 ? launch_norm<float, b16, true>(A, batch, vec, st) : launch_norm<float, float, true>(A, batch, vec, st);
}

}  // namespace
}  // namespace sqnn

extern "C" int sqnn_rmsnorm_fp8(uint32_t batch, uint64_t n, const void *d_x, int x_dtype, int64_t ldx, const void *d_residual,
                                int residual_dtype, int64_t ldr, void *d_h, int64_t ldh, const void *d_weight, int weight_dtype,
                                double eps, uint8_t *d_q, int64_t ldq, float *d_scale, int64_t lds, void *d_y, int y_dtype,
                                int64_t ldy, void *cuda_stream)
{
    sqnn::ApiScope scope("sqnn_rmsnorm_fp8");
    return scope.finish(sqnn::rmsnorm_queue(batch, n, d_x, x_dtype, ldx, d_residual, residual_dtype, ldr, d_h, ldh, d_weight,
                                            weight_dtype, eps, d_q, ldq, d_scale, lds, d_y, y_dtype, ldy, (cudaStream_t)cuda_stream),
                        nullptr, (cudaStream_t)cuda_stream);
}
