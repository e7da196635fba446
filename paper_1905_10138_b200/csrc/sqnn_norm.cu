// Root-mean-square norm with the residual's addition and an output in 8 bits with scales.
//
//   h = round(x + r)                                 (r may be absent: h = x), stored in r's type
//   y = h * rstd * w,      rstd = 1 / sqrt(mean(h^2) + eps)
//   s_k = max |y| of 128 columns / 448 as fp32 (2^-126 at least), q = e4m3(y / s_k), ties to even
//
// What the definition says in exact arithmetic is what comes out, number for number: which 8-bit number a value rounds to must not
// hang on the order of a sum, or the same row would quantize differently here and in another implementation.  For that
//   - squares are added in 64 bits, and rstd is a 64-bit number;
//   - p = h 2^k w (2^k: rstd's power of two, so that p neither overflows nor vanishes where h does not) is exact where both are bf16, and
//     else kept with its rounding error e = fma(h 2^k, w, -p), so that the largest |p + e| of a group, and from it the scale, is exact;
//   - y / s is p c with c = rstd / (2^k s) in fp32: five roundings, less than 6 2^-24 off.  It is converted from both ends of what that allows (c (1 -+
//     2^-21)); only where these give two numbers (12 of a million values) is it computed once more in 64 bits.
// Every operand is read once and every result written once; a row stays in registers between its two passes.  8192 rows of 4096, bf16 with
// residual: 58 us (36 us at the copy's rate).  About 25 instructions an element fill 64 % of the issue slots; the rest is latency: a row has two barriers and one
// warp's work between its passes (2.8 of 11.4 warps wait at a barrier for each that issues), and 64 registers leave 32 warps an SM to hide it.  A first form took 108 us:
// a block per row with nothing of the next one on its way, tests of the distance to the border by bits, 64-bit indexes.
#include "sqnn_launch.h"
#include "sqnn_fp8.cuh"

#include <cuda_bf16.h>

#include <atomic>

namespace sqnn {
namespace {

struct NormArgs {
    const void *x, *r, *w;
    void *h, *y;
    uint8_t *q;
    float *s;
    int64_t ldx, ldr, ldh, ldq, lds, ldy;
    double eps, inv_n;
    uint32_t batch, n, y_bf16;
};

template <typename T> SQNN_DEV float to_f32(T v);
template <> SQNN_DEV float to_f32<float>(float v) { return v; }
template <> SQNN_DEV float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// Where a thread's eight elements of a slot lie.  Sixteen threads share a group of 128 columns: with VEC each has eight in a row (16-byte
// accesses; rows on 16-byte boundaries), without it every sixteenth (neighbouring threads on neighbouring elements, any alignment).
template <bool VEC> SQNN_DEV uint32_t first_of(uint32_t unit) { return VEC ? unit * 8 : (unit >> 4) * 128 + (unit & 15); }
template <bool VEC> constexpr uint32_t step_of = VEC ? 1 : 16;

// Eight elements as they were loaded, so that a load can be asked for long before its numbers are looked at.
template <typename T> struct Raw;
template <> struct Raw<float> {
    float4 a, b;
    SQNN_DEV void values(float (&v)[8]) const
    {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    SQNN_DEV void take(const float (&v)[8]) { a = make_float4(v[0], v[1], v[2], v[3]); b = make_float4(v[4], v[5], v[6], v[7]); }
    SQNN_DEV void put(float *p) const { *reinterpret_cast<float4 *>(p) = a; *reinterpret_cast<float4 *>(p + 4) = b; }
    SQNN_DEV void load(const float *p) { a = *reinterpret_cast<const float4 *>(p); b = *reinterpret_cast<const float4 *>(p + 4); }
};
template <> struct Raw<__nv_bfloat16> {
    uint4 a;
    SQNN_DEV void values(float (&v)[8]) const
    {
        const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(u[j] << 16);
            v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
        }
    }
    SQNN_DEV void take(const float (&v)[8])
    {
        a = make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]), bf16x2(v[6], v[7]));
    }
    SQNN_DEV void put(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = a; }
    SQNN_DEV void load(const __nv_bfloat16 *p) { a = *reinterpret_cast<const uint4 *>(p); }
};
// Elements past n read as zero.
template <typename T, bool VEC>
SQNN_DEV void fetch(const T *row, uint32_t i, uint32_t n, float (&v)[8])
{
    if (VEC && i + 8 <= n) {
        Raw<T> raw;
        raw.load(row + i);
        raw.values(v);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            const uint32_t at = i + j * step_of<VEC>;
            v[j] = at < n ? to_f32<T>(row[at]) : 0.0f;
        }
    }
}
SQNN_DEV void put(float *p, float v) { *p = v; }
SQNN_DEV void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
template <typename T, bool VEC>
SQNN_DEV void store(T *row, uint32_t i, uint32_t n, const float (&v)[8])
{
    if (VEC && i + 8 <= n) {
        Raw<T> raw;
        raw.take(v);
        raw.put(row + i);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            const uint32_t at = i + j * step_of<VEC>;
            if (at < n) put(row + at, v[j]);
        }
    }
}

template <typename T, bool VEC>
SQNN_DEV void request(Raw<T> &raw, const T *row, uint32_t unit, uint32_t units, uint32_t n)
{
    const uint32_t i = first_of<VEC>(unit);
    if (VEC && i + 8 <= n) {
        raw.load(row + i);
    } else {
        float v[8];
        fetch<T, VEC>(row, unit < units ? i : n, n, v);
        raw.take(v);
    }
}

// x + r as an fp32 number that rounds to r's type as the exact sum does.  An fp32 sum rounded again to bf16 could be off where it lands on a
// middle, so it is rounded to odd first (the last bit says that something was cut off); two bf16 numbers cannot get there.
template <typename XT, typename RT>
SQNN_DEV float add(float x, float r)
{
    if constexpr (sizeof(RT) == 2 && sizeof(XT) == 4) {
        const float lo = __fadd_rd(x, r), hi = __fadd_ru(x, r);
        return (__float_as_uint(lo) & 1u) ? lo : hi;
    }
    return x + r;
}

// Largest magnitude as (p, e), both with the sign taken out of p; bit patterns order magnitudes with NaN above infinity.
SQNN_DEV void larger(uint32_t &p, float &e, uint32_t q, float f)
{
    if (q > p || (q == p && f > e)) { p = q; e = f; }
}

SQNN_DEV double exp2_double(int k) { return __longlong_as_double((long long)(1023 + k) << 52); }

// 64-bit numbers to fp32 so that a second rounding to eight bits gives what one would: towards zero, with the last bit set if anything was cut off.
SQNN_DEV float round_to_odd(double d)
{
    const float f = (float)d;
    const float cut = fabs((double)f) > fabs(d) ? __uint_as_float(__float_as_uint(f) - 1) : f;
    return (double)cut != d && d == d ? __uint_as_float(__float_as_uint(cut) | 1u) : f;
}

// The eight numbers whose rounding fp32 left open (seldom run, so kept out of the way of the rest).
static __device__ __noinline__ uint2 convert_exactly(float4 a, float4 b, float4 v, float4 w, float scale_h, double c)
{
    const auto one = [&](float x, float y) { return round_to_odd((double)(x * scale_h) * (double)y * c); };
    return make_uint2(to_fp8x2(one(a.x, v.x), one(a.y, v.y)) | (to_fp8x2(one(a.z, v.z), one(a.w, v.w)) << 16),
                      to_fp8x2(one(b.x, w.x), one(b.y, w.y)) | (to_fp8x2(one(b.z, w.z), one(b.w, w.w)) << 16));
}

// A block takes rows in turn; SLOTS slots of eight elements a thread stay in registers, and the next row is on its way while this one is
// finished.  SLOTS = 0: rows longer than that are read a second time, h where it was stored.  MOST = 384 with one slot: three blocks to an SM hide what a
// look ahead would, and take fewer registers.
template <typename XT, typename RT, typename WT, bool RES, uint32_t SLOTS, uint32_t MOST, bool VEC>
__global__ void __launch_bounds__(MOST, MOST == 384 ? 3 : SLOTS == 1 || (SLOTS == 2 && (!VEC || sizeof(XT) + (RES ? sizeof(RT) : 0) <= 4)) ? 2 : 1) k_rmsnorm_fp8(const NormArgs A)
{
    __shared__ double part[16];
    __shared__ double rstd_s;
    constexpr bool EXACT = sizeof(RT) == 2 && sizeof(WT) == 2;     // products of h and w are fp32 numbers
    constexpr uint32_t KEPT = SLOTS ? SLOTS : 1;
    constexpr bool AHEAD = MOST == 512 && SLOTS * (sizeof(XT) + (RES ? sizeof(RT) : 0)) <= 16;      // what registers allow (SLOTS = 0: nothing to ask for)
    constexpr bool KEEP_WEIGHTS = SLOTS > 0 && sizeof(WT) == 2;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, T = blockDim.x, n = A.n, units = (n + 127) / 128 * 16;
    wait_prior_grid();
    launch_dependents();
    Raw<XT> next_x[KEPT];
    Raw<RT> next_r[KEPT];
    Raw<WT> weights[KEPT];
    auto ask = [&](uint32_t row) {
#pragma unroll
        for (uint32_t k = 0; k < KEPT; ++k) {
            request<XT, VEC>(next_x[k], static_cast<const XT *>(A.x) + (int64_t)row * A.ldx, k * T + tid, units, n);
            if (RES) request<RT, VEC>(next_r[k], static_cast<const RT *>(A.r) + (int64_t)row * A.ldr, k * T + tid, units, n);
        }
    };
    if constexpr (SLOTS > 0 && AHEAD) ask(blockIdx.x);
    if constexpr (KEEP_WEIGHTS) {
#pragma unroll
        for (uint32_t k = 0; k < SLOTS; ++k) request<WT, VEC>(weights[k], static_cast<const WT *>(A.w), k * T + tid, units, n);
    }
#pragma unroll 1
    for (uint32_t row32 = blockIdx.x; row32 < A.batch; row32 += gridDim.x) {
        const int64_t row = row32;
        const XT *x = static_cast<const XT *>(A.x) + row * A.ldx;
        const RT *r = static_cast<const RT *>(A.r) + (RES ? row * A.ldr : 0);
        RT *h = static_cast<RT *>(A.h) + (RES ? row * A.ldh : 0);
        float v[KEPT][8];

        double sums[4] = {};
        auto squares = [&](const float (&a)[8]) {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) { const double d = a[j]; sums[j & 3] = fma(d, d, sums[j & 3]); }
        };
        if constexpr (SLOTS > 0) {
            if constexpr (!AHEAD) ask(row32);
#pragma unroll
            for (uint32_t k = 0; k < SLOTS; ++k) {
                const uint32_t unit = k * T + tid;
                next_x[k].values(v[k]);
                if constexpr (RES) {
                    float b[8];
                    next_r[k].values(b);
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) v[k][j] = add<XT, RT>(v[k][j], b[j]);
                    Raw<RT> sum;
                    sum.take(v[k]);
                    sum.values(v[k]);
                    const uint32_t i = first_of<VEC>(unit);
                    if (VEC && i + 8 <= n) sum.put(h + i);
                    else if (unit < units) store<RT, VEC>(h, i, n, v[k]);
                }
            }
            if (AHEAD && row32 + gridDim.x < A.batch) ask(row32 + gridDim.x);
#pragma unroll
            for (uint32_t k = 0; k < SLOTS; ++k) squares(v[k]);
        } else {
            for (uint32_t unit = tid; unit < units; unit += T) {
                const uint32_t i = first_of<VEC>(unit);
                fetch<XT, VEC>(x, i, n, v[0]);
                if constexpr (RES) {
                    float b[8];
                    fetch<RT, VEC>(r, i, n, b);
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) v[0][j] = add<XT, RT>(v[0][j], b[j]);
                    Raw<RT> sum;
                    sum.take(v[0]);
                    sum.values(v[0]);
                    store<RT, VEC>(h, i, n, v[0]);
                }
                squares(v[0]);
            }
        }
        double sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
        for (uint32_t d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) part[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            sum = lane < T / 32 ? part[lane] : 0.0;
#pragma unroll
            for (uint32_t d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (lane == 0) rstd_s = rsqrt(sum * A.inv_n + A.eps);
        }
        __syncthreads();
        const double rstd = rstd_s;
        // 2^k: rstd's power of two as far as it is an fp32 number (rstd zero, infinite or NaN: any will do)
        int k2 = (int)((__double_as_longlong(rstd) >> 52) & 0x7ff) - 1023;
        k2 = k2 < -126 ? -126 : k2 > 127 ? 127 : k2;
        const float scale_h = __uint_as_float((uint32_t)(127 + k2) << 23);
        const double rest = rstd * exp2_double(-k2);                   // rstd / 2^k, exact
        const float rest32 = (float)rest;
        uint8_t *const q = A.q ? A.q + row * A.ldq : nullptr;

        auto finish = [&](uint32_t unit, const float (&a)[8], const Raw<WT> &weight) {        // all threads of a warp, in step
            const bool in = unit < units;
            const uint32_t i = first_of<VEC>(unit);
            float w[8], p[8];
            weight.values(w);
            if (q) {
                double most;
                if constexpr (EXACT) {
                    float top = 0.0f;
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) {
                        p[j] = a[j] * scale_h * w[j];
                        asm("{\n .reg .f32 m;\n abs.f32 m, %1;\n max.NaN.f32 %0, %0, m;\n}\n" : "+f"(top) : "f"(p[j]));
                    }
#pragma unroll
                    for (uint32_t d = 8; d; d >>= 1) {                 // the sixteen threads of the group
                        const float o = __shfl_xor_sync(0xffffffffu, top, d);
                        asm("max.NaN.f32 %0, %0, %1;\n" : "+f"(top) : "f"(o));
                    }
                    most = (double)top * rest;
                } else {
                    uint32_t top = 0;
                    float top_e = 0.0f;
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) {
                        const float b = a[j] * scale_h;
                        p[j] = b * w[j];
                        const float e = fmaf(b, w[j], -p[j]);
                        larger(top, top_e, __float_as_uint(p[j]) & 0x7fffffffu, p[j] < 0.0f ? -e : e);
                    }
#pragma unroll
                    for (uint32_t d = 8; d; d >>= 1) {
                        const uint32_t o = __shfl_xor_sync(0xffffffffu, top, d);
                        const float f = __shfl_xor_sync(0xffffffffu, top_e, d);
                        larger(top, top_e, o, f);
                    }
                    most = ((double)__uint_as_float(top) + (top < 0x7f800000u ? (double)top_e : 0.0)) * rest;
                }
                float s = (float)(most * (1.0 / (double)FP8_MAX));
                s = s < 0x1p-126f ? 0x1p-126f : s;                     // (NaN stays)
                const float c = rest32 * __frcp_rn(s), c_lo = c * (1.0f - 0x1p-21f), c_hi = c * (1.0f + 0x1p-21f);
                uint32_t lo[4], hi[4];
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    lo[j] = to_fp8x2(p[2 * j] * c_lo, p[2 * j + 1] * c_lo);
                    hi[j] = to_fp8x2(p[2 * j] * c_hi, p[2 * j + 1] * c_hi);
                }
                const uint2 all_hi = make_uint2(hi[0] | (hi[1] << 16), hi[2] | (hi[3] << 16));
                uint2 all = make_uint2(lo[0] | (lo[1] << 16), lo[2] | (lo[3] << 16));
                // (c is no fp32 number in rows below 2^-129 whose group is zero, or nearly)
                if (all.x != all_hi.x || all.y != all_hi.y || c_hi > 0x1.fffffep127f)
                    all = convert_exactly(make_float4(a[0], a[1], a[2], a[3]), make_float4(a[4], a[5], a[6], a[7]), make_float4(w[0], w[1], w[2], w[3]),
                                          make_float4(w[4], w[5], w[6], w[7]), scale_h, rest / (double)s);
                if (in) {
                    if (VEC && i + 8 <= n) {
                        *reinterpret_cast<uint2 *>(q + i) = all;
                    } else {
#pragma unroll
                        for (uint32_t j = 0; j < 8; ++j) {
                            const uint32_t at = i + j * step_of<VEC>;
                            if (at < n) q[at] = (uint8_t)((j < 4 ? all.x : all.y) >> (8 * (j & 3)));
                        }
                    }
                    if ((unit & 15) == 0) A.s[row * A.lds + (unit >> 4)] = s;
                }
            }
            if (A.y && in) {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) p[j] = a[j] * scale_h * w[j] * rest32;
                if (A.y_bf16) store<__nv_bfloat16, VEC>(static_cast<__nv_bfloat16 *>(A.y) + row * A.ldy, i, n, p);
                else store<float, VEC>(static_cast<float *>(A.y) + row * A.ldy, i, n, p);
            }
        };
        if constexpr (SLOTS > 0) {
#pragma unroll
            for (uint32_t k = 0; k < SLOTS; ++k) {
                if constexpr (!KEEP_WEIGHTS) request<WT, VEC>(weights[k], static_cast<const WT *>(A.w), k * T + tid, units, n);
                finish(k * T + tid, v[k], weights[k]);
            }
        } else {
            for (uint32_t base = 0; base < units; base += T) {
                const uint32_t unit = base + tid;
                if (unit < units) {                                    // h as this thread stored it, or x
                    if (RES) fetch<RT, VEC>(h, first_of<VEC>(unit), n, v[0]);
                    else fetch<XT, VEC>(x, first_of<VEC>(unit), n, v[0]);
                } else {
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) v[0][j] = 0.0f;
                }
                request<WT, VEC>(weights[0], static_cast<const WT *>(A.w), unit, units, n);
                finish(unit, v[0], weights[0]);
            }
        }
    }
}

// One slot of eight elements a thread, as far as 512 threads go, else as many as a row needs.  Many rows of which a thread loads no more than four bytes an
// element, on 16-byte boundaries: two slots, so that the reductions weigh less (8192 x 4096, bf16 with residual: one slot 59 us, two 56, four 71; at 2000 rows
// 17.3 and 18.7; 8000 x 2944 52 and 46, 2000 x 2944 16.3 and 15.4).  fp32 or unaligned rows have no registers to spare for two (8000 x 3001, fp32 and bf16 residual, bf16 y: 96 us
// with one, 166 with two; 8000 x 4096 66 and 76).  Where unaligned rows need two slots, two blocks to an SM (2000 x 5001, the same types: 58 us, one block 88).  The bound of 64
// registers that this takes makes the two-slot forms spill (fp32 and unaligned ones up to 212 bytes a thread); other sizes and types of them were not measured apart.
template <typename XT, typename RT, typename WT, bool RES>
int launch_norm(const NormArgs &A, uint32_t batch, bool vec, cudaStream_t st)
{
    const uint32_t units = (A.n + 127) / 128 * 16, most = 512;
    const uint32_t least = units <= most ? 1 : units <= 2 * most ? 2 : units <= 4 * most ? 4 : 0;
    const bool light = vec && sizeof(XT) + (RES ? sizeof(RT) : 0) <= 4;
    const bool many = batch >= (units <= 384 ? 4 : 16) * (uint32_t)sm_count();
    const uint32_t slots = least == 1 && light && many && units > 128 ? 2 : least;
    const uint32_t per = slots ? (units + slots - 1) / slots : most;
    const uint32_t threads = (per + 31) / 32 * 32;
#define SQNN_NORM_PICK(S, T) (vec ? k_rmsnorm_fp8<XT, RT, WT, RES, S, T, true> : k_rmsnorm_fp8<XT, RT, WT, RES, S, T, false>)
    auto k = slots == 1 ? threads <= 384 ? SQNN_NORM_PICK(1, 384) : SQNN_NORM_PICK(1, 512) : slots == 2 ? SQNN_NORM_PICK(2, 512)
           : slots == 4 ? SQNN_NORM_PICK(4, 512) : SQNN_NORM_PICK(0, 512);
#undef SQNN_NORM_PICK
    // as many blocks as run at once (asked for once per kernel, block and device)
    const uint32_t sms = (uint32_t)sm_count();
    uint32_t grid = batch;
    if (batch > sms) {
        static std::atomic<uint32_t> known[64][2][4][16];
        int dev = 0, n = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SQNN_E_CUDA;
        std::atomic<uint32_t> &have = known[dev][vec][slots == 4 ? 3 : slots][threads / 32 - 1];
        uint32_t at_once = have.load(std::memory_order_relaxed);
        if (!at_once) {
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k, (int)threads, 0) != cudaSuccess || n <= 0) return SQNN_E_CUDA;
            have.store(at_once = sms * (uint32_t)n, std::memory_order_relaxed);
        }
        grid = batch < at_once ? batch : at_once;
    }
    return launch_kernel(k, grid, threads, 0, st, A);
}
template <typename XT, typename RT, bool RES>
int launch_norm(const NormArgs &A, uint32_t batch, bool w_bf16, bool vec, cudaStream_t st)
{
    return w_bf16 ? launch_norm<XT, RT, __nv_bfloat16, RES>(A, batch, vec, st) : launch_norm<XT, RT, float, RES>(A, batch, vec, st);
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
    const NormArgs A{d_x, d_residual, d_weight, d_h, d_y, d_q, d_scale, ldx, ldr, ldh, ldq, lds, ldy, eps, 1.0 / (double)n, batch, (uint32_t)n, y_dtype == SQNN_X_BF16};
    const bool wb = weight_dtype == SQNN_X_BF16;
    using b16 = __nv_bfloat16;
    if (x_dtype == SQNN_X_BF16) {
        if (!d_residual) return launch_norm<b16, b16, false>(A, batch, wb, vec, st);
        return residual_dtype == SQNN_X_BF16 ? launch_norm<b16, b16, true>(A, batch, wb, vec, st) : launch_norm<b16, float, true>(A, batch, wb, vec, st);
    }
    if (!d_residual) return launch_norm<float, float, false>(A, batch, wb, vec, st);
    return residual_dtype == SQNN_X_BF16 ? launch_norm<float, b16, true>(A, batch, wb, vec, st) : launch_norm<float, float, true>(A, batch, wb, vec, st);
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
