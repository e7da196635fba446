// A mixture-of-experts layer of 8-bit weights for a few tokens, in two kernels.
//
//   logits = x R^T;  the top_k largest (ties to the lowest index), p their softmax
//   y = sum over a token's experts e of p_e D_e (silu(G_e x) * (U_e x)),    silu(a) = a / (1 + exp(-a))
//
// Few tokens reach many experts, so nearly every weight is used for one or two tokens: the layer is bound by reading the chosen experts'
// weights once.  They go from global memory to registers (a warp keeps several 16-byte loads per lane in flight), become fp16 there (exact)
// and are the A operand of mma.sync m16n8k16: 16 rows by 16 columns, up to eight tokens as the columns of B.  (mma.sync, not tcgen05: a
// stage in shared memory would only add a step to a stream that is used once, and the rate of mma.sync is several times what memory asks for.)
// The columns of a chunk of 64 are dealt to the MMAs so that a lane's 16 bytes of a row are its share of four of them.
//
// Activations are scaled by a power of two per chunk of 64 columns and token so that the largest lies below 2^15, and cut into fp16
// pieces: bf16 numbers are exact in one (down to 2^-40 of the chunk's largest), fp32 numbers leave 2^-22 with two.  Sums are fp32, per chunk in the MMA, then
// scaled by the weights' and the activations' scale and added to 32-bit sums.
//
// k_moe_up:   every cluster works out the routing for itself (its CTAs share the experts' logits through distributed shared memory), then the CTAs
//             share all (expert, 8 rows of G and the same 8 of U); a CTA's warps share the columns of up to 16 such units at a time.
// k_moe_down: a CTA has 16 rows of all chosen experts' D; its warps share (expert, chunk of columns) evenly; each sums into its own
//             accumulators, which are added up in warp order.
// No atomics on sums: results are the same from run to run.
#include "sqnn_launch.h"
#include "sqnn_fp8.cuh"
#include "sqnn_cluster.cuh"

#include <cuda_bf16.h>

#include <atomic>

namespace sqnn {
namespace {

constexpr uint32_t WARPS = 16, THREADS = WARPS * 32;
constexpr uint32_t CLUSTER = 4;           // CTAs that share the routing's work
constexpr uint32_t CHUNK = 64;            // columns per step of a warp
constexpr uint32_t AHEAD = 6;             // steps whose weights are in flight
constexpr uint32_t MAX_TOKENS = SQNN_MOE_MAX_TOKENS, MAX_EXPERTS = SQNN_MOE_MAX_EXPERTS, MAX_TOP_K = SQNN_MOE_MAX_TOP_K;
constexpr uint32_t MAX_PAIRS = MAX_TOKENS * MAX_TOP_K;
constexpr uint32_t MAX_ENTRIES = MAX_EXPERTS + MAX_PAIRS / 8;     // chosen experts, those with many tokens several times

struct MoeArgs {
    const void *x, *router;
    const uint8_t *gate_up, *down;
    const float *gate_up_scale, *down_scale;
    void *y;
    float *h;                     // workspace: [tokens * top_k][pitch]
    int32_t *ids;                 // workspace: [tokens * top_k]
    float *probs;
    int32_t *ids_out;
    float *probs_out;
    int64_t ldx, ldr, ldy;
    int64_t gu_expert, gu_half, gu_row, d_expert, d_row;          // strides
    uint32_t tokens, experts, top_k, hidden, inner, pitch;
    uint32_t renormalize, x_vec, r_vec, y_bf16;
};

// ---- routing tables in shared memory

struct Routing {
    int32_t ids[MAX_PAIRS];
    float probs[MAX_PAIRS];
    uint32_t mask[MAX_EXPERTS][2];        // tokens of an expert
    uint32_t entry[MAX_ENTRIES];          // expert | group of tokens << 16
    uint32_t totals[WARPS];
    uint32_t entries;
};
constexpr uint32_t ROUTING_BYTES = (sizeof(Routing) + 127) / 128 * 128;

// From ids to the list of (expert, group of up to `per` of its tokens), ascending.  All threads; ends with a barrier.
SQNN_DEV void list_entries(Routing &R, const MoeArgs &M, uint32_t per)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (uint32_t i = tid; i < 2 * M.experts; i += THREADS) (&R.mask[0][0])[i] = 0;
    __syncthreads();
    for (uint32_t i = tid; i < M.tokens * M.top_k; i += THREADS) {
        const uint32_t t = i / M.top_k;
        atomicOr(&R.mask[R.ids[i]][t >> 5], 1u << (t & 31));
    }
    __syncthreads();
    static_assert(MAX_EXPERTS <= THREADS, "an expert per thread");
    const uint32_t mine = tid < M.experts ? __popc(R.mask[tid][0]) + __popc(R.mask[tid][1]) : 0, groups = (mine + per - 1) / per;
    uint32_t sum = groups;
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == 31) R.totals[warp] = sum;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < WARPS; ++w) {
        if (w < warp) before += R.totals[w];
        all += R.totals[w];
    }
    for (uint32_t g = 0; g < groups; ++g) R.entry[before + sum - groups + g] = tid | (g << 16);
    if (tid == 0) R.entries = all;
    __syncthreads();
}
// The n-th token of an expert, MAX_TOKENS if it has fewer.
SQNN_DEV uint32_t token_of(const Routing &R, uint32_t expert, uint32_t n)
{
    uint32_t lo = R.mask[expert][0], hi = R.mask[expert][1];
    for (uint32_t i = 0; i < n; ++i) {
        if (lo) lo &= lo - 1;
        else hi &= hi - 1;                                       // (0 stays 0)
    }
    return lo ? (uint32_t)__ffs((int)lo) - 1 : hi ? 31 + (uint32_t)__ffs((int)hi) : MAX_TOKENS;
}
// Which of a token's experts this one is: its row of h.
SQNN_DEV uint32_t pair_of(const Routing &R, const MoeArgs &M, uint32_t token, uint32_t expert)
{
    uint32_t s = 0;
    while (s + 1 < M.top_k && R.ids[token * M.top_k + s] != (int32_t)expert) ++s;
    return token * M.top_k + s;
}

// ---- loads

SQNN_DEV uint4 stream16(const uint8_t *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// 16 bytes of a row from byte `at` on; bytes from `n` on are zero (rows start on 16-byte boundaries, but the last may end with its data).
SQNN_DEV uint4 row16(const uint8_t *row, uint32_t at, uint32_t n)
{
    if (at + 16 <= n) return stream16(row + at);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t j = 0; j < 16; ++j)
        if (at + j < n) w[j >> 2] |= (uint32_t)row[at + j] << (8 * (j & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 16 elements of a row of activations from element `at` on as fp32; elements from `n` on are zero.
SQNN_DEV void values16(const float *row, uint32_t at, uint32_t n, bool vec, float (&v)[16])
{
    if (vec && at + 16 <= n) {
#pragma unroll
        for (uint32_t j = 0; j < 16; j += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(row + at + j);
            v[j] = f.x; v[j + 1] = f.y; v[j + 2] = f.z; v[j + 3] = f.w;
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 16; ++j) v[j] = at + j < n ? row[at + j] : 0.0f;
    }
}
SQNN_DEV void values16(const __nv_bfloat16 *row, uint32_t at, uint32_t n, bool vec, float (&v)[16])
{
    if (vec && at + 16 <= n) {
#pragma unroll
        for (uint32_t j = 0; j < 16; j += 8) {
            const uint4 f = *reinterpret_cast<const uint4 *>(row + at + j);
            const uint32_t u[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                v[j + 2 * i] = __uint_as_float(u[i] << 16);
                v[j + 2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 16; ++j) v[j] = at + j < n ? __bfloat162float(row[at + j]) : 0.0f;
    }
}

// ---- the multiplication of one chunk

SQNN_DEV uint32_t fp8x2_to_f16x2(uint32_t two)
{
    uint32_t v;
    asm("{\n .reg .b16 t;\n cvt.u16.u32 t, %1;\n cvt.rn.f16x2.e4m3x2 %0, t;\n}\n" : "=r"(v) : "r"(two));
    return v;
}
SQNN_DEV uint32_t f16x2(float lo, float hi)
{
    uint32_t v;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(v) : "f"(hi), "f"(lo));
    return v;
}
SQNN_DEV float f16_lo(uint32_t v) { float f; asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.f32.f16 %0, l;\n}\n" : "=f"(f) : "r"(v)); return f; }
SQNN_DEV float f16_hi(uint32_t v) { float f; asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.f32.f16 %0, h;\n}\n" : "=f"(f) : "r"(v)); return f; }
SQNN_DEV void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// B operand of a chunk: this lane's 16 columns of its token (lane / 4), in one or two pieces.
template <bool EXACT16>
struct Columns {
    uint32_t hi[8], lo[EXACT16 ? 1 : 8];
    float back;                   // what undoes the scaling
    SQNN_DEV void make(const float (&v)[16])
    {
        uint32_t top = 0;
#pragma unroll
        for (uint32_t j = 0; j < 16; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const uint32_t e = max(top >> 23, 15u);                  // 255 for infinities and NaN: finite numbers stay finite beside them
        const float s = __uint_as_float((268u - e) << 23);       // 2^(14 - (e - 127))
        back = __uint_as_float((e - 14u) << 23);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            const float a = v[2 * j] * s, b = v[2 * j + 1] * s;
            hi[j] = f16x2(a, b);
            if constexpr (!EXACT16) lo[j] = f16x2(a - f16_lo(hi[j]), b - f16_hi(hi[j]));
        }
    }
};

// c += (16 rows x 64 columns of weights) . B
template <bool EXACT16>
SQNN_DEV void multiply(float (&c)[4], const uint4 &top, const uint4 &bottom, const Columns<EXACT16> &B)
{
    const uint32_t r[4] = {top.x, top.y, top.z, top.w}, q[4] = {bottom.x, bottom.y, bottom.z, bottom.w};
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t a[4] = {fp8x2_to_f16x2(r[j]), fp8x2_to_f16x2(q[j]), fp8x2_to_f16x2(r[j] >> 16), fp8x2_to_f16x2(q[j] >> 16)};
        mma_f16(c, a, B.hi[2 * j], B.hi[2 * j + 1]);
        if constexpr (!EXACT16) mma_f16(c, a, B.lo[2 * j], B.lo[2 * j + 1]);
    }
}

// ---- routing

SQNN_DEV void row_values8(const float *row, uint32_t at, uint32_t n, bool vec, float (&v)[8])
{
    if (vec && at + 8 <= n) {
        const float4 a = *reinterpret_cast<const float4 *>(row + at), b = *reinterpret_cast<const float4 *>(row + at + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) v[j] = at + j < n ? row[at + j] : 0.0f;
    }
}
SQNN_DEV void row_values8(const __nv_bfloat16 *row, uint32_t at, uint32_t n, bool vec, float (&v)[8])
{
    if (vec && at + 8 <= n) {
        const uint4 f = *reinterpret_cast<const uint4 *>(row + at);
        const uint32_t u[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) v[j] = at + j < n ? __bfloat162float(row[at + j]) : 0.0f;
    }
}

// Logits of this CTA's experts (every CLUSTER-th) into the shared memory of all CTAs of the cluster.  Eight products at a time in fp32,
// their sums in 64 bits: which experts a token goes to must not hang on the order of a sum.
template <typename XT>
SQNN_DEV void logits_of_cluster(const MoeArgs &M, double *logits)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = cluster_rank();
    constexpr uint32_t GROUP = 4;                                // tokens that share a read of an expert's row
    const uint32_t groups = (M.tokens + GROUP - 1) / GROUP, mine = (M.experts - rank + CLUSTER - 1) / CLUSTER;
    const XT *const x = static_cast<const XT *>(M.x), *const router = static_cast<const XT *>(M.router);
    for (uint32_t i = warp; i < mine * groups; i += WARPS) {
        const uint32_t e = rank + CLUSTER * (i / groups), t0 = i % groups * GROUP;
        double sum[GROUP] = {};
        for (uint32_t at = lane * 8; at < M.hidden; at += 256) {
            float r[8];
            row_values8(router + (int64_t)e * M.ldr, at, M.hidden, M.r_vec, r);
#pragma unroll
            for (uint32_t t = 0; t < GROUP; ++t) {
                if (t0 + t < M.tokens) {
                    float v[8], s = 0.0f;
                    row_values8(x + (int64_t)(t0 + t) * M.ldx, at, M.hidden, M.x_vec, v);
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) s = fmaf(r[j], v[j], s);
                    sum[t] += (double)s;
                }
            }
        }
#pragma unroll
        for (uint32_t t = 0; t < GROUP; ++t) {
#pragma unroll
            for (uint32_t d = 16; d; d >>= 1) sum[t] += __shfl_xor_sync(0xffffffffu, sum[t], d);
            if (t0 + t < M.tokens && lane < CLUSTER) peer_store(peer_addr(smem_addr(logits + (t0 + t) * M.experts + e), lane), sum[t]);
        }
    }
}

// The top_k experts of each token and their shares; a warp per token.  NaN counts as the largest, so that there are always top_k different ones.
SQNN_DEV void choose(const MoeArgs &M, const double *logits, Routing &R)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const double INF = __longlong_as_double(0x7ff0000000000000ll);
    for (uint32_t t = warp; t < M.tokens; t += WARPS) {
        const double *l = logits + t * M.experts;
        uint32_t taken = 0;                                      // bit j: expert lane + 32 j
        double first = 0.0;
        float total = 0.0f, mine = 0.0f;                         // lane s keeps the share of the s-th expert
        for (uint32_t s = 0; s < M.top_k; ++s) {
            double best = -INF;
            uint32_t at = MAX_EXPERTS;
            for (uint32_t j = 0, e = lane; e < M.experts; ++j, e += 32) {
                if (taken >> j & 1) continue;
                double v = l[e];
                v = v != v ? INF : v;
                if (at == MAX_EXPERTS || v > best) { best = v; at = e; }
            }
#pragma unroll
            for (uint32_t d = 16; d; d >>= 1) {
                const double v = __shfl_xor_sync(0xffffffffu, best, d);
                const uint32_t a = __shfl_xor_sync(0xffffffffu, at, d);
                if (a != MAX_EXPERTS && (at == MAX_EXPERTS || v > best || (v == best && a < at))) { best = v; at = a; }
            }
            if ((at & 31) == lane) taken |= 1u << (at >> 5);
            const double raw = l[at];
            if (s == 0) first = raw;
            const float p = expf((float)(raw - first));
            if (lane == s) { mine = p; R.ids[t * M.top_k + s] = (int32_t)at; }
            total += p;
        }
        if (!M.renormalize) {
            total = 0.0f;
            for (uint32_t e = lane; e < M.experts; e += 32) total += expf((float)(l[e] - first));
#pragma unroll
            for (uint32_t d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
        }
        if (lane < M.top_k) R.probs[t * M.top_k + lane] = mine / total;
    }
}

// ---- first kernel: routing, then h = silu(G x) * (U x) for every (token, expert)

template <typename XT, uint32_t NT>
__global__ void __launch_bounds__(THREADS, 1) k_moe_up(const MoeArgs M)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Routing &R = *reinterpret_cast<Routing *>(smem_raw);
    double *const logits = reinterpret_cast<double *>(smem_raw + ROUTING_BYTES); // [tokens][experts]; after the routing:
    float *const parts = reinterpret_cast<float *>(smem_raw + ROUTING_BYTES);    // [round's parity][warp][its first or second unit][sum][lane]
    auto part = [&](uint32_t parity, uint32_t w, uint32_t which, uint32_t j) -> float * { return parts + ((((parity * WARPS + w) * 2 + which) * 4 * NT + j) << 5); };
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    constexpr bool EXACT16 = sizeof(XT) == 2;
    wait_prior_grid();
    launch_dependents();
    cluster_sync();                                              // all CTAs of the cluster run: their shared memory may be written
    logits_of_cluster<XT>(M, logits);
    cluster_sync();
    choose(M, logits, R);
    __syncthreads();
    if (blockIdx.x == 0)
        for (uint32_t i = tid; i < M.tokens * M.top_k; i += THREADS) {
            M.ids[i] = R.ids[i];
            M.probs[i] = R.probs[i];
            if (M.ids_out) M.ids_out[i] = R.ids[i];
            if (M.probs_out) M.probs_out[i] = R.probs[i];
        }
    list_entries(R, M, 8 * NT);

    const uint32_t groups = (M.inner + 7) / 8, units = R.entries * groups, chunks = (M.hidden + CHUNK - 1) / CHUNK;
    const uint32_t u0 = (uint32_t)((uint64_t)units * blockIdx.x / gridDim.x), u1 = (uint32_t)((uint64_t)units * (blockIdx.x + 1) / gridDim.x);
    const uint32_t iblocks = (M.inner + FP8_BLOCK - 1) / FP8_BLOCK, hblocks = (M.hidden + FP8_BLOCK - 1) / FP8_BLOCK;
    const XT *const x = static_cast<const XT *>(M.x);

    // A warp's way through the rounds: chunk `c` of unit `u`, `left` chunks to go in this round.
    struct Walk { uint32_t round0, u, c, left; };
    auto enter = [&](Walk &w, uint32_t round0) {                 // the warp's share of the round that begins at unit round0
        w.round0 = round0;
        w.left = 0;
        if (round0 >= u1) return;
        const uint32_t total = min(WARPS, u1 - round0) * chunks, a = total * warp / WARPS, b = total * (warp + 1) / WARPS;
        w.u = round0 + a / chunks;
        w.c = a % chunks;
        w.left = b - a;
    };
    auto next = [&](Walk &w) {                                   // -> false at the end of the round
        if (++w.c == chunks) { w.c = 0; ++w.u; }
        return --w.left != 0;
    };
    struct Ring { uint4 gate, up; float sg, su; };
    Ring ring[AHEAD];
    Walk ahead;
    auto request = [&](Ring &r) {                                // the weights of the chunk `ahead` stands at
        if (ahead.round0 >= u1) return;
        const uint32_t n = ahead.u / groups, e = R.entry[n] & 0xffffu, row8 = (ahead.u - n * groups) * 8, row = min(row8 + g, M.inner - 1);
        const uint8_t *p = M.gate_up + (int64_t)e * M.gu_expert + (int64_t)row * M.gu_row;
        const uint32_t at = ahead.c * CHUNK + t4 * 16;
        r.gate = row16(p, at, M.hidden);
        r.up = row16(p + M.gu_half, at, M.hidden);
        const float *s = M.gate_up_scale + ((uint64_t)(2 * e) * iblocks + row8 / FP8_BLOCK) * hblocks + ahead.c / (FP8_BLOCK / CHUNK);
        r.sg = __ldg(s);
        r.su = __ldg(s + (uint64_t)iblocks * hblocks);
        if (!next(ahead))
            do enter(ahead, ahead.round0 + WARPS);
            while (ahead.left == 0 && ahead.round0 < u1);
    };
    enter(ahead, u0);
    while (ahead.left == 0 && ahead.round0 < u1) enter(ahead, ahead.round0 + WARPS);
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j) request(ring[j]);

    uint32_t slot = 0, parity = 0;
    for (uint32_t round0 = u0; round0 < u1; round0 += WARPS, parity ^= 1) {
        Walk w;
        enter(w, round0);
        const uint32_t first_unit = w.u;
        float acc[NT][4];
#pragma unroll
        for (uint32_t k = 0; k < NT; ++k) acc[k][0] = acc[k][1] = acc[k][2] = acc[k][3] = 0.0f;
        auto put = [&](uint32_t which) {
#pragma unroll
            for (uint32_t k = 0; k < NT; ++k)
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    part(parity, warp, which, 4 * k + j)[lane] = acc[k][j];
                    acc[k][j] = 0.0f;
                }
        };
        const XT *rows[NT];
        bool have[NT];
        auto tokens_of = [&](uint32_t unit) {
            const uint32_t en = R.entry[unit / groups], e = en & 0xffffu, g0 = (en >> 16) * 8 * NT;
#pragma unroll
            for (uint32_t k = 0; k < NT; ++k) {
                const uint32_t t = token_of(R, e, g0 + 8 * k + g);
                have[k] = t < MAX_TOKENS;
                rows[k] = x + (int64_t)(have[k] ? t : 0) * M.ldx;
            }
        };
        if (w.left) tokens_of(w.u);
        bool more = w.left != 0;
        while (more) {
#pragma unroll
            for (uint32_t j = 0; j < AHEAD; ++j) {
                if (!more || slot != j) continue;                // (uniform; a round may end anywhere in the ring)
                float sg, su;
                uint4 gate, up;
                gate = ring[j].gate; up = ring[j].up; sg = ring[j].sg; su = ring[j].su;
                request(ring[j]);
#pragma unroll
                for (uint32_t k = 0; k < NT; ++k) {
                    float v[16];
                    if (have[k]) values16(rows[k], w.c * CHUNK + t4 * 16, M.hidden, M.x_vec, v);
                    else
#pragma unroll
                        for (uint32_t i = 0; i < 16; ++i) v[i] = 0.0f;
                    Columns<EXACT16> B;
                    B.make(v);
                    float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    multiply(c, gate, up, B);
                    const float b0 = __shfl_sync(0xffffffffu, B.back, 8 * t4), b1 = __shfl_sync(0xffffffffu, B.back, 8 * t4 + 4);
                    acc[k][0] = fmaf(c[0], sg * b0, acc[k][0]);
                    acc[k][1] = fmaf(c[1], sg * b1, acc[k][1]);
                    acc[k][2] = fmaf(c[2], su * b0, acc[k][2]);
                    acc[k][3] = fmaf(c[3], su * b1, acc[k][3]);
                }
                const uint32_t unit = w.u;
                more = next(w);
                slot = slot + 1 == AHEAD ? 0 : slot + 1;
                if (!more || w.u != unit) put(unit - first_unit);
                if (more && w.u != unit) tokens_of(w.u);
            }
        }
        __syncthreads();
        // a warp per unit: its parts in warp order, the gate, and out to h
        if (warp < min(WARPS, u1 - round0)) {
            const uint32_t unit = round0 + warp, count = min(WARPS, u1 - round0), total = count * chunks;
            float sum[NT][4];
#pragma unroll
            for (uint32_t k = 0; k < NT; ++k) sum[k][0] = sum[k][1] = sum[k][2] = sum[k][3] = 0.0f;
            for (uint32_t q = 0; q < WARPS; ++q) {
                const uint32_t a = total * q / WARPS, b = total * (q + 1) / WARPS;
                if (a >= b || b <= warp * chunks || a >= (warp + 1) * chunks) continue;
                const uint32_t which = warp - a / chunks;
#pragma unroll
                for (uint32_t k = 0; k < NT; ++k)
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) sum[k][j] += part(parity, q, which, 4 * k + j)[lane];
            }
            const uint32_t en = R.entry[unit / groups], e = en & 0xffffu, g0 = (en >> 16) * 8 * NT, row = unit % groups * 8 + g;
#pragma unroll
            for (uint32_t k = 0; k < NT; ++k)
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) {
                    const uint32_t t = token_of(R, e, g0 + 8 * k + 2 * t4 + j);
                    if (t < MAX_TOKENS && row < M.inner) {
                        const float a = sum[k][j];
                        M.h[(uint64_t)pair_of(R, M, t, e) * M.pitch + row] = a / (1.0f + expf(-a)) * sum[k][2 + j];
                    }
                }
        }
    }
    // no CTA leaves while another one of its cluster may still write to it: all such writes were before the second cluster_sync
}

// ---- second kernel: y = sum p D h

template <uint32_t NT>
__global__ void __launch_bounds__(THREADS, 1) k_moe_down(const MoeArgs M)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Routing &R = *reinterpret_cast<Routing *>(smem_raw);
    float *const sums = reinterpret_cast<float *>(smem_raw + ROUTING_BYTES);     // [warp][token][16 rows]
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const uint32_t row0 = blockIdx.x * 16;
    float *const mine = sums + (uint64_t)warp * M.tokens * 16;
    for (uint32_t i = lane; i < M.tokens * 16; i += 32) mine[i] = 0.0f;
    wait_prior_grid();
    launch_dependents();
    for (uint32_t i = tid; i < M.tokens * M.top_k; i += THREADS) {
        R.ids[i] = M.ids[i];
        R.probs[i] = M.probs[i];
    }
    __syncthreads();
    list_entries(R, M, 8 * NT);
    const uint32_t chunks = (M.inner + CHUNK - 1) / CHUNK, total = R.entries * chunks;
    const uint32_t q0 = (uint32_t)((uint64_t)total * warp / WARPS), q1 = (uint32_t)((uint64_t)total * (warp + 1) / WARPS);
    const uint32_t iblocks = (M.inner + FP8_BLOCK - 1) / FP8_BLOCK, hblocks = (M.hidden + FP8_BLOCK - 1) / FP8_BLOCK;
    const uint32_t ra = min(row0 + g, M.hidden - 1), rb = min(row0 + g + 8, M.hidden - 1);

    struct Ring { uint4 a, b; float s; };
    Ring ring[AHEAD];
    uint32_t ahead_n = q0 / chunks, ahead_c = q0 % chunks, ahead_q = q0;
    auto request = [&](Ring &r) {
        if (ahead_q >= q1) return;
        const uint32_t e = R.entry[ahead_n] & 0xffffu;
        const uint8_t *p = M.down + (int64_t)e * M.d_expert;
        const uint32_t at = ahead_c * CHUNK + t4 * 16;
        r.a = row16(p + (int64_t)ra * M.d_row, at, M.inner);
        r.b = row16(p + (int64_t)rb * M.d_row, at, M.inner);
        r.s = __ldg(M.down_scale + ((uint64_t)e * hblocks + row0 / FP8_BLOCK) * iblocks + ahead_c / (FP8_BLOCK / CHUNK));
        ++ahead_q;
        if (++ahead_c == chunks) { ahead_c = 0; ++ahead_n; }
    };
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j) request(ring[j]);

    uint32_t n = q0 / chunks, c_at = q0 % chunks;
    float acc[NT][4];
    const float *rows[NT];
    bool have[NT];
    auto begin = [&]() {
        const uint32_t en = R.entry[n], e = en & 0xffffu, g0 = (en >> 16) * 8 * NT;
#pragma unroll
        for (uint32_t k = 0; k < NT; ++k) {
            acc[k][0] = acc[k][1] = acc[k][2] = acc[k][3] = 0.0f;
            const uint32_t t = token_of(R, e, g0 + 8 * k + g);
            have[k] = t < MAX_TOKENS;
            rows[k] = M.h + (have[k] ? (uint64_t)pair_of(R, M, t, e) * M.pitch : 0);
        }
    };
    auto end = [&]() {                                           // an expert's part goes to the warp's sums
        const uint32_t en = R.entry[n], e = en & 0xffffu, g0 = (en >> 16) * 8 * NT;
#pragma unroll
        for (uint32_t k = 0; k < NT; ++k)
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {
                const uint32_t t = token_of(R, e, g0 + 8 * k + 2 * t4 + j);
                if (t < MAX_TOKENS) {
                    const float p = R.probs[pair_of(R, M, t, e)];
                    float *const s = mine + t * 16 + g;
                    s[0] = fmaf(p, acc[k][j], s[0]);
                    s[8] = fmaf(p, acc[k][2 + j], s[8]);
                }
            }
        __syncwarp();
    };
    if (q0 < q1) begin();
    for (uint32_t q = q0; q < q1;) {
#pragma unroll
        for (uint32_t j = 0; j < AHEAD; ++j) {
            if (q >= q1) break;
            const uint4 a = ring[j].a, b = ring[j].b;
            const float s = ring[j].s;
            request(ring[j]);
#pragma unroll
            for (uint32_t k = 0; k < NT; ++k) {
                float v[16];
                if (have[k]) values16(rows[k], c_at * CHUNK + t4 * 16, M.inner, true, v);
                else
#pragma unroll
                    for (uint32_t i = 0; i < 16; ++i) v[i] = 0.0f;
                Columns<false> B;
                B.make(v);
                float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                multiply(c, a, b, B);
                const float b0 = __shfl_sync(0xffffffffu, B.back, 8 * t4) * s, b1 = __shfl_sync(0xffffffffu, B.back, 8 * t4 + 4) * s;
                acc[k][0] = fmaf(c[0], b0, acc[k][0]);
                acc[k][1] = fmaf(c[1], b1, acc[k][1]);
                acc[k][2] = fmaf(c[2], b0, acc[k][2]);
                acc[k][3] = fmaf(c[3], b1, acc[k][3]);
            }
            ++q;
            if (++c_at == chunks || q == q1) {
                end();
                if (c_at == chunks) { c_at = 0; ++n; }
                if (q < q1) begin();
            }
        }
    }
    __syncthreads();
    for (uint32_t i = tid; i < M.tokens * 16; i += THREADS) {
        const uint32_t t = i >> 4, row = row0 + (i & 15);
        float s = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < WARPS; ++w) s += sums[(uint64_t)w * M.tokens * 16 + i];
        if (row < M.hidden) {
            const int64_t at = (int64_t)t * M.ldy + row;
            if (M.y_bf16) static_cast<__nv_bfloat16 *>(M.y)[at] = __float2bfloat16_rn(s);
            else static_cast<float *>(M.y)[at] = s;
        }
    }
}

// ---- host

struct MoeShape { uint32_t pairs, pitch; size_t h_bytes, ids_bytes, bytes; };
MoeShape moe_shape(uint32_t tokens, uint32_t top_k, uint64_t inner)
{
    MoeShape s;
    s.pairs = tokens * top_k;
    s.pitch = (uint32_t)((inner + 31) / 32 * 32);
    s.h_bytes = ((size_t)s.pairs * s.pitch * 4 + 255) / 256 * 256;
    s.ids_bytes = ((size_t)s.pairs * 4 + 255) / 256 * 256;
    s.bytes = s.h_bytes + 2 * s.ids_bytes;
    return s;
}

template <typename XT, uint32_t NT>
int launch_moe(const MoeArgs &M, cudaStream_t st)
{
    auto up = k_moe_up<XT, NT>;
    auto down = k_moe_down<NT>;
    const size_t logits = (size_t)M.tokens * M.experts * sizeof(double), parts = (size_t)2 * WARPS * 2 * 4 * NT * 32 * sizeof(float);
    const size_t smem_up = ROUTING_BYTES + (logits > parts ? logits : parts), smem_down = ROUTING_BYTES + (size_t)WARPS * M.tokens * 16 * sizeof(float);
    if (ensure_dynamic_smem(reinterpret_cast<const void *>(up), smem_up) != SQNN_OK) return SQNN_E_CUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CLUSTER;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CLUSTER);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem_up;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    // as many CTAs as run at once in whole clusters, asked for once per device (threads and registers decide, not shared memory: one per SM)
    static std::atomic<int> known[64];
    int dev = 0, clusters = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SQNN_E_CUDA;
    if (dev < 64) clusters = known[dev].load(std::memory_order_relaxed);
    if (clusters == 0) {
        if (cudaOccupancyMaxActiveClusters(&clusters, up, &cfg) != cudaSuccess || clusters <= 0) return SQNN_E_CUDA;
        if (dev < 64) known[dev].store(clusters, std::memory_order_relaxed);
    }
    cfg.gridDim = dim3((uint32_t)clusters * CLUSTER);
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, up, M) != cudaSuccess) return SQNN_E_CUDA;
    return launch_kernel(down, (M.hidden + 15) / 16, THREADS, smem_down, st, M);
}

int moe_queue(const sqnn_moe *L, uint32_t tokens, const void *d_x, int x_dtype, int64_t ldx, void *d_y, int y_dtype, int64_t ldy,
              int32_t *d_ids, float *d_probs, void *d_workspace, size_t workspace_bytes, cudaStream_t st)
{
    const auto known_type = [](int t) { return t == SQNN_X_F32 || t == SQNN_X_BF16; };
    const auto aligned_to = [](const void *p, uintptr_t size) { return ((uintptr_t)p & (size - 1)) == 0; };
    if (!L || !d_x || !d_y || tokens == 0) return SQNN_E_INVALID_ARG;
    if (!L->router || !L->gate_up || !L->gate_up_scale || !L->down || !L->down_scale) return SQNN_E_INVALID_ARG;
    if (L->experts == 0 || L->top_k == 0 || L->top_k > L->experts || L->hidden == 0 || L->inner == 0) return SQNN_E_INVALID_ARG;
    if (!known_type(x_dtype) || !known_type(y_dtype)) return SQNN_E_INVALID_ARG;
    if (tokens > SQNN_MOE_MAX_TOKENS || L->experts > SQNN_MOE_MAX_EXPERTS || L->top_k > SQNN_MOE_MAX_TOP_K || tokens * L->experts > SQNN_MOE_MAX_LOGITS ||
        L->hidden > (1u << 20) || L->inner > (1u << 20))
        return SQNN_E_UNSUPPORTED;
    const int64_t hidden = L->hidden, inner = L->inner;
    const uintptr_t xs = x_dtype == SQNN_X_BF16 ? 2 : 4, ys = y_dtype == SQNN_X_BF16 ? 2 : 4;
    if (ldx < hidden || ldy < hidden || L->router_row < hidden || L->gate_up_row < hidden || L->down_row < inner || L->gate_up_half < 0 ||
        L->gate_up_expert < 0 || L->down_expert < 0)
        return SQNN_E_INVALID_ARG;
    if (!aligned_to(d_x, xs) || !aligned_to(L->router, xs) || !aligned_to(d_y, ys) || !aligned_to(L->gate_up_scale, 4) || !aligned_to(L->down_scale, 4) ||
        !aligned_to(d_ids, 4) || !aligned_to(d_probs, 4))
        return SQNN_E_INVALID_ARG;
    if (!aligned_to(L->gate_up, 16) || !aligned_to(L->down, 16) || ((L->gate_up_row | L->gate_up_half | L->gate_up_expert | L->down_row | L->down_expert) & 15))
        return SQNN_E_UNSUPPORTED;
    const MoeShape shape = moe_shape(tokens, L->top_k, L->inner);
    if (!d_workspace || workspace_bytes < shape.bytes || !aligned_to(d_workspace, 256)) return SQNN_E_WORKSPACE;
    MoeArgs M = {};
    M.x = d_x; M.router = L->router; M.gate_up = L->gate_up; M.down = L->down;
    M.gate_up_scale = L->gate_up_scale; M.down_scale = L->down_scale;
    M.y = d_y;
    M.h = static_cast<float *>(d_workspace);
    M.ids = reinterpret_cast<int32_t *>(static_cast<uint8_t *>(d_workspace) + shape.h_bytes);
    M.probs = reinterpret_cast<float *>(static_cast<uint8_t *>(d_workspace) + shape.h_bytes + shape.ids_bytes);
    M.ids_out = d_ids; M.probs_out = d_probs;
    M.ldx = ldx; M.ldr = L->router_row; M.ldy = ldy;
    M.gu_expert = L->gate_up_expert; M.gu_half = L->gate_up_half; M.gu_row = L->gate_up_row;
    M.d_expert = L->down_expert; M.d_row = L->down_row;
    M.tokens = tokens; M.experts = L->experts; M.top_k = L->top_k; M.hidden = L->hidden; M.inner = L->inner; M.pitch = shape.pitch;
    M.renormalize = L->renormalize;
    M.x_vec = aligned_to(d_x, 16) && (ldx * (int64_t)xs) % 16 == 0;
    M.r_vec = aligned_to(L->router, 16) && (L->router_row * (int64_t)xs) % 16 == 0;
    M.y_bf16 = y_dtype == SQNN_X_BF16;
    // up to eight tokens of an expert are multiplied together, from nine tokens on up to sixteen
    if (x_dtype == SQNN_X_BF16) return tokens <= 8 ? launch_moe<__nv_bfloat16, 1>(M, st) : launch_moe<__nv_bfloat16, 2>(M, st);
    return tokens <= 8 ? launch_moe<float, 1>(M, st) : launch_moe<float, 2>(M, st);
}

}  // namespace
}  // namespace sqnn

extern "C" size_t sqnn_moe_workspace_bytes(uint32_t tokens, uint32_t top_k, uint32_t inner)
{
    if (tokens > SQNN_MOE_MAX_TOKENS || top_k > SQNN_MOE_MAX_TOP_K) return 0;
    return sqnn::moe_shape(tokens, top_k, inner).bytes;
}

extern "C" int sqnn_moe_fp8(const sqnn_moe *layer, uint32_t tokens, const void *d_x, int x_dtype, int64_t ldx, void *d_y, int y_dtype, int64_t ldy,
                            int32_t *d_ids, float *d_probs, void *d_workspace, size_t workspace_bytes, void *cuda_stream)
{
    sqnn::ApiScope scope("sqnn_moe_fp8");
    return scope.finish(sqnn::moe_queue(layer, tokens, d_x, x_dtype, ldx, d_y, y_dtype, ldy, d_ids, d_probs, d_workspace, workspace_bytes,
                                        (cudaStream_t)cuda_stream),
                        nullptr, (cudaStream_t)cuda_stream);
}
