// A mixture-of-experts layer of 8-bit weights for a few tokens, in two kernels.
//
//   logits = x R^T;  the top_k largest (ties to the lowest index), p their softmax
//   y = sum over a token's experts e of p_e D_e (silu(G_e x) * (U_e x)),    silu(a) = a / (1 + exp(-a))
//
// Few tokens reach many experts, so nearly every weight is used for one or two tokens: the layer is bound by reading the chosen experts'
// weights once.  A warp takes 16 rows (or twice 16) by 128 columns at a time: one lane has TMA copy them into the warp's own ring in shared memory,
// several steps ahead; ldmatrix gives every lane four neighbouring bytes of a row, they become fp16 (exact) and are the A operand
// of mma.sync m16n8k16 with up to eight tokens as the columns of B.  (mma.sync, not tcgen05: weights that are used once gain nothing
// from a tile that many warps share, and the rate of mma.sync is several times what memory asks for.  Weights read straight into registers, 62 us
// for one token and 8 of 64 experts of 2048 x 1024: the unrolled code did not fit the instruction cache.  A ring filled by 16-byte copies of
// every lane, 38 us: 230 to 280 instructions per kilobyte or two, most of them addresses.  This form: 26.3 us.)
// The 16 columns of an MMA are dealt so that its k slots 2 t, 2 t + 1, 2 t + 8, 2 t + 9 are columns 4 t .. 4 t + 3, and B is stored
// in the order that gives a lane its share of four MMAs in 32 bytes: position 16 t + 4 j + i of 64 holds column 16 j + 4 t + i.
//
// Activations are scaled by a power of two so that the largest lies between 2^14 and 2^15, and cut into fp16 pieces, which end at 2^-24: bf16 numbers, in one piece,
// are exact down to 2^-31 of the largest, fp32 numbers, in two, are left with 2^-23 of themselves off, or 2^-39 of the largest (as bf16 numbers are below).  (A
// third MMA would bring the last bit; the weights have four.)  x is scaled per token, the inner values, whose largest nobody knows before all are there, per token and
// MMA: a unit of the first kernel is the 16 inner values of one MMA of the second.
// Sums are fp32 in the MMA (cut to it, not rounded), then scaled and added to 32-bit sums.
//
// k_moe_up:   every cluster works out the routing for itself (its CTAs share the experts' logits through distributed shared memory; 18 tokens of 128 experts: a third of
//             the call), then the CTAs share all units (expert, 16 rows of G and the same of U); a CTA's warps share the columns of up to 16 units at a time.
// k_moe_down: a CTA, or a cluster of two or four, has 16 or 32 rows of all chosen experts' D; the warps share (expert, 128 columns) evenly; each sums into its own
//             accumulators, which are added up in warp and rank order.
// No atomics on sums: results are the same from run to run.
#include "sqnn_launch.h"
#include "sqnn_fp8.cuh"
#include "sqnn_cluster.cuh"
#include "sqnn_tc.cuh"

#include <cuda_bf16.h>

#include <atomic>

namespace sqnn {
namespace {

constexpr uint32_t WARPS = 16, THREADS = WARPS * 32;              // first kernel
constexpr uint32_t STREAMS = 8;           // its warps that stream weights
constexpr uint32_t MAX_DOWN_WARPS = 12;   // second kernel: all stream; 8 where there is no room for the sums and rings of 12
constexpr uint32_t CLUSTER = 4;           // CTAs that share the routing's work
constexpr uint32_t STEP = FP8_BLOCK;      // columns per step of a warp
constexpr uint32_t GROUP = 8;             // tokens multiplied together
constexpr uint32_t MAX_TOKENS = SQNN_MOE_MAX_TOKENS, MAX_EXPERTS = SQNN_MOE_MAX_EXPERTS, MAX_TOP_K = SQNN_MOE_MAX_TOP_K;
constexpr uint32_t MAX_PAIRS = MAX_TOKENS * MAX_TOP_K;
constexpr uint32_t MAX_ENTRIES = MAX_EXPERTS + MAX_PAIRS;         // chosen experts, those with many tokens several times
constexpr size_t SMEM_BYTES = 224 * 1024, DOWN_SMEM_BYTES = 216 * 1024;    // (the second kernel has 8 KB of static variables)
constexpr uint32_t UP_DEPTH = 4, UP_SLOT = 2 * 16 * STEP;         // first kernel's ring: 16 rows of G and of U
constexpr uint32_t PARTS_BYTES = STREAMS * 2 * 8 * 32 * 4;        // [warp][its first or second unit][sum][lane]
constexpr uint32_t H_BLOCK = 2 * 2 * STEP + 4 * (STEP / 16);      // inner values of a token, 128 columns: two pieces and eight scales
constexpr uint32_t H_PITCH = H_BLOCK + 16;                        // the same in shared memory: neighbouring tokens in other banks
constexpr uint32_t MAX_DOWN_DEPTH = 8;
constexpr uint64_t WAIT_LIMIT_CYCLES = 4000000000ull;
constexpr uint32_t ALL = 0xffffffffu;
constexpr uint32_t NEAR_ENTRIES = 64;     // entries that the second kernel has in shared memory

// An entry of the list of chosen experts, as the second kernel needs it.
struct Entry {
    uint32_t expert, count;               // count <= GROUP tokens
    uint32_t token[GROUP];
    uint32_t pair[GROUP];                 // rows of h
    float prob[GROUP];
};

struct MoeArgs {
    const void *x, *router;
    const uint8_t *gate_up, *down;
    const float *gate_up_scale, *down_scale;
    void *y;
    uint8_t *h;                   // workspace: a row of blocks per (token, choice)
    Entry *list;                  // workspace
    uint32_t *list_size;
    int32_t *ids_out;
    float *probs_out;
    int64_t ldx, ldr, ldy;
    uint32_t gu_expert, gu_half, d_expert;                        // in rows
    uint32_t tokens, experts, top_k, hidden, inner;
    uint32_t h_row;               // bytes per row of h
    uint32_t renormalize, x_vec, r_vec, y_bf16;
    uint32_t x_row, x_rows;       // first kernel: bytes per staged row of x, how many there is room for
    uint32_t per;                 // tokens per entry in the first kernel
    uint32_t depth, slot;         // second kernel's ring
    uint32_t split;               // its CTAs (a cluster) that share a run of rows
    uint32_t skip_loads;          // test only: no weights are asked for
    uint64_t wait_limit;
    uint32_t *status;
};

// ---- routing tables in shared memory

struct Routing {
    int32_t ids[MAX_PAIRS];
    float probs[MAX_PAIRS];               // before they are divided
    uint32_t mask[MAX_EXPERTS][2];        // tokens of an expert
    uint32_t entry[MAX_ENTRIES];          // expert | group of tokens << 16
    uint32_t totals[WARPS];
    uint32_t entries;
    uint32_t largest[MAX_TOKENS];         // magnitude of a token's largest activation, as bits
    uint32_t spread[MAX_TOKENS];          // the largest sum of magnitudes of products among a token's logits, or more: fp32 as bits
    float total[MAX_TOKENS];              // what its shares are divided by
};
constexpr uint32_t ROUTING_BYTES = (sizeof(Routing) + 127) / 128 * 128;

SQNN_DEV uint32_t tokens_of(const Routing &R, uint32_t expert) { return __popc(R.mask[expert][0]) + __popc(R.mask[expert][1]); }
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

// ---- the multiplication of one chunk

SQNN_DEV uint32_t f16x2(float lo, float hi)
{
    uint32_t v;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(v) : "f"(hi), "f"(lo));
    return v;
}
SQNN_DEV float f16_lo(uint32_t v) { float f; asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.f32.f16 %0, l;\n}\n" : "=f"(f) : "r"(v)); return f; }
SQNN_DEV float f16_hi(uint32_t v) { float f; asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.f32.f16 %0, h;\n}\n" : "=f"(f) : "r"(v)); return f; }
SQNN_DEV void mma_f16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)     // c = a b
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
SQNN_DEV void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The power of two that brings a magnitude of this biased exponent below 2^15, and its inverse.  (255, infinities and NaN: finite numbers stay finite
// beside them.)
SQNN_DEV uint32_t exponent_of(uint32_t magnitude) { return max(magnitude >> 23, 15u); }
SQNN_DEV float scale_of(uint32_t e) { return __uint_as_float((268u - e) << 23); }       // 2^(14 - (e - 127))
SQNN_DEV float back_of(uint32_t e) { return __uint_as_float((e - 14u) << 23); }

SQNN_DEV void bulk_load(uint32_t sdst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n"
                 :: "r"(sdst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
SQNN_DEV uint4 shared16(uint32_t sa)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(sa) : "memory");
    return v;
}
SQNN_DEV float shared4(uint32_t sa)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v) : "r"(sa) : "memory");
    return v;
}
// Four 8 x 16-byte matrices: lane 8 i + r gives the address of row r of matrix i and gets bytes 4 (lane % 4) .. + 3 of row lane / 4 of each.
SQNN_DEV uint4 matrices(uint32_t sa)
{
    uint4 v;
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(sa) : "memory");
    return v;
}
// Where a lane's row for matrices() lies in a tile of 16 rows by 128 bytes with the 128-byte swizzle (on a 1024-byte boundary): matrices of rows 0 - 7 and 8 - 15
// of 16 columns, then of the next 16; `^ (p << 5)` for columns 32 p on.
SQNN_DEV uint32_t matrix_row(uint32_t lane) { return ((lane & 7) + (lane & 8)) * STEP + (((lane >> 4) ^ (lane & 7)) << 4); }
// A operand of an MMA from a lane's four bytes of row g and of row g + 8.
SQNN_DEV void weights_of(uint32_t (&a)[4], uint32_t top, uint32_t bottom)
{
    asm("{\n .reg .b16 tl, th, bl, bh;\n mov.b32 {tl, th}, %4;\n mov.b32 {bl, bh}, %5;\n cvt.rn.f16x2.e4m3x2 %0, tl;\n cvt.rn.f16x2.e4m3x2 %1, bl;\n"
        " cvt.rn.f16x2.e4m3x2 %2, th;\n cvt.rn.f16x2.e4m3x2 %3, bh;\n}\n" : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(top), "r"(bottom));
}

// ---- routing

// Logits of this CTA's experts (every CLUSTER-th), as keys, and how far off they may be, into the shared memory of all CTAs of the cluster, and the tokens'
// largest activations.  Waits for the cluster before it writes to others.
//
// Which experts a token goes to must not hang on the order of a sum.  Few logits are near one another, so all are summed in fp32 over a few products at a time (and
// these sums in 64 bits), beside them the magnitudes of the products, and choose() computes those once more in 64 bits that lie within the error of a chosen
// one.  (All products in 64 bits: 16 000 cycles of an SM's 64-bit units for 16 tokens and 64 experts of 4096 columns, where this takes 11 600.)  With A the sum of
// magnitudes:
//   - bf16: an MMA adds 16 exact products, each cut off below 2^-25 of the largest (as measured), and cuts the sum to 24 bits: at most 5 2^-23 of their magnitudes.  Two
//     additions of such sums, 2^-24 each, make one of 64 columns: 6 2^-23 A.  A itself comes from such MMAs, at most 2^-11 A too small.
//   - fp32: eight fused multiply-adds, 2^-24 each: 8 2^-24 A; A at most 2^-17 A too small.
//   - what lies below 2^-126 may be lost: 2^-125 for each column.  Where a sum passes fp32's range nothing is known.
// `scratch`: 24 KB.
template <typename XT> constexpr float SLACK = sizeof(XT) == 2 ? 0x1.81p-21f : 0x1.01p-21f;
constexpr uint32_t INFINITE = 0x7f800000u, UNKNOWN = 0x7f000000u;         // (2^127: a logit that has passed the range has an A above that)
constexpr uint32_t ORDINARY = 67u << 23;                         // 2^-60
// 64-bit floating numbers as integers of the same order; NaN comes last.  And back.
SQNN_DEV int64_t key_of(double v)
{
    if (v != v) return 0x7fffffffffffffffll;
    const int64_t b = __double_as_longlong(v == 0.0 ? 0.0 : v);
    return b ^ ((b >> 63) & 0x7fffffffffffffffll);
}
SQNN_DEV double value_of(int64_t k) { return __longlong_as_double(k ^ ((k >> 63) & 0x7fffffffffffffffll)); }
SQNN_DEV void send_logit(int64_t *keys, uint32_t experts, uint32_t token, uint32_t expert, double v)
{
    const uint32_t at = smem_addr(keys + token * experts + expert);
    const int64_t key = key_of(v);
#pragma unroll
    for (uint32_t r = 0; r < CLUSTER; ++r) peer_store(peer_addr(at, r), key);
}
SQNN_DEV void send_spread(Routing &R, uint32_t token, uint32_t bits)     // (NaN is larger than infinity)
{
    const uint32_t at = smem_addr(R.spread + token);
#pragma unroll
    for (uint32_t r = 0; r < CLUSTER; ++r) peer_max(peer_addr(at, r), bits);
}
SQNN_DEV void mma_bf16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)     // c = a b
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
SQNN_DEV void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bf16 numbers of a row from `at` on, zero from `n` on.  (What is seldom run is kept out of line, here and below: the kernels run once
// through most of their code, and fetching instructions is what that costs.)
static __device__ __noinline__ uint4 ragged8(const __nv_bfloat16 *row, uint32_t at, uint32_t n)
{
    const uint16_t *const p = reinterpret_cast<const uint16_t *>(row);
    uint32_t v[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
        v[j] = (at + 2 * j < n ? p[at + 2 * j] : 0u) | (at + 2 * j + 1 < n ? (uint32_t)p[at + 2 * j + 1] << 16 : 0u);
    return make_uint4(v[0], v[1], v[2], v[3]);
}
static __device__ __noinline__ float4 ragged4(const float *row, uint32_t at, uint32_t n)
{
    return make_float4(at < n ? row[at] : 0.0f, at + 1 < n ? row[at + 1] : 0.0f, at + 2 < n ? row[at + 2] : 0.0f, at + 3 < n ? row[at + 3] : 0.0f);
}
SQNN_DEV void load16(const __nv_bfloat16 *p, uint32_t (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p), b = *reinterpret_cast<const uint4 *>(p + 8);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
SQNN_DEV void ragged16(const __nv_bfloat16 *row, uint32_t at, uint32_t n, uint32_t (&v)[8])
{
    const uint4 a = ragged8(row, at, n), b = ragged8(row, at + 8, n);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
SQNN_DEV void load8(const float *p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
SQNN_DEV void unpack8(const uint4 &f, float (&v)[8])
{
    const uint32_t u[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
SQNN_DEV void load8(const __nv_bfloat16 *p, float (&v)[8]) { unpack8(*reinterpret_cast<const uint4 *>(p), v); }
SQNN_DEV void row_values8(const float *row, uint32_t at, uint32_t n, bool vec, float (&v)[8])
{
    if (vec && at + 8 <= n) {
        load8(row + at, v);
    } else {
        float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f), b = a;
        if (at < n) {
            a = ragged4(row, at, n);
            b = ragged4(row, at + 4, n);
        }
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
SQNN_DEV void row_values8(const __nv_bfloat16 *row, uint32_t at, uint32_t n, bool vec, float (&v)[8])
{
    unpack8(vec && at + 8 <= n ? *reinterpret_cast<const uint4 *>(row + at) : at < n ? ragged8(row, at, n) : make_uint4(0, 0, 0, 0), v);
}

// bf16: on the tensor cores, 16 experts by 8 tokens by 64 columns (four MMAs of their own, products exact) at a time.  The columns of a tile are shared by as
// many warps as there are to spare.
SQNN_DEV void logits_of_cluster(const MoeArgs &M, int64_t *keys, double *scratch, Routing &R, const __nv_bfloat16 *x, const __nv_bfloat16 *router)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3, rank = cluster_rank();
    // (a CTA without experts still looks at the tokens)
    const uint32_t mine = (M.experts - rank + CLUSTER - 1) / CLUSTER, n_tiles = (M.tokens + 7) / 8, tiles = (max(mine, 1u) + 15) / 16 * n_tiles;
    const uint32_t parts = tiles < WARPS ? WARPS / tiles : 1, steps = (M.hidden + 63) / 64;
    float *const totals = reinterpret_cast<float *>(scratch + WARPS * 128);
    const bool vec = M.x_vec && M.r_vec;
    if (parts == 1) cluster_wait();
#pragma unroll 1
    for (uint32_t i = warp; i < tiles * parts; i += WARPS) {
        const uint32_t tile = i / parts, part = i - tile * parts, e0 = tile / n_tiles * 16, t0 = tile % n_tiles * 8;
        const __nv_bfloat16 *const ra = router + (int64_t)min(rank + CLUSTER * (e0 + g), M.experts - 1) * M.ldr;
        const __nv_bfloat16 *const rb = router + (int64_t)min(rank + CLUSTER * (e0 + g + 8), M.experts - 1) * M.ldr;
        const __nv_bfloat16 *const xr = x + (int64_t)min(t0 + g, M.tokens - 1) * M.ldx;
        double sum[4] = {};
        float total[4] = {};                                     // of magnitudes
        uint32_t top = 0, na[8], nb[8], nv[8];
        auto ask = [&](uint32_t c) {                             // (one test for all, so that all are under way together)
            const uint32_t at = c * 64 + t4 * 16;
            if (vec && at + 16 <= M.hidden) {
                load16(ra + at, na);
                load16(rb + at, nb);
                load16(xr + at, nv);
            } else {
                ragged16(ra, at, M.hidden, na);
                ragged16(rb, at, M.hidden, nb);
                ragged16(xr, at, M.hidden, nv);
            }
        };
        const uint32_t c0 = steps * part / parts, c1 = steps * (part + 1) / parts;
        ask(c0);                                                 // (more parts than steps: columns of another's, or zeros, that nobody looks at)
#pragma unroll 1
        for (uint32_t c = c0; c < c1; ++c) {
            uint32_t a[8], b[8], v[8];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) { a[j] = na[j]; b[j] = nb[j]; v[j] = nv[j]; }
            if (c + 1 < c1) ask(c + 1);
            float s[4][4];
            constexpr uint32_t MAGNITUDE = 0x7fff7fffu;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint32_t x0 = v[2 * j] & MAGNITUDE, x1 = v[2 * j + 1] & MAGNITUDE;
                mma_bf16_first(s[j], a[2 * j], b[2 * j], a[2 * j + 1], b[2 * j + 1], v[2 * j], v[2 * j + 1]);
                mma_bf16(total, a[2 * j] & MAGNITUDE, b[2 * j] & MAGNITUDE, a[2 * j + 1] & MAGNITUDE, b[2 * j + 1] & MAGNITUDE, x0, x1);
                top = __vmaxu2(top, __vmaxu2(x0, x1));
            }
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) sum[j] += (double)((s[0][j] + s[1][j]) + (s[2][j] + s[3][j]));
        }
        if (e0 == 0) {
            top = max(top & 0xffffu, top >> 16) << 16;
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            if (t4 == 0 && t0 + g < M.tokens) atomicMax(&R.largest[t0 + g], top);
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t e = e0 + g + (j >> 1) * 8, t = t0 + 2 * t4 + (j & 1);
            if (parts > 1) scratch[i * 128 + j * 32 + lane] = sum[j];
            else if (e < mine && t < M.tokens) send_logit(keys, M.experts, t, rank + CLUSTER * e, sum[j]);
        }
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {                       // the largest of 16 experts
            uint32_t most = max(__float_as_uint(total[k]), __float_as_uint(total[2 + k]));      // (experts past the last repeat it)
#pragma unroll
            for (uint32_t d = 4; d < 32; d <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
            const uint32_t t = 2 * t4 + k;
            if (g == 0 && parts > 1) totals[i * 8 + t] = __uint_as_float(most);
            else if (g == 0 && t0 + t < M.tokens) send_spread(R, t0 + t, most);
        }
    }
    if (parts == 1) return;
    __syncthreads();
    cluster_wait();                                              // all CTAs of the cluster run: their shared memory may be written
#pragma unroll 1
    for (uint32_t i4 = tid; i4 < tiles * 512; i4 += THREADS) {    // four threads per sum
        const uint32_t i = i4 / 4, tile = i / 128, j = i / 32 & 3, l = i & 31, e = tile / n_tiles * 16 + (l >> 2) + (j >> 1) * 8, t = tile % n_tiles * 8 + 2 * (l & 3) + (j & 1);
        double sum = 0.0;
        for (uint32_t p = i4 & 3; p < parts; p += 4) sum += scratch[(tile * parts + p) * 128 + (i & 127)];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if ((i4 & 3) == 0 && e < mine && t < M.tokens) send_logit(keys, M.experts, t, rank + CLUSTER * e, sum);
    }
    const uint32_t item = tid / 4 - THREADS / 8;                 // a token's parts in a tile, by the largest expert of each; four threads
    if (item < tiles * 8) {
        const uint32_t tile = item / 8, t = tile % n_tiles * 8 + item % 8;
        float total = 0.0f;
        for (uint32_t p = tid & 3; p < parts; p += 4) total += totals[(tile * parts + p) * 8 + item % 8];
        total += __shfl_xor_sync(0xffffffffu, total, 1);
        total += __shfl_xor_sync(0xffffffffu, total, 2);
        if ((tid & 3) == 0 && t < M.tokens) send_spread(R, t, __float_as_uint(total));
    }
}

// fp32: a warp has OWN experts, four tokens and a share of the columns; eight products at a time.  OWN is four where there are enough of them: each row of x
// and of the router comes from L2 (the SM's memory is all taken; 18 tokens, 7 of 128 experts, 1200 x 128: 97 us for the call with one, 64 with four).  Functions of their
// own, so that the registers they need are not missing elsewhere.
template <uint32_t OWN, bool VEC>
static __device__ __noinline__ void logits_by(uint32_t tokens, uint32_t experts, uint32_t hidden, const float *x, int64_t ldx, const float *router, int64_t ldr, int64_t *keys,
                                              double *scratch, Routing &R)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank();
    constexpr uint32_t SHARE = 4, SUMS = OWN * SHARE;            // SHARE: tokens that share a read of an expert's row
    const uint32_t mine = (experts - rank + CLUSTER - 1) / CLUSTER, groups = (tokens + SHARE - 1) / SHARE, tasks = (max(mine, 1u) + OWN - 1) / OWN * groups;
    const uint32_t parts = tasks < WARPS ? WARPS / tasks : 1, steps = (hidden + 255) / 256;
    // this lane's eight of 256 columns: neighbours, or (rows off 16-byte boundaries) every 32nd
    auto values = [&](const float *row, uint32_t c, float (&v)[8]) {
        if constexpr (VEC) {
            row_values8(row, c * 256 + lane * 8, hidden, true, v);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                const uint32_t at = c * 256 + j * 32 + lane;
                v[j] = at < hidden ? row[at] : 0.0f;
            }
        }
    };
    const auto expert_row = [&](uint32_t e) { return router + (int64_t)min(rank + CLUSTER * e, experts - 1) * ldr; };
    const auto token_row = [&](uint32_t t) { return x + (int64_t)min(t, tokens - 1) * ldx; };
    constexpr bool AT_ONCE = OWN == 1 && VEC;                    // the rows of x too (where registers allow)
    float *const totals = reinterpret_cast<float *>(scratch + WARPS * SUMS);
    if (parts == 1) cluster_wait();
#pragma unroll 1
    for (uint32_t i = warp; i < tasks * parts; i += WARPS) {
        const uint32_t task = i / parts, part = i - task * parts, own = task / groups * OWN, t0 = task % groups * SHARE;
        double sum[SUMS] = {};
        float total[SHARE] = {};                                 // of magnitudes, or more: the largest of eight of x times the largest expert's eight of the router
        uint32_t top[SHARE] = {};
#pragma unroll (OWN == 1 && !VEC ? 2 : 1)
        for (uint32_t c = steps * part / parts; c < steps * (part + 1) / parts; ++c) {
            float r[OWN][8], rows[AT_ONCE ? SHARE : 1][8];
            if (VEC && c * 256 + lane * 8 + 8 <= hidden) {       // (one test for all, so that all are under way together)
#pragma unroll
                for (uint32_t o = 0; o < OWN; ++o) load8(expert_row(own + o) + c * 256 + lane * 8, r[o]);
#pragma unroll
                for (uint32_t t = 0; AT_ONCE && t < SHARE; ++t) load8(token_row(t0 + t) + c * 256 + lane * 8, rows[t]);
            } else {
#pragma unroll
                for (uint32_t o = 0; o < OWN; ++o) values(expert_row(own + o), c, r[o]);
#pragma unroll
                for (uint32_t t = 0; AT_ONCE && t < SHARE; ++t) values(token_row(t0 + t), c, rows[t]);
            }
            float eight = 0.0f;
#pragma unroll
            for (uint32_t o = 0; o < OWN; ++o) {
                float s = 0.0f;
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) s += fabsf(r[o][j]);
                eight = fmaxf(eight, s);                         // (NaN is seen in its logit)
            }
#pragma unroll
            for (uint32_t t = 0; t < SHARE; ++t) {
                float v[8];
                if constexpr (AT_ONCE) {
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) v[j] = rows[t][j];
                } else {
                    values(token_row(t0 + t), c, v);
                }
                uint32_t most = 0;
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
                top[t] = max(top[t], most);
                total[t] = fmaf(eight, __uint_as_float(most), total[t]);
#pragma unroll
                for (uint32_t o = 0; o < OWN; ++o) {
                    float s = 0.0f;
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) s = fmaf(r[o][j], v[j], s);
                    sum[o * SHARE + t] += (double)s;
                }
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < SUMS; ++k)
#pragma unroll
            for (uint32_t d = 16; d; d >>= 1) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], d);
#pragma unroll
        for (uint32_t t = 0; t < SHARE; ++t) {
            const uint32_t most = __reduce_max_sync(0xffffffffu, top[t]);
#pragma unroll
            for (uint32_t d = 16; d; d >>= 1) total[t] += __shfl_xor_sync(0xffffffffu, total[t], d);
            if (lane == 0 && t0 + t < tokens) {
                if (own == 0) atomicMax(&R.largest[t0 + t], most);
                if (parts > 1) totals[i * SHARE + t] = total[t];
                else send_spread(R, t0 + t, __float_as_uint(total[t]));
#pragma unroll
                for (uint32_t o = 0; o < OWN; ++o) {
                    if (parts > 1) scratch[i * SUMS + o * SHARE + t] = sum[o * SHARE + t];
                    else if (own + o < mine) send_logit(keys, experts, t0 + t, rank + CLUSTER * (own + o), sum[o * SHARE + t]);
                }
            }
        }
    }
    if (parts == 1) return;
    __syncthreads();
    cluster_wait();
    if (tid < tasks * SUMS) {
        const uint32_t task = tid / SUMS, k = tid % SUMS, t = task % groups * SHARE + k % SHARE, e = task / groups * OWN + k / SHARE;
        if (t < tokens && e < mine) {
            double sum = 0.0;
            float total = 0.0f;
            for (uint32_t p = 0; p < parts; ++p) {
                sum += scratch[(task * parts + p) * SUMS + k];
                total += totals[(task * parts + p) * SHARE + k % SHARE];
            }
            send_logit(keys, experts, t, rank + CLUSTER * e, sum);
            if (k < SHARE) send_spread(R, t, __float_as_uint(total));
        }
    }
}
SQNN_DEV void logits_of_cluster(const MoeArgs &M, int64_t *keys, double *scratch, Routing &R, const float *x, const float *router)
{
    const bool few = (M.experts + CLUSTER - 1) / CLUSTER * ((M.tokens + 3) / 4) <= 2 * WARPS;
    if (M.x_vec && M.r_vec) {
        if (few) logits_by<1, true>(M.tokens, M.experts, M.hidden, x, M.ldx, router, M.ldr, keys, scratch, R);
        else logits_by<4, true>(M.tokens, M.experts, M.hidden, x, M.ldx, router, M.ldr, keys, scratch, R);
    } else {
        if (few) logits_by<1, false>(M.tokens, M.experts, M.hidden, x, M.ldx, router, M.ldr, keys, scratch, R);
        else logits_by<4, false>(M.tokens, M.experts, M.hidden, x, M.ldx, router, M.ldr, keys, scratch, R);
    }
}

// A token's logits that lie within `slack` of another one among the top_k, once more in 64 bits.  (The last of these counts as near itself: what is near a chosen one
// from below is near the last, and so is that chosen one.)  All lanes of a warp.
template <typename XT>
static __device__ __noinline__ void settle_logits(const XT *x, const XT *router, int64_t ldr, uint32_t hidden, uint32_t experts, uint32_t top_k, bool vec,
                                                  int64_t *row, const int64_t *best, const int32_t *ids, double slack)
{
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll 1
    for (uint32_t e0 = 0; e0 < experts; e0 += 32) {
        const uint32_t e = e0 + lane;
        bool near = false;
        if (e < experts) {
            const double v = value_of(row[e]);
#pragma unroll 1
            for (uint32_t s = 0; s < top_k; ++s) near |= (ids[s] != (int32_t)e || s + 1 == top_k) && !(fabs(v - value_of(best[s])) > slack);
        }
#pragma unroll 1
        for (uint32_t left = __ballot_sync(0xffffffffu, near); left; left &= left - 1) {
            const uint32_t n = e0 + (uint32_t)__ffs((int)left) - 1;
            const XT *const r = router + (int64_t)n * ldr;
            double sum = 0.0;
            if (vec) {
#pragma unroll 4
                for (uint32_t at = lane * 8; at + 8 <= hidden; at += 256) {
                    float a[8], b[8];
                    load8(x + at, a);
                    load8(r + at, b);
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) sum = fma((double)a[j], (double)b[j], sum);
                }
            }
#pragma unroll 4
            for (uint32_t at = (vec ? hidden & ~7u : 0u) + lane; at < hidden; at += 32) sum = fma((double)(float)x[at], (double)(float)r[at], sum);
#pragma unroll
            for (uint32_t d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (lane == 0) row[n] = key_of(sum);
        }
        __syncwarp();
    }
}

// From logits to the top_k experts of each token, their shares, and the list of (expert, group of up to `per` of its tokens), ascending.  NaN counts as the
// largest, so that there are always top_k different experts.  All threads; masks are zero before, ends with a barrier.  `chosen`: 8 KB.
template <typename XT>
SQNN_DEV void choose(const MoeArgs &M, int64_t *keys, int64_t *chosen, Routing &R)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // a warp per token: the largest key top_k times, by the upper half, the lower half, the index; the lane that has it notes it down
    for (uint32_t t = warp; t < M.tokens; t += WARPS) {
        int2 *const row = reinterpret_cast<int2 *>(keys + t * M.experts);
        int64_t *const best = chosen + t * M.top_k;
        int32_t *const ids = R.ids + t * M.top_k;
        constexpr int32_t TAKEN = -0x7fffffff - 1;               // below all keys
        constexpr int64_t LOWEST = -0x7fffffffffffffffll - 1;    // such a key
#pragma unroll 1
        for (bool settled = false;; settled = true) {
#pragma unroll 1
            for (uint32_t s = 0; s < M.top_k; ++s) {
                int2 top = make_int2(0, TAKEN);
                uint32_t at = MAX_EXPERTS;
                for (uint32_t e = lane; e < M.experts; e += 32) {
                    const int2 k = row[e];
                    if (k.y > top.y || (k.y == top.y && (uint32_t)k.x > (uint32_t)top.x)) { top = k; at = e; }
                }
                const int32_t upper = __reduce_max_sync(0xffffffffu, top.y);
                bool mine = top.y == upper;
                const uint32_t who = __ballot_sync(0xffffffffu, mine);
                if (who & (who - 1)) {
                    const uint32_t lower = __reduce_max_sync(0xffffffffu, mine ? (uint32_t)top.x : 0u);
                    mine = mine && (uint32_t)top.x == lower;
                    const uint32_t lowest = __reduce_min_sync(0xffffffffu, mine ? at : MAX_EXPERTS);     // (by all lanes)
                    mine = mine && at == lowest;
                }
                if (mine) {
                    *reinterpret_cast<int2 *>(best + s) = top;
                    ids[s] = (int32_t)at;
                    row[at] = make_int2(0, TAKEN);
                }
            }
            __syncwarp();
            // Equal or nearly equal ones among these?  (Logits of zeros are zero, those of a router that leaves nothing of a token count as zero; of infinities and
            // NaN nothing better is to be had.)
            const uint32_t largest = R.largest[t], spread = R.spread[t];
            if (settled || largest == 0 || largest >= INFINITE || (spread == 0 && largest >= ORDINARY)) break;
            const float slack = __uint_as_float(spread < UNKNOWN ? spread : INFINITE) * (2 * SLACK<XT>) + 0x1p-124f * (float)M.hidden;
            int64_t left = LOWEST;                                    // the largest that is left, lane by lane
            for (uint32_t e = lane; e < M.experts; e += 32) left = max(left, keys[t * M.experts + e]);
            const double last = value_of(best[M.top_k - 1]);
            bool near = left != LOWEST && !(last - value_of(left) > slack);
            if (lane + 1 < M.top_k) near |= !(value_of(best[lane]) - value_of(best[lane + 1]) > slack);
            if (!__any_sync(0xffffffffu, near)) break;
            if (lane < M.top_k) (keys + t * M.experts)[ids[lane]] = best[lane];
            __syncwarp();
            settle_logits<XT>(static_cast<const XT *>(M.x) + (int64_t)t * M.ldx, static_cast<const XT *>(M.router), M.ldr, M.hidden, M.experts, M.top_k, M.x_vec && M.r_vec,
                              keys + t * M.experts, best, ids, slack);
        }
        const double first = value_of(best[0]);
        float sum = 0.0f;
        if (lane < M.top_k) {
            sum = expf((float)(value_of(best[lane]) - first));
            R.probs[t * M.top_k + lane] = sum;
            atomicOr(&R.mask[ids[lane]][t >> 5], 1u << (t & 31));
        }
        if (!M.renormalize)
            for (uint32_t e = lane; e < M.experts; e += 32)
                if (row[e].y != TAKEN) sum += expf((float)(value_of(keys[t * M.experts + e]) - first));
#pragma unroll
        for (uint32_t d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) R.total[t] = sum;
    }
    fence_async_smem();                                          // the rings' copies come after all that was written where they go, here last
    __syncthreads();
    static_assert(MAX_EXPERTS <= THREADS, "an expert per thread");
    const uint32_t groups = tid < M.experts ? (tokens_of(R, tid) + M.per - 1) / M.per : 0;
    uint32_t upto = groups;
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += v;
    }
    if (lane == 31) R.totals[warp] = upto;
    __syncthreads();
    uint32_t before = 0, count = 0;
#pragma unroll
    for (uint32_t w = 0; w < WARPS; ++w) {
        if (w < warp) before += R.totals[w];
        count += R.totals[w];
    }
    for (uint32_t g = 0; g < groups; ++g) R.entry[before + upto - groups + g] = tid | (g << 16);
    if (tid == 0) R.entries = count;
    __syncthreads();
}

// ---- first kernel: routing, then h = silu(G x) * (U x) for every (token, expert)

// A warp's waits: bounded; once one has given up, its block asks for and waits for nothing any more, and stores nothing.
struct Waits {
    volatile uint32_t *abort_flag;
    uint32_t *status;
    uint64_t limit;
    SQNN_DEV void wait(uint32_t bar, uint32_t parity) const
    {
        mbar_wait_warp(bar, parity, abort_flag, status, limit);  // (returns at once after a wait that gave up)
        __syncwarp();
    }
};

// The units of all entries form one line, cut into equal runs, one per CTA.  A run is gone through in windows, as many whole entries as
// there is room for their tokens in shared memory, and a window in rounds of up to STREAMS units, whose columns the warps share evenly.
struct Walk {
    uint32_t u, c, left;          // unit, step, and steps to go in this round
    uint32_t round0, round_n;     // the round's units
    uint32_t window0, window1;    // the window's units
};

// EARLY: there is room for all tokens of the call, so they are staged once, a row each, and there are no windows.
template <typename XT, bool EARLY>
__global__ void __launch_bounds__(THREADS, 1) k_moe_up(const __grid_constant__ CUtensorMap weights, const MoeArgs M)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    constexpr uint32_t PIECES = sizeof(XT) == 2 ? 1 : 2;
    __shared__ uint64_t bars[STREAMS * UP_DEPTH];
    __shared__ uint32_t abort_word;
    // [rings][routing][partial sums of two rounds][rows of x]; the keys of the logits, [tokens][experts], lie where the rings are later
    const uint32_t skew = (1024u - (smem_addr(smem_raw) & 1023u)) & 1023u;
    uint8_t *const smem = smem_raw + skew;
    static_assert(WARPS == 2 * STREAMS, "half of the warps stream, half join");
    static_assert(SQNN_MOE_MAX_LOGITS * sizeof(int64_t) <= STREAMS * UP_DEPTH * UP_SLOT, "room for the logits");
    Routing &R = *reinterpret_cast<Routing *>(smem + STREAMS * UP_DEPTH * UP_SLOT);
    int64_t *const keys = reinterpret_cast<int64_t *>(smem);
    float *const parts = reinterpret_cast<float *>(smem + STREAMS * UP_DEPTH * UP_SLOT + ROUTING_BYTES);
    uint8_t *const x_rows = reinterpret_cast<uint8_t *>(parts) + 2 * PARTS_BYTES;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const Waits W{&abort_word, M.status, M.wait_limit};
    if (tid < STREAMS * UP_DEPTH) mbar_init(smem_addr(bars + tid), 1);
    if (tid == 0) abort_word = 0;
    if (tid < MAX_TOKENS) R.largest[tid] = R.spread[tid] = 0;
    for (uint32_t i = tid; i < 2 * M.experts; i += THREADS) (&R.mask[0][0])[i] = 0;
    if (tid == 0) asm volatile("prefetch.tensormap [%0];\n" :: "l"(&weights) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    __syncthreads();                                             // the zeros are there before any warp adds a maximum
    wait_prior_grid();
    launch_dependents();
    cluster_arrive();
    logits_of_cluster(M, keys, reinterpret_cast<double *>(parts), R, static_cast<const XT *>(M.x), static_cast<const XT *>(M.router));
    cluster_sync();                                              // (the last time that one CTA writes to another)
    // Tokens, scaled and in fp16, to rows `base` and on: an expert's, from the first-th on, or all.
    const uint32_t steps = (M.hidden + STEP - 1) / STEP, lo_at = steps * STEP * 2;
    auto stage = [&](uint32_t base, uint32_t count, uint32_t expert, uint32_t first) {
        const uint32_t cols8 = steps * (STEP / 8);
#pragma unroll 2
        for (uint32_t i = tid; i < count * cols8; i += THREADS) {
            const uint32_t k = i / cols8, at = (i - k * cols8) * 8, t = expert == ALL ? k : token_of(R, expert, first + k);
            const float s = scale_of(exponent_of(R.largest[t]));
            float v[8];
            row_values8(static_cast<const XT *>(M.x) + (int64_t)t * M.ldx, at, M.hidden, M.x_vec, v);
            uint32_t hi[4], lo[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const float a = v[2 * j] * s, b = v[2 * j + 1] * s;
                hi[j] = f16x2(a, b);
                lo[j] = f16x2(a - f16_lo(hi[j]), b - f16_hi(hi[j]));
            }
            // columns 16 j + 4 t and on, t even: four at position 16 t + 4 j, the next four at 16 (t + 1) + 4 j
            uint8_t *const p = x_rows + (base + k) * M.x_row + (at & ~63u) * 2 + (at & 12u) * 8 + (at >> 4 & 3u) * 8;
            *reinterpret_cast<uint2 *>(p) = make_uint2(hi[0], hi[1]);
            *reinterpret_cast<uint2 *>(p + 32) = make_uint2(hi[2], hi[3]);
            if constexpr (PIECES == 2) {
                *reinterpret_cast<uint2 *>(p + lo_at) = make_uint2(lo[0], lo[1]);
                *reinterpret_cast<uint2 *>(p + lo_at + 32) = make_uint2(lo[2], lo[3]);
            }
        }
    };
    if constexpr (EARLY) stage(0, M.tokens, ALL, 0);
    choose<XT>(M, keys, reinterpret_cast<int64_t *>(parts), R);
    if (blockIdx.x == 0) {                                       // for the caller and for the second kernel
        for (uint32_t i = tid; i < M.tokens * M.top_k; i += THREADS) {
            if (M.ids_out) M.ids_out[i] = R.ids[i];
            if (M.probs_out) M.probs_out[i] = R.probs[i] / R.total[i / M.top_k];
        }
        for (uint32_t i = tid; i < R.entries * GROUP; i += THREADS) {
            const uint32_t n = i / GROUP, k = i % GROUP, en = R.entry[n], e = en & 0xffffu, first = (en >> 16) * M.per, count = min(M.per, tokens_of(R, e) - first);
            Entry &E = M.list[n];
            if (k == 0) { E.expert = e; E.count = count; }
            if (k < count) {
                const uint32_t t = token_of(R, e, first + k), pair = pair_of(R, M, t, e);
                E.token[k] = t;
                E.pair[k] = pair;
                E.prob[k] = R.probs[pair] / R.total[t];
            }
        }
        if (tid == 0) *M.list_size = R.entries;
    }

    const uint32_t per_entry = (M.inner + 15) / 16, units = R.entries * per_entry;     // (below 2^21)
    const uint32_t u0 = units * blockIdx.x / gridDim.x, u1 = units * (blockIdx.x + 1) / gridDim.x;
    const uint32_t iblocks = (M.inner + FP8_BLOCK - 1) / FP8_BLOCK;
    auto tokens_in = [&](uint32_t n) {                           // of entry n
        const uint32_t en = R.entry[n];
        return min(M.per, tokens_of(R, en & 0xffffu) - (en >> 16) * M.per);
    };
    auto enter = [&](Walk &w, uint32_t round0) {
        w.round0 = round0;
        w.left = 0;
        if (round0 >= u1) return;
        if (EARLY) {
            w.window0 = u0;
            w.window1 = u1;
        } else if (round0 >= w.window1) {
            uint32_t n = round0 / per_entry, rows = 0;
            while (n < R.entries && n * per_entry < u1 && rows + tokens_in(n) <= M.x_rows) rows += tokens_in(n++);
            w.window0 = round0;
            w.window1 = min(u1, n * per_entry);
        }
        w.round_n = min(STREAMS, w.window1 - round0);
        if (warp >= STREAMS) return;
        const uint32_t total = w.round_n * steps, a = total * warp / STREAMS, b = total * (warp + 1) / STREAMS, d = a / steps;
        w.u = round0 + d;
        w.c = a - d * steps;
        w.left = b - a;
    };

    // ---- the weights of the step `ahead` stands at, into the ring
    const uint32_t ring = smem_addr(smem) + warp * UP_DEPTH * UP_SLOT, my_bars = smem_addr(bars) + 8 * warp * UP_DEPTH;
    Walk ahead;
    ahead.window1 = ahead.round_n = 0;
    uint32_t weight_row = 0, put_slot = 0, issued = 0;
    const uint64_t once = policy_once();
    auto open_unit = [&]() {
        const uint32_t n = ahead.u / per_entry;
        weight_row = (R.entry[n] & 0xffffu) * M.gu_expert + (ahead.u - n * per_entry) * 16;
    };
    auto next_round = [&]() {                                    // to this warp's first step of the next round that has one
#pragma unroll 1
        do enter(ahead, ahead.round0 + ahead.round_n);
        while (ahead.left == 0 && ahead.round0 < u1);
        if (ahead.round0 < u1) open_unit();
    };
    auto request = [&]() {
        if (ahead.round0 < u1) {
            if (lane == 0 && !M.skip_loads && !*W.abort_flag) {
                const uint32_t bar = my_bars + 8 * put_slot, sa = ring + put_slot * UP_SLOT;
                mbar_expect_tx(bar, UP_SLOT);
                tma_load_2d_once(sa, &weights, bar, (int32_t)(ahead.c * STEP), (int32_t)weight_row, once);
                tma_load_2d_once(sa + UP_SLOT / 2, &weights, bar, (int32_t)(ahead.c * STEP), (int32_t)(weight_row + M.gu_half), once);
                ++issued;
            }
            const bool over = ++ahead.c == steps;
            if (over) { ahead.c = 0; ++ahead.u; }
            if (--ahead.left == 0) next_round();
            else if (over) open_unit();
            put_slot = put_slot + 1 == UP_DEPTH ? 0 : put_slot + 1;
        }
    };
    if (warp < STREAMS) {
        ahead.round0 = u0;
        next_round();
#pragma unroll 1
        for (uint32_t j = 0; j + 1 < UP_DEPTH; ++j) request();
    }

    // A unit of a round that is over, by a warp of the second half: its parts in warp order, the gate, and out to h.  These warps work a round behind
    // the others, which have gone on.
    auto join = [&](uint32_t round0, uint32_t round_n, const float *from) {
        const uint32_t k0 = warp - STREAMS;
        if (__any_sync(0xffffffffu, k0 >= round_n || *W.abort_flag)) return;     // (all lanes or none)
        const uint32_t unit = round0 + k0, total = round_n * steps;
        float sum[8] = {};
        for (uint32_t q = 0; q < STREAMS; ++q) {
            const uint32_t a = total * q / STREAMS, b = total * (q + 1) / STREAMS;
            if (a >= b || b <= k0 * steps || a >= (k0 + 1) * steps) continue;
            const float *const p = from + ((q * 2 + (k0 - a / steps)) * 8) * 32 + lane;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) sum[j] += p[j * 32];
        }
        const uint32_t n = unit / per_entry, en = R.entry[n], e = en & 0xffffu, q = unit - n * per_entry, count = tokens_in(n);
        const uint32_t i = q * 16 + g;                       // rows i and i + 8
        // where a row's value goes: 16 (row / 4 % 4) + 4 (q % 4) + row % 4 of its 64
        const uint32_t at = q / (STEP / 16) * H_BLOCK + ((q & 4) * 16 + (g >> 2) * 16 + (q & 3) * 4 + (g & 3)) * 2;
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            const float a = sum[k], b = sum[2 + k];
            const float va = i < M.inner ? a / (1.0f + expf(-a)) * sum[4 + k] : 0.0f;
            const float vb = i + 8 < M.inner ? b / (1.0f + expf(-b)) * sum[6 + k] : 0.0f;
            uint32_t top = max(__float_as_uint(va) & 0x7fffffffu, __float_as_uint(vb) & 0x7fffffffu);
#pragma unroll
            for (uint32_t d = 4; d < 32; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
            const uint32_t ex = exponent_of(top);
            const float s = scale_of(ex);
            // (infinity minus infinity: nothing is left of what has passed fp32's range)
            const uint32_t hi = f16x2(va * s, vb * s), lo = top == 0x7f800000u ? 0u : f16x2(va * s - f16_lo(hi), vb * s - f16_hi(hi));
            const uint32_t column = 2 * t4 + k;
            if (column < count) {
                const uint32_t t = token_of(R, e, (en >> 16) * M.per + column);
                uint8_t *const row = M.h + (uint64_t)pair_of(R, M, t, e) * M.h_row;
                *reinterpret_cast<uint16_t *>(row + at) = (uint16_t)hi;
                *reinterpret_cast<uint16_t *>(row + at + 64) = (uint16_t)(hi >> 16);
                *reinterpret_cast<uint16_t *>(row + at + 256) = (uint16_t)lo;
                *reinterpret_cast<uint16_t *>(row + at + 320) = (uint16_t)(lo >> 16);
                if (g == 0) *reinterpret_cast<float *>(row + q / 8 * H_BLOCK + 512 + (q & 7) * 4) = back_of(ex);
                if (q + 1 == per_entry)                      // the rest of the last block is zero
                    for (uint32_t z = q + 1; z & 7; ++z) {
                        const uint32_t to = z / 8 * H_BLOCK + ((z & 4) * 16 + (g >> 2) * 16 + (z & 3) * 4 + (g & 3)) * 2;
                        *reinterpret_cast<uint16_t *>(row + to) = *reinterpret_cast<uint16_t *>(row + to + 64) = 0;
                        *reinterpret_cast<uint16_t *>(row + to + 256) = *reinterpret_cast<uint16_t *>(row + to + 320) = 0;
                        if (g == 0) *reinterpret_cast<float *>(row + z / 8 * H_BLOCK + 512 + (z & 7) * 4) = 0.0f;
                    }
            }
        }
    };
    Walk w;
    w.window1 = w.round_n = 0;
    uint32_t done0 = 0, done_n = 0, parity = 0;                  // the round before
    uint32_t get_slot = 0, get_parity = 0;
    const uint32_t row_at = matrix_row(lane);
    const float *unit_scale = nullptr;                           // the unit's scales of G; those of U `to_up` further on
    const uint64_t to_up = (uint64_t)iblocks * steps;
    uint32_t next_sg = 0, next_su = 0;                           // asked for a step before they are needed
    auto ask_scales = [&]() {
        next_sg = ldg_ahead(reinterpret_cast<const uint32_t *>(unit_scale + w.c));
        next_su = ldg_ahead(reinterpret_cast<const uint32_t *>(unit_scale + to_up + w.c));
    };
    auto scales_of_unit = [&]() {
        const uint32_t n = w.u / per_entry, e = R.entry[n] & 0xffffu, q = w.u - n * per_entry;
        unit_scale = M.gate_up_scale + ((uint64_t)(2 * e) * iblocks + q / (FP8_BLOCK / 16)) * steps;
        ask_scales();
    };
#pragma unroll 1
    for (uint32_t round0 = u0; round0 < u1; round0 += w.round_n) {
        const bool fresh = round0 >= w.window1;
        enter(w, round0);
        if (w.left) scales_of_unit();
        if (!EARLY && fresh) {                                   // the window's tokens
            const uint32_t n1 = (w.window1 + per_entry - 1) / per_entry;
            uint32_t base = 0;
            for (uint32_t n = w.window0 / per_entry; n < n1; ++n) {
                const uint32_t en = R.entry[n], count = tokens_in(n);
                stage(base, count, en & 0xffffu, (en >> 16) * M.per);
                base += count;
            }
            __syncthreads();
        }
        // ---- the second half joins the round before, the first half takes its steps of this one
        if (warp >= STREAMS) {
            if (done_n) join(done0, done_n, parts + (parity ^ 1) * (PARTS_BYTES / 4));
        } else {
            const uint32_t first_unit = w.u;
            float acc[8] = {};
            uint32_t x_at = 0;
            float b0 = 0.0f, b1 = 0.0f;
            auto begin = [&]() {                                 // where the tokens of the unit's entry are, and their scales
                const uint32_t n0 = w.window0 / per_entry, n = w.u / per_entry, en = R.entry[n], e = en & 0xffffu, first = (en >> 16) * M.per, count = tokens_in(n);
                uint32_t row = EARLY ? token_of(R, e, first + min(g, count - 1)) : min(g, count - 1);
                for (uint32_t k = n0; !EARLY && k < n; ++k) row += tokens_in(k);
                x_at = smem_addr(x_rows) + row * M.x_row + t4 * 32;                          // columns without a token repeat the last one; nobody looks at them
                b0 = back_of(exponent_of(R.largest[token_of(R, e, first + min(2 * t4, count - 1))]));
                b1 = back_of(exponent_of(R.largest[token_of(R, e, first + min(2 * t4 + 1, count - 1))]));
            };
            if (w.left) begin();
#pragma unroll 1
            while (w.left) {
                W.wait(my_bars + 8 * get_slot, get_parity);
                const uint32_t sa = ring + get_slot * UP_SLOT + row_at, xa = x_at + w.c * (STEP * 2);
                const float sg = __uint_as_float(settle(next_sg)), su = __uint_as_float(settle(next_su));
                bool end = --w.left == 0;
                const uint32_t unit = w.u;
                if (++w.c == steps) { w.c = 0; ++w.u; end = true; }
                if (!end) ask_scales();
                else if (w.left) scales_of_unit();
                float cg[2][4], cu[2][4];
#pragma unroll
                for (uint32_t p = 0; p < 4; ++p) {               // 32 columns
                    const uint4 hi = shared16(xa + (p >> 1) * 128 + (p & 1) * 16);
                    uint4 lo;
                    if constexpr (PIECES == 2) lo = shared16(xa + lo_at + (p >> 1) * 128 + (p & 1) * 16);
                    const uint4 wg = matrices((sa) ^ (p << 5)), wu = matrices((sa + UP_SLOT / 2) ^ (p << 5));
                    uint32_t a[4];
                    weights_of(a, wg.x, wg.y);
                    if (p < 2) mma_f16_first(cg[p & 1], a, hi.x, hi.y);
                    else mma_f16(cg[p & 1], a, hi.x, hi.y);
                    if constexpr (PIECES == 2) mma_f16(cg[p & 1], a, lo.x, lo.y);
                    weights_of(a, wu.x, wu.y);
                    if (p < 2) mma_f16_first(cu[p & 1], a, hi.x, hi.y);
                    else mma_f16(cu[p & 1], a, hi.x, hi.y);
                    if constexpr (PIECES == 2) mma_f16(cu[p & 1], a, lo.x, lo.y);
                    weights_of(a, wg.z, wg.w);
                    mma_f16(cg[p & 1], a, hi.z, hi.w);
                    if constexpr (PIECES == 2) mma_f16(cg[p & 1], a, lo.z, lo.w);
                    weights_of(a, wu.z, wu.w);
                    mma_f16(cu[p & 1], a, hi.z, hi.w);
                    if constexpr (PIECES == 2) mma_f16(cu[p & 1], a, lo.z, lo.w);
                }
                __syncwarp();                                    // the slot has been read
                // (three steps ahead: into the slot before this one, free since the last step)
                request();
                if (++get_slot == UP_DEPTH) { get_slot = 0; get_parity ^= 1; }
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    acc[j] = fmaf(cg[0][j] + cg[1][j], sg * (j & 1 ? b1 : b0), acc[j]);
                    acc[4 + j] = fmaf(cu[0][j] + cu[1][j], su * (j & 1 ? b1 : b0), acc[4 + j]);
                }
                if (end) {
                    float *const p = parts + parity * (PARTS_BYTES / 4) + ((warp * 2 + (unit - first_unit)) * 8) * 32 + lane;
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) { p[j * 32] = acc[j]; acc[j] = 0.0f; }
                    if (w.left) begin();
                }
            }
        }
        __syncthreads();
        done0 = round0;
        done_n = w.round_n;
        parity ^= 1;
    }
    if (warp >= STREAMS && done_n) join(done0, done_n, parts + (parity ^ 1) * (PARTS_BYTES / 4));
    __syncthreads();
    // after a wait that gave up: copies in flight must land before the block's shared memory goes away
    if (warp < STREAMS && lane == 0 && *W.abort_flag)
        for (uint32_t s = 0; s < UP_DEPTH; ++s) {
            const uint32_t uses = (issued + UP_DEPTH - 1 - s) / UP_DEPTH;
            if (uses) mbar_drain(my_bars + 8 * s, (uses - 1) & 1u, M.wait_limit);
        }
}

// ---- second kernel: y = sum p D h

template <uint32_t ROWS, uint32_t DOWN_WARPS, bool SPLIT>
__global__ void __launch_bounds__(DOWN_WARPS * 32, 1) k_moe_down(const __grid_constant__ CUtensorMap weights, const MoeArgs M)
{
    constexpr uint32_t TILES = ROWS / 16, W_BYTES = ROWS * STEP;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ uint64_t bars[DOWN_WARPS * MAX_DOWN_DEPTH];
    __shared__ Entry near[NEAR_ENTRIES];
    __shared__ uint32_t abort_word, list_size;
    // [ring of weights][ring of inner values][sums: warp, token, row]
    const uint32_t skew = (1024u - (smem_addr(smem_raw) & 1023u)) & 1023u, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    uint8_t *const smem = smem_raw + skew;
    const uint32_t h_slot = M.slot - W_BYTES, ring = smem_addr(smem) + warp * M.depth * W_BYTES;
    const uint32_t h_ring = smem_addr(smem) + DOWN_WARPS * M.depth * W_BYTES + warp * M.depth * h_slot, my_bars = smem_addr(bars) + 8 * warp * MAX_DOWN_DEPTH;
    float *const sums = reinterpret_cast<float *>(smem + (size_t)DOWN_WARPS * M.depth * M.slot);
    float *const mine = sums + warp * M.tokens * ROWS;
    const uint32_t rank = SPLIT ? cluster_rank() : 0, row0 = (SPLIT ? blockIdx.x / M.split : blockIdx.x) * ROWS;
    const Waits W{&abort_word, M.status, M.wait_limit};
    for (uint32_t i = lane; i < M.tokens * ROWS; i += 32) mine[i] = 0.0f;
    if (lane < M.depth) mbar_init(my_bars + 8 * lane, 1);
    if (tid == 0) abort_word = 0;
    if (tid == 0) asm volatile("prefetch.tensormap [%0];\n" :: "l"(&weights) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    __syncthreads();
    wait_prior_grid();
    launch_dependents();
    asm volatile("fence.proxy.async.global;\n" ::: "memory");    // the copies below read what the first kernel stored
    // the list is read before its length is known, as far as it may reach: one trip to memory
    for (uint32_t i = tid; i < min(M.tokens * M.top_k, NEAR_ENTRIES) * (uint32_t)(sizeof(Entry) / 4); i += DOWN_WARPS * 32)
        reinterpret_cast<uint32_t *>(near)[i] = reinterpret_cast<const uint32_t *>(M.list)[i];
    if (tid == 0) list_size = *M.list_size;
    __syncthreads();
    auto entry = [&](uint32_t n) -> const Entry & { return n < NEAR_ENTRIES ? near[n] : M.list[n]; };
    const uint32_t steps = (M.inner + STEP - 1) / STEP, total = list_size * steps;
    const uint32_t part = rank * DOWN_WARPS + warp, parts = SPLIT ? M.split * DOWN_WARPS : DOWN_WARPS;
    const uint32_t q0 = total * part / parts, q1 = total * (part + 1) / parts;

    // ---- a step's weights and its tokens' inner values into the rings
    uint32_t ahead_n = q0 / steps, ahead_c = q0 - ahead_n * steps, ahead_q = q0, put_slot = 0, issued = 0;
    uint32_t weight_row = 0, ahead_count = 0;
    const uint64_t once = policy_once();
    const uint8_t *h_row = nullptr;                              // of token `lane`
    auto open_entry = [&]() {
        const Entry &E = entry(ahead_n);
        ahead_count = E.count;
        weight_row = E.expert * M.d_expert + row0;
        h_row = M.h + (uint64_t)E.pair[lane < ahead_count ? lane : 0] * M.h_row;
    };
    auto request = [&]() {
        if (ahead_q < q1) {
            const uint32_t bar = my_bars + 8 * put_slot;
            const bool go = !M.skip_loads && !*W.abort_flag;
            if (lane == 0 && go) {
                mbar_expect_tx(bar, W_BYTES + ahead_count * H_BLOCK);
                tma_load_2d_once(ring + put_slot * W_BYTES, &weights, bar, (int32_t)(ahead_c * STEP), (int32_t)weight_row, once);
                ++issued;
            }
            const bool all_go = __shfl_sync(0xffffffffu, (int)go, 0) != 0;
            if (lane < ahead_count && all_go) bulk_load(h_ring + put_slot * h_slot + lane * H_PITCH, h_row + (uint64_t)ahead_c * H_BLOCK, H_BLOCK, bar);
            ++ahead_q;
            if (++ahead_c == steps) {
                ahead_c = 0;
                ++ahead_n;
                if (ahead_q < q1) open_entry();
            }
            put_slot = put_slot + 1 == M.depth ? 0 : put_slot + 1;
        }
    };
    if (q0 < q1) open_entry();
#pragma unroll 1
    for (uint32_t j = 0; j + 1 < M.depth; ++j) request();

    uint32_t n = q0 / steps, c_at = q0 - n * steps, get_slot = 0, get_parity = 0, count = 0;
    const uint32_t row_at = matrix_row(lane);
    float acc[TILES][4] = {};
    // of the entry at hand and of the next one; D's scale is asked for a step before it is needed
    uint32_t next_expert = 0, next_count = 0;
    const float *entry_scale = nullptr;
    uint32_t next_s = 0;
    auto scales_of = [&](uint32_t expert) { return M.down_scale + ((uint64_t)expert * ((M.hidden + FP8_BLOCK - 1) / FP8_BLOCK) + row0 / FP8_BLOCK) * steps; };
    auto look_ahead = [&]() {
        if ((uint64_t)(n + 1) * steps < q1) {
            next_expert = entry(n + 1).expert;
            next_count = entry(n + 1).count;
        }
    };
    if (q0 < q1) {
        count = entry(n).count;
        entry_scale = scales_of(entry(n).expert);
        next_s = ldg_ahead(reinterpret_cast<const uint32_t *>(entry_scale + c_at));
        look_ahead();
    }
#pragma unroll 1
    for (uint32_t q = q0; q < q1; ++q) {
        W.wait(my_bars + 8 * get_slot, get_parity);
        const uint32_t sa = ring + get_slot * W_BYTES + row_at, b = h_ring + get_slot * h_slot + min(g, count - 1) * H_PITCH + t4 * 32;
        const uint32_t f_at = h_ring + get_slot * h_slot + 512, f0_at = f_at + min(2 * t4, count - 1) * H_PITCH, f1_at = f_at + min(2 * t4 + 1, count - 1) * H_PITCH;
        const float s = __uint_as_float(settle(next_s));
        if (c_at + 1 == steps) entry_scale = scales_of(next_expert) - steps;
        if (q + 1 < q1) next_s = ldg_ahead(reinterpret_cast<const uint32_t *>(entry_scale + c_at + 1));
        if (c_at + 1 == steps) entry_scale += steps;
        float part[TILES][4] = {};                               // of this step, before D's scale
#pragma unroll
        for (uint32_t p = 0; p < 4; ++p) {                       // 32 columns
            const uint4 hi = shared16(b + (p >> 1) * 128 + (p & 1) * 16), lo = shared16(b + 256 + (p >> 1) * 128 + (p & 1) * 16);
            const float f0[2] = {shared4(f0_at + p * 8), shared4(f0_at + p * 8 + 4)}, f1[2] = {shared4(f1_at + p * 8), shared4(f1_at + p * 8 + 4)};
#pragma unroll
            for (uint32_t r = 0; r < TILES; ++r) {
                const uint4 w = matrices((sa + r * (16 * STEP)) ^ (p << 5));
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) {
                    uint32_t a[4];
                    weights_of(a, j ? w.z : w.x, j ? w.w : w.y);
                    float c[4];
                    mma_f16_first(c, a, j ? hi.z : hi.x, j ? hi.w : hi.y);
                    mma_f16(c, a, j ? lo.z : lo.x, j ? lo.w : lo.y);
                    part[r][0] = fmaf(c[0], f0[j], part[r][0]);
                    part[r][1] = fmaf(c[1], f1[j], part[r][1]);
                    part[r][2] = fmaf(c[2], f0[j], part[r][2]);
                    part[r][3] = fmaf(c[3], f1[j], part[r][3]);
                }
            }
        }
        __syncwarp();                                            // the slot has been read
        request();
        if (++get_slot == M.depth) { get_slot = 0; get_parity ^= 1; }
#pragma unroll
        for (uint32_t r = 0; r < TILES; ++r)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) acc[r][j] = fmaf(part[r][j], s, acc[r][j]);
        if (++c_at == steps || q + 1 == q1) {                    // the entry's part goes to the warp's sums
            const Entry &E = entry(n);
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k)
                if (2 * t4 + k < count) {
                    const float p = E.prob[2 * t4 + k];
                    float *const to = mine + E.token[2 * t4 + k] * ROWS + g;
#pragma unroll
                    for (uint32_t r = 0; r < TILES; ++r) {
                        to[16 * r] = fmaf(p, acc[r][k], to[16 * r]);
                        to[16 * r + 8] = fmaf(p, acc[r][2 + k], to[16 * r + 8]);
                    }
                }
#pragma unroll
            for (uint32_t r = 0; r < TILES; ++r) acc[r][0] = acc[r][1] = acc[r][2] = acc[r][3] = 0.0f;
            __syncwarp();
            if (c_at == steps) {
                c_at = 0;
                ++n;
                count = next_count;
                look_ahead();
            }
        }
    }
    __syncthreads();
    if (*W.abort_flag) {                                         // copies in flight must land before the block's shared memory goes away
        if (lane == 0)
            for (uint32_t s = 0; s < M.depth; ++s) {
                const uint32_t uses = (issued + M.depth - 1 - s) / M.depth;
                if (uses) mbar_drain(my_bars + 8 * s, (uses - 1) & 1u, M.wait_limit);
            }
        if (!SPLIT) return;                                      // (the others of a cluster look at the flag)
    }
    auto write = [&](uint32_t i, float s) {
        const uint32_t row = row0 + i % ROWS;
        if (row >= M.hidden) return;
        const int64_t at = (int64_t)(i / ROWS) * M.ldy + row;
        if (M.y_bf16) static_cast<__nv_bfloat16 *>(M.y)[at] = __float2bfloat16_rn(s);
        else static_cast<float *>(M.y)[at] = s;
    };
    for (uint32_t i = tid; i < M.tokens * ROWS; i += DOWN_WARPS * 32) {
        float s = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < DOWN_WARPS; ++w) s += sums[w * M.tokens * ROWS + i];
        if (!SPLIT) write(i, s);
        else sums[i] = s;                                        // (nobody else reads this place)
    }
    if constexpr (!SPLIT) return;
    __syncwarp();
    cluster_sync();                                              // all CTAs' sums are there; each adds up a share, in rank order
    bool whole = true;
    for (uint32_t r = 0; r < M.split; ++r) whole = whole && peer_load(peer_addr(smem_addr(&abort_word), r)) == 0;
    for (uint32_t i = rank * DOWN_WARPS * 32 + tid; whole && i < M.tokens * ROWS; i += parts * 32) {
        float s = 0.0f;
        for (uint32_t r = 0; r < M.split; ++r) s += __uint_as_float(peer_load(peer_addr(smem_addr(sums + i), r)));
        write(i, s);
    }
    cluster_sync();                                              // shared memory outlives its readers
}

// ---- host

struct MoeShape { uint32_t h_row; size_t h_bytes, bytes; };
MoeShape moe_shape(uint32_t tokens, uint32_t top_k, uint64_t inner)
{
    MoeShape s;
    const size_t pairs = (size_t)tokens * top_k;
    s.h_row = (uint32_t)((inner + STEP - 1) / STEP * H_BLOCK);
    s.h_bytes = (pairs * s.h_row + 255) / 256 * 256;
    s.bytes = s.h_bytes + 256 + (pairs * sizeof(Entry) + 255) / 256 * 256;       // an entry has a token at least
    return s;
}

// Whether the second kernel has room for a ring of two slots, whatever the call: the sums of all tokens, slots of full groups.
constexpr bool room_for_down(uint32_t rows, uint32_t warps)
{
    return 1024 + warps * (MAX_TOKENS * rows * 4 + 2 * (rows * STEP + GROUP * H_PITCH)) <= DOWN_SMEM_BYTES;
}

template <typename XT>
int launch_moe(MoeArgs M, const sqnn_moe *L, cudaStream_t st)
{
    // first kernel: what the ring and the partial sums leave holds rows of x
    const uint32_t cols = (M.hidden + STEP - 1) / STEP * STEP, pieces = sizeof(XT) == 2 ? 1 : 2;
    const size_t fixed = 1024 + STREAMS * UP_DEPTH * UP_SLOT + ROUTING_BYTES + 2 * PARTS_BYTES;
    M.x_row = cols * 2 * pieces + 16;                            // 16 bytes past a multiple of 128: neighbouring rows in neighbouring banks
    M.x_rows = (uint32_t)((SMEM_BYTES - fixed) / M.x_row);
    if (M.x_rows == 0) return SQNN_E_UNSUPPORTED;
    M.per = M.x_rows < GROUP ? M.x_rows : GROUP;
    auto up = M.tokens <= M.x_rows ? k_moe_up<XT, true> : k_moe_up<XT, false>;
    // second kernel: 32 rows per CTA where that still makes two CTAs for three SMs; as deep a ring as there is room for
    const uint32_t rows = 3 * ((M.hidden + 31) / 32) >= 2 * (uint32_t)sm_count() ? 32 : 16;
    M.slot = rows * STEP + (M.tokens < M.per ? M.tokens : M.per) * H_PITCH;
    // 12 warps with a ring of two slots (16 tokens, 64 experts of 1536, top 8, hidden 4096: 209 us in short runs) are faster than 8 with four (213), but do not
    // always fit; 8 with two do, and so do 12 where a CTA has 16 rows
    const auto depth_of = [&](uint32_t warps) { return (uint32_t)((DOWN_SMEM_BYTES - 1024 - (size_t)warps * M.tokens * rows * 4) / (warps * M.slot)); };
    static_assert(room_for_down(16, MAX_DOWN_WARPS) && room_for_down(32, 8), "a ring of two slots whatever the call");
    const uint32_t warps = depth_of(MAX_DOWN_WARPS) >= 2 ? MAX_DOWN_WARPS : 8;
    M.depth = depth_of(warps) < MAX_DOWN_DEPTH ? depth_of(warps) : MAX_DOWN_DEPTH;
    const size_t smem_down = 1024 + (size_t)warps * (M.tokens * rows * 4 + M.depth * M.slot);
    const auto down = rows == 16 ? k_moe_down<16, MAX_DOWN_WARPS, false> : warps == 8 ? k_moe_down<32, 8, false> : k_moe_down<32, MAX_DOWN_WARPS, false>;
    const auto down_split = k_moe_down<16, MAX_DOWN_WARPS, true>;
    CUtensorMap gu_map, d_map;
    if (!byte_rows_map(&gu_map, L->gate_up, M.hidden, (uint64_t)(M.experts - 1) * M.gu_expert + M.gu_half + M.inner, L->gate_up_row, 16) ||
        !byte_rows_map(&d_map, L->down, M.inner, (uint64_t)(M.experts - 1) * M.d_expert + M.hidden, L->down_row, rows))
        return SQNN_E_CUDA;
    if (ensure_dynamic_smem(reinterpret_cast<const void *>(up), SMEM_BYTES) != SQNN_OK) return SQNN_E_CUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CLUSTER;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CLUSTER);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM_BYTES;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    // as many CTAs as run at once in whole clusters, asked for once per device
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
    // Few runs of rows: a cluster shares one, as far as all clusters run at once and each warp has three steps or more (29 tokens, 7 of 8 experts, hidden 367,
    // inner 3264: 121 us by one CTA a run, 73 by four; 5 tokens, 3 of 12, 1000 and 500, two steps a warp: 20.5 and 21.3).
    const uint32_t runs = (M.hidden + rows - 1) / rows, steps = (M.inner + STEP - 1) / STEP, reached = M.tokens * M.top_k < M.experts ? M.tokens * M.top_k : M.experts;
    cudaLaunchConfig_t cfg_down = cfg;
    cudaLaunchAttribute attr_down[2] = {attr[0], attr[1]};
    cfg_down.attrs = attr_down;
    cfg_down.blockDim = dim3(warps * 32);
    M.split = 1;
    if (rows == 16) {
        static std::atomic<int> known_down[64][2];
        for (uint32_t s = 4; s > 1 && M.split == 1; s /= 2) {            // (three: 46 us where two take 42)
            if (runs * s > (uint32_t)sm_count() || reached * steps < 3 * s * warps) continue;
            int at_once = dev < 64 ? known_down[dev][s / 4].load(std::memory_order_relaxed) : 0;
            if (at_once == 0) {
                if (ensure_dynamic_smem(reinterpret_cast<const void *>(down_split), DOWN_SMEM_BYTES) != SQNN_OK) return SQNN_E_CUDA;
                attr_down[0].val.clusterDim.x = s;
                cfg_down.gridDim = dim3(s);
                cfg_down.numAttrs = 1;
                cfg_down.dynamicSmemBytes = DOWN_SMEM_BYTES;
                if (cudaOccupancyMaxActiveClusters(&at_once, down_split, &cfg_down) != cudaSuccess || at_once <= 0) return SQNN_E_CUDA;
                if (dev < 64) known_down[dev][s / 4].store(at_once, std::memory_order_relaxed);
            }
            if (runs <= (uint32_t)at_once) M.split = s;
        }
    }
    if (cudaLaunchKernelEx(&cfg, up, gu_map, M) != cudaSuccess) return SQNN_E_CUDA;
    if (M.split == 1) return launch_kernel(down, runs, warps * 32, smem_down, st, d_map, M);
    if (ensure_dynamic_smem(reinterpret_cast<const void *>(down_split), smem_down) != SQNN_OK) return SQNN_E_CUDA;
    attr_down[0].val.clusterDim.x = M.split;
    cfg_down.gridDim = dim3(runs * M.split);
    cfg_down.numAttrs = 2;
    cfg_down.dynamicSmemBytes = smem_down;
    return cudaLaunchKernelEx(&cfg_down, down_split, d_map, M) == cudaSuccess ? SQNN_OK : SQNN_E_CUDA;
}

int moe_queue(const sqnn_moe *L, uint32_t tokens, const void *d_x, int x_dtype, int64_t ldx, void *d_y, int y_dtype, int64_t ldy,
              int32_t *d_ids, float *d_probs, void *d_workspace, size_t workspace_bytes, uint32_t *d_status, cudaStream_t st)
{
    const auto known_type = [](int t) { return t == SQNN_X_F32 || t == SQNN_X_BF16; };
    const auto aligned_to = [](const void *p, uintptr_t size) { return ((uintptr_t)p & (size - 1)) == 0; };
    if (!L || !d_x || !d_y || tokens == 0) return SQNN_E_INVALID_ARG;
    if (!L->router || !L->gate_up || !L->gate_up_scale || !L->down || !L->down_scale) return SQNN_E_INVALID_ARG;
    if (L->experts == 0 || L->top_k == 0 || L->top_k > L->experts || L->hidden == 0 || L->inner == 0) return SQNN_E_INVALID_ARG;
    if (!known_type(x_dtype) || !known_type(y_dtype)) return SQNN_E_INVALID_ARG;
    if (tokens > SQNN_MOE_MAX_TOKENS || L->experts > SQNN_MOE_MAX_EXPERTS || L->top_k > SQNN_MOE_MAX_TOP_K || tokens * L->experts > SQNN_MOE_MAX_LOGITS ||
        L->hidden > SQNN_MOE_MAX_WIDTH || L->inner > SQNN_MOE_MAX_WIDTH)
        return SQNN_E_UNSUPPORTED;
    const int64_t hidden = L->hidden, inner = L->inner;
    const uintptr_t xs = x_dtype == SQNN_X_BF16 ? 2 : 4, ys = y_dtype == SQNN_X_BF16 ? 2 : 4;
    if (ldx < hidden || ldy < hidden || L->router_row < hidden || L->gate_up_row < hidden || L->down_row < inner || L->gate_up_half < 0 ||
        L->gate_up_expert < 0 || L->down_expert < 0)
        return SQNN_E_INVALID_ARG;
    if (!aligned_to(d_x, xs) || !aligned_to(L->router, xs) || !aligned_to(d_y, ys) || !aligned_to(L->gate_up_scale, 4) || !aligned_to(L->down_scale, 4) ||
        !aligned_to(d_ids, 4) || !aligned_to(d_probs, 4))
        return SQNN_E_INVALID_ARG;
    if (!aligned_to(L->gate_up, 16) || !aligned_to(L->down, 16) || ((L->gate_up_row | L->down_row) & 15)) return SQNN_E_UNSUPPORTED;
    // the weights of all experts are rows of one matrix to the copies
    const int64_t most_rows = 1ll << 30, most_elements = 1ll << 50;      // (what is multiplied below stays within 64 bits)
    if (L->gate_up_expert > most_elements || L->gate_up_half > most_elements || L->down_expert > most_elements ||
        L->gate_up_half % L->gate_up_row || L->gate_up_expert % L->gate_up_row || L->down_expert % L->down_row || L->gate_up_row > (1ll << 30) || L->down_row > (1ll << 30) ||
        L->gate_up_expert / L->gate_up_row * L->experts + L->gate_up_half / L->gate_up_row + inner > most_rows || L->down_expert / L->down_row * L->experts + hidden > most_rows)
        return SQNN_E_UNSUPPORTED;
    const MoeShape shape = moe_shape(tokens, L->top_k, L->inner);
    if (!d_workspace || workspace_bytes < shape.bytes || !aligned_to(d_workspace, 256)) return SQNN_E_WORKSPACE;
    MoeArgs M = {};
    M.x = d_x; M.router = L->router;
    M.gate_up_scale = L->gate_up_scale; M.down_scale = L->down_scale;
    M.y = d_y;
    M.h = static_cast<uint8_t *>(d_workspace);
    M.list_size = reinterpret_cast<uint32_t *>(M.h + shape.h_bytes);
    M.list = reinterpret_cast<Entry *>(M.h + shape.h_bytes + 256);
    M.ids_out = d_ids; M.probs_out = d_probs;
    M.ldx = ldx; M.ldr = L->router_row; M.ldy = ldy;
    M.gu_expert = (uint32_t)(L->gate_up_expert / L->gate_up_row); M.gu_half = (uint32_t)(L->gate_up_half / L->gate_up_row);
    M.d_expert = (uint32_t)(L->down_expert / L->down_row);
    M.tokens = tokens; M.experts = L->experts; M.top_k = L->top_k; M.hidden = L->hidden; M.inner = L->inner;
    M.h_row = shape.h_row;
    const DebugKnobs dbg = debug_knobs();
    M.skip_loads = (dbg.flags & 16u) ? 1u : 0u;
    M.wait_limit = dbg.wait_cycles ? dbg.wait_cycles : WAIT_LIMIT_CYCLES;
    M.status = d_status;
    M.renormalize = L->renormalize;
    M.x_vec = aligned_to(d_x, 16) && (ldx * (int64_t)xs) % 16 == 0;
    M.r_vec = aligned_to(L->router, 16) && (L->router_row * (int64_t)xs) % 16 == 0;
    M.y_bf16 = y_dtype == SQNN_X_BF16;
    return x_dtype == SQNN_X_BF16 ? launch_moe<__nv_bfloat16>(M, L, st) : launch_moe<float>(M, L, st);
}

}  // namespace
}  // namespace sqnn

extern "C" size_t sqnn_moe_workspace_bytes(uint32_t tokens, uint32_t top_k, uint32_t inner)
{
    if (tokens > SQNN_MOE_MAX_TOKENS || top_k > SQNN_MOE_MAX_TOP_K || inner > SQNN_MOE_MAX_WIDTH) return 0;
    return sqnn::moe_shape(tokens, top_k, inner).bytes;
}

extern "C" int sqnn_moe_fp8(const sqnn_moe *layer, uint32_t tokens, const void *d_x, int x_dtype, int64_t ldx, void *d_y, int y_dtype, int64_t ldy,
                            int32_t *d_ids, float *d_probs, void *d_workspace, size_t workspace_bytes, uint32_t *d_status,
                            void *cuda_stream)
{
    sqnn::ApiScope scope("sqnn_moe_fp8");
    return scope.finish(sqnn::moe_queue(layer, tokens, d_x, x_dtype, ldx, d_y, y_dtype, ldy, d_ids, d_probs, d_workspace, workspace_bytes,
                                        d_status, (cudaStream_t)cuda_stream),
                        d_status, (cudaStream_t)cuda_stream);
}
