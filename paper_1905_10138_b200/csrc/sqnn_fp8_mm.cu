// Product of 8-bit weights with a scale per 128 x 128 block and 8-bit activations with a scale per row and 128 columns.
//
//   Y[b][r] = sum_k sx[b][k] sw[r / 128][k] sum_{c in block k} W[r][c] X[b][c]
//
// The inner sums run on tcgen05.mma (kind::f8f6f4, fp32 accumulators in tensor memory), one block k of 128 columns at a time; the
// scales differ from block to block, so each block's sums are read back, scaled and added to a 32-bit accumulator in registers while
// the tensor cores work on the next blocks in other columns of tensor memory.
//
// Three forms, by who lies along the 128 lanes:
//   - batches up to 64: the weights' rows are the lanes, the batch the 16 to 64 columns.  Bound by reading the weights.  A lane's
//     weights share one scale (its block of 128 rows), the activations' scales go by column.
//   - else the batch's rows are the lanes and 128 weight rows the columns: a lane has one scale per block,
//   - or, for large products, two CTAs on neighbouring SMs share a tile of 256 by 256 (cta_group::2): each brings its own 128 batch rows and half of
//     the weights' rows, so that a byte in shared memory serves twice as many products.  (At 128 by 128 the operands of a block take the
//     whole of shared memory's bandwidth.)
// Few tiles: the CTAs of a cluster share one, each taking a range of the blocks k; each sends its sums to the CTAs that own a share of the
// columns, through distributed shared memory, and these add them up in the order of the ranks.  No workspace, no atomics: results are the same
// from run to run.
//
// Measured, us (floor at the copy's and the tensor cores' measured rates): 4096 x 9216 batch 1 9.9 (5.8), batch 64 12.7 (6.0); 4096 x 16384 batch 512 42.5 (20.6) in
// short runs and 49 in loops of a second, where the chip is at its 1000 W and the clock at 1.69 GHz; batch 4096 275 (164) and 314 (at 1.49 GHz).  Small batches are bound by
// how soon the loads start and by the end of the call (start, exchange of sums) beside the stream; large ones by the two accumulators that take turns (per two
// blocks 600 cycles of MMA, and reading, scaling and signalling 1200 that overlap only in part) and, in long loops, by power.
#include "sqnn_launch.h"
#include "sqnn_fp8.cuh"
#include "sqnn_fp8_plan.h"
#include "sqnn_cluster.cuh"
#include "sqnn_tc.cuh"

#include <cuda_bf16.h>

#include <atomic>

namespace sqnn {

namespace {

constexpr uint32_t LANES = 128;           // rows of the lane operand per tile
constexpr uint32_t KB = FP8_BLOCK;        // columns per step: one block of scales, one 128-byte swizzled row
constexpr uint32_t CHUNK = 16;            // blocks whose scales are fetched together
constexpr uint32_t MAX_STAGES = 12;
constexpr uint64_t WAIT_LIMIT_CYCLES = 4000000000ull;

struct Fp8Args {
    const float *ws, *xs;         // scales of weights and activations
    void *y;
    int64_t ldws, ldxs, ldy;
    uint32_t m, batch;
    uint32_t kblocks;             // blocks of 128 columns per row
    uint32_t tiles, col_tiles;    // tiles in all; tiles along the columns
    uint32_t split;               // CTAs per tile (= cluster size)
    uint32_t quarters, first;     // tiles are quarters of the pair's tiles (`col_tiles` of them along the columns) from `first` on
    uint32_t stages;
    uint32_t y_bf16, vec, vec4;   // rows of Y on 16-byte boundaries; on those of four elements
    uint32_t xs_vec;              // rows of the activations' scales on 16-byte boundaries
    uint32_t skip_loads;          // test only: the loader issues no loads
    uint64_t wait_limit;
    uint32_t *status;
};

// Four tcgen05.mma (K = 32 each) over the 128 columns of a stage and two commits: the stage is free, the accumulator is full.
SQNN_DEV void mma_block(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t free_stage, uint32_t acc_full)
{
#define SQNN_MMA(A, B, P) " @e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], " A ", " B ", %3, " P ";\n"
    asm volatile("{\n .reg .pred e, f, t;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n"
                 " elect.sync _|e, 0xffffffff;\n setp.ne.b32 f, %3, %3;\n setp.eq.b32 t, %3, %3;\n"
                 " add.u64 a1, %1, 2;\n add.u64 a2, %1, 4;\n add.u64 a3, %1, 6;\n"
                 " add.u64 b1, %2, 2;\n add.u64 b2, %2, 4;\n add.u64 b3, %2, 6;\n"
                 SQNN_MMA("%1", "%2", "f") SQNN_MMA("a1", "b1", "t") SQNN_MMA("a2", "b2", "t") SQNN_MMA("a3", "b3", "t")
                 " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n"
                 " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n}\n"
                 :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(free_stage), "r"(acc_full) : "memory");
#undef SQNN_MMA
}
// The same for a pair of CTAs (M = 256: 128 lanes of each; B: half of the columns from each); the commits signal both.
SQNN_DEV void mma_block_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t free_stage, uint32_t acc_full, uint32_t mask)
{
#define SQNN_MMA(A, B, P) " @e tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], " A ", " B ", %3, " P ";\n"
    asm volatile("{\n .reg .pred e, f, t;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n .reg .b16 m;\n cvt.u16.u32 m, %6;\n"
                 " elect.sync _|e, 0xffffffff;\n setp.ne.b32 f, %3, %3;\n setp.eq.b32 t, %3, %3;\n"
                 " add.u64 a1, %1, 2;\n add.u64 a2, %1, 4;\n add.u64 a3, %1, 6;\n"
                 " add.u64 b1, %2, 2;\n add.u64 b2, %2, 4;\n add.u64 b3, %2, 6;\n"
                 SQNN_MMA("%1", "%2", "f") SQNN_MMA("a1", "b1", "t") SQNN_MMA("a2", "b2", "t") SQNN_MMA("a3", "b3", "t")
                 " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], m;\n"
                 " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%4], m;\n}\n"
                 :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(free_stage), "r"(acc_full), "r"(mask) : "memory");
#undef SQNN_MMA
}
SQNN_DEV void commit_pair(uint32_t bar)
{
    asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
                 " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" :: "r"(bar) : "memory");
}
// Instruction descriptor: D fp32, A and B e4m3, both K-major.
SQNN_DEV uint32_t instr_desc_fp8(uint32_t m, uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((m >> 4) << 24); }

// acc (two fp32 numbers) += t * s
SQNN_DEV void fma2(uint64_t &acc, uint32_t lo, uint32_t hi, uint64_t s)
{
    asm("{\n .reg .b64 t;\n mov.b64 t, {%1, %2};\n fma.rn.f32x2 %0, t, %3, %0;\n}\n" : "+l"(acc) : "r"(lo), "r"(hi), "l"(s));
}
SQNN_DEV uint64_t pair(float lo, float hi)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(v) : "f"(lo), "f"(hi));
    return v;
}
// A thread's sums, two to a register pair.
template <uint32_t COLS>
struct Sums {
    uint64_t v[COLS / 2];
    SQNN_DEV void clear()
    {
#pragma unroll
        for (uint32_t j = 0; j < COLS / 2; ++j) v[j] = 0ull;
    }
    SQNN_DEV float operator[](uint32_t j) const
    {
        float2 f;
        asm("mov.b64 {%0, %1}, %2;\n" : "=f"(f.x), "=f"(f.y) : "l"(v[j / 2]));
        return j & 1 ? f.y : f.x;
    }
};

// Four neighbouring elements of a row of Y, as many of them as `room` allows.
SQNN_DEV void put4(const Fp8Args &M, int64_t at, uint32_t room, const float4 &v)
{
    if (M.vec4 && room >= 4) {
        if (M.y_bf16) *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(M.y) + at) = make_uint2(bf16x2(v.x, v.y), bf16x2(v.z, v.w));
        else *reinterpret_cast<float4 *>(static_cast<float *>(M.y) + at) = v;
    } else {
        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (j < room) {
                if (M.y_bf16) static_cast<__nv_bfloat16 *>(M.y)[at + j] = __float2bfloat16_rn(e[j]);
                else static_cast<float *>(M.y)[at + j] = e[j];
            }
    }
}

// A warp's 32 rows of a tile (a lane each, batch rows from b0 on), COLS columns from r0 on.  Rows on 16-byte boundaries are written by their lanes, others go through
// `turn` (shared memory of the warp) 32 columns at a time, so that a store is 32 neighbouring elements.
constexpr uint32_t TURN_FLOATS = 32 * 33;
template <uint32_t COLS>
SQNN_DEV void store_rows(const Fp8Args &M, const Sums<COLS> &acc, uint32_t b0, uint32_t r0, uint32_t lane, float *turn)
{
    if (r0 >= M.m) return;
    const uint32_t b = b0 + lane;
    const int64_t at = (int64_t)b * M.ldy + r0;
    if (M.vec && M.y_bf16 && r0 + COLS <= M.m) {
        if (b >= M.batch) return;
        uint4 *const p = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(M.y) + at);
#pragma unroll
        for (uint32_t j = 0; j < COLS; j += 8)
            p[j / 8] = make_uint4(bf16x2(acc[j], acc[j + 1]), bf16x2(acc[j + 2], acc[j + 3]), bf16x2(acc[j + 4], acc[j + 5]), bf16x2(acc[j + 6], acc[j + 7]));
    } else if (M.vec4) {
        if (b >= M.batch) return;
#pragma unroll
        for (uint32_t j = 0; j < COLS; j += 4)
            if (r0 + j < M.m) put4(M, at + j, M.m - (r0 + j), make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]));
    } else {
        const uint32_t rows = b0 < M.batch ? min(32u, M.batch - b0) : 0;
#pragma unroll
        for (uint32_t c = 0; c < COLS; c += 32) {
#pragma unroll
            for (uint32_t j = 0; j < 32; ++j) turn[lane * 33 + j] = acc[c + j];
            __syncwarp();
            if (r0 + c + lane < M.m)
                for (uint32_t i = 0; i < rows; ++i) {
                    const int64_t to = (int64_t)(b0 + i) * M.ldy + r0 + c + lane;
                    if (M.y_bf16) static_cast<__nv_bfloat16 *>(M.y)[to] = __float2bfloat16_rn(turn[i * 33 + lane]);
                    else static_cast<float *>(M.y)[to] = turn[i * 33 + lane];
                }
            __syncwarp();
        }
    }
}

template <uint32_t N> constexpr uint32_t promoters_of = N >= 128 ? 8 : 4;   // warps that scale and add: four per 128 lanes and half of the columns
template <uint32_t N> constexpr uint32_t buffers_of = N == 16 || N == 128 ? 4 : 2;      // accumulators in tensor memory
template <uint32_t N> constexpr uint32_t tmem_cols_of = N * buffers_of<N>;  // 64 to 512: a power of two
template <uint32_t N> constexpr uint32_t threads_of_fp8 = promoters_of<N> * 32 + 64;

// Scales of CHUNK blocks in shared memory, double-buffered: by lane or column, then those of the weights' blocks of rows.  A chunk is asked for
// while the one before is in use and stored when its turn comes.
template <bool SWAP, uint32_t N>
struct Scales {
    static constexpr uint32_t ROWS = SWAP ? N : LANES, PITCH = ROWS + 4, WBLOCKS = N == 256 ? 2 : 1, THREADS = promoters_of<N> * 32;
    static constexpr uint32_t FOURS = ROWS * (CHUNK / 4), EACH = (FOURS + THREADS - 1) / THREADS;
    static constexpr uint32_t FLOATS = 2 * CHUNK * PITCH;
    float *buf;                   // [2][CHUNK][PITCH]
    float4 x[EACH];
    float w;
    // asks for blocks [k0, k0 + CHUNK), those below k1; k0 is a multiple of four
    SQNN_DEV void fetch(const Fp8Args &M, uint32_t row0, uint32_t wblock, uint32_t k0, uint32_t k1, uint32_t tid)
    {
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            const uint32_t f = i * THREADS + tid, row = row0 + f / (CHUNK / 4), k = k0 + f % (CHUNK / 4) * 4;
            x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (f >= FOURS || row >= M.batch || k >= k1) continue;
            const float *const p = M.xs + (int64_t)row * M.ldxs + k;
            if (M.xs_vec && k + 4 <= k1) {
                x[i] = *reinterpret_cast<const float4 *>(p);
            } else {
                x[i].x = p[0];
                if (k + 1 < k1) x[i].y = p[1];
                if (k + 2 < k1) x[i].z = p[2];
                if (k + 3 < k1) x[i].w = p[3];
            }
        }
        const uint32_t j = tid / CHUNK, k = k0 + tid % CHUNK;
        w = j < WBLOCKS && (wblock + j) * FP8_BLOCK < M.m && k < k1 ? M.ws[(int64_t)(wblock + j) * M.ldws + k] : 0.0f;
    }
    SQNN_DEV void store(uint32_t which, uint32_t tid) const
    {
        float *const b = buf + which * CHUNK * PITCH;
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            const uint32_t f = i * THREADS + tid, row = f / (CHUNK / 4), k = f % (CHUNK / 4) * 4;
            if (f < FOURS) {
                b[k * PITCH + row] = x[i].x;
                b[(k + 1) * PITCH + row] = x[i].y;
                b[(k + 2) * PITCH + row] = x[i].z;
                b[(k + 3) * PITCH + row] = x[i].w;
            }
        }
        if (tid < CHUNK * WBLOCKS) b[tid % CHUNK * PITCH + ROWS + tid / CHUNK] = w;
    }
    SQNN_DEV const float *at(uint32_t which, uint32_t k) const { return buf + (which * CHUNK + k) * PITCH; }
};

// Columns of a tile that one of `split` CTAs adds up.
SQNN_HD uint32_t share_of(uint32_t n, uint32_t split) { return ((n + split - 1) / split + 3) / 4 * 4; }

// This thread's sums (lane `row`, columns col0 on) to the CTAs that add them up.  Their buffers: per source and four columns 128 lanes of four floats; with SWAP
// per source and column 128 lanes.
template <bool SWAP, uint32_t COLS>
SQNN_DEV void send_sums(const Sums<COLS> &acc, uint32_t buffer_sa, uint32_t share, uint32_t source, uint32_t row, uint32_t col0, uint32_t peer0, uint32_t peer_step)
{
    uint32_t owner = col0 / share, at = col0 - owner * share, base = peer_addr(buffer_sa, peer0 + owner * peer_step);
#pragma unroll
    for (uint32_t j = 0; j < COLS; j += 4) {
        if constexpr (SWAP) {
            const uint32_t to = base + ((source * share + at) * LANES + row) * 4;
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) peer_store(to + LANES * 4 * i, acc[j + i]);
        } else {
            peer_store4(base + ((source * share + at) / 4 * LANES + row) * 16, make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]));
        }
        at += 4;
        if (at == share) {
            at = 0;
            ++owner;
            if (j + 4 < COLS) base = peer_addr(buffer_sa, peer0 + owner * peer_step);
        }
    }
}
// Adds up a CTA's share of a tile and writes it: `own` is its place among the CTAs of the tile, row0 and col0 the tile's first lane and column.
template <bool SWAP, uint32_t N, uint32_t THREADS>
SQNN_DEV void add_sums(const Fp8Args &M, const float *buffer, uint32_t share, uint32_t own, uint32_t row0, uint32_t col0, uint32_t tid)
{
    const uint32_t first = own * share, cols = first < N ? min(share, N - first) : 0;
    if constexpr (SWAP) {
        for (uint32_t f = tid; f < cols * (LANES / 4); f += THREADS) {
            const uint32_t c = f / (LANES / 4), r = f % (LANES / 4) * 4;
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (uint32_t q = 0; q < M.split; ++q) {
                const float4 v = *reinterpret_cast<const float4 *>(buffer + (q * share + c) * LANES + r);
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
            const uint32_t b = col0 + first + c, at = row0 + r;
            if (b < M.batch && at < M.m) put4(M, (int64_t)b * M.ldy + at, M.m - at, sum);
        }
    } else {
        const uint32_t fours = cols / 4;
        for (uint32_t f = tid; f < fours * LANES; f += THREADS) {
            const uint32_t r = f / fours, c = (f - r * fours) * 4;
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (uint32_t q = 0; q < M.split; ++q) {
                const float4 v = *reinterpret_cast<const float4 *>(buffer + ((q * share + c) / 4 * LANES + r) * 4);
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
            const uint32_t b = row0 + r, at = col0 + first + c;
            if (b < M.batch && at < M.m) put4(M, (int64_t)b * M.ldy + at, M.m - at, sum);
        }
    }
}

SQNN_DEV void tmem_request(uint32_t taddr, uint32_t (&v)[16]) { tmem_request16(taddr, v); }
SQNN_DEV void tmem_request(uint32_t taddr, uint32_t (&v)[32]) { tmem_request32(taddr, v); }
// acc += t * scale of this block.  A thread's COLS columns come in pieces, each asked for before the arithmetic of the one before; `release` is called
// when the last one has arrived.  (Single fma take fewer cycles than fma.rn.f32x2, 385 against 525 a block of 128
// columns with nothing else running, but did not fit the registers here.)
template <bool SWAP, uint32_t COLS, typename F>
SQNN_DEV void promote(Sums<COLS> &acc, uint32_t tmem_at, const float *s, float lane_s, const F &release)
{
    constexpr uint32_t PIECE = COLS == 64 ? 32 : 16, PIECES = COLS / PIECE;
    uint32_t d[2][PIECE];
    tmem_request(tmem_at, d[0]);
#pragma unroll
    for (uint32_t c = 0; c < PIECES; ++c) {
        tmem_ld_wait(d[c & 1]);
        if (c + 1 < PIECES) tmem_request(tmem_at + (c + 1) * PIECE, d[(c + 1) & 1]);
        else release();
#pragma unroll
        for (uint32_t j = 0; j < PIECE; j += 2) {
            float f0 = lane_s, f1 = lane_s;
            if constexpr (SWAP) {
                const float2 x = *reinterpret_cast<const float2 *>(s + c * PIECE + j);
                f0 *= x.x;
                f1 *= x.y;
            }
            fma2(acc.v[(c * PIECE + j) / 2], d[c & 1][j], d[c & 1][j + 1], pair(f0, f1));
        }
    }
}

// One tile per CTA or cluster.
template <bool SWAP, uint32_t N>
__global__ void __launch_bounds__(threads_of_fp8<N>, 1)
k_fp8_mm(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap col_map, const Fp8Args M)
{
    constexpr uint32_t PW = promoters_of<N>, BUFS = buffers_of<N>, COLS = N * 4 / PW;     // COLS: columns per promoting thread
    constexpr uint32_t A_BYTES = LANES * KB, B_BYTES = N * KB, STAGE = A_BYTES + B_BYTES;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * MAX_STAGES + 2 * 4 + 2];
    __shared__ uint32_t tmem_slot, abort_word, given_up[8];
    volatile uint32_t *abort_flag = &abort_word;
    bool started = false;                                        // the cluster's first barrier has been waited for
    bool held = true;                                            // (the issuer's) the tensor memory
    const uint32_t full = smem_addr(bars), empty = full + 8 * MAX_STAGES, acc_full = empty + 8 * MAX_STAGES, acc_empty = acc_full + 8 * 4;
    const uint32_t chunk_bar = acc_empty + 8 * 4, over = chunk_bar + 8;   // scales are there; after a timeout: the MMAs are over
    // [stages][scales][sums of the tile's CTAs]
    const uint32_t stages_sa = (smem_addr(smem_raw) + 1023u) & ~1023u;
    float *const after = reinterpret_cast<float *>(smem_raw + (stages_sa - smem_addr(smem_raw)) + M.stages * STAGE);
    Scales<SWAP, N> sc;
    sc.buf = after;
    float *const sums = after + Scales<SWAP, N>::FLOATS;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = M.split > 1 ? cluster_rank() : 0, tile = blockIdx.x / M.split;
    uint32_t tl = tile / M.col_tiles, tc = tile - tl * M.col_tiles;
    if (!SWAP && M.quarters) {
        const uint32_t whole = M.first + tile / 4;
        tl = whole / M.col_tiles;
        tc = 2 * (whole - tl * M.col_tiles) + (tile & 1);
        tl = 2 * tl + (tile >> 1 & 1);
    }
    const uint32_t k_begin = M.kblocks * rank / M.split, k_end = M.kblocks * (rank + 1) / M.split;
    const uint32_t k_first = k_begin & ~3u;                      // where the first chunk of scales begins
    // first batch row of the scales, first block of weight rows
    const uint32_t row0 = SWAP ? tc * N : tl * LANES, wblock = SWAP ? tl : tc * (N / FP8_BLOCK);

    if (warp == PW + 1) {
        tmem_alloc(&tmem_slot, tmem_cols_of<N>);
    } else if (warp == PW) {
        if (lane < M.stages) { mbar_init(full + 8 * lane, 1); mbar_init(empty + 8 * lane, 1); }
        if (lane < BUFS) { mbar_init(acc_full + 8 * lane, 1); mbar_init(acc_empty + 8 * lane, PW); }
        if (lane == 0) {
            mbar_init(chunk_bar, PW);
            mbar_init(over, 1);
            abort_word = 0;
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    launch_dependents();                                         // after the allocation: see k_gemv_tc
    if (M.split > 1) cluster_arrive();                           // waited for before anything is written to another CTA
    wait_prior_grid();

    if (warp < PW) {
        // ------------------------------ scaling and adding up ------------------------------
        const uint32_t quad = warp & 3, half = warp >> 2, lane_row = quad * 32 + lane;
        const uint32_t tmem_at = tmem_base + ((quad * 32) << 16) + half * COLS;
        uint32_t it = 0, chunk_no = 0;
        Sums<COLS> acc;
        acc.clear();
        sc.fetch(M, row0, wblock, k_first, k_end, tid);
        for (uint32_t k0 = k_first; k0 < k_end; k0 += CHUNK, ++chunk_no) {
            // this chunk is there and the one before done with, for all of these warps (a bounded wait: a plain barrier would keep a
            // warp for good once another one has given up)
            sc.store(chunk_no & 1, tid);
            __syncwarp();
            if (lane == 0) mbar_arrive(chunk_bar);
            if (!mbar_wait_warp(chunk_bar, chunk_no & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
            if (k0 + CHUNK < k_end) sc.fetch(M, row0, wblock, k0 + CHUNK, k_end, tid);
            const uint32_t count = min(CHUNK, k_end - k0);
            for (uint32_t k = max(k0, k_begin) - k0; k < count; ++k, ++it) {
                const uint32_t buf = it % BUFS;
                const float *s = sc.at(chunk_no & 1, k);
                const float ws = s[Scales<SWAP, N>::ROWS], lane_s = SWAP ? ws : s[lane_row] * ws;
                if (!mbar_wait_warp(acc_full + 8 * buf, (it / BUFS) & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
                tc_fence_after();
                promote<SWAP, COLS>(acc, tmem_at + buf * N, s, lane_s, [&]() {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty + 8 * buf);
                });
            }
        }
        // ------------------------------ the tile's results ------------------------------
        if (M.split > 1) {
            cluster_wait();
            started = true;
            send_sums<SWAP, COLS>(acc, smem_addr(sums), share_of(N, M.split), rank, lane_row, half * COLS, 0, 1);
        } else if constexpr (SWAP) {
            const uint32_t r = wblock * FP8_BLOCK + lane_row;
            if (r < M.m) {
#pragma unroll
                for (uint32_t j = 0; j < COLS; ++j) {
                    if (row0 + j >= M.batch) break;
                    const int64_t at = (int64_t)(row0 + j) * M.ldy + r;
                    if (M.y_bf16) static_cast<__nv_bfloat16 *>(M.y)[at] = __float2bfloat16_rn(acc[j]);
                    else static_cast<float *>(M.y)[at] = acc[j];
                }
            }
        } else {
            // (all steps are over: the stages are free)
            store_rows<COLS>(M, acc, row0 + quad * 32, wblock * FP8_BLOCK + half * COLS, lane, after - M.stages * (STAGE / 4) + warp * TURN_FLOATS);
        }
    } else if (warp == PW) {
        // ------------------------------ operands by TMA ------------------------------
        if (lane == 0 && !M.skip_loads) {
            uint32_t stage = 0, use = 0;
            bool ok = true;
            for (uint32_t k = k_begin; k < k_end; ++k) {
                if (use > 0 && !mbar_wait(empty + 8 * stage, (use - 1) & 1u, abort_flag, M.status, M.wait_limit)) { ok = false; break; }
                const uint32_t bar = full + 8 * stage, at = stages_sa + stage * STAGE;
                mbar_expect_tx(bar, STAGE);
                tma_load_2d(at, &lane_map, bar, (int32_t)(k * KB), (int32_t)(tl * LANES));
                tma_load_2d(at + A_BYTES, &col_map, bar, (int32_t)(k * KB), (int32_t)(tc * N));
                if (++stage == M.stages) { stage = 0; ++use; }
            }
            // after a wait that gave up: copies in flight must land before the block's shared memory goes away
            if (!ok)
                for (uint32_t s = 0; s < M.stages; ++s) {
                    const uint32_t issued = use + (s < stage ? 1u : 0u);
                    if (issued) mbar_drain(full + 8 * s, (issued - 1) & 1u, M.wait_limit);
                }
        }
    } else {
        // ------------------------------ MMA issuer (a converged warp) ------------------------------
        const uint32_t idesc = instr_desc_fp8(128, N);
        const uint64_t desc0 = smem_desc_sw128(stages_sa);
        uint32_t stage = 0, parity = 0, it = 0;
        for (uint32_t k = k_begin; k < k_end; ++k, ++it) {
            const uint32_t buf = it % BUFS, use = it / BUFS;
            if (!mbar_wait_warp(full + 8 * stage, parity, abort_flag, M.status, M.wait_limit)) goto leave;
            if (use > 0 && !mbar_wait_warp(acc_empty + 8 * buf, (use - 1) & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
            tc_fence_after();
            const uint64_t a = desc0 + stage * (STAGE >> 4);
            mma_block(tmem_base + buf * N, a, a + (A_BYTES >> 4), idesc, empty + 8 * stage, acc_full + 8 * buf);
            if (++stage == M.stages) { stage = 0; parity ^= 1u; }
        }
        // The columns are given back before this CTA waits for others of its cluster, which may be waiting for columns themselves, on an SM that
        // another kernel shares.
        for (uint32_t buf = 0; buf < BUFS && buf < it; ++buf)
            if (!mbar_wait_warp(acc_empty + 8 * buf, ((it - buf + BUFS - 1) / BUFS - 1) & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
        tc_fence_after();
        tmem_dealloc(tmem_base, tmem_cols_of<N>);
        held = false;
    }
leave:
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*abort_flag) {                                           // (the same for all: nobody waits any more)
        if (warp == PW + 1 && held) {                            // tensor and shared memory must outlive the MMAs that were issued
            mma_commit(over);
            mbar_drain(over, 0, M.wait_limit);
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (warp == PW + 1 && held) tmem_dealloc(tmem_base, tmem_cols_of<N>);
    }
    if (M.split > 1) {
        if (!started) cluster_wait();
        if (tid < M.split) peer_store(peer_addr(smem_addr(given_up + rank), tid), __uint_as_float(*abort_flag));
        cluster_sync();                                          // all sums are here
        bool whole = true;                                       // a CTA whose wait gave up leaves the tile unwritten
        for (uint32_t q = 0; q < M.split; ++q) whole = whole && given_up[q] == 0;
        if (whole) add_sums<SWAP, N, threads_of_fp8<N>>(M, sums, share_of(N, M.split), rank, SWAP ? wblock * FP8_BLOCK : row0, SWAP ? row0 : wblock * FP8_BLOCK, tid);
    }
}

// Tiles of 256 batch rows by 256 weight rows, each by a pair of CTAs (ranks 2 p and 2 p + 1 of a cluster of `split` pairs): this one's 128 batch rows are its
// lanes; it loads them and 128 of the weights' rows.  The even CTA issues the MMAs of both; loads of both count on its barriers.
constexpr uint32_t PAIR_N = 256, PAIR_PW = 8, PAIR_BUFS = 2, PAIR_COLS = 128, PAIR_STAGE = 2 * LANES * KB, PAIR_THREADS = threads_of_fp8<PAIR_N>;
__global__ void __launch_bounds__(PAIR_THREADS, 1)
k_fp8_mm_pair(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const Fp8Args M)
{
    constexpr uint32_t PW = PAIR_PW, BUFS = PAIR_BUFS, COLS = PAIR_COLS, N = PAIR_N, THREADS = PAIR_THREADS;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * MAX_STAGES + 2 * BUFS + 2];
    __shared__ uint32_t tmem_slot, abort_word, given_up[8];
    volatile uint32_t *abort_flag = &abort_word;
    const uint32_t full = smem_addr(bars), empty = full + 8 * MAX_STAGES, acc_full = empty + 8 * MAX_STAGES, acc_empty = acc_full + 8 * BUFS;
    const uint32_t chunk_bar = acc_empty + 8 * BUFS, over = chunk_bar + 8;
    // [stages; after the last step: sums of the tile's CTAs][scales][for rows of Y off 16-byte boundaries]
    const uint32_t stages_sa = (smem_addr(smem_raw) + 1023u) & ~1023u;
    float *const sums = reinterpret_cast<float *>(smem_raw + (stages_sa - smem_addr(smem_raw)));
    Scales<false, N> sc;
    sc.buf = sums + M.stages * (PAIR_STAGE / 4);
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank(), part = rank >> 1, side = rank & 1, leader = rank & ~1u;
    const uint32_t first_tile = blockIdx.x / (2 * M.split), tile_step = gridDim.x / (2 * M.split);
    Sums<COLS> acc;
    const uint32_t k_begin = M.kblocks * part / M.split, k_end = M.kblocks * (part + 1) / M.split;
    const uint32_t k_first = k_begin & ~3u;

    if (warp == PW + 1) {
        tmem_alloc_pair(&tmem_slot, 512);
    } else if (warp == PW) {
        if (lane < M.stages) { mbar_init(full + 8 * lane, 1); mbar_init(empty + 8 * lane, 1); }
        if (lane < BUFS) { mbar_init(acc_full + 8 * lane, 1); mbar_init(acc_empty + 8 * lane, 2 * PW); }
        if (lane == 0) { mbar_init(chunk_bar, PW); mbar_init(over, 1); abort_word = 0; }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    launch_dependents();                                         // after the allocation: see k_gemv_tc
    cluster_sync();                                              // the barriers of all CTAs of the cluster are there
    wait_prior_grid();

    if (warp < PW) {
        // ------------------------------ scaling and adding up ------------------------------
        const uint32_t quad = warp & 3, half = warp >> 2, lane_row = quad * 32 + lane;
        const uint32_t tmem_at = tmem_base + ((quad * 32) << 16) + half * COLS, lead_empty = peer_addr(acc_empty, leader);
        uint32_t it = 0, chunk_no = 0;
        auto ask = [&](uint32_t tile, uint32_t k0) {
            const uint32_t tl = tile / M.col_tiles, tc = tile - tl * M.col_tiles;
            sc.fetch(M, tl * 256 + side * LANES, tc * (N / FP8_BLOCK), k0, k_end, tid);
        };
        ask(first_tile, k_first);
        for (uint32_t tile = first_tile; tile < M.tiles; tile += tile_step) {
            const uint32_t tl = tile / M.col_tiles, tc = tile - tl * M.col_tiles;
            acc.clear();
            for (uint32_t k0 = k_first; k0 < k_end; k0 += CHUNK, ++chunk_no) {
                sc.store(chunk_no & 1, tid);                     // (as in k_fp8_mm)
                __syncwarp();
                if (lane == 0) mbar_arrive(chunk_bar);
                if (!mbar_wait_warp(chunk_bar, chunk_no & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
                if (k0 + CHUNK < k_end) ask(tile, k0 + CHUNK);
                else if (tile + tile_step < M.tiles) ask(tile + tile_step, k_first);
                const uint32_t count = min(CHUNK, k_end - k0);
                for (uint32_t k = max(k0, k_begin) - k0; k < count; ++k, ++it) {
                    const uint32_t buf = it % BUFS;
                    const float *s = sc.at(chunk_no & 1, k);
                    const float lane_s = s[lane_row] * s[LANES + half];
                    if (!mbar_wait_warp(acc_full + 8 * buf, (it / BUFS) & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
                    tc_fence_after();
                    promote<false, COLS>(acc, tmem_at + buf * N, s, lane_s, [&]() {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) peer_arrive(lead_empty + 8 * buf);
                    });
                }
            }
            if (M.split == 1) store_rows<COLS>(M, acc, tl * 256 + side * LANES + quad * 32, tc * N + half * COLS, lane, sc.buf + Scales<false, N>::FLOATS + warp * TURN_FLOATS);
        }
    } else if (warp == PW) {
        // ------------------------------ operands by TMA ------------------------------
        if (lane == 0 && !M.skip_loads) {
            const uint32_t lead_full = peer_addr(full, leader);
            uint32_t stage = 0, use = 0;
            bool ok = true;
            for (uint32_t tile = first_tile; tile < M.tiles && ok; tile += tile_step) {
                const uint32_t tl = tile / M.col_tiles, tc = tile - tl * M.col_tiles;
                for (uint32_t k = k_begin; k < k_end; ++k) {
                    if (use > 0 && !mbar_wait(empty + 8 * stage, (use - 1) & 1u, abort_flag, M.status, M.wait_limit)) { ok = false; break; }
                    const uint32_t at = stages_sa + stage * PAIR_STAGE;
                    if (side == 0) mbar_expect_tx(full + 8 * stage, 2 * PAIR_STAGE);
                    tma_load_2d_pair(at, &x_map, lead_full + 8 * stage, (int32_t)(k * KB), (int32_t)(tl * 256 + side * LANES));
                    tma_load_2d_pair(at + PAIR_STAGE / 2, &w_map, lead_full + 8 * stage, (int32_t)(k * KB), (int32_t)(tc * N + side * LANES));
                    if (++stage == M.stages) { stage = 0; ++use; }
                }
            }
            // after a wait that gave up: copies in flight must land before the block's shared memory goes away.  (They count on the other CTA's barriers,
            // which need not complete any more: a millisecond is a thousand times what a copy takes.)
            if (!ok)
                for (const long long t0 = clock64(); clock64() - t0 < 2000000;) {}
        }
    } else if (warp == PW + 1 && side == 0) {
        // ------------------------------ MMA issuer (a converged warp of the even CTA) ------------------------------
        const uint32_t idesc = instr_desc_fp8(256, N), mask = 3u << leader;
        const uint64_t desc0 = smem_desc_sw128(stages_sa);
        uint32_t stage = 0, parity = 0, it = 0;
        for (uint32_t tile = first_tile; tile < M.tiles; tile += tile_step) {
            for (uint32_t k = k_begin; k < k_end; ++k, ++it) {
                const uint32_t buf = it % BUFS, use = it / BUFS;
                if (!mbar_wait_warp(full + 8 * stage, parity, abort_flag, M.status, M.wait_limit)) goto leave;
                if (use > 0 && !mbar_wait_warp(acc_empty + 8 * buf, (use - 1) & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
                tc_fence_after();
                const uint64_t a = desc0 + stage * (PAIR_STAGE >> 4);
                mma_block_pair(tmem_base + buf * N, a, a + (PAIR_STAGE / 2 >> 4), idesc, empty + 8 * stage, acc_full + 8 * buf, mask);
                if (++stage == M.stages) { stage = 0; parity ^= 1u; }
            }
        }
    }
leave:
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*abort_flag && side == 0) {                              // tensor and shared memory must outlive the MMAs that were issued
        if (warp == PW + 1) {
            commit_pair(over);
            mbar_drain(over, 0, M.wait_limit);
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    }
    if (M.split > 1 && tid < 2 * M.split) peer_store(peer_addr(smem_addr(given_up + rank), tid), __uint_as_float(*abort_flag));
    cluster_sync();                                              // all CTAs of the cluster are past their last step and their last signal
    if (M.split > 1) {                                           // one tile per cluster
        bool whole = true;                                       // a CTA whose wait gave up leaves the tile unwritten
        for (uint32_t q = 0; q < 2 * M.split; ++q) whole = whole && given_up[q] == 0;
        const uint32_t tl = first_tile / M.col_tiles, tc = first_tile - tl * M.col_tiles, share = share_of(N, M.split);
        if (whole && warp < PW) send_sums<false, COLS>(acc, stages_sa, share, part, (warp & 3) * 32 + lane, (warp >> 2) * COLS, side, 2);
        cluster_sync();                                          // all sums are here
        if (whole) add_sums<false, N, THREADS>(M, sums, share, part, tl * 256 + side * LANES, tc * N, tid);
    }
    if (warp == PW + 1) tmem_dealloc_pair(tmem_base, 512);
}

int launch_clusters(const void *kernel, const CUtensorMap &first, const CUtensorMap &second, const Fp8Args &M, uint32_t grid, uint32_t cluster, uint32_t threads,
                    size_t smem, cudaStream_t st)
{
    if (ensure_dynamic_smem(kernel, smem) != SQNN_OK) return SQNN_E_CUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    void *args[3] = {const_cast<CUtensorMap *>(&first), const_cast<CUtensorMap *>(&second), const_cast<Fp8Args *>(&M)};
    return cudaLaunchKernelExC(&cfg, kernel, args) == cudaSuccess ? SQNN_OK : SQNN_E_CUDA;
}

struct Operands {
    const void *w, *x;
    int64_t ldw, ldx;
    uint64_t n;
};

// How many clusters of each size run at once: asked for once per kernel and device.  (A table and no lock: a small product's kernel takes 3 us.)
struct AtOnce {
    std::atomic<uint32_t> known[64][9];
    uint32_t operator()(int dev, const void *kernel, uint32_t cluster, uint32_t threads, size_t smem)
    {
        uint32_t n = known[dev][cluster].load(std::memory_order_relaxed);
        if (n) return n;
        // (all of the SM's memory as shared memory: left to itself the runtime may set aside what one CTA needs)
        if (ensure_dynamic_smem(kernel, smem) != SQNN_OK ||
            cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess)
            return 0;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = cluster;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(cluster);
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int v = 0;
        if (cudaOccupancyMaxActiveClusters(&v, kernel, &cfg) != cudaSuccess || v <= 0) return 0;
        known[dev][cluster].store((uint32_t)v, std::memory_order_relaxed);
        return (uint32_t)v;
    }
};
template <bool SWAP, uint32_t N>
size_t smem_of(uint32_t split, uint32_t stages)
{
    const size_t sums = split > 1 ? (size_t)split * share_of(N, split) * LANES * 4 : 0;
    return 1024 + (size_t)stages * (LANES + N) * KB + Scales<SWAP, N>::FLOATS * sizeof(float) + sums;
}
template <bool SWAP, uint32_t N>
int launch_fp8(Fp8Args M, const Operands &O, uint32_t wanted, int dev, cudaStream_t st)
{
    constexpr uint32_t stages = 4;
    static AtOnce at_once;
    const uint32_t lane_rows = SWAP ? M.m : M.batch, col_rows = SWAP ? M.batch : M.m;
    const void *const kernel = reinterpret_cast<const void *>(k_fp8_mm<SWAP, N>);
    if (!M.quarters) {
        M.col_tiles = (col_rows + N - 1) / N;
        M.tiles = (lane_rows + LANES - 1) / LANES * M.col_tiles;
    }
    M.stages = stages;
    M.split = split_for(M.tiles, wanted, M.kblocks < 8 ? M.kblocks : 8,
                        [&](uint32_t s) {
                            const size_t smem = smem_of<SWAP, N>(s, stages);
                            return clusters_at_once(at_once(dev, kernel, s, threads_of_fp8<N>, smem), s, (uint32_t)sm_count(), ctas_per_sm(smem, tmem_cols_of<N>));
                        });
    CUtensorMap wmap, xmap;
    if (!byte_rows_map(&wmap, O.w, O.n, M.m, O.ldw, SWAP ? LANES : N) || !byte_rows_map(&xmap, O.x, O.n, M.batch, O.ldx, SWAP ? N : LANES)) return SQNN_E_CUDA;
    return launch_clusters(kernel, SWAP ? wmap : xmap, SWAP ? xmap : wmap, M, M.tiles * M.split, M.split, threads_of_fp8<N>,
                           smem_of<SWAP, N>(M.split, stages), st);
}

int launch_pair(Fp8Args M, const Operands &O, int dev, cudaStream_t st)
{
    static AtOnce known[2];                                      // (five and six stages)
    const void *const kernel = reinterpret_cast<const void *>(k_fp8_mm_pair);
    M.col_tiles = (M.m + PAIR_N - 1) / PAIR_N;
    M.tiles = (M.batch + 255) / 256 * M.col_tiles;
    M.stages = M.vec4 ? 6 : 5;
    const size_t smem = 1024 + (size_t)M.stages * PAIR_STAGE + Scales<false, PAIR_N>::FLOATS * sizeof(float) + (M.vec4 ? 0 : PAIR_PW * TURN_FLOATS * sizeof(float));
    const auto at_once = [&](uint32_t s) { return known[M.vec4](dev, kernel, 2 * s, threads_of_fp8<PAIR_N>, smem); };
    M.split = split_for(M.tiles, (uint32_t)sm_count() / 2 * 4 / 5, M.kblocks < 4 ? M.kblocks : 4, at_once);
    const uint32_t pairs = at_once(1);
    if (pairs == 0) return SQNN_E_CUDA;
    CUtensorMap wmap, xmap;
    if (!byte_rows_map(&wmap, O.w, O.n, M.m, O.ldw, LANES) || !byte_rows_map(&xmap, O.x, O.n, M.batch, O.ldx, LANES)) return SQNN_E_CUDA;
    // Tiles of a last round that would leave most pairs idle are done as quarters, a CTA or a cluster each, by a kernel of their own (us, without / with, in turn on
    // one chip: 4096 x 9216 batch 1300, 22 of 96 tiles, 78.1 / 68.2; 2560 x 4096 batch 2048, 6 of 80, 41.5 / 33.7; 34 of 256 tiles: 4096 x 9216 batch 4096 157.8 / 154.5,
    // 4096 x 16384 284 to 305 / 275 to 283; but 8192 x 1024 batch 2048 37 / 39, so short rows keep to two thirds of the SMs).
    const uint32_t last = M.split == 1 && M.tiles > pairs ? M.tiles % pairs : 0;
    const bool tail = last > 0 && 4 * last <= (M.kblocks < 64 ? (uint32_t)sm_count() * 2 / 3 : (uint32_t)sm_count());
    if (tail) M.tiles -= last;
    const uint32_t clusters = M.split > 1 || M.tiles < pairs ? M.tiles : pairs;
    const int rc = launch_clusters(kernel, xmap, wmap, M, clusters * 2 * M.split, 2 * M.split, threads_of_fp8<PAIR_N>, smem, st);
    if (rc != SQNN_OK || !tail) return rc;
    M.quarters = 1;
    M.first = M.tiles;
    M.tiles = 4 * last;
    return launch_fp8<false, 128>(M, O, (uint32_t)sm_count() * 4 / 5, dev, st);
}

int fp8_matmul_queue(uint64_t m, uint64_t n, uint32_t batch, const uint8_t *d_w, int64_t ldw, const float *d_w_scale, int64_t ldws,
                     const uint8_t *d_x, int64_t ldx, const float *d_x_scale, int64_t ldxs, void *d_y, int y_dtype, int64_t ldy,
                     uint32_t *d_status, cudaStream_t st)
{
    if (m == 0 || n == 0 || batch == 0 || !d_w || !d_w_scale || !d_x || !d_x_scale || !d_y) return SQNN_E_INVALID_ARG;
    if (y_dtype != SQNN_X_F32 && y_dtype != SQNN_X_BF16) return SQNN_E_INVALID_ARG;
    if (m > (1ull << 30) || n > (1ull << 30) || batch > (1u << 30)) return SQNN_E_UNSUPPORTED;
    const int64_t rows = (int64_t)m, cols = (int64_t)n, kblocks = (cols + FP8_BLOCK - 1) / FP8_BLOCK;
    if (ldw < cols || ldx < cols || ldws < kblocks || ldxs < kblocks || ldy < rows) return SQNN_E_INVALID_ARG;
    if (((uintptr_t)d_w_scale & 3) || ((uintptr_t)d_x_scale & 3) || ((uintptr_t)d_y & (y_dtype == SQNN_X_BF16 ? 1 : 3))) return SQNN_E_INVALID_ARG;
    if (((uintptr_t)d_w & 15) || ((uintptr_t)d_x & 15) || (ldw & 15) || (ldx & 15)) return SQNN_E_UNSUPPORTED;   // TMA: 16-byte base and pitch
    if (ldw >= (1ll << 40) || ldx >= (1ll << 40)) return SQNN_E_UNSUPPORTED;
    const DebugKnobs dbg = debug_knobs();
    Fp8Args M = {};
    M.ws = d_w_scale; M.xs = d_x_scale; M.y = d_y;
    M.ldws = ldws; M.ldxs = ldxs; M.ldy = ldy;
    M.m = (uint32_t)m; M.batch = batch; M.kblocks = (uint32_t)kblocks;
    M.y_bf16 = y_dtype == SQNN_X_BF16;
    M.vec = ((uintptr_t)d_y & 15) == 0 && (ldy * (M.y_bf16 ? 2 : 4)) % 16 == 0;
    M.skip_loads = (dbg.flags & 8u) ? 1u : 0u;
    M.wait_limit = dbg.wait_cycles ? dbg.wait_cycles : WAIT_LIMIT_CYCLES;
    M.status = d_status;
    M.vec4 = ((uintptr_t)d_y % (M.y_bf16 ? 8 : 16)) == 0 && ldy % 4 == 0;
    M.xs_vec = ((uintptr_t)d_x_scale & 15) == 0 && ldxs % 4 == 0;
    const Operands O{d_w, d_x, ldw, ldx, n};
    const uint64_t w_tiles = (m + LANES - 1) / LANES, x_tiles = ((uint64_t)batch + LANES - 1) / LANES;
    if (w_tiles * x_tiles > 0x7fffffffull / 8) return SQNN_E_UNSUPPORTED;
    const uint32_t sms = (uint32_t)sm_count();
    // Small batches: a quarter more CTAs than SMs keep enough weights on their way; those with more columns are one to an SM.  The pair's larger
    // tiles gain from about as many 128 x 128 tiles on as there are SMs (us, pair / one CTA per tile, in turn on one chip: 4096 x 16384 batch 512 42.5 / 48.0, 8192 x
    // 1024 batch 2048 35.4 / 40.3, 4096 x 9216 batch 4096 155 / 187; 6000 x 3000 batch 200 17.0 / 11.6, 2048 x 2048 batch 256 14.6 / 9.8).
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SQNN_E_CUDA;
    if (batch <= 16) return launch_fp8<true, 16>(M, O, sms * 5 / 4, dev, st);
    if (batch <= 32) return launch_fp8<true, 32>(M, O, sms * 5 / 4, dev, st);
    if (batch <= 64) return launch_fp8<true, 64>(M, O, sms * 4 / 5, dev, st);
    if (batch <= 128 || m <= 128 || w_tiles * x_tiles < sms * 4 / 5) return launch_fp8<false, 128>(M, O, sms * 4 / 5, dev, st);
    return launch_pair(M, O, dev, st);
}

}  // namespace
}  // namespace sqnn

extern "C" int sqnn_fp8_matmul(uint64_t m, uint64_t n, uint32_t batch, const uint8_t *d_w, int64_t ldw, const float *d_w_scale,
                               int64_t ldws, const uint8_t *d_x, int64_t ldx, const float *d_x_scale, int64_t ldxs, void *d_y,
                               int y_dtype, int64_t ldy, uint32_t *d_status, void *cuda_stream)
{
    sqnn::ApiScope scope("sqnn_fp8_matmul");
    return scope.finish(sqnn::fp8_matmul_queue(m, n, batch, d_w, ldw, d_w_scale, ldws, d_x, ldx, d_x_scale, ldxs, d_y, y_dtype, ldy,
                                               d_status, (cudaStream_t)cuda_stream),
                        d_status, (cudaStream_t)cuda_stream);
}
