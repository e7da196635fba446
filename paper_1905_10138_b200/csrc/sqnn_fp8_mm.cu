// Product of 8-bit weights with a scale per 128 x 128 block and 8-bit activations with a scale per row and 128 columns.
//
//   Y[b][r] = sum_k sx[b][k] sw[r / 128][k] sum_{c in block k} W[r][c] X[b][c]
//
// The inner sums run on tcgen05.mma (kind::f8f6f4, fp32 accumulators in tensor memory), one block k of 128 columns at a time; the
// scales differ from block to block, so each block's sums are read back, scaled and added to a 32-bit accumulator in registers while
// the tensor cores work on the next blocks in other columns of tensor memory.
//
// Two forms, by who lies along the 128 lanes:
//   - small batches (SWAP): the weights' rows are the lanes, the batch the 16 to 64 columns.  Bound by reading the weights.  A lane's
//     weights share one scale (its block of 128 rows), the activations' scales go by column.
//   - else the batch's rows are the lanes and 128 or 256 weight rows the columns: a lane has one scale per block.
// Few tiles: the CTAs of a cluster share one, each taking a range of the blocks k, and add their accumulators up through
// distributed shared memory in the order of their rank.  No workspace, no atomics: results are the same from run to run.
#include "sqnn_launch.h"
#include "sqnn_fp8.cuh"
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
    uint32_t stages;
    uint32_t y_bf16, vec;         // vec: rows of Y on 16-byte boundaries
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
                 " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n"
                 " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n}\n"
                 :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(free_stage), "r"(acc_full) : "memory");
#undef SQNN_MMA
}
// Instruction descriptor: D fp32, A and B e4m3, both K-major, M = 128, N = n.
SQNN_DEV uint32_t instr_desc_fp8(uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((128u >> 4) << 24); }

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
SQNN_DEV float2 unpair(uint64_t v)
{
    float2 f;
    asm("mov.b64 {%0, %1}, %2;\n" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}

SQNN_DEV uint32_t bf16x2(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return reinterpret_cast<const uint32_t &>(b);
}
// Four neighbouring elements of a row of Y, as many of them as `room` allows.
SQNN_DEV void put4(const Fp8Args &M, int64_t at, uint32_t room, const float4 &v)
{
    if (M.vec && room >= 4) {
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

template <uint32_t N> constexpr uint32_t promoters_of = N >= 128 ? 8 : 4;   // warps that scale and add: four per 128 lanes and half of the columns
template <uint32_t N> constexpr uint32_t buffers_of = N == 256 ? 2 : 4;     // accumulators in tensor memory
template <uint32_t N> constexpr uint32_t tmem_cols_of = N * buffers_of<N>;  // 64 to 512: a power of two
template <uint32_t N> constexpr uint32_t threads_of_fp8 = promoters_of<N> * 32 + 64;
constexpr uint32_t scale_floats(bool swap, uint32_t n) { return 2 * CHUNK * (swap ? n + 4 : LANES + 4); }

// Scales of CHUNK blocks in shared memory, double-buffered: by lane or column, then those of the weights' blocks of rows.
template <bool SWAP, uint32_t N>
struct Scales {
    static constexpr uint32_t ROWS = SWAP ? N : LANES, PITCH = ROWS + 4, WBLOCKS = N == 256 ? 2 : 1;
    float *buf;                   // [2][CHUNK][PITCH]
    // queues the copies of blocks [k0, k0 + CHUNK), those below k1
    SQNN_DEV void fetch(const Fp8Args &M, uint32_t which, uint32_t row0, uint32_t wblock, uint32_t k0, uint32_t k1, uint32_t tid, uint32_t threads) const
    {
        float *b = buf + which * CHUNK * PITCH;
        for (uint32_t i = tid; i < ROWS * CHUNK; i += threads) {
            const uint32_t row = i / CHUNK, k = i % CHUNK;
            if (row0 + row < M.batch && k0 + k < k1) cp_async4(b + k * PITCH + row, M.xs + (int64_t)(row0 + row) * M.ldxs + (k0 + k));
        }
        if (tid < CHUNK * WBLOCKS) {
            const uint32_t j = tid / CHUNK, k = tid % CHUNK;
            if ((wblock + j) * FP8_BLOCK < M.m && k0 + k < k1) cp_async4(b + k * PITCH + ROWS + j, M.ws + (int64_t)(wblock + j) * M.ldws + (k0 + k));
        }
        cp_async_commit();
    }
    SQNN_DEV const float *at(uint32_t which, uint32_t k) const { return buf + (which * CHUNK + k) * PITCH; }
};

template <bool SWAP, uint32_t N>
__global__ void __launch_bounds__(threads_of_fp8<N>, 1)
k_fp8_mm(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap col_map, const Fp8Args M)
{
    constexpr uint32_t PW = promoters_of<N>, BUFS = buffers_of<N>, COLS = N * 4 / PW;     // COLS: columns per promoting thread
    constexpr uint32_t A_BYTES = LANES * KB, B_BYTES = N * KB, STAGE = A_BYTES + B_BYTES;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * MAX_STAGES + 2 * 4 + 2];
    __shared__ uint32_t tmem_slot, abort_word;
    volatile uint32_t *abort_flag = &abort_word;
    const uint32_t full = smem_addr(bars), empty = full + 8 * MAX_STAGES, acc_full = empty + 8 * MAX_STAGES, acc_empty = acc_full + 8 * 4;
    const uint32_t chunk_bar = acc_empty + 8 * 4, over = chunk_bar + 8;   // scales are there; after a timeout: the MMAs are over
    const uint32_t stages_sa = (smem_addr(smem_raw) + 1023u) & ~1023u;
    float *const parts = reinterpret_cast<float *>(smem_raw + (stages_sa - smem_addr(smem_raw)));   // after the last step: partial sums
    const Scales<SWAP, N> sc{parts + M.stages * STAGE / 4};
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = M.split > 1 ? cluster_rank() : 0, first_tile = blockIdx.x / M.split, tile_step = gridDim.x / M.split;
    const uint32_t k_begin = (uint32_t)((uint64_t)M.kblocks * rank / M.split), k_end = (uint32_t)((uint64_t)M.kblocks * (rank + 1) / M.split);

    if (warp == PW + 1) {
        tmem_alloc(&tmem_slot, tmem_cols_of<N>);
    } else if (warp == PW) {
        if (lane < M.stages) { mbar_init(full + 8 * lane, 1); mbar_init(empty + 8 * lane, 1); }
        if (lane < BUFS) { mbar_init(acc_full + 8 * lane, 1); mbar_init(acc_empty + 8 * lane, PW); }
        if (lane == 0) { mbar_init(chunk_bar, PW); mbar_init(over, 1); abort_word = 0; }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    launch_dependents();                                         // after the allocation: see k_gemv_tc
    wait_prior_grid();

    if (warp < PW) {
        // ------------------------------ scaling and adding up ------------------------------
        const uint32_t quad = warp & 3, half = warp >> 2, lane_row = quad * 32 + lane;
        const uint32_t tmem_at = tmem_base + ((quad * 32) << 16) + half * COLS;
        uint32_t it = 0, chunk_no = 0;
        // tile -> first batch row of its scales, first block of weight rows
        auto rows_of = [&](uint32_t tile, uint32_t &row0, uint32_t &wblock) {
            const uint32_t tl = tile / M.col_tiles, tc = tile - tl * M.col_tiles;
            row0 = SWAP ? tc * N : tl * LANES;
            wblock = SWAP ? tl : tc * (N / FP8_BLOCK);
        };
        if (first_tile < M.tiles) {
            uint32_t row0, wblock;
            rows_of(first_tile, row0, wblock);
            sc.fetch(M, 0, row0, wblock, k_begin, k_end, tid, PW * 32);
        }
        for (uint32_t tile = first_tile; tile < M.tiles; tile += tile_step) {
            uint64_t acc[COLS / 2];
#pragma unroll
            for (uint32_t j = 0; j < COLS / 2; ++j) acc[j] = 0ull;
            uint32_t row0, wblock;
            rows_of(tile, row0, wblock);
            for (uint32_t k0 = k_begin; k0 < k_end; k0 += CHUNK, ++chunk_no) {
                // this chunk is there and the one before done with, for all of these warps (a bounded wait: a plain barrier would keep
                // a warp for good once another one has given up)
                cp_async_wait_all();
                __syncwarp();
                if (lane == 0) mbar_arrive(chunk_bar);
                if (!mbar_wait_warp(chunk_bar, chunk_no & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
                if (k0 + CHUNK < k_end) {
                    sc.fetch(M, (chunk_no + 1) & 1, row0, wblock, k0 + CHUNK, k_end, tid, PW * 32);
                } else if (tile + tile_step < M.tiles) {
                    uint32_t r, w;
                    rows_of(tile + tile_step, r, w);
                    sc.fetch(M, (chunk_no + 1) & 1, r, w, k_begin, k_end, tid, PW * 32);
                }
                const uint32_t count = min(CHUNK, k_end - k0);
                for (uint32_t k = 0; k < count; ++k, ++it) {
                    const uint32_t buf = it % BUFS;
                    const float *s = sc.at(chunk_no & 1, k);
                    const float ws = s[Scales<SWAP, N>::ROWS + (SWAP ? 0 : half * COLS / FP8_BLOCK)];
                    const float lane_s = SWAP ? ws : s[lane_row] * ws;
                    if (!mbar_wait_warp(acc_full + 8 * buf, (it / BUFS) & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
                    tc_fence_after();
                    if constexpr (COLS >= 32) {
#pragma unroll
                        for (uint32_t c = 0; c < COLS; c += 32) {
                            uint32_t d[32];
                            tmem_ld32(tmem_at + buf * N + c, d);
#pragma unroll
                            for (uint32_t j = 0; j < 16; ++j) {
                                uint64_t f;
                                if constexpr (SWAP) {
                                    const float2 x = *reinterpret_cast<const float2 *>(s + c + 2 * j);
                                    f = pair(x.x * lane_s, x.y * lane_s);
                                } else {
                                    f = pair(lane_s, lane_s);
                                }
                                fma2(acc[c / 2 + j], d[2 * j], d[2 * j + 1], f);
                            }
                        }
                    } else {
                        uint32_t d[16];
                        tmem_ld16(tmem_at + buf * N, d);
#pragma unroll
                        for (uint32_t j = 0; j < 8; ++j) {
                            const float2 x = *reinterpret_cast<const float2 *>(s + 2 * j);
                            fma2(acc[j], d[2 * j], d[2 * j + 1], pair(x.x * lane_s, x.y * lane_s));
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty + 8 * buf);
                }
            }
            // ------------------------------ the tile's results ------------------------------
            if (M.split > 1) {                                   // one tile per cluster: to shared memory, summed below
                if constexpr (SWAP) {
#pragma unroll
                    for (uint32_t j = 0; j < COLS / 2; ++j) {
                        const float2 v = unpair(acc[j]);
                        parts[(2 * j) * LANES + lane_row] = v.x;
                        parts[(2 * j + 1) * LANES + lane_row] = v.y;
                    }
                } else {
                    float *p = parts + lane_row * (N + 4) + half * COLS;
#pragma unroll
                    for (uint32_t j = 0; j < COLS / 2; j += 2) {
                        const float2 u = unpair(acc[j]), v = unpair(acc[j + 1]);
                        *reinterpret_cast<float4 *>(p + 2 * j) = make_float4(u.x, u.y, v.x, v.y);
                    }
                }
            } else if constexpr (SWAP) {
                const uint32_t r = wblock * FP8_BLOCK + lane_row;
                if (r < M.m) {
#pragma unroll
                    for (uint32_t j = 0; j < COLS / 2; ++j) {
                        const float2 v = unpair(acc[j]);
                        const uint32_t b = row0 + 2 * j;
                        const int64_t at = (int64_t)b * M.ldy + r;
                        if (M.y_bf16) {
                            if (b < M.batch) static_cast<__nv_bfloat16 *>(M.y)[at] = __float2bfloat16_rn(v.x);
                            if (b + 1 < M.batch) static_cast<__nv_bfloat16 *>(M.y)[at + M.ldy] = __float2bfloat16_rn(v.y);
                        } else {
                            if (b < M.batch) static_cast<float *>(M.y)[at] = v.x;
                            if (b + 1 < M.batch) static_cast<float *>(M.y)[at + M.ldy] = v.y;
                        }
                    }
                }
            } else if (row0 + lane_row < M.batch) {
                const uint32_t r0 = wblock * FP8_BLOCK + half * COLS;
                const int64_t at = (int64_t)(row0 + lane_row) * M.ldy + r0;
#pragma unroll
                for (uint32_t j = 0; j < COLS / 2; j += 2) {
                    const float2 u = unpair(acc[j]), v = unpair(acc[j + 1]);
                    if (r0 + 2 * j < M.m) put4(M, at + 2 * j, M.m - (r0 + 2 * j), make_float4(u.x, u.y, v.x, v.y));
                }
            }
        }
    } else if (warp == PW) {
        // ------------------------------ operands by TMA ------------------------------
        if (lane == 0 && !M.skip_loads) {
            uint32_t stage = 0, use = 0;
            bool ok = true;
            for (uint32_t tile = first_tile; tile < M.tiles && ok; tile += tile_step) {
                const uint32_t tl = tile / M.col_tiles, tc = tile - tl * M.col_tiles;
                for (uint32_t k = k_begin; k < k_end; ++k) {
                    if (use > 0 && !mbar_wait(empty + 8 * stage, (use - 1) & 1u, abort_flag, M.status, M.wait_limit)) { ok = false; break; }
                    const uint32_t bar = full + 8 * stage, at = stages_sa + stage * STAGE;
                    mbar_expect_tx(bar, STAGE);
                    tma_load_2d(at, &lane_map, bar, (int32_t)(k * KB), (int32_t)(tl * LANES));
                    tma_load_2d(at + A_BYTES, &col_map, bar, (int32_t)(k * KB), (int32_t)(tc * N));
                    if (++stage == M.stages) { stage = 0; ++use; }
                }
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
        const uint32_t idesc = instr_desc_fp8(N);
        const uint64_t desc0 = smem_desc_sw128(stages_sa);
        uint32_t stage = 0, parity = 0, it = 0;
        for (uint32_t tile = first_tile; tile < M.tiles; tile += tile_step) {
            for (uint32_t k = k_begin; k < k_end; ++k, ++it) {
                const uint32_t buf = it % BUFS, use = it / BUFS;
                if (use > 0 && !mbar_wait_warp(acc_empty + 8 * buf, (use - 1) & 1u, abort_flag, M.status, M.wait_limit)) goto leave;
                if (!mbar_wait_warp(full + 8 * stage, parity, abort_flag, M.status, M.wait_limit)) goto leave;
                tc_fence_after();
                const uint64_t a = desc0 + stage * (STAGE >> 4);
                mma_block(tmem_base + buf * N, a, a + (A_BYTES >> 4), idesc, empty + 8 * stage, acc_full + 8 * buf);
                if (++stage == M.stages) { stage = 0; parity ^= 1u; }
            }
        }
    }
leave:
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*abort_flag) {                                           // (the same for all: nobody waits any more)
        if (warp == PW + 1) {                                    // tensor and shared memory must outlive the MMAs that were issued
            mma_commit(over);
            mbar_drain(over, 0, M.wait_limit);
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    }
    if (warp == PW + 1) tmem_dealloc(tmem_base, tmem_cols_of<N>);
    if (M.split > 1) {
        cluster_sync();
        // each CTA adds up its share of the tile; a CTA whose wait gave up leaves the tile unwritten
        bool whole = true;
        const uint32_t parts_sa = stages_sa, abort_sa = smem_addr(&abort_word);
        for (uint32_t q = 0; q < M.split; ++q) whole = whole && peer_load(peer_addr(abort_sa, q)) == 0;
        if (whole && first_tile < M.tiles) {
            const uint32_t tl = first_tile / M.col_tiles, tc = first_tile - tl * M.col_tiles;
            constexpr uint32_t FOURS = LANES * N / 4;
            const uint32_t f1 = FOURS * (rank + 1) / M.split;
            for (uint32_t f = FOURS * rank / M.split + tid; f < f1; f += threads_of_fp8<N>) {
                const uint32_t b = SWAP ? f / (LANES / 4) : f / (N / 4), r = 4 * (SWAP ? f % (LANES / 4) : f % (N / 4));
                const uint32_t at = parts_sa + 4 * (SWAP ? b * LANES + r : b * (N + 4) + r);
                float4 sum = peer_load4(peer_addr(at, 0));
                for (uint32_t q = 1; q < M.split; ++q) {
                    const float4 v = peer_load4(peer_addr(at, q));
                    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                }
                const uint32_t row = (SWAP ? tc * N : tl * LANES) + b, col = (SWAP ? tl * LANES : tc * N) + r;
                if (row < M.batch && col < M.m) put4(M, (int64_t)row * M.ldy + col, M.m - col, sum);
            }
        }
        cluster_sync();                                          // nobody leaves while others read its shared memory
    }
}

// Raises nothing when it fails; `rows` x n bytes with `ld` bytes from row to row, boxes of `box_rows` x 128 bytes, swizzled.
bool make_map(CUtensorMap *map, const void *p, uint64_t n, uint64_t rows, int64_t ld, uint32_t box_rows)
{
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return false;
    const cuuint64_t gdim[2] = {(cuuint64_t)n, (cuuint64_t)rows};
    const cuuint64_t gstride[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {KB, box_rows};
    const cuuint32_t estride[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(p), gdim, gstride, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool SWAP, uint32_t N>
int launch_fp8(Fp8Args M, const void *w, int64_t ldw, const void *x, int64_t ldx, uint64_t n, uint32_t split, size_t budget, cudaStream_t st)
{
    constexpr uint32_t STAGE = (LANES + N) * KB;
    const uint32_t lane_rows = SWAP ? M.m : M.batch, col_rows = SWAP ? M.batch : M.m;
    M.col_tiles = (col_rows + N - 1) / N;
    M.tiles = (lane_rows + LANES - 1) / LANES * M.col_tiles;
    M.split = split;
    const size_t scales = scale_floats(SWAP, N) * sizeof(float);
    const size_t room = budget - 1024 - scales;
    M.stages = (uint32_t)(room / STAGE < MAX_STAGES ? room / STAGE : MAX_STAGES);
    const size_t smem = 1024 + (size_t)M.stages * STAGE + scales;
    CUtensorMap wmap, xmap;
    if (!make_map(&wmap, w, n, M.m, ldw, SWAP ? LANES : N) || !make_map(&xmap, x, n, M.batch, ldx, SWAP ? N : LANES)) return SQNN_E_CUDA;
    auto kernel = k_fp8_mm<SWAP, N>;
    if (ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), smem) != SQNN_OK) return SQNN_E_CUDA;
    const uint32_t sms = (uint32_t)sm_count();
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split > 1 ? M.tiles * split : M.tiles < sms ? M.tiles : sms);
    cfg.blockDim = dim3(threads_of_fp8<N>);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, SWAP ? wmap : xmap, SWAP ? xmap : wmap, M) == cudaSuccess ? SQNN_OK : SQNN_E_CUDA;
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
    const uint32_t sms = (uint32_t)sm_count();
    const uint64_t lane_tiles_w = (m + LANES - 1) / LANES;
    auto split_for = [&](uint64_t tiles, uint64_t slots) {
        uint64_t s = tiles ? slots / tiles : 1;
        if (s > 8) s = 8;
        if (s > (uint64_t)kblocks) s = (uint64_t)kblocks;
        return (uint32_t)(s < 1 ? 1 : s);
    };
    constexpr size_t HALF = 112 * 1024, WHOLE = 224 * 1024;
    if (batch <= 64) {
        const uint32_t split = split_for(lane_tiles_w, 2 * sms);
        if (batch <= 16) return launch_fp8<true, 16>(M, d_w, ldw, d_x, ldx, n, split, HALF, st);
        if (batch <= 32) return launch_fp8<true, 32>(M, d_w, ldw, d_x, ldx, n, split, HALF, st);
        return launch_fp8<true, 64>(M, d_w, ldw, d_x, ldx, n, split, HALF, st);
    }
    const uint64_t lane_tiles = ((uint64_t)batch + LANES - 1) / LANES, wide = lane_tiles * ((m + 255) / 256), narrow = lane_tiles * lane_tiles_w;
    if (wide > 0x7fffffffull || narrow > 0x7fffffffull) return SQNN_E_UNSUPPORTED;
    if (wide >= sms) return launch_fp8<false, 256>(M, d_w, ldw, d_x, ldx, n, 1, WHOLE, st);
    return launch_fp8<false, 128>(M, d_w, ldw, d_x, ldx, n, split_for(narrow, sms), WHOLE, st);
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
