// e4m3 operands with a scale for each block of 128: their quantisation and the dense layer over them.
#include <cuda_runtime.h>
#include <cuda.h>
#include <cstring>
#include <type_traits>
#include "tt_ptx.cuh"
#include "tt_f8.cuh"

namespace tt {

// ---- quantisation ---------------------------------------------------------------------------------------------------------
//
// s = 2^ceil(log2(max |x| / 448)) comes from the bits of the maximum, x / s is a product with the power 1 / s, so the only rounding is the
// one to e4m3.  Bound by memory: every value is read once and kept in registers between the maximum and the conversion.
// (8192 x 4096 in 16 bits: 19.0 us, 5.3 TB/s, 0.82 of a copy's rate.  A row: 2.5 to 2.8 us, the rate of launches.)

// Rows of activations: a warp has one block of columns of eight rows, of four at a time, so that the scales of a block come out side by side.  Eight
// lanes have a row's block, 8 values of either half each (a warp's loads are whole lines).
template <int TYPE>
__global__ void __launch_bounds__(256) tt_quantize_rows_kernel(const tt_quantize_args a, int blocks, long long tasks) {
    pdl_allow_next();
    pdl_wait_prev();
    const int lane = threadIdx.x & 31;
    const long long task = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (task >= tasks) return;
    typedef typename Element<TYPE>::type T;
    const long long row8 = task / blocks;
    const int block = (int)(task - row8 * blocks), c = block * 128 + 8 * (lane & 7);
    const long long row0 = row8 * 8 + (lane >> 3);
    Eights<TYPE, 2> v[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (row0 + 4 * u < a.m) v[u].load(static_cast<const T*>(a.x) + (row0 + 4 * u) * a.x_row, c, 64, a.kk, true);
        else v[u].zero();
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const long long row = row0 + 4 * u;
        float most = v[u].most();
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) most = __uint_as_float(max(__float_as_uint(most), __float_as_uint(__shfl_xor_sync(0xffffffffu, most, d))));      // (NaN is the largest)
        const bool finite = most < INFINITY;
        if (__any_sync(0xffffffffu, !finite)) {
            most = v[u].finite_most();
#pragma unroll
            for (int d = 4; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        }
        const float s = power_scale(most), inv = power_inverse(s);
        if (row >= a.m) continue;
        uint8_t* q = static_cast<uint8_t*>(a.q) + row * a.q_row;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint2 w = finite ? v[u].template bytes<true>(h, inv) : v[u].template bytes<false>(h, inv);
            const int at = c + 64 * h;
            if (at + 8 <= a.kk) *reinterpret_cast<uint2*>(q + at) = w;
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (at + i < a.kk) q[at + i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
            }
        }
        if ((lane & 7) == 0) a.scales[block * a.s_block + row * a.s_row] = s;
    }
}

// The same where rows do not start on 16 bytes: a lane has every 32nd value of a row's block, so that a warp's loads and stores are whole lines here
// too.  (6012 x 287 in 32 bits: 5.2 us; by eight values a lane, one at a time, 10.9.)
template <int TYPE>
__global__ void __launch_bounds__(256) tt_quantize_lines_kernel(const tt_quantize_args a, int blocks, long long tasks) {
    pdl_allow_next();
    pdl_wait_prev();
    const int lane = threadIdx.x & 31;
    const long long task = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const long long row0 = task / blocks * 8;
    const int block = (int)(task - row0 / 8 * blocks), c = block * 128 + lane, rows = (int)min((long long)a.m - row0, 8ll);
    // As they lie in memory, all under way at once.  16-bit loads that are left out one by one become branches, which wait for each other (8191 x
    // 4095: 83 us), so behind the last column and row it is the last one's value again, which leaves the maximum as it is (36).
    typedef typename std::conditional<TYPE == TT_TYPE_F32, uint32_t, uint16_t>::type Bits;
    const Bits* x = static_cast<const Bits*>(a.x) + row0 * a.x_row;
    uint32_t raw[8][4];
#pragma unroll
    for (int r = 0; r < 8; x += ++r < rows || TYPE == TT_TYPE_F32 ? a.x_row : 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (TYPE == TT_TYPE_F32) raw[r][j] = r < rows && c + 32 * j < a.kk ? x[c + 32 * j] : 0u;
            else raw[r][j] = x[min(c + 32 * j, a.kk - 1)];
        }
    uint8_t* q = static_cast<uint8_t*>(a.q) + row0 * a.q_row + c;
#pragma unroll
    for (int r = 0; r < 8; ++r, q += a.q_row) {
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (TYPE == TT_TYPE_F32) v[j] = __uint_as_float(raw[r][j]);
            else v[j] = up2<TYPE>(raw[r][j]).x;
        }
        float most = finite_max(finite_max(finite_max(finite_max(0.f, v[0]), v[1]), v[2]), v[3]);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        const float s = power_scale(most), inv = power_inverse(s);
        if (r >= rows) continue;
        const uint32_t w = to_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
#pragma unroll
        for (int j = 0; j < 4; ++j) if (c + 32 * j < a.kk) q[32 * j] = (uint8_t)(w >> (8 * j));
        if (lane == r) a.scales[block * a.s_block + (row0 + r) * a.s_row] = s;
    }
}

// Blocks of 128 x 128: a CTA each, a thread has 8 columns of every sixteenth row.  (4096 x 4096 in 16 bits: 11.7 us; weights are quantised once.)
template <int TYPE>
__global__ void __launch_bounds__(256) tt_quantize_blocks_kernel(const tt_quantize_args a, int blocks, int wide) {
    __shared__ float warp_most[8];
    pdl_allow_next();
    pdl_wait_prev();
    typedef typename Element<TYPE>::type T;
    const int rb = (int)blockIdx.x / blocks, kb = (int)blockIdx.x - rb * blocks;
    const int c = kb * 128 + 8 * ((int)threadIdx.x & 15), r0 = rb * 128 + ((int)threadIdx.x >> 4);
    float v[8][8], most = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = r0 + 16 * j;
        const T* x = static_cast<const T*>(a.x) + (long long)r * a.x_row;
        if (r < a.m && wide && c + 8 <= a.kk) load_wide<TYPE, 8>(x + c, v[j]);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = r < a.m && c + i < a.kk ? Element<TYPE>::up(x[c + i]) : 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) most = finite_max(most, v[j][i]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if ((threadIdx.x & 31) == 0) warp_most[threadIdx.x >> 5] = most;
    __syncthreads();
    most = warp_most[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) most = fmaxf(most, warp_most[w]);
    const float s = power_scale(most), inv = power_inverse(s);
    if (threadIdx.x == 0) a.scales[(long long)kb * a.s_block + (long long)rb * a.s_row] = s;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = r0 + 16 * j;
        if (r >= a.m || c >= a.kk) continue;
        uint8_t* q = static_cast<uint8_t*>(a.q) + (long long)r * a.q_row;
        const uint32_t lo = to_e4m3x4(v[j][0] * inv, v[j][1] * inv, v[j][2] * inv, v[j][3] * inv);
        const uint32_t hi = to_e4m3x4(v[j][4] * inv, v[j][5] * inv, v[j][6] * inv, v[j][7] * inv);
        if (wide && c + 8 <= a.kk) *reinterpret_cast<uint2*>(q + c) = make_uint2(lo, hi);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (c + i < a.kk) q[c + i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
        }
    }
}

// ---- the dense layer ------------------------------------------------------------------------------------------------------
//
// D[128 rows, TN] = A B^T by tcgen05.mma kind::f8f6f4 over one block of 128 columns at a time (four steps of 32), each block into the next of
// the accumulators in tensor memory.  The read-out warps take a block's sums, multiply them by its scales and add them up in registers, in 32
// bits, while the tensor core is at the following blocks: the scales may be any values, and no sum is longer than 128 before it
// is added in full precision.
//
// Rows on the 128 lanes are the tokens, or (SWAP) the weights' rows where there are too few tokens to fill them.  `split` CTAs of
// a cluster share a tile's blocks where there are fewer tiles than SMs, leave their sums in shared memory and add up a band of columns each,
// in the order of the splits.  (8 x 4096 x 4096: 5.8 us, 2.9 TB/s with the launch, whose own share is 3 us; 333 x 1000 x 1960: 9.2 us.)

struct DenseF8 {
    const float* a_scale; long long as_row, as_block;     // of operand A's rows (normal: per row, SWAP: per 128 rows)
    const float* b_scale; long long bs_row, bs_block;
    const float* bias; void* y; long long y_row;
    unsigned* status;
    int rows_a, rows_b, blocks, blocks_per_split, split, stages, tiles_a;
    int y_type, act, wide;
    int tiles;                                              // pairs: of 256 x TN
    unsigned idesc;
    unsigned long long wait_ns;
};

constexpr int kF8Threads = 320;                            // warp 0 TMA, warp 1 MMA + tensor memory, warps 2-9 read-out
constexpr unsigned kF8TileA = 128 * 128;
constexpr int kF8MaxStages = 8;
constexpr int kHalfSm = 113 * 1024;

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* tmap, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// apply_act, but for NaN, which stays NaN (a NaN operand is to show).
__device__ __forceinline__ float activate(float v, int act) {
    if (act == TT_ACT_GELU_ERF) return gelu_erf(v);
    if (act != TT_ACT_NONE) v = v < 0.f ? 0.f : v;
    return act == TT_ACT_RELU6 && v > 6.f ? 6.f : v;
}

template <int TN, bool SWAP>
__global__ void __launch_bounds__(kF8Threads, SWAP ? 2 : 1)
tt_dense_f8_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const DenseF8 g) {
    constexpr int kBufs = 512 / TN < 4 ? 512 / TN : 4;     // accumulators
    constexpr int kCols = TN / 2;                          // columns of a read-out warp
    constexpr uint32_t kStage = kF8TileA + TN * 128u;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kF8MaxStages], empty_bar[kF8MaxStages], acc_full[kBufs], acc_empty[kBufs], drained, red_bar;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int* abortp = &abort_flag;
    const int tile_a = (int)blockIdx.x % g.tiles_a, tile_b = (int)blockIdx.x / g.tiles_a;
    const int kb0 = (int)blockIdx.z * g.blocks_per_split, kb1 = min(g.blocks, kb0 + g.blocks_per_split);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // what a CTA of a cluster of `split` adds up in the end: a band of lines of the tile, SWAP: a column of 128 rows each, else a row of TN columns (+ 4)
    constexpr uint32_t kLine = SWAP ? 512u : (TN + 4) * 4u;
    constexpr int kLines = SWAP ? TN : 128;
    const int per = kLines / g.split;
    const uint32_t band_bytes = (uint32_t)per * kLine, landing = base + (uint32_t)g.stages * kStage;
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_b) : "memory");
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < g.stages; ++i) { mbar_init(smem_u32(&full_bar[i]), 1u); mbar_init(smem_u32(&empty_bar[i]), 1u); }
        for (int i = 0; i < kBufs; ++i) { mbar_init(smem_u32(&acc_full[i]), 1u); mbar_init(smem_u32(&acc_empty[i]), 8u); }
        mbar_init(smem_u32(&drained), 1u);
        mbar_init(smem_u32(&red_bar), 1u);
        abort_flag = 0;
        fence_mbar_init();
        if (g.split > 1) mbar_expect_tx(smem_u32(&red_bar), (uint32_t)(g.split - 1) * band_bytes);
        fence_proxy_async_shared();
    }
    __syncthreads();
    if (g.split > 1) cluster_arrive();                      // (this CTA's barriers and landing place exist)
    // Tensor memory is taken behind the wait for the launch in front and before the next one may begin: a CTA that waits for a launch holds none that
    // the launch could be waiting for.  Nor does one hold any while it waits for the peers of its cluster: a peer may be waiting for what another
    // stream's CTA holds on its SM, and that one's own peer for this CTA's.  The copies do not wait for it.
    pdl_wait_prev();
    constexpr uint32_t kTmemCols = kBufs * TN < 32 ? 32 : kBufs * TN;
    uint32_t tmem_base = 0u;
    if (warp > 0) {
        if (warp == 1) {
            tmem_alloc(smem_u32(&tmem_slot), kTmemCols);
            tmem_relinquish();
        }
        tc_fence_before();
        asm volatile("bar.sync 1, %0;" ::"n"(kF8Threads - 32) : "memory");
        tc_fence_after();
        tmem_base = *(volatile uint32_t*)&tmem_slot;
        pdl_allow_next();
    }

    float acc[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
    const int quad = warp & 3, half = (warp - 2) >> 2;      // a warp reads the lanes of its quadrant, one half of the columns
    if (warp == 0) {
        if (elect_one()) {
            int st = 0, used = 0;
            uint32_t ph = 0;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait(smem_u32(&empty_bar[st]), ph ^ 1u, abortp, g.status, 1u, g.wait_ns)) break;
                const uint32_t bar = smem_u32(&full_bar[st]), dst = base + (uint32_t)st * kStage;
                mbar_expect_tx(bar, kStage);
                tma_load_2d(dst, &tmap_a, bar, kb * 128, tile_a * 128);
                tma_load_2d(dst + kF8TileA, &tmap_b, bar, kb * 128, tile_b * TN);
                ++used;
                if (++st == g.stages) { st = 0; ph ^= 1u; }
            }
            // shared memory stays until the last copy into each stage has landed, also when somebody gave up (bounded)
            const unsigned long long t0 = global_timer_ns();
            for (int i = 0; i < g.stages && i < used; ++i) {
                const uint32_t turn = (uint32_t)((used - 1 - i) / g.stages) & 1u;
                while (!mbar_try_wait(smem_u32(&full_bar[i]), turn)) if (global_timer_ns() - t0 > g.wait_ns) break;
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            const uint64_t d0 = make_desc(0u, 128);
            int st = 0, buf = 0;
            uint32_t ph = 0, aph = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                ok = mbar_wait(smem_u32(&acc_empty[buf]), aph ^ 1u, abortp, g.status, 2u, g.wait_ns) &&
                     mbar_wait(smem_u32(&full_bar[st]), ph, abortp, g.status, 3u, g.wait_ns);
                if (!ok) break;
                tc_fence_after();
                const uint32_t a = base + (uint32_t)st * kStage, b = a + kF8TileA;
                const uint64_t da = d0 + (uint64_t)((a & 0x3FFFFu) >> 4), db = d0 + (uint64_t)((b & 0x3FFFFu) >> 4);
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_f8(tmem_base + (uint32_t)(buf * TN), da + 2u * k, db + 2u * k, g.idesc, k > 0 ? 1u : 0u);
                mma_commit(smem_u32(&empty_bar[st]));
                mma_commit(smem_u32(&acc_full[buf]));
                if (++st == g.stages) { st = 0; ph ^= 1u; }
                if (++buf == kBufs) { buf = 0; aph ^= 1u; }
            }
            if (!ok) {                                      // nothing of what was issued is to run on behind this CTA (bounded)
                mma_commit(smem_u32(&drained));
                const unsigned long long t0 = global_timer_ns();
                while (!mbar_try_wait(smem_u32(&drained), 0u)) if (global_timer_ns() - t0 > g.wait_ns) break;
            }
        }
        __syncwarp();
    } else {
        // the scales of the next block are under way while this one's products are waited for
        const int row = tile_a * 128 + quad * 32 + lane;
        const int cb = min(tile_b * TN + half * kCols + lane % kCols, g.rows_b - 1);      // SWAP: the lane's column
        const float* as = g.a_scale + (SWAP ? (long long)tile_a : (long long)min(row, g.rows_a - 1)) * g.as_row;
        const float* bs = g.b_scale + (SWAP ? (long long)cb : (long long)((tile_b * TN) >> 7)) * g.bs_row;
        int buf = 0;
        uint32_t aph = 0;
        float sa = 0.f, sb = 0.f;
        if (kb0 < kb1) { sa = __ldg(as + kb0 * g.as_block); sb = __ldg(bs + kb0 * g.bs_block); }
        for (int kb = kb0; kb < kb1; ++kb) {
            const float s = sa * sb;
            if (kb + 1 < kb1) { sa = __ldg(as + (kb + 1) * g.as_block); sb = __ldg(bs + (kb + 1) * g.bs_block); }
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&acc_full[buf]), aph, abortp, g.status, 4u, g.wait_ns))) break;
            tc_fence_after();
            const uint32_t t = tmem_base + (uint32_t)(buf * TN + half * kCols) + ((uint32_t)(quad * 32) << 16);
            uint32_t r[kCols];
            if constexpr (kCols >= 32) {
#pragma unroll
                for (int j = 0; j < kCols; j += 32) tmem_ld32(t + (uint32_t)j, *reinterpret_cast<uint32_t(*)[32]>(&r[j]));
            } else {
#pragma unroll
                for (int j = 0; j < kCols; j += 8) tmem_ld8(t + (uint32_t)j, &r[j]);
            }
            tmem_wait_ld();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&acc_empty[buf]));
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
                const float sj = SWAP ? __shfl_sync(0xffffffffu, s, j) : s;
                acc[j] = fmaf(__uint_as_float(r[j]), sj, acc[j]);
            }
            if (++buf == kBufs) { buf = 0; aph ^= 1u; }
        }
    }

    // ---- out: y[token][column of the weights] ----
    const int first_col = tile_b * TN + half * kCols;
    // (32 columns of a row, 64 bytes or more, leave as well from their lane as by way of shared memory, and sooner; 64 take 2 us longer that way)
    constexpr bool kAlone = !SWAP && TN <= 32;
    if ((SWAP || kAlone) && g.split == 1) {
        if (warp >= 2 && !*abortp) {
            const int row = tile_a * 128 + quad * 32 + lane;
            if constexpr (SWAP) {
                if (row < g.rows_a) {
                    const float b = g.bias ? __ldg(g.bias + row) : 0.f;
#pragma unroll
                    for (int j = 0; j < kCols; ++j)
                        if (first_col + j < g.rows_b) store_one(g.y, (long long)(first_col + j) * g.y_row + row, g.y_type, activate(acc[j] + b, g.act));
                }
            } else if (row < g.rows_a) {
                const long long at = (long long)row * g.y_row + first_col;
#pragma unroll
                for (int j = 0; j < kCols; ++j) {
                    const float b = g.bias && first_col + j < g.rows_b ? __ldg(g.bias + first_col + j) : 0.f;
                    acc[j] = activate(acc[j] + b, g.act);
                }
                if (g.wide && first_col + kCols <= g.rows_b) {
                    if (g.y_type == TT_TYPE_F32) store_wide<TT_TYPE_F32, kCols>(static_cast<float*>(g.y) + at, acc);
                    else if (g.y_type == TT_TYPE_F16) store_wide<TT_TYPE_F16, kCols>(static_cast<__half*>(g.y) + at, acc);
                    else store_wide<TT_TYPE_BF16, kCols>(static_cast<__nv_bfloat16*>(g.y) + at, acc);
                } else {
#pragma unroll
                    for (int j = 0; j < kCols; ++j) if (first_col + j < g.rows_b) store_one(g.y, at + j, g.y_type, acc[j]);
                }
            }
        }
    } else {
        // Sums to shared memory (the pipeline is idle: the last block's products are done with it), every peer's band of them to it in one copy
        // (loads from a peer's shared memory run at some 10 bytes a cycle), and this CTA's band added up as the others' arrive.  A tile that is
        // not split goes this way too, so that rows leave as rows.
        const uint32_t me = (uint32_t)blockIdx.z;
        if (warp >= 2) {
            const uint32_t r = (uint32_t)(quad * 32 + lane);
            if constexpr (SWAP) {
#pragma unroll
                for (int j = 0; j < kCols; ++j) st_shared_f32(base + (uint32_t)(half * kCols + j) * kLine + r * 4u, acc[j]);
            } else {
#pragma unroll
                for (int j = 0; j < kCols; j += 4) st_shared_v4(base + r * kLine + (uint32_t)(half * kCols + j) * 4u, acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
            }
            fence_proxy_async_shared();
            tc_fence_before();
            asm volatile("bar.sync 2, 288;" ::: "memory");
        } else if (warp == 1) {
            __syncwarp();
            asm volatile("bar.sync 2, 288;" ::: "memory");
            tc_fence_after();
            tmem_dealloc(tmem_base, kTmemCols);
        }
        __syncwarp();
        if (g.split > 1) cluster_wait();                    // the peers are there
        if (warp == 2 && lane < g.split && lane != (int)me && !*abortp) {
            const uint32_t slot = me < (uint32_t)lane ? me : me - 1u;
            bulk_copy_to_peer(map_to_peer(landing + slot * band_bytes, (uint32_t)lane), base + (uint32_t)lane * band_bytes, band_bytes, map_to_peer(smem_u32(&red_bar), (uint32_t)lane));
        }
        __syncwarp();
        if (warp >= 2 && (g.split == 1 ? !*abortp : __all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&red_bar), 0u, abortp, g.status, 5u, g.wait_ns)))) {
            constexpr int kQuads = SWAP ? 32 : TN / 4;       // four values at a time
            for (int e = (int)threadIdx.x - 64; e < per * kQuads; e += 256) {
                const int in = e / kQuads, c = 4 * (e - in * kQuads), line = (int)me * per + in;
                const int token = (SWAP ? tile_b * TN : tile_a * 128) + line, col = (SWAP ? tile_a * 128 : tile_b * TN) + c;
                const int tokens = SWAP ? g.rows_b : g.rows_a, cols = SWAP ? g.rows_a : g.rows_b;
                if (token >= tokens || col >= cols) continue;
                float v[4] = {0.f, 0.f, 0.f, 0.f};
                for (uint32_t p = 0; p < (uint32_t)g.split; ++p) {          // (in the order of the splits)
                    const float4 f = ld_shared_v4f((p == me ? base + me * band_bytes : landing + (p < me ? p : p - 1u) * band_bytes) + (uint32_t)in * kLine + (uint32_t)c * 4u);
                    v[0] += f.x; v[1] += f.y; v[2] += f.z; v[3] += f.w;
                }
                const long long at = (long long)token * g.y_row + col;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float b = g.bias && col + i < cols ? __ldg(g.bias + col + i) : 0.f;
                    v[i] = activate(v[i] + b, g.act);
                }
                if (g.wide && col + 4 <= cols) {
                    if (g.y_type == TT_TYPE_F32) *reinterpret_cast<float4*>(static_cast<float*>(g.y) + at) = make_float4(v[0], v[1], v[2], v[3]);
                    else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.y) + at) =
                        g.y_type == TT_TYPE_F16 ? make_uint2(down2<TT_TYPE_F16>(v[0], v[1]), down2<TT_TYPE_F16>(v[2], v[3]))
                                                : make_uint2(down2<TT_TYPE_BF16>(v[0], v[1]), down2<TT_TYPE_BF16>(v[2], v[3]));
                } else {
                    for (int i = 0; i < 4 && col + i < cols; ++i) store_one(g.y, at + i, g.y_type, v[i]);
                }
            }
        }
        if (g.split > 1) {
            __syncwarp();
            cluster_arrive();                               // nobody leaves while a copy may be on its way to it
            cluster_wait();
        }
    }
    if ((SWAP || kAlone) && g.split == 1) {
        tc_fence_before();
        __syncthreads();
        if (warp == 1) {
            __syncwarp();
            tc_fence_after();
            tmem_dealloc(tmem_base, kTmemCols);
        }
    }
}

// The same for many tokens: pairs of CTAs walk tiles of 256 x TN persistently.  Each CTA has 128 rows of A and half of B's in shared memory,
// tcgen05.mma.cta_group::2 reads both CTAs', so an SM takes in (128 + TN / 2) * 128 bytes for 128 * TN * 128 products: 64 bytes a cycle at the tensor
// core's rate, which is what an SM can get from the L2 (a 128 x 128 tile of one CTA needs twice that).  Two accumulators; the
// sixteen read-out warps have a quarter of a block's sums each, 4 warps a scheduler, so that one waits for tensor memory while another adds.
// (8192 x 4096 x 4096: 127 us at full clocks, 2.2 PFLOP/s; 150 us, 1.8 PFLOP/s, when repeated until the power limit sets the clock.  The read-out is
// the bound: a compare and a select more for each block of it are 7 us, and the tensor cores are busy for 58 % of the time.  At 256 columns a thread
// spills 49 words.)
constexpr int kPairThreads = 128 + 512;                    // a warpgroup of TMA and MMA, four of read-out (96 registers each at launch; 32 and 112)
constexpr unsigned kPairStaging = 16 * 4096;                // a block of 32 rows x 128 bytes for each read-out warp
constexpr int kPairSmem = 230400;
constexpr int kBand = 16;

__device__ __forceinline__ void mma_f8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const void* tmap, uint32_t bar_cluster, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(tmap), "r"(bar_cluster), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_store_2d(const void* tmap, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tmap), "r"(src), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
                   "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(taddr));
}

// mbar_arrive_remote where no ordinary memory access has to be seen: what is given back is tensor memory, whose loads have been waited for.  (With
// release semantics the arrival took 1100 to 1800 cycles of the warp.)
__device__ __forceinline__ void mbar_arrive_remote_relaxed(uint32_t bar, uint32_t rank) {
    asm volatile(
        "{\n\t.reg .b32 ra;\n\t"
        "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
        "mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [ra];\n\t}"
        ::"r"(bar), "r"(rank) : "memory");
}

template <int TN>
__global__ void __launch_bounds__(kPairThreads, 1)
tt_dense_f8_pair_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const __grid_constant__ CUtensorMap tmap_y, const DenseF8 g) {
    constexpr int kCols = TN / 4;                          // columns of a read-out warp
    constexpr uint32_t kStage = kF8TileA + TN / 2 * 128u;
    constexpr int kParts = TN / 128, kBufs = 4 / kParts;   // a block's sums come in parts of 128 columns, half of B's rows of each CTA's
    constexpr int kReaders = 16 / kParts;                  // read-out warps of a part
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kF8MaxStages], empty_bar[kF8MaxStages], acc_full[4], acc_empty[4];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int* abortp = &abort_flag;
    const uint32_t rank = cluster_ctarank();
    const int unit = (int)blockIdx.x / 2, n_units = (int)gridDim.x / 2;
    const int my_tiles = g.tiles > unit ? (g.tiles - unit + n_units - 1) / n_units : 0;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_b) : "memory");
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < g.stages; ++i) { mbar_init(smem_u32(&full_bar[i]), 1u); mbar_init(smem_u32(&empty_bar[i]), 1u); }
        for (int i = 0; i < 4; ++i) { mbar_init(smem_u32(&acc_full[i]), 1u); mbar_init(smem_u32(&acc_empty[i]), 2u * kReaders); }
        abort_flag = 0;
        fence_mbar_init();
        fence_proxy_async_shared();
    }
    pdl_wait_prev();                                        // (before tensor memory is taken, see above)
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                     // the peer's barriers exist before anything arrives on them
    tc_fence_after();
    const uint32_t tmem_base = *(volatile uint32_t*)&tmem_slot;
    pdl_allow_next();
    // Tiles in bands of kBand of 256 rows, so that the pairs at work share rows of A and of B alike.
    const int tiles_b = g.tiles / g.tiles_a;
    const auto place = [&](int t, int& tm, int& tn) {
        const int band = t / (kBand * tiles_b), in = t - band * kBand * tiles_b, high = min(kBand, g.tiles_a - band * kBand);
        tn = in / high;
        tm = band * kBand + in - tn * high;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
        if (warp == 0 && elect_one()) {
            int st = 0;
            uint32_t ph = 0;
            long long issued = 0;
            bool ok = true;
            for (int i = 0; i < my_tiles && ok; ++i) {
                int tm, tn;
                place(unit + i * n_units, tm, tn);
                const int a0 = (2 * tm + (int)rank) * 128, b0 = tn * TN + (int)rank * (TN / 2);
                for (int kb = 0; kb < g.blocks; ++kb) {
                    ok = bounded_wait(&empty_bar[st], ph ^ 1u, abortp, g.status, 1u, g.wait_ns);
                    if (!ok) break;
                    const uint32_t dst = base + (uint32_t)st * kStage;
                    if (rank == 0) mbar_expect_tx(smem_u32(&full_bar[st]), 2u * kStage);
                    const uint32_t bar = map_to_peer(smem_u32(&full_bar[st]), 0u);       // the pair's loads all report to rank 0
                    tma_load_2d_pair(dst, &tmap_a, bar, kb * 128, a0);
                    tma_load_2d_pair(dst + kF8TileA, &tmap_b, bar, kb * 128, b0);
                    ++issued;
                    if (++st == g.stages) { st = 0; ph ^= 1u; }
                }
            }
            if (!ok || *abortp) {
                // let copies in flight land before shared memory is given back (bounded); the other CTA's report to rank 0, it gives them time
                const unsigned long long t0 = global_timer_ns();
                if (rank == 0) {
                    for (long long it = issued > g.stages ? issued - g.stages : 0; it < issued; ++it)
                        while (!mbar_try_wait(smem_u32(&full_bar[it % g.stages]), (uint32_t)(it / g.stages) & 1u)) if (global_timer_ns() - t0 > 2000000ull) break;
                } else {
                    while (global_timer_ns() - t0 < 2000000ull) { }
                }
            }
        }
        if (warp == 1 && rank == 0 && elect_one()) {
            const uint64_t d0 = make_desc(0u, 128);
            int st = 0, buf = 0;
            uint32_t ph = 0, aph = 0;
            bool ok = true;
            for (int i = 0; i < my_tiles && ok; ++i)
                for (int kb = 0; kb < g.blocks; ++kb) {
                    ok = bounded_wait(&full_bar[st], ph, abortp, g.status, 3u, g.wait_ns);
                    const uint32_t a = base + (uint32_t)st * kStage, b = a + kF8TileA;
                    const uint64_t da = d0 + (uint64_t)((a & 0x3FFFFu) >> 4), db = d0 + (uint64_t)((b & 0x3FFFFu) >> 4);
#pragma unroll
                    for (int h = 0; h < kParts; ++h) {
                        ok = ok && bounded_wait<true>(&acc_empty[buf * kParts + h], aph ^ 1u, abortp, g.status, 2u, g.wait_ns);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f8_pair(tmem_base + (uint32_t)((buf * kParts + h) * 128), da + 2u * k, db + (uint64_t)(h * (64 * 128 / 16)) + 2u * k, g.idesc, k > 0 ? 1u : 0u);
                        mma_commit_cg<2>(smem_u32(&acc_full[buf * kParts + h]));
                    }
                    if (!ok) break;
                    mma_commit_cg<2>(smem_u32(&empty_bar[st]));
                    if (++st == g.stages) { st = 0; ph ^= 1u; }
                    if (++buf == kBufs) { buf = 0; aph ^= 1u; }
                }
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
        // four warps have 128 lanes x kCols columns of the tile; of a part's columns the first half is of this pair's first CTA's rows of B
        const int quad = warp & 3, group = (warp - 4) >> 2, part = kParts == 2 ? group >> 1 : 0, at0 = kParts == 2 ? (group & 1) * 64 : group * kCols;
        const int c0 = kParts == 2 ? (group & 1) * 128 + part * 64 : at0;
        const uint32_t staging = base + (uint32_t)g.stages * kStage + (uint32_t)(warp - 4) * 4096u;
        const uint32_t lanes = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(part * 128 + at0);
        int buf = 0;
        uint32_t aph = 0;
        bool ok = true;
        for (int i = 0; i < my_tiles; ++i) {
            int tm, tn;
            place(unit + i * n_units, tm, tn);
            const int row0 = (2 * tm + (int)rank) * 128 + quad * 32, col0 = tn * TN + c0;
            const float* as = g.a_scale + (long long)min(row0 + lane, g.rows_a - 1) * g.as_row;
            const float* bs = g.b_scale + (long long)(min(col0, g.rows_b - 1) >> 7) * g.bs_row;
            float acc[kCols];
#pragma unroll
            for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
            float sa = __ldg(as), sb = __ldg(bs);
            for (int kb = 0; kb < g.blocks; ++kb) {
                const float s = sa * sb;
                if (kb + 1 < g.blocks) { sa = __ldg(as += g.as_block); sb = __ldg(bs += g.bs_block); }
                ok = ok && __all_sync(0xffffffffu, bounded_wait(&acc_full[buf * kParts + part], aph, abortp, g.status, 4u, g.wait_ns));
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = lanes + (uint32_t)(buf * kParts * 128);
                // (sixteen at a time: there are four warps a scheduler to take turns, and no registers for more)
#pragma unroll
                for (int j = 0; j < kCols; j += 16) {
                    uint32_t r[16];
                    tmem_ld16(at + (uint32_t)j, r);
                    tmem_wait_ld();
                    if (j + 16 >= kCols) {
                        // (the accumulator is free again)
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_remote_relaxed(smem_u32(&acc_empty[buf * kParts + part]), 0u);
                    }
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        const float2 f = fma_pair(make_float2(__uint_as_float(r[k]), __uint_as_float(r[k + 1])), make_float2(s, s), make_float2(acc[j + k], acc[j + k + 1]));
                        acc[j + k] = f.x;
                        acc[j + k + 1] = f.y;
                    }
                }
                if (++buf == kBufs) { buf = 0; aph ^= 1u; }
            }
            if (!ok) break;
            if (g.bias) {
#pragma unroll
                for (int part32 = 0; part32 < kCols; part32 += 32) {
                    const float b = __ldg(g.bias + min(col0 + part32 + lane, g.rows_b - 1));
#pragma unroll
                    for (int j = 0; j < 32; ++j) acc[part32 + j] += __shfl_sync(0xffffffffu, b, j);
                }
            }
            if (g.act == TT_ACT_GELU_ERF) {
#pragma unroll
                for (int j = 0; j < kCols; ++j) acc[j] = gelu_erf(acc[j]);
            } else if (g.act != TT_ACT_NONE) {
#pragma unroll
                for (int j = 0; j < kCols; ++j) acc[j] = activate(acc[j], g.act);
            }
            // Blocks of 32 rows through shared memory, swizzled as the tensor map has it, and out by TMA; where rows are no multiples of 16 bytes, a
            // row at a time (a lane's own row would be 32 places at once).
            const int per = g.y_type == TT_TYPE_F32 ? 32 : kCols;           // columns of a block: 128 bytes of them, or 64 (kCols 32 in 16 bits)
#pragma unroll
            for (int piece = 0; piece < kCols / 32; ++piece) {
                if (piece > 0 && g.y_type != TT_TYPE_F32) break;
                const int col = col0 + piece * per;
                if (lane == 0) bulk_stores_pending<0>();
                __syncwarp();
                if (g.y_type == TT_TYPE_F32) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4)
                        st_shared_v4(staging + (uint32_t)lane * 128u + ((uint32_t)((j >> 2) ^ (lane & 7)) << 4), acc[32 * piece + j], acc[32 * piece + j + 1], acc[32 * piece + j + 2], acc[32 * piece + j + 3]);
                } else {
#pragma unroll
                    for (int j = 0; j < kCols; j += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = g.y_type == TT_TYPE_F16 ? down2<TT_TYPE_F16>(acc[j + 2 * e], acc[j + 2 * e + 1]) : down2<TT_TYPE_BF16>(acc[j + 2 * e], acc[j + 2 * e + 1]);
                        const uint32_t x = kCols == 64 ? (uint32_t)(lane & 7) : (uint32_t)((lane >> 1) & 3);
                        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(staging + (uint32_t)lane * (kCols * 2u) + (((uint32_t)(j >> 3) ^ x) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                    }
                }
                if (g.wide) {
                    fence_proxy_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        if (row0 < g.rows_a && col < g.rows_b) tma_store_2d(&tmap_y, staging, col, row0);
                        bulk_stores_commit();
                    }
                } else {
                    __syncwarp();
                    if (g.y_type == TT_TYPE_F32) {
                        float* y = static_cast<float*>(g.y) + (long long)row0 * g.y_row + col + lane;
#pragma unroll 1
                        for (int r = 0; r < 32; r += 8, y += 8 * g.y_row) {
                            float v[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] = ld_shared_f32(staging + (uint32_t)(r + k) * 128u + ((uint32_t)((lane >> 2) ^ k) << 4) + 4u * (uint32_t)(lane & 3));
#pragma unroll
                            for (int k = 0; k < 8; ++k) if (row0 + r + k < g.rows_a && col + lane < g.rows_b) y[k * g.y_row] = v[k];
                        }
                    } else {
                        // A lane has two values, a word of memory, or the second and the next lane's first where rows begin between two words.
                        constexpr int kWords = kCols / 2, kRows = 32 / kWords;
                        const int l = lane % kWords, sub = lane / kWords, n = g.rows_b - col;
                        uint16_t* y = static_cast<uint16_t*>(g.y) + (long long)(row0 + sub) * g.y_row + col + 2 * l;
#pragma unroll 1
                        for (int r = sub; r < 32; r += 8 * kRows, y += 8 * kRows * g.y_row) {
                            uint32_t w[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const int at = r + k * kRows, x = kCols == 64 ? at & 7 : (at >> 1) & 3;
                                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[k]) : "r"(staging + (uint32_t)at * (kCols * 2u) + ((uint32_t)((l >> 2) ^ x) << 4) + 4u * (uint32_t)(l & 3)) : "memory");
                            }
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                uint16_t* p = y + k * kRows * g.y_row;
                                const uint32_t next = __shfl_down_sync(0xffffffffu, w[k], 1, kWords);
                                if (row0 + r + k * kRows >= g.rows_a) continue;
                                if ((reinterpret_cast<uintptr_t>(p) & 2u) == 0u) {
                                    if (2 * l + 1 < n) *reinterpret_cast<uint32_t*>(p) = w[k];
                                    else if (2 * l < n) *p = (uint16_t)w[k];
                                } else {
                                    if (l < kWords - 1 && 2 * l + 2 < n) *reinterpret_cast<uint32_t*>(p + 1) = __funnelshift_r(w[k], next, 16);
                                    else if (2 * l + 1 < n) p[1] = (uint16_t)(w[k] >> 16);
                                    if (l == 0 && n > 0) *p = (uint16_t)w[k];
                                }
                            }
                        }
                    }
                    __syncwarp();
                }
            }
        }
        if (lane == 0) bulk_stores_pending<0>();             // shared memory stays until the last store has read it
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                     // the pair stays together until neither CTA touches the other
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

template <int TN, bool SWAP>
static cudaError_t launch_dense_f8(const CUtensorMap& ta, const CUtensorMap& tb, DenseF8 g, void* stream) {
    constexpr int kStageBytes = (int)kF8TileA + TN * 128;
    static OncePerDevice raised;
    const cudaError_t ready = raised([] { return cudaFuncSetAttribute(tt_dense_f8_kernel<TN, SWAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDynSmemLimit); });
    if (ready != cudaSuccess) return ready;
    // SWAP takes half of an SM's shared memory: two CTAs fit, of this launch or the next one's, whose set-up then runs while this one's sums are
    // joined; their columns of tensor memory fit together.  The other form takes all columns and so most of the shared memory: beside a CTA that
    // holds some it would wait for them, and CTAs of two clusters that wait so for each other would do it forever.
    const int landing = g.split > 1 ? (SWAP ? TN * 512 : 128 * (TN + 4) * 4) / g.split * (g.split - 1) : 0;      // the peers' bands
    const int fits = ((SWAP ? kHalfSm : kDynSmemLimit) - 1024 - landing) / kStageBytes;
    g.stages = fits < kF8MaxStages ? fits : kF8MaxStages;
    const int tiles_b = (g.rows_b + TN - 1) / TN;
    return launch(tt_dense_f8_kernel<TN, SWAP>, dim3((unsigned)(g.tiles_a * tiles_b), 1, (unsigned)g.split), kF8Threads, 1024 + (size_t)g.stages * kStageBytes + landing, g.split, stream, ta, tb, g);
}

// The forms that the layer is built in, and what they cost, in microseconds on a B200: fitted to 30 layers of 8 to 8192 tokens, 128 to 14336 columns
// and 1000 to 8192 products under every form and split.  A launch takes kLaunch; a block of 128 products of a tile takes `block` (what the L2 gives an SM
// is the bound); the exchange of splits and the way out are a tile's; what does not fit the SMs at once comes later, and with the next CTA's set-up.
struct F8Form { bool swap; int tn, pair; float block, exchange, out; };
constexpr F8Form kF8Forms[] = {
    {true, 16, 0, 0.215f, 0.3f, 0.1f}, {true, 32, 0, 0.22f, 0.5f, 0.2f}, {true, 64, 0, 0.29f, 1.5f, 0.4f},
    {false, 32, 0, 0.215f, 0.5f, 0.3f}, {false, 64, 0, 0.30f, 1.3f, 0.6f}, {false, 128, 0, 0.36f, 3.2f, 2.0f},
    {false, 128, 1, 0.345f, 0.f, 0.8f}, {false, 256, 1, 0.47f, 0.f, 1.5f}};
struct F8Choice { F8Form form; int split; };
static F8Choice choose_f8(long long m, long long n, int blocks) {
    constexpr float kLaunch = 4.6f, kNextCta = 3.0f;
    F8Choice best{kF8Forms[7], 1};
    float least = 3.4e38f;
    for (const F8Form& f : kF8Forms) {
        const long long rows = f.swap ? n : m, cols = f.swap ? m : n, high = f.pair ? 256 : 128;
        const long long tiles = (rows + high - 1) / high * ((cols + f.tn - 1) / f.tn);
        for (int split = 1; split <= (f.pair ? 1 : 8); split *= 2) {
            if (split > 1 && (split * 2 > blocks || tiles * split > kSms)) break;
            const long long at_once = f.pair ? kSms / 2 : kSms, rounds = (tiles * split + at_once - 1) / at_once;
            const float tile = (float)((blocks + split - 1) / split) * f.block + (split > 1 ? f.exchange : f.out);
            const float us = kLaunch + (float)rounds * tile + (f.pair ? 0.f : (float)(rounds - 1) * kNextCta);
            if (us < least) { least = us; best = F8Choice{f, split}; }
        }
    }
    return best;
}

template <int TN>
static cudaError_t launch_dense_f8_pair(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& ty, DenseF8 g, void* stream) {
    constexpr int kStageBytes = (int)kF8TileA + TN / 2 * 128;
    static OncePerDevice raised;
    const cudaError_t ready = raised([] { return cudaFuncSetAttribute(tt_dense_f8_pair_kernel<TN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem); });
    if (ready != cudaSuccess) return ready;
    const int fits = (kPairSmem - 1024 - (int)kPairStaging) / kStageBytes;
    g.stages = fits < kF8MaxStages ? fits : kF8MaxStages;
    g.tiles_a = (g.rows_a + 255) / 256;
    g.tiles = g.tiles_a * ((g.rows_b + TN - 1) / TN);
    g.idesc = (1u << 4) | ((128u >> 3) << 17) | ((256u >> 4) << 24);
    const int units = g.tiles < kSms / 2 ? g.tiles : kSms / 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2u * (unsigned)units, 1, 1); cfg.blockDim = dim3(kPairThreads, 1, 1);
    cfg.dynamicSmemBytes = kPairSmem; cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, tt_dense_f8_pair_kernel<TN>, ta, tb, ty, g);
}

}  // namespace tt

using namespace tt;

constexpr int kMostRows = 0x7fffff00;                       // of an axis: tiles reach behind its end
constexpr int64_t kMostPitch = 1ll << 40;                   // bytes from row to row that a tensor map takes

extern "C" tt_status tt_quantize(const tt_quantize_args* a, void* stream) {
    if (!a || !known_type(a->x_type) || a->m < 0 || a->kk < 0 || a->m > kMostRows || a->kk > kMostRows || (a->block_rows != 1 && a->block_rows != kF8Block)) return TT_ERR_INVALID_ARG;
    if (a->m == 0 || a->kk == 0) return TT_OK;
    const int64_t bytes = type_bytes(a->x_type);
    if (!a->x || !a->q || !a->scales || a->x_row < a->kk || a->q_row < a->kk || a->s_row < 0 || a->s_block < 0) return TT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(a->x) % (uintptr_t)bytes || reinterpret_cast<uintptr_t>(a->scales) % 4) return TT_ERR_INVALID_ARG;
    const int wide = on16(a->x) && a->x_row * bytes % 16 == 0 && reinterpret_cast<uintptr_t>(a->q) % 8 == 0 && a->q_row % 8 == 0;
    const int blocks = (a->kk + kF8Block - 1) / kF8Block;
    if (a->block_rows == kF8Block) {
        const long long grid = (long long)blocks * ((a->m + kF8Block - 1) / kF8Block);
        if (grid > 0x7fffffff) return TT_ERR_INVALID_ARG;
        const auto kern = a->x_type == TT_TYPE_F32 ? tt_quantize_blocks_kernel<TT_TYPE_F32> : a->x_type == TT_TYPE_F16 ? tt_quantize_blocks_kernel<TT_TYPE_F16> : tt_quantize_blocks_kernel<TT_TYPE_BF16>;
        return status_of(launch(kern, dim3((unsigned)grid, 1, 1), 256, 0, 1, stream, *a, blocks, wide));
    }
    // (few tasks: a warp to a CTA, so that they are spread over the SMs)
    const long long tasks = (a->m + 7ll) / 8 * blocks, grid_threads = tasks < 8ll * kSms ? 32 : 256, grid = (tasks * 32 + grid_threads - 1) / grid_threads;
    if (grid > 0x7fffffff) return TT_ERR_INVALID_ARG;
    if (!wide) {
        const auto kern = a->x_type == TT_TYPE_F32 ? tt_quantize_lines_kernel<TT_TYPE_F32> : a->x_type == TT_TYPE_F16 ? tt_quantize_lines_kernel<TT_TYPE_F16> : tt_quantize_lines_kernel<TT_TYPE_BF16>;
        return status_of(launch(kern, dim3((unsigned)grid, 1, 1), (int)grid_threads, 0, 1, stream, *a, blocks, tasks));
    }
    const auto kern = a->x_type == TT_TYPE_F32 ? tt_quantize_rows_kernel<TT_TYPE_F32> : a->x_type == TT_TYPE_F16 ? tt_quantize_rows_kernel<TT_TYPE_F16> : tt_quantize_rows_kernel<TT_TYPE_BF16>;
    return status_of(launch(kern, dim3((unsigned)grid, 1, 1), (int)grid_threads, 0, 1, stream, *a, blocks, tasks));
}

extern "C" tt_status tt_dense_quantized(const tt_dense_quantized_args* a, void* stream) {
    if (!a || !known_type(a->y_type) || a->m < 0 || a->nn < 0 || a->kk < 0 || a->m > kMostRows || a->nn > kMostRows || a->kk > kMostRows || a->act < TT_ACT_NONE || a->act > TT_ACT_GELU_ERF) return TT_ERR_INVALID_ARG;
    if (a->m == 0 || a->nn == 0) return TT_OK;
    if (a->kk == 0) return TT_ERR_INVALID_ARG;             // (there is no sum to take)
    if (!a->x || !a->w || !a->x_scale || !a->w_scale || !a->y || !a->status) return TT_ERR_INVALID_ARG;
    if (a->x_row < a->kk || a->w_row < a->kk || a->y_row < a->nn || a->xs_row < 0 || a->xs_block < 0 || a->ws_row < 0 || a->ws_block < 0) return TT_ERR_INVALID_ARG;
    const int64_t bytes = type_bytes(a->y_type);
    if (!on16(a->x) || !on16(a->w) || a->x_row % 16 || a->w_row % 16 || a->x_row >= kMostPitch || a->w_row >= kMostPitch || a->y_row >= kMostPitch / bytes) return TT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(a->y) % (uintptr_t)bytes || reinterpret_cast<uintptr_t>(a->x_scale) % 4 || reinterpret_cast<uintptr_t>(a->w_scale) % 4 ||
        reinterpret_cast<uintptr_t>(a->bias) % 4 || reinterpret_cast<uintptr_t>(a->status) % 4) return TT_ERR_INVALID_ARG;
    DenseF8 g{};
    g.bias = a->bias; g.y = a->y; g.y_row = a->y_row; g.status = a->status; g.y_type = a->y_type; g.act = a->act;
    g.wide = on16(a->y) && a->y_row * bytes % 16 == 0;
    g.blocks = (a->kk + kF8Block - 1) / kF8Block;
    g.wait_ns = 1000000000ull;
    const F8Choice choice = choose_f8(a->m, a->nn, g.blocks);
    const bool swap = choice.form.swap;
    const int tn = choice.form.tn;
    g.rows_a = swap ? a->nn : a->m; g.rows_b = swap ? a->m : a->nn;
    g.tiles_a = (g.rows_a + 127) / 128;
    if ((long long)g.tiles_a * ((g.rows_b + tn - 1) / tn) > 0x7fffffff) return TT_ERR_INVALID_ARG;
    g.split = choice.split;
    g.blocks_per_split = (g.blocks + g.split - 1) / g.split;
    g.idesc = (1u << 4) | ((unsigned)(tn >> 3) << 17) | ((unsigned)(kHwTileM >> 4) << 24);
    if (swap) {
        g.a_scale = a->w_scale; g.as_row = a->ws_row; g.as_block = a->ws_block; g.b_scale = a->x_scale; g.bs_row = a->xs_row; g.bs_block = a->xs_block;
    } else {
        g.a_scale = a->x_scale; g.as_row = a->xs_row; g.as_block = a->xs_block; g.b_scale = a->w_scale; g.bs_row = a->ws_row; g.bs_block = a->ws_block;
    }
    CUtensorMap ta, tb, ty{};
    tt_status s = swap ? encode_bytes(&ta, a->w, a->kk, a->nn, a->w_row, 128) : encode_bytes(&ta, a->x, a->kk, a->m, a->x_row, 128);
    if (s == TT_OK) s = swap ? encode_bytes(&tb, a->x, a->kk, a->m, a->x_row, tn) : encode_bytes(&tb, a->w, a->kk, a->nn, a->w_row, choice.form.pair ? tn / 2 : tn);
    if (s != TT_OK) return s;
    if (choice.form.pair) {
        g.wide = g.wide && a->nn * bytes % 16 == 0;        // (a TMA store clips in pieces of 16 bytes)
        if (g.wide) s = encode_output(&ty, a->y, (int)bytes, a->nn, a->m, a->y_row, a->y_type == TT_TYPE_F32 ? 32 : tn / 4);
        if (s != TT_OK) return s;
        return status_of(tn == 256 ? launch_dense_f8_pair<256>(ta, tb, ty, g, stream) : launch_dense_f8_pair<128>(ta, tb, ty, g, stream));
    }
    if (swap) return status_of(tn == 16 ? launch_dense_f8<16, true>(ta, tb, g, stream) : tn == 32 ? launch_dense_f8<32, true>(ta, tb, g, stream) : launch_dense_f8<64, true>(ta, tb, g, stream));
    return status_of(tn == 32 ? launch_dense_f8<32, false>(ta, tb, g, stream) : tn == 64 ? launch_dense_f8<64, false>(ta, tb, g, stream) : launch_dense_f8<128, false>(ta, tb, g, stream));
}
