// Attention of prompts over the paged e4m3 cache: many rows (queries of the heads that share a key head) for each key, so the products and the
// exponentials are the bound, not the cache's bytes.
//
// Built for heads of 64 and 128 values; what a shorter head lacks (32, 96) is zeros, which the copies and the queries' warps fill in.
// A CTA has two tiles of 128 rows and walks the keys 128 at a time.  Four warps bring keys and values from the pages, turn them into 16-bit floating
// point (exactly) and leave them as operand tiles, which serve both tiles of rows.  S = Q K^T goes to tensor memory; two threads of the
// softmax warps have a row of it, take its maximum, and leave P = 2^(s - m) in S's place as the first operand of O += P V, whose sums stay
// in tensor memory.  While one tile's softmax runs, the tensor core is at the other tile's products.
//   O is multiplied only when a maximum has grown by more than 2^8 since it was last: P may be up to 2^8 times what it
// would be, which 16 bits have room for (it is brought to 2^15 at most, and what is 2^-21 of the largest has all of its bits; with 2^11 and 2^-18
// a column of small values beside one key of nearly all the weight was off by more than a rounding), and the row's sum has
// the same factor.  A page's scale of values is in
// P too, as a part of the exponent, over the largest scale so far.  Where that is of a page that some rows do not see, it may be so much larger than what
// they do see that nothing would be left of their P: `used` of such a row is lower by the power of two between them, and P as much higher.  (A difference
// of less than 2^5 is left alone.  That steps are told so by the pages' warp, in a number that they look at anyway, is for speed: a branch of its own
// in front of the maxima cost 13 us of 254.)
//   Two prompts of 2048 tokens behind as many, 32 heads over 8 of 128: 252 us, 817 TFLOP/s of 16-bit products, half of the tensor cores' rate.  A step
// of 128 keys takes 3500 to 3900 cycles: the products 2050, the exponentials 2050 and the shared memory 2560, and a tile's chain (its softmax, then the
// product that takes P and the one that makes the next scores) 3500, which is the bound.  The way in and out are 11000 and 6000 cycles of a CTA.
// (Scores of the second 64 keys while P of the first is being made: 370 us, as the queries are read twice.  A part of the exponentials as polynomials:
// slower, they are not the bound.)
//   NaN in values that only some rows of the tile see (the steps at the edge of what is visible) are taken out of the product and put into
// the outputs of the rows that do: a column's first such token (at the upper edge; its last one at the lower) decides.
#include <cuda_runtime.h>
#include <climits>
#include "tt_cache.cuh"

namespace tt {

constexpr int kPromptThreads = 768;         // warps 0-7 and 8-15 softmax of a tile each, 16-19 keys and values, 20 MMA and tensor memory, 21 pages, scales and copies
constexpr int kSoftmax = 512;               // threads of the softmax, two to a row
constexpr unsigned long long kPromptWait = 1000000000ull;                    // nanoseconds that a wait takes at most
constexpr uint32_t kAtom = 128u * 128u;     // 128 rows of 64 values

__device__ __forceinline__ void mma_f16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st8u(uint32_t taddr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]));
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, float v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "f"(v) : "memory");
}
__device__ __forceinline__ float tmem_ld1(uint32_t taddr) {
    float v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=f"(v) : "r"(taddr) : "memory");
    return v;
}
__device__ __forceinline__ float max_of(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 ld_shared_v2f(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
// Registers of a warpgroup from here on.  768 threads begin with 80 each (61440): 96 for the softmax's four, 56 and 40 for the others make 61440.
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Named barriers: 1 the softmax and the warps of keys and values, 2 the softmax and the MMA warp (at the end), 4 and 5 a tile's softmax.
__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void named_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// What the softmax needs to know of a step's eight groups of 16 tokens.
struct alignas(8) StepScales {
    float key[8], shift[8], back[8];
    float ref, shrink;                      // the largest scale of values so far; the one before over it, with a minus if rows are to be looked at on their own:
    uint8_t value[8]; int common;           // the exponents of the values' scales (255: not finite), and of the largest so far that all rows of the tile see
};
__device__ __forceinline__ int exponent_of(float scale) { return __float_as_int(scale) >> 23 & 255; }

// Splits of a tile that have anything to do.
__device__ __forceinline__ int prompt_splits(const Attend& g, const TileView& view) {
    return view.hi > view.lo ? (int)((unsigned)(view.hi - view.lo / kPromptTokens * kPromptTokens + g.chunk - 1) / (unsigned)g.chunk) : 1;
}

template <int D>
struct PromptShape {
    static constexpr int kAtoms = D / 64;
    static constexpr uint32_t kTile = kAtoms * kAtom;                    // bytes of 128 rows of queries, keys or values
    static constexpr uint32_t kBytes = 1024u + 7u * kTile;               // two of each, and the bytes of the next keys and values
    static constexpr uint32_t kScores = 0, kOut = 256;                   // columns of tensor memory: S (and P) of both tiles, O of both
};

template <int D>
__global__ void __launch_bounds__(kPromptThreads, 1) tt_attend_prompt_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ Attend g) {
    typedef PromptShape<D> S;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_ready[2][2], o_done[2], raw_full[2], raw_empty[2], drained;
    __shared__ StepScales scales[4];
    __shared__ int nan_first[D], nan_last[D], nan_any;
    __shared__ uint8_t sizes[kPromptRows];                                // of the queries' rows: the exponents of what they were multiplied by (then row_ref, see there)
    __shared__ uint32_t tmem_slot;
    __shared__ int late[6];                                               // what the way out needs (the softmax has no registers to keep it in)
    __shared__ int abort_flag;

    const tt_cache& c = g.a.cache;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, head = blockIdx.y;
    volatile int* abortp = &abort_flag;
    pdl_wait_prev();
    TileView view;
    const long long unit = (long long)gridDim.x - 1 - blockIdx.x;       // (the last tiles see the most; all heads' last ones first: 253 us for 249)
    if (!view_tile(g, kPromptRows, unit, view)) return;
    const int base_token = view.lo / kPromptTokens * kPromptTokens;
    const int active = prompt_splits(g, view);
    if ((int)blockIdx.z >= active) return;
    const int from = base_token + (int)blockIdx.z * g.chunk, to = view.hi - from > g.chunk ? from + g.chunk : view.hi;
    const int steps = to > from ? (to - from - 1) / kPromptTokens + 1 : 0;
    const int tiles = view.rows > 128 ? 2 : 1;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, k_s = base + 2u * S::kTile, v_s = base + 4u * S::kTile;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&q_full), 16u);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&k_full[i]), 5u); mbar_init(smem_u32(&v_full[i]), 4u);
            mbar_init(smem_u32(&k_empty[i]), 1u); mbar_init(smem_u32(&v_empty[i]), 1u);
            mbar_init(smem_u32(&s_full[i]), 1u); mbar_init(smem_u32(&p_ready[i][0]), 8u); mbar_init(smem_u32(&p_ready[i][1]), 8u); mbar_init(smem_u32(&o_done[i]), 1u);
        }
        mbar_init(smem_u32(&raw_full[0]), 1u); mbar_init(smem_u32(&raw_full[1]), 1u);
        mbar_init(smem_u32(&raw_empty[0]), 4u); mbar_init(smem_u32(&raw_empty[1]), 4u);
        mbar_init(smem_u32(&drained), 1u);
        abort_flag = nan_any = 0;
        late[0] = view.start + view.t0; late[1] = view.h0; late[2] = view.rows; late[3] = active; late[4] = view.before + view.t0; late[5] = view.hi;
        fence_mbar_init();
        fence_proxy_async_shared();
    }
    if ((int)threadIdx.x < D) { nan_first[threadIdx.x] = INT_MAX; nan_last[threadIdx.x] = INT_MIN; }
    if (warp == 20) {
        tmem_alloc(smem_u32(&tmem_slot), 512u);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t*)&tmem_slot;
    pdl_allow_next();                                                     // (the next launch may take tensor memory: this CTA has its own)

    // a softmax thread's row
    const int tile = warp >> 3, half = (warp >> 2) & 1, r = tile * 128 + (int)(threadIdx.x & 127);      // (a half of its columns)
    float top = -INFINITY, used = 0.f, sum = 0.f;                         // maximum; the one that O and the sum are relative to
    bool fine = true;

    if (warp < 16) {
        registers_up<96>();
        // ---------------- queries: a row as 16-bit floating point with a maximum of 2^14..2^15 ----------------
        // Eight lanes have a row, a warp 16 rows of its tile: what it loads lies side by side.  (The two prompts above: a thread a
        // row, in queries and outputs, 317 us; four values a lane 257; so 250.)
        const auto stage = [&](auto type) {
            constexpr int TYPE = decltype(type)::value, kPieces = D / 64;
            const int row0 = tile * 128 + (warp & 7) * 16 + (lane >> 3);
            int t = (view.h0 + row0) / g.group, h = view.h0 + row0 - t * g.group;
            long long at = ((long long)view.start + view.t0 + t) * g.a.q_token + (long long)(head * g.group + h) * g.a.q_head + 8 * (lane & 7);
            Eights<TYPE, kPieces> x[4];
            const auto load = [&](auto wide) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
#pragma unroll
                    for (int p = 0; p < kPieces; ++p) x[k].raw[p] = row0 + 4 * k < view.rows && 64 * p + 8 * (lane & 7) < c.d ? raw_eight(g.a.q, at + 64 * p, decltype(wide)::value) : make_uint4(0u, 0u, 0u, 0u);
                    h += 4; at += 4 * g.a.q_head;
                    while (h >= g.group) { h -= g.group; at += g.a.q_token - g.group * g.a.q_head; }
                }
            };
            // (a branch for all loads: one for each makes them wait for each other)
            if (g.q_wide == 2) load(std::integral_constant<int, 2>());
            else if (g.q_wide == 1) load(std::integral_constant<int, 1>());
            else load(std::integral_constant<int, 0>());
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float most = x[k].most();
                if (!(most < INFINITY)) most = x[k].finite_most();
#pragma unroll
                for (int d = 1; d < 8; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
                const int ex = most > 0.f ? (__float_as_int(most) >> 23) : 127 + 14, size = min(254, max(1, 127 + 14 + 127 - ex));
                const float up = __int_as_float(size << 23 | (g.scale_log2 < 0.f ? 1 << 31 : 0));      // (the factor of the scores is positive: their maximum is the products')
                const int row = row0 + 4 * k, lr = row & 127;
#pragma unroll
                for (int p = 0; p < kPieces; ++p) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) { const float2 v = x[k].pair(4 * p + e); w[e] = down2<TT_TYPE_F16>(v.x * up, v.y * up); }
                    const int i = 8 * p + (lane & 7);
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(q_s + (uint32_t)tile * S::kTile + (uint32_t)(i % S::kAtoms) * kAtom + (uint32_t)lr * 128u + ((uint32_t)((i / S::kAtoms) ^ (lr & 7)) << 4)),
                                 "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
                if ((lane & 7) == 0) sizes[row] = (uint8_t)size;
            }
        };
        if (g.a.type == TT_TYPE_F16) stage(std::integral_constant<int, TT_TYPE_F16>());
        else stage(std::integral_constant<int, TT_TYPE_BF16>());
        fence_proxy_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&q_full));
        named_sync(4 + tile, 256);
        const float factor = fabsf(g.scale_log2) / __int_as_float((int)sizes[r] << 23);
        // From here on it is the exponent of the largest scale that the row has seen, looked after where rows are apart.  (Both threads of a row put the
        // same there, and a step's barrier is between theirs and the next step's.)
        volatile uint8_t* const row_ref = &sizes[r];
        named_sync(4 + tile, 256);
        *row_ref = 0;

        // ---------------- softmax ----------------
        const volatile int* out = late;
        // the row's position, and the tokens lo .. hi - 1 that it sees (looked up again wherever they are needed)
        struct Seen { int pos, lo, hi; };
        const auto seen_by_row = [&] {
            const int pos = out[4] + (out[1] + r) / g.group;
            return Seen{pos, g.a.window > 0 ? pos + 1 - g.a.window : 0, g.a.causal ? min(out[5], pos + 1) : out[5]};
        };
        const uint32_t s_t = tmem + ((uint32_t)((warp & 3) * 32) << 16) + S::kScores + (uint32_t)tile * 128u;
        const uint32_t o_t = tmem + ((uint32_t)((warp & 3) * 32) << 16) + S::kOut + (uint32_t)(tile * D);
        if (tile < tiles) {
            for (int i = 0; i < steps; ++i) {
                // (a warp that gives up goes on, without waiting: the others of its tile meet it below)
                fine = fine && __all_sync(0xffffffffu, bounded_wait(&s_full[tile], (uint32_t)i & 1u, abortp, g.a.status, 31u, kPromptWait));
                tc_fence_after();
                const int t = from + i * kPromptTokens;
                const bool whole = t >= view.whole_lo && t + kPromptTokens <= view.whole_hi;
                // This half has columns 32 * half .. + 31 and the 32 that are 64 further on (so both halves' first 32 let a product begin); of a
                // place k, `column` is relative to 32 * half, and the row sees columns j_lo .. j_hi - 1.
                const auto column = [](int k) { return k < 32 ? k : k + 32; };
                uint32_t v[64];
#pragma unroll
                for (int h = 0; h < 2; ++h) tmem_ld32(s_t + 32u * (uint32_t)half + 64u * h, *reinterpret_cast<uint32_t(*)[32]>(&v[32 * h]));
                tmem_wait_ld();
                if (!whole) {
                    const Seen s = seen_by_row();
                    const int j_lo = s.lo - t - 32 * half, j_hi = s.hi - t - 32 * half;
#pragma unroll
                    for (int k = 0; k < 64; ++k) v[k] = column(k) >= j_lo && column(k) < j_hi ? v[k] : 0xff800000u;      // (-inf)
                }
                const uint32_t info = smem_u32(&scales[i & 3]) + 8u * (uint32_t)half;
                const auto four_of = [&](uint32_t at) { const float2 a = ld_shared_v2f(at), b = ld_shared_v2f(at + 16u); return make_float4(a.x, a.y, b.x, b.y); };
                float4 keys = four_of(info);
                float m[4];
#pragma unroll
                for (int gr = 0; gr < 4; ++gr) m[gr] = fmaxf(__uint_as_float(v[16 * gr]), __uint_as_float(v[16 * gr + 1]));
#pragma unroll
                for (int k = 2; k < 16; k += 2)
#pragma unroll
                    for (int gr = 0; gr < 4; ++gr) m[gr] = max_of(m[gr], __uint_as_float(v[16 * gr + k]), __uint_as_float(v[16 * gr + k + 1]));
                // (a factor of 0, of a page of zeros, would make NaN of -inf: the smallest one does as well; NaN stays)
                const auto factor_of = [&](float key) { return max_or_nan(factor * key, 1.17549435e-38f); };
                keys = make_float4(factor_of(keys.x), factor_of(keys.y), factor_of(keys.z), factor_of(keys.w));
                float mx = max_of(fmaxf(m[0] * keys.x, m[1] * keys.y), m[2] * keys.z, m[3] * keys.w);
                // The halves tell each other their maxima in tensor memory, in a column that its writer has read and that nobody but the reader writes next.
                tmem_st1(s_t + (half ? 32u : 16u), mx);
                tmem_wait_st();
                tc_fence_before();
                named_sync(4 + tile, 256);
                tc_fence_after();
                const float seen = top;
                top = max_of(top, mx, tmem_ld1(s_t + (half ? 16u : 32u)));
                // O and the sum follow the maximum when it is 2^8 ahead, and the largest scale at once
                const float shrink = ld_shared_f32(smem_u32(&scales[i & 3].shrink));
                const bool first = seen != top && seen == -INFINITY;      // the row's first visible token is in this step
                const bool move = top > used + 8.f || first || shrink != 1.f;
                if (__any_sync(0xffffffffu, move)) {
                    float now = top;
                    if (__float_as_int(shrink) < 0) {
                        const Seen s = seen_by_row();
                        int own = max((int)*row_ref, scales[i & 3].common);
                        // (a scale that is not finite reaches the rows that see its page by their factor, and no others)
#pragma unroll 1
                        for (int k = 0; k < 8; ++k) {
                            const int value = scales[i & 3].value[k];
                            const bool sees = t + 16 * k < s.hi && t + 16 * k + 16 > s.lo;
                            if (sees && value < 255) own = max(own, value);
                            else if ((k >> 1 & 1) == half) {
                                const float f = sees ? __int_as_float(0x7fffffff) : 1.17549435e-38f;
                                const int gr = (k & 1) + 2 * (k >> 2);
                                keys = make_float4(gr == 0 ? f : keys.x, gr == 1 ? f : keys.y, gr == 2 ? f : keys.z, gr == 3 ? f : keys.w);
                            }
                        }
                        *row_ref = (uint8_t)own;
                        now -= (float)min(100, max(0, exponent_of(scales[i & 3].ref) - own));
                    }
                    if (top == -INFINITY) now = 0.f;
                    const float alpha = seen != -INFINITY ? exp2_fast(used - now) : 0.f;
                    const float scale_o = alpha * fabsf(shrink);
                    used = now;
                    sum *= alpha;
                    if (i > 0 && half == 0) {                             // (in front of the first half of P, which lets the product begin)
                        fine = fine && __all_sync(0xffffffffu, bounded_wait(&o_done[tile], (uint32_t)(i - 1) & 1u, abortp, g.a.status, 32u, kPromptWait));
                        tc_fence_after();
#pragma unroll 1
                        for (int h = 0; h < D; h += 16) {                 // (few at a time: the scores are in registers)
                            uint32_t o[16];
                            tmem_ld8(o_t + (uint32_t)h, o);
                            tmem_ld8(o_t + (uint32_t)h + 8u, o + 8);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * scale_o);
                            tmem_st8u(o_t + (uint32_t)h, o);
                            tmem_st8u(o_t + (uint32_t)h + 8u, o + 8);
                        }
                    }
                }
                const float4 shift = four_of(info + 32u), back = four_of(info + 64u);
#pragma unroll
                for (int gr = 0; gr < 4; ++gr) {
                    const float f = gr == 0 ? keys.x : gr == 1 ? keys.y : gr == 2 ? keys.z : keys.w;
                    const float add = (gr == 0 ? shift.x : gr == 1 ? shift.y : gr == 2 ? shift.z : shift.w) - used;
                    float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    uint32_t p[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float2 e = fma_pair(make_float2(__uint_as_float(v[16 * gr + 2 * k]), __uint_as_float(v[16 * gr + 2 * k + 1])), make_float2(f, f), make_float2(add, add));
                        e.x = exp2_fast(e.x);
                        e.y = exp2_fast(e.y);
                        part[k & 1] = add_pair(part[k & 1], e);
                        p[k] = down2<TT_TYPE_F16>(e.x, e.y);
                    }
                    part[0] = add_pair(part[0], part[1]);
                    sum = fmaf(part[0].x + part[0].y, gr == 0 ? back.x : gr == 1 ? back.y : gr == 2 ? back.z : back.w, sum);
                    tmem_st8u(s_t + 16u * (uint32_t)half + (gr < 2 ? 8u * gr : 16u + 8u * gr), p);
                    if (gr & 1) {
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&p_ready[tile][gr >> 1]));
                    }
                }
            }
        }
        // ---------------- out ----------------
        named_sync(1, kSoftmax + 128);                                               // (every NaN of the steps at the edges has been noted)
        const int token0 = out[0], h0 = out[1], rows = out[2], active = out[3];
        const bool mine = r < rows;
        const long long place = unit * c.heads + head;
        constexpr int kPart = kPromptRows * (D + 2);                     // O by eight columns of all rows, then the rows' maxima and sums
        if (tile < tiles) {
            if (steps > 0 && fine) fine = __all_sync(0xffffffffu, bounded_wait(&o_done[tile], (uint32_t)(steps - 1) & 1u, abortp, g.a.status, 32u, kPromptWait));
            tc_fence_after();
            if (steps > 0) {
                // the row's sum: both halves', by way of the scores' columns (every product that read them is done)
                tmem_st1(s_t + (half ? 64u : 32u), sum);
                tmem_wait_st();
                tc_fence_before();
                named_sync(4 + tile, 256);
                tc_fence_after();
                sum += tmem_ld1(s_t + (half ? 32u : 64u));
            }
            const Seen s = seen_by_row();
            const int row_pos = s.pos;
            const bool none = steps == 0 || s.hi <= max(s.lo, from) || s.lo >= to;      // the row sees nothing here
            // O is in units of 2^7 and the largest scale; a split's part stays relative to its sum
            const float ref = steps > 0 ? ld_shared_f32(smem_u32(&scales[(steps - 1) & 3].ref)) : 0.f;
            const float unit_o = 0.0078125f * (active == 1 ? 1.f / sum : 1.f);      // (the scale apart: 2^-126 times this is no normal number)
            float* left = g.partial + (place * g.splits + blockIdx.z) * kPart + 8 * r;
            const uint32_t line = q_s + (uint32_t)tile * S::kTile + (uint32_t)(r & 127) * (2u * D);      // (where the queries were)
#pragma unroll 1
            for (int h = half * (D / 2); h < (half + 1) * (D / 2); h += 16) {
                uint32_t v[16];
                if (steps > 0) {
                    tmem_ld8(o_t + (uint32_t)h, v);
                    tmem_ld8(o_t + (uint32_t)h + 8u, v + 8);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int j = 0; j < 16; j += 8) {
                    const int n = h + j, first = n % 64 / 8 * 8 * S::kAtoms + n / 64 * 8;      // the place of columns n .. n + 7 in the head
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = none ? 0.f : __uint_as_float(v[j + e]) * unit_o * ref;
                    if (nan_any) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (nan_first[first + e] <= row_pos || (g.a.window > 0 && nan_last[first + e] > row_pos - g.a.window)) x[e] = __int_as_float(0x7fffffff);
                    }
                    if (active == 1) {
                        const bool f16 = g.a.type == TT_TYPE_F16;
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = f16 ? down2<TT_TYPE_F16>(x[2 * e], x[2 * e + 1]) : down2<TT_TYPE_BF16>(x[2 * e], x[2 * e + 1]);
                        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(line + (((uint32_t)(first >> 3) ^ (uint32_t)(r & 7)) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                    } else if (mine && fine) {
                        *reinterpret_cast<float4*>(left + first * kPromptRows) = make_float4(x[0], x[1], x[2], x[3]);
                        *reinterpret_cast<float4*>(left + first * kPromptRows + 4) = make_float4(x[4], x[5], x[6], x[7]);
                    }
                }
            }
            if (active > 1 && mine && fine && half == 0) *reinterpret_cast<float2*>(g.partial + (place * g.splits + blockIdx.z) * kPart + (long long)kPromptRows * D + 2 * r) = make_float2(used, none ? 0.f : sum);
            if (active == 1) {
                named_sync(4 + tile, 256);
                // rows of a tile to its warps, so that what a warp stores lies side by side
                constexpr int kAcross = D / 8, kAtOnce = 32 / kAcross;
                const int i = lane % kAcross;
                int row = tile * 128 + (warp & 7) * 16 + lane / kAcross, t = (h0 + row) / g.group, h = h0 + row - t * g.group;
                long long at = ((long long)token0 + t) * g.a.y_token + (long long)(head * g.group + h) * g.a.y_head + 8 * i;
#pragma unroll 4
                for (int k = 0; k < 16; k += kAtOnce, row += kAtOnce) {
                    uint32_t w[4];
                    read_shared<16>(q_s + (uint32_t)row * (2u * D) + (((uint32_t)i ^ (uint32_t)(row & 7)) << 4), w);
                    if (row < rows && 8 * i < c.d && fine) {
                        uint16_t* y = static_cast<uint16_t*>(g.a.y) + at;
                        if (g.y_wide == 2) *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
                        else if (g.y_wide) {
                            *reinterpret_cast<uint2*>(y) = make_uint2(w[0], w[1]);
                            *reinterpret_cast<uint2*>(y + 4) = make_uint2(w[2], w[3]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                        }
                    }
#pragma unroll
                    for (int next = 0; next < kAtOnce; ++next) {
                        at += g.a.y_head;
                        if (++h == g.group) { h = 0; at += g.a.y_token - g.group * g.a.y_head; }
                    }
                }
            }
        }
        tc_fence_before();
        __syncwarp();
        named_arrive(2, kSoftmax + 32);                                             // (the tensor memory has been read)
    } else if (warp < 20) {
        registers_down<56>();
        // ---------------- keys and values: pages -> operand tiles ----------------
        // A step's bytes arrive by TMA, a step ahead.  Eight lanes have a token; the four warps take the 16 tokens of a group at a time, and a lane turns
        // kPiece values into one 16-byte chunk of each atom's line (all banks at once): value kPiece * lane + 8 a + e of a head is value e of chunk
        // `lane` of atom a, and the queries and the outputs are ordered alike.
        constexpr int kPiece = 8 * S::kAtoms;
        const int dt = (int)threadIdx.x - kSoftmax, piece = dt & 7, sub = dt >> 3;
        constexpr uint32_t kGroup = 128u * kPiece;                                               // bytes of a group of 16 tokens
        const uint32_t raw = base + 6u * S::kTile + (uint32_t)(dt * kPiece);                    // (keys; the values' behind them)
        const uint32_t chunk = (uint32_t)sub * 128u + ((((uint32_t)piece) ^ ((uint32_t)sub & 7u)) << 4);
        const auto put = [&](uint32_t tile_s, int group, const uint32_t (&w)[kPiece / 4]) {
#pragma unroll
            for (int a = 0; a < S::kAtoms; ++a) {
                uint32_t h[4];
                f16_pairs_of_e4m3(w[2 * a], h[0], h[1]);
                f16_pairs_of_e4m3(w[2 * a + 1], h[2], h[3]);
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(tile_s + chunk + (uint32_t)a * kAtom + (uint32_t)group * 2048u), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
            }
        };
        // the last step's tokens behind `to`, and those in front of what any row sees, may be anything: zeros
        const auto bytes_of = [&](int w, int p, int t, bool edge, uint32_t (&x)[kPiece / 4]) {
            read_shared<kPiece>(raw + (uint32_t)(8 * w + p) * kGroup, x);
            if (edge) {
                const int tok = t + 16 * p + sub;
                if (tok < view.lo || tok >= to) {
#pragma unroll
                    for (int q = 0; q < kPiece / 4; ++q) x[q] = 0u;
                }
            }
        };
        for (int i = 0; i < steps && fine; ++i) {
            const int t = from + i * kPromptTokens, buf = i & 1;
            const bool edge = t < view.lo || t + kPromptTokens > to;
            const auto wait = [&](uint64_t* bar, uint32_t parity, unsigned where) { return bounded_wait(bar, parity, abortp, g.a.status, where, kPromptWait); };
            fine = __all_sync(0xffffffffu, wait(&k_empty[buf], ((uint32_t)(i >> 1) & 1u) ^ 1u, 33u) && wait(&raw_full[0], (uint32_t)i & 1u, 40u));
            if (!fine) break;
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                uint32_t w[kPiece / 4];
                bytes_of(0, p, t, edge, w);
                put(k_s + (uint32_t)buf * S::kTile, p, w);
            }
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) { mbar_arrive(smem_u32(&raw_empty[0])); mbar_arrive(smem_u32(&k_full[buf])); }
            fine = __all_sync(0xffffffffu, wait(&v_empty[buf], ((uint32_t)(i >> 1) & 1u) ^ 1u, 34u) && wait(&raw_full[1], (uint32_t)i & 1u, 41u));
            if (!fine) break;
            const bool low = t < view.whole_lo, high = g.a.causal && t + kPromptTokens > view.whole_hi;
            if (low || high) {
#pragma unroll 1
                for (int p = 0; p < 8; ++p) {
                    uint32_t w[kPiece / 4];
                    bytes_of(1, p, t, edge, w);
#pragma unroll
                    for (int q = 0; q < kPiece / 4; ++q) {
                        const uint32_t n = nan_bytes(w[q]);
                        if (n == 0u) continue;
                        nan_any = 1;
                        for (int e = 0; e < 4; ++e)
                            if ((n >> (8 * e)) & 0x80u) {
                                if (high) atomicMin(&nan_first[kPiece * piece + 4 * q + e], t + 16 * p + sub);
                                else atomicMax(&nan_last[kPiece * piece + 4 * q + e], t + 16 * p + sub);
                            }
                        w[q] &= ~((n >> 7) * 0xffu);
                    }
                    put(v_s + (uint32_t)buf * S::kTile, p, w);
                }
            } else {
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    uint32_t w[kPiece / 4];
                    bytes_of(1, p, t, edge, w);
                    put(v_s + (uint32_t)buf * S::kTile, p, w);
                }
            }
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) { mbar_arrive(smem_u32(&raw_empty[1])); mbar_arrive(smem_u32(&v_full[buf])); }
        }
        named_arrive(1, kSoftmax + 128);
    } else {
        registers_down<40>();
        if (warp == 21 && steps > 0) {
            // ---------------- pages, scales, copies ----------------
            // lane g of the first eight has the page of a step's group g, and its scales; what is looked up is used a step later
            const int* table = c.table + view.b * c.table_row;
            const int shift = 31 - __clz(c.block), box = min(c.block, kPromptTokens);                // tokens of a box
            const uint32_t raw0 = base + 6u * S::kTile;
            // (a box is copied as a whole, by its first group's page: it is held if any of its tokens is)
            const auto held = [&](int i) { const int t = from + i * kPromptTokens + (16 * (lane & 7) & ~(box - 1)); return i < steps && t + box > view.lo && t < to; };
            const auto page_of = [&](int i) { return held(i) ? table[(from + i * kPromptTokens + 16 * (lane & 7)) >> shift] : -1; };
            const auto good = [&](int i, int pg) {
                if ((unsigned)pg < (unsigned)c.pages) return pg;
                if (held(i)) report_invalid(g.a.status);
                return -1;                                                // (a box outside of the tensor is zeros)
            };
            const auto scale_of = [&](int pg, int w) { return pg >= 0 ? c.scale[w][pg * c.s_page[w] + head * c.s_head[w]] : 0.f; };
            const auto wait = [&](uint64_t* bar, uint32_t parity, unsigned where) { return __all_sync(0xffffffffu, bounded_wait(bar, parity, abortp, g.a.status, where, kPromptWait)); };
            const auto fetch = [&](int i, int pages, int w) {
                if (lane == 0) mbar_expect_tx(smem_u32(&raw_full[w]), 128u * (uint32_t)D);
                for (int p = 0; p < kPromptTokens; p += box) {
                    const int pg = __shfl_sync(0xffffffffu, pages, p >> 4);
                    if (lane == 0) tma_load_4d(raw0 + (uint32_t)(w * 128 + p) * (uint32_t)D, w ? &tmap_v : &tmap_k, smem_u32(&raw_full[w]), 0, (from + i * kPromptTokens + p) & (c.block - 1), head, pg);
                }
            };
            int page = good(0, page_of(0)), page1 = page_of(1);
            float ks = scale_of(page, 0), vs = scale_of(page, 1), most = 0.f;      // most: the largest scale of values so far
            int common = 0;
            fetch(0, page, 0);
            fetch(0, page, 1);
            for (int i = 0; i < steps; ++i) {
                const int buf = i & 1, page2 = page_of(i + 2), next = good(i + 1, page1);
                const float ks1 = scale_of(next, 0), vs1 = scale_of(next, 1);
                // the scales, before the keys report: what lay here four steps ago has been read
                if (!wait(&k_empty[buf], ((uint32_t)(i >> 1) & 1u) ^ 1u, 42u)) break;
                const float value = vs < INFINITY ? vs : 0.f;
                float m = value;
#pragma unroll
                for (int d = 4; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                const float before = most;
                most = fmaxf(most, m);
                const int group_t = from + i * kPromptTokens + 16 * (lane & 7), exponent = vs < INFINITY ? exponent_of(vs) : 255;
                common = max(common, __reduce_max_sync(0xffffffffu, group_t < view.whole_hi && group_t + 16 > view.whole_lo && exponent < 255 ? exponent : 0));
                const bool odd = __any_sync(0xffffffffu, exponent == 255 || !(ks < INFINITY));
                if (lane < 8) {
                    StepScales& sc = scales[i & 3];
                    // (a share of less than 2^-100 of the largest scale is taken as that: a row's sum has all probabilities of 2^-33 and more)
                    const float unit = most > 0.f ? fmaxf(__fdividef(value, most), 7.888609052210118e-31f) : 1.f, lg = value == most ? 0.f : log2f(unit);
                    sc.key[lane] = ks;
                    sc.shift[lane] = lg + 7.f;
                    sc.back[lane] = exp2_fast(-lg) * 0.0078125f;
                    sc.value[lane] = (uint8_t)exponent;
                    if (lane == 0) {
                        const float shrink = before == most ? 1.f : __fdividef(before, most);
                        sc.ref = most;
                        sc.shrink = odd || exponent_of(most) > common + 4 ? -shrink : shrink;
                        sc.common = common;
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&k_full[buf]));
                if (i + 1 < steps) {
                    if (!wait(&raw_empty[0], (uint32_t)i & 1u, 43u)) break;
                    fetch(i + 1, next, 0);
                    if (!wait(&raw_empty[1], (uint32_t)i & 1u, 44u)) break;
                    fetch(i + 1, next, 1);
                }
                page1 = page2;
                ks = ks1;
                vs = vs1;
            }
            // shared memory stays until the copies have landed, also when somebody gave up (bounded)
            const unsigned long long t0 = global_timer_ns();
            while (*abortp && global_timer_ns() - t0 < 2000000ull) { }
        }
        // ---------------- MMA issuer ----------------
        if (warp == 20 && steps > 0 && elect_one()) {
            constexpr uint32_t kIdescS = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
            constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);     // values: the columns are the contiguous axis
            const uint64_t dk = make_desc(0u, 128);
            // an MN-major tile: groups of eight tokens 1024 bytes apart, the next 64 columns an atom's 16 KB further on
            const uint64_t dv = (uint64_t)(kAtom >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | 1ull << 46 | 2ull << 61;
            const auto at = [](uint32_t a) { return (uint64_t)((a & 0x3FFFFu) >> 4); };
            const auto wait = [&](uint64_t* bar, uint32_t parity, unsigned where) { return bounded_wait(bar, parity, abortp, g.a.status, where, kPromptWait); };
            const auto scores = [&](int tl, int buf) {
                const uint64_t a = dk + at(q_s + (uint32_t)tl * S::kTile), b = dk + at(k_s + (uint32_t)buf * S::kTile);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_f16(tmem + S::kScores + (uint32_t)tl * 128u, a + (uint64_t)((k >> 2) * (kAtom >> 4) + 2 * (k & 3)), b + (uint64_t)((k >> 2) * (kAtom >> 4) + 2 * (k & 3)), kIdescS, k > 0 ? 1u : 0u);
                mma_commit(smem_u32(&s_full[tl]));
            };
            bool ok = wait(&q_full, 0u, 35u) && wait(&k_full[0], 0u, 36u);
            if (ok) {
                tc_fence_after();
                for (int tl = 0; tl < tiles; ++tl) scores(tl, 0);
                mma_commit(smem_u32(&k_empty[0]));
            }
            for (int i = 0; i < steps && ok; ++i) {
                const int buf = i & 1, next = (i + 1) & 1;
                for (int tl = 0; tl < tiles && ok; ++tl) {
                    // (the first half of P is multiplied while the second is being written)
                    ok = (tl > 0 || wait(&v_full[buf], (uint32_t)(i >> 1) & 1u, 38u)) && wait(&p_ready[tl][0], (uint32_t)i & 1u, 37u);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t b = dv + at(v_s + (uint32_t)buf * S::kTile);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_f16_ta(tmem + S::kOut + (uint32_t)(tl * D), tmem + S::kScores + (uint32_t)(tl * 128 + 8 * k), b + (uint64_t)(128 * k), kIdescO, i > 0 || k > 0 ? 1u : 0u);
                    ok = wait(&p_ready[tl][1], (uint32_t)i & 1u, 37u);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 4; k < 8; ++k)
                        mma_f16_ta(tmem + S::kOut + (uint32_t)(tl * D), tmem + S::kScores + (uint32_t)(tl * 128 + 8 * k), b + (uint64_t)(128 * k), kIdescO, i > 0 || k > 0 ? 1u : 0u);
                    mma_commit(smem_u32(&o_done[tl]));
                    if (tl == tiles - 1) mma_commit(smem_u32(&v_empty[buf]));
                    if (i + 1 < steps) {
                        // the next scores take P's place, behind the product that reads it
                        ok = tl > 0 || wait(&k_full[next], (uint32_t)((i + 1) >> 1) & 1u, 39u);
                        if (!ok) break;
                        tc_fence_after();
                        scores(tl, next);
                        if (tl == tiles - 1) mma_commit(smem_u32(&k_empty[next]));
                    }
                }
            }
            // nothing of what was issued is to run on behind this CTA, also when somebody gave up (bounded)
            mma_commit(smem_u32(&drained));
            const unsigned long long t0 = global_timer_ns();
            while (!mbar_try_wait(smem_u32(&drained), 0u)) if (global_timer_ns() - t0 > kPromptWait) break;
        }
        if (warp == 20) {
            __syncwarp();
            named_sync(2, kSoftmax + 32);
            tc_fence_after();
            tmem_dealloc(tmem, 512u);
        }
    }
}

// The splits of a tile together, kBandRows of its rows a CTA, in the order of the splits.  A kernel of its own: what one SM reads of another's results
// comes at 14 bytes a cycle, and a split of a tile is 130 KB.  (Two prompts of 300
// tokens over 8000, 4 heads over one of 128: 40 us; joined by the last CTA of a tile 79.)
constexpr int kBandRows = 16;
template <int D>
__global__ void __launch_bounds__(128) tt_attend_join_kernel(const Attend g) {
    __shared__ float share[kPromptSplits * kBandRows];
    pdl_allow_next();
    pdl_wait_prev();
    const tt_cache& c = g.a.cache;
    constexpr int kBands = kPromptRows / kBandRows, kPart = kPromptRows * (D + 2);
    const int head = blockIdx.y, row0 = (int)blockIdx.x % kBands * kBandRows;
    const long long unit = blockIdx.x / kBands;
    TileView view;
    if (!view_tile(g, kPromptRows, unit, view)) return;
    const int active = prompt_splits(g, view), rows = min(kBandRows, view.rows - row0);
    if (active == 1 || rows <= 0) return;
    const float* parts = g.partial + (unit * c.heads + head) * g.splits * kPart;
    // eight lanes have a row: its maxima and sums of the splits
    const int r = (int)threadIdx.x >> 3, l = (int)threadIdx.x & 7;
    constexpr int kOwn = kPromptSplits / 8;
    float2 ml[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        if (l + 8 * k < active && r < rows) ml[k] = *reinterpret_cast<const float2*>(parts + (long long)(l + 8 * k) * kPart + kPromptRows * D + 2 * (row0 + r));
    }
    float mx = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) if (ml[k].y != 0.f) mx = fmaxf(mx, ml[k].x);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        ml[k].x = ml[k].y != 0.f ? exp2_fast(ml[k].x - mx) : 0.f;
        if (ml[k].y != 0.f) sum += ml[k].y * ml[k].x;
    }
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) share[(l + 8 * k) * kBandRows + r] = ml[k].x * inv;
    __syncthreads();
    join_splits<128>(rows * (D / 4), active,
        [&](int e, int z) { const int rr = row0 + e / (D / 4), i = 4 * (e % (D / 4)); return reinterpret_cast<const float4*>(parts + (long long)z * kPart + (i >> 3) * (8 * kPromptRows) + 8 * rr + (i & 4)); },
        [&](int e, int z) { return share[z * kBandRows + e / (D / 4)]; },
        [&](int e, const float (&v)[4]) {
            const int rr = view.h0 + row0 + e / (D / 4), i = 4 * (e % (D / 4)), t = rr / g.group;
            if (i < c.d) store_four(g.a.y, (view.start + view.t0 + (long long)t) * g.a.y_token + (long long)(head * g.group + rr - t * g.group) * g.a.y_head + i, g.a.type, g.y_wide, v);
        });
}

template <int D>
static cudaError_t launch_prompt(const Attend& g, long long units, void* stream) {
    typedef PromptShape<D> S;
    static OncePerDevice raised;
    const cudaError_t ready = raised([] { return cudaFuncSetAttribute(tt_attend_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kBytes); });
    if (ready != cudaSuccess) return ready;
    CUtensorMap maps[2];
    const tt_cache& c = g.a.cache;
    for (int w = 0; w < 2; ++w) {
        // (without pages nothing is read: the map is of any memory)
        const tt_status st = g.max_length > 0 ? encode_pages(&maps[w], c.data[w], c.d, c.block, c.heads, c.pages, c.token[w], c.head[w], c.page[w], D, false, c.block)
                                              : encode_pages(&maps[w], reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(g.a.y) & ~uintptr_t(15)), c.d, c.block, 1, 1, c.d, c.d, c.d, D, false, c.block);
        if (st != TT_OK) return cudaErrorInvalidValue;
    }
    const cudaError_t e = launch(tt_attend_prompt_kernel<D>, dim3((unsigned)units, (unsigned)g.a.cache.heads, (unsigned)g.splits), kPromptThreads, S::kBytes, 1, stream, maps[0], maps[1], g);
    if (e != cudaSuccess || g.splits == 1) return e;
    return launch(tt_attend_join_kernel<D>, dim3((unsigned)units * (kPromptRows / kBandRows), (unsigned)g.a.cache.heads, 1), 128, 0, 1, stream, g);
}
cudaError_t launch_attend_prompt(const Attend& g, long long units, void* stream) {
    return prompt_head(g.a.cache.d) == 64 ? launch_prompt<64>(g, units, stream) : launch_prompt<128>(g, units, stream);
}

}  // namespace tt
