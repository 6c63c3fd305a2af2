// Attention of prompts over the paged e4m3 cache: many rows (queries of the heads that share a key head) for each key, so the products and the
// exponentials are the bound, not the cache's bytes.
//
// A CTA has two tiles of 128 rows and walks the keys 128 at a time.  Four warps bring keys and values from the pages, turn them into 16-bit floating
// point (exactly) and leave them as operand tiles, which serve both tiles of rows.  S = Q K^T goes to tensor memory; a thread of the softmax warps
// has one row of it, takes its maximum, and leaves P = 2^(s - m) in S's place as the first operand of O += P V, whose sums stay
// in tensor memory.  While one tile's softmax runs, the tensor core is at the other tile's products.
//   O is multiplied only when a maximum has grown by more than 2^8 since it was last: P may be up to 2^8 times what it
// would be, which 16 bits have room for (it is brought to 2^15 at most), and the row's sum has the same factor.  A page's scale of values is in
// P too, as the part of the exponent, over the largest scale so far.
//   NaN in values that only some rows of the tile see (the steps at the edge of what is visible) are taken out of the product and put into
// the outputs of the rows that do: a column's first such token (at the upper edge; its last one at the lower) decides.
#include <cuda_runtime.h>
#include <climits>
#include "tt_cache.cuh"

namespace tt {

constexpr int kPromptThreads = 512;         // warps 0-3 and 4-7 softmax of a tile each, 8-11 keys and values, 12 MMA and tensor memory
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
// 32 columns from here on.
__device__ __forceinline__ void tmem_st32u(uint32_t taddr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                   "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
                   "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]));
}
__device__ __forceinline__ float max_of(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ void tmem_ld8u(uint32_t taddr, uint32_t* v) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(taddr) : "memory");
}
// N bytes to shared memory, or N zeros.
template <int N>
__device__ __forceinline__ void copy_async_or_zero(uint32_t dst, const void* src, bool copy) {
    const int bytes = copy ? N : 0;
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(bytes), "n"(N) : "memory");
}
// Registers of a warpgroup from here on.  512 threads begin with 128 each (65536): 184 for the softmax's
// two, 96 and 40 for the others make 64512.
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Named barriers: 1 the softmax and the warps of keys and values, 2 the softmax and the MMA warp (at the end), 3 the softmax alone.
__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void named_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// What the softmax needs to know of a step's eight groups of 16 tokens.
struct alignas(16) StepScales { float key[8], shift[8], back[8]; float ref; };

template <int D>
struct PromptShape {
    static constexpr int kAtoms = D / 64;
    static constexpr uint32_t kTile = kAtoms * kAtom;                    // bytes of 128 rows of queries, keys or values
    static constexpr uint32_t kBytes = 1024u + 7u * kTile;               // two of each, and the bytes of the next keys and values
    static constexpr uint32_t kScores = 0, kOut = 256;                   // columns of tensor memory: S (and P) of both tiles, O of both
};

template <int D>
__global__ void __launch_bounds__(kPromptThreads, 1) tt_attend_prompt_kernel(const __grid_constant__ Attend g) {
    typedef PromptShape<D> S;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_ready[2][2], o_done[2], drained;
    __shared__ StepScales scales[4];
    __shared__ int nan_first[D], nan_last[D];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, last_one;

    const tt_cache& c = g.a.cache;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, head = blockIdx.y;
    volatile int* abortp = &abort_flag;
    pdl_wait_prev();
    TileView view;
    const long long unit = (long long)gridDim.x - 1 - blockIdx.x;       // (the last tiles see the most)
    if (!view_tile(g, kPromptRows, unit, view)) return;
    const int base_token = view.lo / kPromptTokens * kPromptTokens;
    const int active = view.hi > view.lo ? (view.hi - base_token + g.chunk - 1) / g.chunk : 1;
    if ((int)blockIdx.z >= active) return;
    const int from = base_token + (int)blockIdx.z * g.chunk, to = min(view.hi, from + g.chunk);
    const int steps = to > from ? (to - from + kPromptTokens - 1) / kPromptTokens : 0;
    const int tiles = view.rows > 128 ? 2 : 1;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, k_s = base + 2u * S::kTile, v_s = base + 4u * S::kTile;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&q_full), 8u);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&k_full[i]), 4u); mbar_init(smem_u32(&v_full[i]), 4u);
            mbar_init(smem_u32(&k_empty[i]), 1u); mbar_init(smem_u32(&v_empty[i]), 1u);
            mbar_init(smem_u32(&s_full[i]), 1u); mbar_init(smem_u32(&p_ready[i][0]), 4u); mbar_init(smem_u32(&p_ready[i][1]), 4u); mbar_init(smem_u32(&o_done[i]), 1u);
        }
        mbar_init(smem_u32(&drained), 1u);
        abort_flag = 0;
        fence_mbar_init();
        fence_proxy_async_shared();
    }
    if ((int)threadIdx.x < D) { nan_first[threadIdx.x] = INT_MAX; nan_last[threadIdx.x] = INT_MIN; }
    if (warp == 12) {
        tmem_alloc(smem_u32(&tmem_slot), 512u);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t*)&tmem_slot;
    pdl_allow_next();                                                     // (the next launch may take tensor memory: this CTA has its own)

    // a softmax thread's row
    const int tile = warp >> 2, r = (int)threadIdx.x & 255;
    const bool mine = warp < 8 && r < view.rows;
    const int row_t = view.t0 + (view.h0 + r) / g.group, row_h = head * g.group + (view.h0 + r) % g.group;
    float top = -INFINITY, used = 0.f, sum = 0.f, ref = 0.f;              // maximum; the one that O and the sum are relative to; the unit of O
    bool fine = true;

    if (warp < 8) {
        registers_up<184>();
        // ---------------- queries: a row as 16-bit floating point with a maximum of 2^14..2^15 ----------------
        const int lr = r & 127;
        const long long at = (view.start + (long long)row_t) * g.a.q_token + (long long)row_h * g.a.q_head;
        float most = 0.f;
        if (mine) {
#pragma unroll 8
            for (int i = 0; i < D; i += 4) {
                float v[4];
                load_four(g.a.q, at + i, g.a.type, g.q_wide, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = finite_max(most, v[e]);
            }
        }
        const int ex = most > 0.f ? (__float_as_int(most) >> 23) : 127 + 14;
        const float size = __int_as_float((min(254, max(1, 127 + 14 + 127 - ex))) << 23);
        const float up = g.scale_log2 < 0.f ? -size : size;               // (the factor of the scores is positive: their maximum is the products')
        const float factor = fabsf(g.scale_log2) / size;
        const uint32_t line = q_s + (uint32_t)tile * S::kTile + (uint32_t)lr * 128u;
#pragma unroll 8
        for (int i = 0; i < D; i += 4) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (mine) load_four(g.a.q, at + i, g.a.type, g.q_wide, v);
            const uint32_t to_ = line + (uint32_t)(i / 8 % S::kAtoms) * kAtom + (((uint32_t)(i / (8 * S::kAtoms)) ^ (uint32_t)(lr & 7)) << 4) + (uint32_t)(i & 4) * 2u;
            st_shared_u32(to_, down2<TT_TYPE_F16>(v[0] * up, v[1] * up));
            st_shared_u32(to_ + 4u, down2<TT_TYPE_F16>(v[2] * up, v[3] * up));
        }
        fence_proxy_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&q_full));

        // ---------------- softmax ----------------
        const int row_pos = view.before + row_t;                          // the row sees tokens row_lo .. row_hi - 1
        const int row_hi = g.a.causal ? min(view.hi, row_pos + 1) : view.hi, row_lo = g.a.window > 0 ? row_pos + 1 - g.a.window : 0;
        if (tile < tiles) {
            const uint32_t s_t = tmem + ((uint32_t)((warp & 3) * 32) << 16) + S::kScores + (uint32_t)tile * 128u;
            const uint32_t o_t = tmem + ((uint32_t)((warp & 3) * 32) << 16) + S::kOut + (uint32_t)(tile * D);
            for (int i = 0; i < steps; ++i) {
                if (!__all_sync(0xffffffffu, bounded_wait(&s_full[tile], (uint32_t)i & 1u, abortp, g.a.status, 31u, kPromptWait))) { fine = false; break; }
                tc_fence_after();
                const int t = from + i * kPromptTokens;
                const bool whole = t >= view.whole_lo && t + kPromptTokens <= view.whole_hi;
                const int j_lo = row_lo - t, j_hi = row_hi - t;           // the row sees columns j_lo .. j_hi - 1
                uint32_t v[128];
#pragma unroll
                for (int h = 0; h < 4; ++h) tmem_ld32(s_t + 32u * h, *reinterpret_cast<uint32_t(*)[32]>(&v[32 * h]));
                tmem_wait_ld();
                if (!whole) {
#pragma unroll
                    for (int k = 0; k < 128; ++k) v[k] = k >= j_lo && k < j_hi ? v[k] : 0xff800000u;      // (-inf)
                }
                float key[8], shift[8], back[8];
                const uint32_t info = smem_u32(&scales[i & 3]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 a = ld_shared_v4f(info + 16u * h), b = ld_shared_v4f(info + 32u + 16u * h), d = ld_shared_v4f(info + 64u + 16u * h);
                    key[4 * h] = a.x; key[4 * h + 1] = a.y; key[4 * h + 2] = a.z; key[4 * h + 3] = a.w;
                    shift[4 * h] = b.x; shift[4 * h + 1] = b.y; shift[4 * h + 2] = b.z; shift[4 * h + 3] = b.w;
                    back[4 * h] = d.x; back[4 * h + 1] = d.y; back[4 * h + 2] = d.z; back[4 * h + 3] = d.w;
                }
                float mx = top, m[8];
#pragma unroll
                for (int gr = 0; gr < 8; ++gr) m[gr] = fmaxf(__uint_as_float(v[16 * gr]), __uint_as_float(v[16 * gr + 1]));
#pragma unroll
                for (int k = 2; k < 16; k += 2)
#pragma unroll
                    for (int gr = 0; gr < 8; ++gr) m[gr] = max_of(m[gr], __uint_as_float(v[16 * gr + k]), __uint_as_float(v[16 * gr + k + 1]));
#pragma unroll
                for (int gr = 0; gr < 8; ++gr) {
                    // (a factor of 0, of a page of zeros, would make NaN of -inf: the smallest one does as well)
                    key[gr] = fmaxf(factor * key[gr], 1.17549435e-38f);
                    mx = fmaxf(mx, m[gr] * key[gr]);
                }
                const float seen = top;
                top = mx;
                // O and the sum follow the maximum when it is 2^8 ahead, and the largest scale at once
                const float new_ref = ld_shared_f32(info + 96u);
                const bool first = seen != top && seen == -INFINITY;      // the row's first visible token is in this step
                const bool move = top > used + 8.f || first || ref != new_ref;
                if (__any_sync(0xffffffffu, move)) {
                    const float now = top == -INFINITY ? 0.f : top;
                    const float alpha = seen != -INFINITY ? exp2_fast(used - now) : 0.f;
                    const float scale_o = ref == new_ref ? alpha : alpha * __fdividef(ref, new_ref);
                    used = now;
                    sum *= alpha;
                    ref = new_ref;
                    if (i > 0) {
                        if (!__all_sync(0xffffffffu, bounded_wait(&o_done[tile], (uint32_t)(i - 1) & 1u, abortp, g.a.status, 32u, kPromptWait))) { fine = false; break; }
                        tc_fence_after();
#pragma unroll 1
                        for (int h = 0; h < D; h += 16) {                 // (few at a time: the scores are in registers)
                            uint32_t o[16];
                            tmem_ld8u(o_t + (uint32_t)h, o);
                            tmem_ld8u(o_t + (uint32_t)h + 8u, o + 8);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * scale_o);
                            tmem_st8u(o_t + (uint32_t)h, o);
                            tmem_st8u(o_t + (uint32_t)h + 8u, o + 8);
                        }
                    }
                }
                // exponentials of a group while the sums and the conversion of the one before are under way
                float2 e[2][8];
                uint32_t p[32];
#pragma unroll
                for (int gr = 0; gr < 9; ++gr) {
                    if (gr < 8) {
                        const float f = key[gr], add = shift[gr] - used;
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            e[gr & 1][k] = fma_pair(make_float2(__uint_as_float(v[16 * gr + 2 * k]), __uint_as_float(v[16 * gr + 2 * k + 1])), make_float2(f, f), make_float2(add, add));
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (gr < 8) { e[gr & 1][k].x = exp2_fast(e[gr & 1][k].x); e[gr & 1][k].y = exp2_fast(e[gr & 1][k].y); }
                        if (gr > 0) p[8 * ((gr - 1) & 3) + k] = down2<TT_TYPE_F16>(e[(gr - 1) & 1][k].x, e[(gr - 1) & 1][k].y);
                    }
                    if (gr > 0) {
                        float2 (&d)[8] = e[(gr - 1) & 1];
                        const float2 a = add_pair(add_pair(add_pair(d[0], d[1]), add_pair(d[2], d[3])), add_pair(add_pair(d[4], d[5]), add_pair(d[6], d[7])));
                        sum = fmaf(a.x + a.y, back[gr - 1], sum);
                    }
                    if (gr == 4 || gr == 8) {
                        constexpr int kHalf[9] = {0, 0, 0, 0, 0, 0, 0, 0, 1};
                        const int h = kHalf[gr];
                        tmem_st32u(s_t + 32u * h, p);
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&p_ready[tile][h]));
                    }
                }
            }
        }
        // ---------------- out ----------------
        named_sync(1, 384);                                               // (every NaN of the steps at the edges has been noted)
        const long long place = unit * c.heads + head;
        constexpr int kPart = kPromptRows * (D + 2);
        const auto store = [&](int rr, int i, const float (&v)[4]) {
            const int tt = (view.h0 + rr) / g.group;
            store_four(g.a.y, (view.start + view.t0 + (long long)tt) * g.a.y_token + (long long)(head * g.group + (view.h0 + rr) % g.group) * g.a.y_head + i, g.a.type, g.y_wide, v);
        };
        if (tile < tiles) {
            if (steps > 0 && fine) fine = __all_sync(0xffffffffu, bounded_wait(&o_done[tile], (uint32_t)(steps - 1) & 1u, abortp, g.a.status, 32u, kPromptWait));
            tc_fence_after();
            if (fine) {
                const uint32_t o_t = tmem + ((uint32_t)((warp & 3) * 32) << 16) + S::kOut + (uint32_t)(tile * D);
                const int pos = row_pos;
                const bool none = steps == 0 || row_hi <= max(row_lo, from) || row_lo >= to;      // the row sees nothing here
                // O is in units of 2^7 and the largest scale; a split's part stays relative to its sum
                const float unit_o = ref * 0.0078125f * (active == 1 ? 1.f / sum : 1.f);
                float* left = g.partial + (place * g.splits + blockIdx.z) * kPart + (long long)r * D;
#pragma unroll 1
                for (int h = 0; h < D; h += 32) {
                    uint32_t v[32];
                    if (steps > 0) {
                        tmem_ld32(o_t + (uint32_t)h, v);
                        tmem_wait_ld();
                    }
                    if (mine) {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const int n = h + j, first = n % 64 / 8 * 8 * S::kAtoms + n / 64 * 8 + n % 8;      // the place of column n in the head
                            float x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                x[e] = none ? 0.f : __uint_as_float(v[j + e]) * unit_o;
                                if (nan_first[first + e] <= pos || (g.a.window > 0 && nan_last[first + e] > pos - g.a.window)) x[e] = __int_as_float(0x7fffffff);
                            }
                            if (active == 1) store(r, first, x);
                            else *reinterpret_cast<float4*>(left + first) = make_float4(x[0], x[1], x[2], x[3]);
                        }
                    }
                    __syncwarp();
                }
                if (active > 1 && mine) *reinterpret_cast<float2*>(g.partial + (place * g.splits + blockIdx.z) * kPart + (long long)kPromptRows * D + 2 * r) = make_float2(used, none ? 0.f : sum);
            }
        }
        tc_fence_before();
        __syncwarp();
        named_arrive(2, 288);                                             // (the tensor memory has been read)
        if (active == 1) return;

        // ---------------- the splits together, by the last CTA of the tile ----------------
        __threadfence();
        named_sync(3, 256);
        if (threadIdx.x == 0) last_one = atomicAdd(g.counters + place, 1u) == (unsigned)active - 1u;
        named_sync(3, 256);
        if (!last_one) return;
        __threadfence();
        const float* parts = g.partial + place * g.splits * kPart;
        float* share = reinterpret_cast<float*>(smem_raw);               // [split][row]
        if (mine) {
            float mx = -INFINITY, l = 0.f;
            for (int z = 0; z < active; ++z) {
                const float2 ml = __ldcg(reinterpret_cast<const float2*>(parts + (long long)z * kPart + kPromptRows * D + 2 * r));
                if (ml.y != 0.f) mx = fmaxf(mx, ml.x);
            }
            for (int z = 0; z < active; ++z) {
                const float2 ml = __ldcg(reinterpret_cast<const float2*>(parts + (long long)z * kPart + kPromptRows * D + 2 * r));
                const float k = ml.y != 0.f ? exp2_fast(ml.x - mx) : 0.f;
                if (ml.y != 0.f) l += ml.y * k;
                share[z * kPromptRows + r] = k;
            }
            const float inv = l != 0.f ? 1.f / l : 0.f;
            for (int z = 0; z < active; ++z) share[z * kPromptRows + r] *= inv;
        }
        named_sync(3, 256);
        for (int e = threadIdx.x; e < view.rows * (D / 4); e += 256) {
            const int rr = e / (D / 4), i = 4 * (e - rr * (D / 4));
            float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int z = 0; z < active; ++z) {
                const float4 f = __ldcg(reinterpret_cast<const float4*>(parts + (long long)z * kPart + (long long)rr * D + i));
                const float w = share[z * kPromptRows + rr];
                v[0] = fmaf(f.x, w, v[0]); v[1] = fmaf(f.y, w, v[1]); v[2] = fmaf(f.z, w, v[2]); v[3] = fmaf(f.w, w, v[3]);
            }
            store(rr, i, v);
        }
        if (threadIdx.x == 0) g.counters[place] = 0u;                    // ready for the next call
    } else if (warp < 12) {
        registers_down<96>();
        // ---------------- keys and values: pages -> operand tiles ----------------
        // Eight lanes have a token; the four warps take the 16 tokens of a group at a time.  A lane copies kPiece values a step ahead into a place of
        // its own, and turns them into one 16-byte chunk of each atom's line (all banks at once): value kPiece * lane + 8 a + e of a head is
        // value e of chunk `lane` of atom a, and the queries and the outputs are ordered alike.
        constexpr int kPiece = 8 * S::kAtoms;
        const int dt = (int)threadIdx.x - 256, piece = dt & 7, sub = dt >> 3;
        const uint8_t* keys = static_cast<const uint8_t*>(c.data[0]) + head * c.head[0] + sub * c.token[0] + kPiece * piece;
        const uint8_t* vals = static_cast<const uint8_t*>(c.data[1]) + head * c.head[1] + sub * c.token[1] + kPiece * piece;
        const int* table = c.table + view.b * c.table_row;
        const int shift = 31 - __clz(c.block);
        const uint32_t raw = base + 6u * S::kTile + (uint32_t)(dt * kPiece);                     // (keys; the values' behind them)
        constexpr uint32_t kGroup = 128u * kPiece;                                               // bytes of a group of 16 tokens there
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
        const auto fetch = [&](int i, int pages, const uint8_t* data, int w) {
            const int t = from + i * kPromptTokens;
            if (i < steps) {
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    const int pg = __shfl_sync(0xffffffffu, pages, p), first = t + 16 * p, tok = first + sub;
                    const bool any = pg >= 0 && tok >= view.lo && tok < to;                      // (else zeros)
                    const uint8_t* at = any ? data + (pg * c.page[w] + (first & (c.block - 1)) * c.token[w]) : data;
                    copy_async_or_zero<kPiece>(raw + (uint32_t)w * 8u * kGroup + (uint32_t)p * kGroup, at, any);
                }
            }
            cp_async_commit();
        };
        // lane g of the first eight has the page of a step's group g, and its scales
        const auto page_of = [&](int i) {
            const int t = from + i * kPromptTokens + 16 * (lane & 7);
            if (i >= steps || t + 15 < view.lo || t >= to) return -1;
            const int pg = table[t >> shift];
            if ((unsigned)pg < (unsigned)c.pages) return pg;
            report_invalid(g.a.status);
            return -1;
        };
        const auto scale_of = [&](int pg, int w) { return pg >= 0 ? c.scale[w][pg * c.s_page[w] + head * c.s_head[w]] : 0.f; };
        float most = 0.f;                                                 // the largest scale of values so far
        int page = page_of(0), page1 = page_of(1);
        float ks = scale_of(page, 0), vs = scale_of(page, 1);
        fetch(0, page, keys, 0);
        fetch(0, page, vals, 1);
        for (int i = 0; i < steps; ++i) {
            const int t = from + i * kPromptTokens, buf = i & 1;
            const int page2 = page_of(i + 2);
            const float ks1 = scale_of(page1, 0), vs1 = scale_of(page1, 1);
            if (!__all_sync(0xffffffffu, bounded_wait(&k_empty[buf], ((uint32_t)(i >> 1) & 1u) ^ 1u, abortp, g.a.status, 33u, kPromptWait))) break;
            if (warp == 8) {
                // the scales, before the keys report: what lay here four steps ago has been read
                float m = vs;
#pragma unroll
                for (int d = 4; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                most = fmaxf(most, m);
                if (lane < 8) {
                    StepScales& sc = scales[i & 3];
                    // (a share of less than 2^-40 of the largest scale is taken as that)
                    const float unit = most > 0.f ? fmaxf(__fdividef(vs, most), 9.094947017729282e-13f) : 1.f, lg = vs == most ? 0.f : log2f(unit);
                    sc.key[lane] = ks;
                    sc.shift[lane] = lg + 7.f;
                    sc.back[lane] = exp2_fast(-lg) * 0.0078125f;
                    if (lane == 0) sc.ref = most;
                }
            }
            cp_async_wait<1>();
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                uint32_t w[kPiece / 4];
                read_shared<kPiece>(raw + (uint32_t)p * kGroup, w);
                put(k_s + (uint32_t)buf * S::kTile, p, w);
            }
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&k_full[buf]));
            fetch(i + 1, page1, keys, 0);
            if (!__all_sync(0xffffffffu, bounded_wait(&v_empty[buf], ((uint32_t)(i >> 1) & 1u) ^ 1u, abortp, g.a.status, 34u, kPromptWait))) break;
            cp_async_wait<1>();
            const bool low = t < view.whole_lo, high = g.a.causal && t + kPromptTokens > view.whole_hi;
            if (low || high) {
#pragma unroll 1
                for (int p = 0; p < 8; ++p) {
                    uint32_t w[kPiece / 4];
                    read_shared<kPiece>(raw + (uint32_t)(8 + p) * kGroup, w);
#pragma unroll
                    for (int q = 0; q < kPiece / 4; ++q) {
                        const uint32_t n = nan_bytes(w[q]);
                        if (n == 0u) continue;
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
                    read_shared<kPiece>(raw + (uint32_t)(8 + p) * kGroup, w);
                    put(v_s + (uint32_t)buf * S::kTile, p, w);
                }
            }
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&v_full[buf]));
            fetch(i + 1, page1, vals, 1);
            page1 = page2;
            ks = ks1;
            vs = vs1;
        }
        cp_async_wait<0>();
        named_arrive(1, 384);
    } else {
        registers_down<40>();
        // ---------------- MMA issuer ----------------
        if (warp == 12 && steps > 0 && elect_one()) {
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
        if (warp == 12) {
            __syncwarp();
            named_sync(2, 288);
            tc_fence_after();
            tmem_dealloc(tmem, 512u);
        }
    }
}

bool prompt_built_for(int d) { return d == 64 || d == 128; }

template <int D>
static cudaError_t launch_prompt(const Attend& g, long long units, void* stream) {
    typedef PromptShape<D> S;
    static OncePerDevice raised;
    const cudaError_t ready = raised([] { return cudaFuncSetAttribute(tt_attend_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kBytes); });
    if (ready != cudaSuccess) return ready;
    return launch(tt_attend_prompt_kernel<D>, dim3((unsigned)units, (unsigned)g.a.cache.heads, (unsigned)g.splits), kPromptThreads, S::kBytes, 1, stream, g);
}
cudaError_t launch_attend_prompt(const Attend& g, long long units, void* stream) {
    return g.a.cache.d == 64 ? launch_prompt<64>(g, units, stream) : launch_prompt<128>(g, units, stream);
}

}  // namespace tt
