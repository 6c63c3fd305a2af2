// The paged e4m3 cache: what its kernels share.
#pragma once
#include "tt_ptx.cuh"
#include "tt_f8.cuh"
#include <type_traits>

namespace tt {

__device__ __forceinline__ void report_invalid(unsigned* status) { atomicCAS(status, 0u, (unsigned)TT_ERR_INVALID_ARG); }

// Work that is dealt by sequences of unknown sizes: sequence b owns the units begin(starts[b], b) and up (as many as it can need at most).  The
// whole warp looks for a unit's, 32 places at a time (a lane on its own would take the logarithm of the batch in loads, one after the other).
// False if the unit is in front of all (the starts do not rise from 0).
template <class BEGIN>
__device__ __forceinline__ bool sequence_of(const int* starts, int batch, const BEGIN& begin_of, long long unit, int& b, long long& first) {
    const int lane = threadIdx.x & 31;
    const auto begin = [&](int i) { return (long long)begin_of(starts[i], i); };
    if (batch <= 128) {                                      // all places at once
        int in = __popc(__ballot_sync(0xffffffffu, lane < batch && begin(lane) <= unit));
        if (batch > 32) {
#pragma unroll
            for (int i = 32; i < 128; i += 32) in += __popc(__ballot_sync(0xffffffffu, i + lane < batch && begin(i + lane) <= unit));
        }
        b = max(0, in - 1);
    } else {
        int n = batch;                                       // it is one of b .. b + n - 1
        b = 0;
        while (n > 1) {
            const int step = (n + 31) / 32, i = b + lane * step;
            const unsigned in = __ballot_sync(0xffffffffu, lane * step < n && begin(i) <= unit);
            const int last = in ? 31 - __clz((int)in) : 0;   // (places rise; whatever they hold, the result is one of the batch)
            n = min(step, n - last * step);
            b += last * step;
        }
    }
    first = begin(b);
    return first <= unit;
}

// The splits of a tile together: element e of the tile's `elements` vectors of four is the sum over splits of part(e, z) * share(e, z).  A thread has
// 16 of them under way at a time, none behind another.
template <int THREADS, class PART, class SHARE, class STORE>
__device__ __forceinline__ void join_splits(int elements, int splits, const PART& part, const SHARE& share, const STORE& store) {
    const auto go = [&](auto at_once) {
        constexpr int E = decltype(at_once)::value, Z = 16 / E;
        for (int e0 = threadIdx.x; e0 < elements; e0 += E * THREADS) {
            float v[E][4];
#pragma unroll
            for (int k = 0; k < E; ++k) v[k][0] = v[k][1] = v[k][2] = v[k][3] = 0.f;
            for (int z0 = 0; z0 < splits; z0 += Z) {
                float4 f[E][Z];
#pragma unroll
                for (int k = 0; k < E; ++k)
#pragma unroll
                    for (int z = 0; z < Z; ++z) {
                        f[k][z] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (e0 + k * THREADS < elements && z0 + z < splits) f[k][z] = __ldcg(part(e0 + k * THREADS, z0 + z));
                    }
#pragma unroll
                for (int k = 0; k < E; ++k)
#pragma unroll
                    for (int z = 0; z < Z; ++z)
                        if (e0 + k * THREADS < elements && z0 + z < splits) {
                            const float w = share(e0 + k * THREADS, z0 + z);
                            v[k][0] = fmaf(f[k][z].x, w, v[k][0]); v[k][1] = fmaf(f[k][z].y, w, v[k][1]);
                            v[k][2] = fmaf(f[k][z].z, w, v[k][2]); v[k][3] = fmaf(f[k][z].w, w, v[k][3]);
                        }
            }
#pragma unroll
            for (int k = 0; k < E; ++k) if (e0 + k * THREADS < elements) store(e0 + k * THREADS, v[k]);
        }
    };
    if (splits <= 4) go(std::integral_constant<int, 4>());
    else if (splits <= 8) go(std::integral_constant<int, 2>());
    else go(std::integral_constant<int, 1>());
}

constexpr int kStep = 16;                   // tokens of a step: pages are multiples of it

// An attention call, as one of its kernels takes it.
struct Attend {
    tt_cache_attention_args a;
    int group, rows;                        // query heads of a key head; rows of a tile
    int chunk, splits, max_length;          // tokens of a split, most splits
    int span, share;                        // tokens that a tile can see; CTAs that all tokens are dealt to
    int least, most;                        // rows of the sequences that the kernel takes
    int by_sequence;                        // no more than one tile each: tile b is sequence b's
    int q_wide, y_wide;                     // values of q, of y at a time: four (1) or eight (2)
    float scale_log2;                       // the scale times log2(e)
    unsigned* counters; float* partial;
};
constexpr int kPromptRows = 256;            // rows of a tile of tt_attend_prompt_kernel
constexpr int kPromptSplits = 16;           // its most splits of a sequence
constexpr int kPromptCtas = 128;            // CTAs of it that tiles are split for
constexpr int kPromptTokens = 128;          // tokens of a step of it
constexpr int prompt_head(int d) { return d <= 64 ? 64 : 128; }      // what tt_attend_prompt_kernel is built for that holds a head of d
constexpr bool prompt_built_for(int d) { return d <= 128; }
cudaError_t launch_attend_prompt(const Attend& g, long long units, void* stream);

// What a tile of rows has to do with the tokens of its sequence: false if there is nothing (or an error, which is reported).
struct TileView {
    int b, start, rows;                     // sequence, its first token in the batch, the tile's rows
    int t0, h0;                             // the first row: token (of the new ones) and head (of the group)
    int before;                             // tokens in front of the new ones (negative: the first queries see nothing)
    int lo, hi;                             // tokens that any row sees
    int whole_lo, whole_hi;                 // tokens that every row sees
};
__device__ __forceinline__ bool view_tile(const Attend& g, int tile_rows, long long unit, TileView& v) {
    const tt_cache& c = g.a.cache;
    long long first_unit = unit;
    bool found = true;
    if (g.by_sequence) v.b = (int)unit;
    else found = sequence_of(g.a.starts, c.batch, [&](int start, int b) { return (long long)start * g.group / tile_rows + b; }, unit, v.b, first_unit);
    v.start = g.a.starts[v.b];
    const int count = g.a.starts[v.b + 1] - v.start, length = g.a.lengths[v.b];
    if (found && count == 0) return false;
    if (!found || count < 0 || v.start < 0 || v.start + (long long)count > g.a.tokens || length < 0 || length > g.max_length || (g.a.max_count > 0 && count > g.a.max_count)) {
        if (threadIdx.x == 0) report_invalid(g.a.status);
        return false;
    }
    const long long row0 = (unit - first_unit) * tile_rows, all = (long long)count * g.group;
    if (row0 >= all || all < g.least || all > g.most) return false;
    v.rows = (int)min((long long)tile_rows, all - row0);
    v.t0 = (int)((unsigned)row0 / (unsigned)g.group);       // (all rows of a sequence are less than 2^31)
    v.h0 = (int)(row0 - (long long)v.t0 * g.group);
    const int t1 = v.t0 + (v.h0 + v.rows - 1) / g.group;
    v.before = length - count;
    v.lo = g.a.window > 0 ? max(0, v.before + v.t0 + 1 - g.a.window) : 0;
    v.hi = g.a.causal ? max(0, min(length, v.before + t1 + 1)) : length;
    v.whole_lo = g.a.window > 0 ? max(0, v.before + t1 + 1 - g.a.window) : 0;
    v.whole_hi = g.a.causal ? max(0, min(length, v.before + v.t0 + 1)) : length;
    return true;
}

__device__ __forceinline__ float exp2_fast(float x) {      // 2^x to two units in the last place; 0 below 2^-126
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <int N>
__device__ __forceinline__ void read_shared(uint32_t addr, uint32_t (&v)[N / 4]) {
    if constexpr (N == 16) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
    else if constexpr (N == 8) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(addr) : "memory");
    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[0]) : "r"(addr) : "memory");
}
// A non-zero byte for each e4m3 byte of the word that is NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// Four 16-bit values as they lie in memory, and as 32-bit ones.
__device__ __forceinline__ uint2 raw_four(const void* p, long long i, int wide) {
    const uint16_t* x = static_cast<const uint16_t*>(p) + i;
    if (wide) return *reinterpret_cast<const uint2*>(x);
    return make_uint2((uint32_t)x[0] | (uint32_t)x[1] << 16, (uint32_t)x[2] | (uint32_t)x[3] << 16);
}
__device__ __forceinline__ uint4 raw_eight(const void* p, long long i, int wide) {
    if (wide == 2) return *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    const uint2 a = raw_four(p, i, wide), b = raw_four(p, i + 4, wide);
    return make_uint4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void four_of(uint2 u, int type, float (&v)[4]) {
    const float2 a = type == TT_TYPE_F16 ? up2<TT_TYPE_F16>(u.x) : up2<TT_TYPE_BF16>(u.x), b = type == TT_TYPE_F16 ? up2<TT_TYPE_F16>(u.y) : up2<TT_TYPE_BF16>(u.y);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
__device__ __forceinline__ void store_four(void* p, long long i, int type, int wide, const float (&v)[4]) {
    if (wide) {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) =
            type == TT_TYPE_F16 ? make_uint2(down2<TT_TYPE_F16>(v[0], v[1]), down2<TT_TYPE_F16>(v[2], v[3])) : make_uint2(down2<TT_TYPE_BF16>(v[0], v[1]), down2<TT_TYPE_BF16>(v[2], v[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) store_one(p, i + e, type, v[e]);
    }
}

}  // namespace tt
