// Rotary positions: pairs of a head's values turned by an angle proportional to the token's position.
//
// The phase of pair i at position p is p * turns[i] modulo 2^64, turns[i] being its frequency in turns per position as a fraction of 2^64: an
// integer product that wraps as an angle does, so a position of 2^20 is as exact as the first one (in 32-bit floating point its angle would
// be off by 2^20 * 2^-24).  The top 32 bits, signed, are the angle in half turns for sincospi.
//
// A thread has the pairs of one 16-byte piece of a head (or of two, in the layout of halves), takes their sines once, and goes through every
// head_step-th head with them: bound by memory, as long as the sines (some 40 instructions a pair) are shared by enough heads.
#include <cuda_runtime.h>
#include <cmath>
#include "tt_ptx.cuh"
#include "tt_f8.cuh"

namespace tt {

struct Rotary {
    tt_rotary_args a;
    int units, rot_units;                   // pieces of a head, those of them that are turned
    int head_step;                          // threads that share a token's piece
    long long threads;
};

// A pair's sine and cosine at position p.
__device__ __forceinline__ void rotary_turn(long long p, unsigned long long turns, float factor, bool inverse, float& c, float& s) {
    const unsigned long long phase = (unsigned long long)p * turns;
    const float half_turns = (float)(int)(phase >> 32) * 4.656612873077392578125e-10f;      // 2^-31
    sincospif(half_turns, &s, &c);
    c *= factor;
    s *= inverse ? -factor : factor;
}

// V values a piece: 16 bytes, or one (one pair, where values lie at no better than their own size).
template <int TYPE, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(128) tt_rotary_kernel(const Rotary g) {
    pdl_allow_next();
    pdl_wait_prev();
    typedef typename Element<TYPE>::type T;
    constexpr int kPairs = V == 1 ? 1 : INTERLEAVED ? V / 2 : V;       // pairs of a piece
    constexpr int kLoad = V == 1 ? 2 : INTERLEAVED ? V : 2 * V;        // ... and its values
    const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= g.threads) return;
    const int unit = (int)(t % g.units);
    const long long rest = t / g.units;
    const int h0 = (int)(rest % g.head_step), token = (int)(rest / g.head_step), half = g.a.rot >> 1;
    const bool turned = unit < g.rot_units;
    float c[kPairs], s[kPairs];
    if (turned) {
        const long long p = g.a.position_bits == 64 ? static_cast<const long long*>(g.a.positions)[token] : (long long)static_cast<const int*>(g.a.positions)[token];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) rotary_turn(p, g.a.turns[unit * kPairs + i], g.a.factor, g.a.inverse != 0, c[i], s[i]);
    }
    const int all = g.a.heads[0] + g.a.heads[1];
    if (turned) {
        const int at = INTERLEAVED ? unit * 2 * kPairs : unit * kPairs;            // the piece's first value; of halves, the second part's at + half
#pragma unroll 2
        for (int h = h0; h < all; h += g.head_step) {
            const int w = h >= g.a.heads[0] ? 1 : 0, hh = h - (w ? g.a.heads[0] : 0);
            const T* x = static_cast<const T*>(g.a.x[w]) + (long long)token * g.a.x_token[w] + (long long)hh * g.a.x_head[w] + at;
            T* y = static_cast<T*>(g.a.y[w]) + (long long)token * g.a.y_token[w] + (long long)hh * g.a.y_head[w] + at;
            float v[kLoad];
            if constexpr (V == 1) {
                v[0] = Element<TYPE>::up(x[0]);
                v[1] = Element<TYPE>::up(x[INTERLEAVED ? 1 : half]);
                y[0] = Element<TYPE>::down(v[0] * c[0] - v[1] * s[0]);
                y[INTERLEAVED ? 1 : half] = Element<TYPE>::down(v[1] * c[0] + v[0] * s[0]);
            } else if constexpr (INTERLEAVED) {
                load_wide<TYPE, V>(x, v);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float a = v[2 * i], b = v[2 * i + 1];
                    v[2 * i] = a * c[i] - b * s[i];
                    v[2 * i + 1] = b * c[i] + a * s[i];
                }
                store_wide<TYPE, V>(y, v);
            } else {
                float a[V], b[V];
                load_wide<TYPE, V>(x, a);
                load_wide<TYPE, V>(x + half, b);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float u = a[i] * c[i] - b[i] * s[i];
                    b[i] = b[i] * c[i] + a[i] * s[i];
                    a[i] = u;
                }
                store_wide<TYPE, V>(y, a);
                store_wide<TYPE, V>(y + half, b);
            }
        }
    } else {
        const int at = g.a.rot + (unit - g.rot_units) * V;
#pragma unroll 4
        for (int h = h0; h < all; h += g.head_step) {
            const int w = h >= g.a.heads[0] ? 1 : 0, hh = h - (w ? g.a.heads[0] : 0);
            const T* x = static_cast<const T*>(g.a.x[w]) + (long long)token * g.a.x_token[w] + (long long)hh * g.a.x_head[w] + at;
            T* y = static_cast<T*>(g.a.y[w]) + (long long)token * g.a.y_token[w] + (long long)hh * g.a.y_head[w] + at;
            if constexpr (V == 1) *y = *x;
            else *reinterpret_cast<uint4*>(y) = *reinterpret_cast<const uint4*>(x);
        }
    }
}

template <int TYPE>
static cudaError_t launch_rotary(Rotary& g, bool wide, void* stream) {
    constexpr int V = 16 / type_bytes(TYPE);
    void (*kern)(const Rotary);
    if (wide) kern = g.a.interleaved ? tt_rotary_kernel<TYPE, V, true> : tt_rotary_kernel<TYPE, V, false>;
    else kern = g.a.interleaved ? tt_rotary_kernel<TYPE, 1, true> : tt_rotary_kernel<TYPE, 1, false>;
    return launch(kern, dim3((unsigned)((g.threads + 127) / 128), 1, 1), 128, 0, 1, stream, g);
}

}  // namespace tt

using namespace tt;

extern "C" tt_status tt_rotary(const tt_rotary_args* a, void* stream) {
    if (!a || !known_type(a->type) || (a->position_bits != 32 && a->position_bits != 64) || a->tokens < 0 || a->heads[0] < 0 || a->heads[1] < 0 || a->d < 0 ||
        a->rot < 0 || a->rot > a->d || a->rot % 2) return TT_ERR_INVALID_ARG;
    if (a->tokens == 0 || a->heads[0] + (long long)a->heads[1] == 0 || a->d == 0) return TT_OK;
    if (a->heads[0] > 65536 || a->heads[1] > 65536 || a->d > 65536) return TT_ERR_INVALID_ARG;
    if (a->rot > 0 && (!a->positions || !a->turns || reinterpret_cast<uintptr_t>(a->positions) % (uintptr_t)(a->position_bits / 8) || reinterpret_cast<uintptr_t>(a->turns) % 8))
        return TT_ERR_INVALID_ARG;
    const int bytes = type_bytes(a->type), V = 16 / bytes;
    bool wide = a->d % V == 0 && a->rot % (a->interleaved ? V : 2 * V) == 0, in_place = true;
    for (int w = 0; w < 2; ++w) {
        if (a->heads[w] == 0) continue;
        if (!a->x[w] || !a->y[w]) return TT_ERR_INVALID_ARG;
        if (reinterpret_cast<uintptr_t>(a->x[w]) % (uintptr_t)bytes || reinterpret_cast<uintptr_t>(a->y[w]) % (uintptr_t)bytes) return TT_ERR_INVALID_ARG;
        for (const int64_t stride : {a->x_token[w], a->x_head[w], a->y_token[w], a->y_head[w]}) {
            if (stride < 0) return TT_ERR_INVALID_ARG;
            wide = wide && stride % V == 0;
        }
        wide = wide && reinterpret_cast<uintptr_t>(a->x[w]) % 16 == 0 && reinterpret_cast<uintptr_t>(a->y[w]) % 16 == 0;
        in_place = in_place && a->x[w] == a->y[w] && a->x_token[w] == a->y_token[w] && a->x_head[w] == a->y_head[w];
    }
    Rotary g{};
    g.a = *a;
    const int v = wide ? V : 1;
    g.rot_units = a->interleaved ? a->rot / (wide ? V : 2) : a->rot / 2 / v;
    g.units = g.rot_units + (in_place ? 0 : (a->d - a->rot) / v);
    if (g.units == 0) return TT_OK;
    // As many threads share a token's piece as it takes to give every SM a few warps, and no more: each takes the sines again.
    const int all = a->heads[0] + a->heads[1];
    const long long one = (long long)a->tokens * g.units;
    g.head_step = 1;
    while (g.head_step < all && one * g.head_step < (long long)kSms * 1024) g.head_step *= 2;
    if (g.head_step > all) g.head_step = all;
    g.threads = one * g.head_step;
    if ((g.threads + 127) / 128 > 0x7fffffff) return TT_ERR_INVALID_ARG;
    return status_of(a->type == TT_TYPE_F32 ? launch_rotary<TT_TYPE_F32>(g, wide, stream) : a->type == TT_TYPE_F16 ? launch_rotary<TT_TYPE_F16>(g, wide, stream)
                                                                                                                 : launch_rotary<TT_TYPE_BF16>(g, wide, stream));
}

extern "C" tt_status tt_rotary_turns(const double* frequencies, size_t n, uint64_t* turns) {
    if (n > 0 && (!frequencies || !turns)) return TT_ERR_INVALID_ARG;
    for (size_t i = 0; i < n; ++i) {
        if (!std::isfinite(frequencies[i])) return TT_ERR_INVALID_ARG;
        // the fraction of a turn, in the 64 bits of an extended mantissa
        long double t = (long double)frequencies[i] / (2.0L * 3.14159265358979323846264338327950288L);
        t -= std::floor(t);
        const long double scaled = std::nearbyint(std::ldexp(t, 64));
        turns[i] = scaled >= 18446744073709551616.0L ? 0 : (uint64_t)scaled;
    }
    return TT_OK;
}
