// Rotary positions: pairs of a head's values turned by an angle proportional to the token's position.
//
// The phase of pair i at position p is p * turns[i] modulo 2^64, turns[i] being its frequency in turns per position as a fraction of 2^64: an
// integer product that wraps as an angle does, so a position of 2^20 is as exact as the first one (in 32-bit floating point its angle would
// be off by 2^20 * 2^-24).  The top 32 bits, signed, are the angle in half turns for sincospi.
//
// A thread has the pairs of one 16-byte piece of a head (or of two, in the layout of halves), takes their sines once, and goes through every
// head_step-th head with them: bound by memory, as long as the sines (some 40 instructions a pair) are shared by enough heads.  (8192 tokens, 40 heads
// of 128, half of each turned: 29.4 us, 5.7 TB/s, 0.88 of a copy's rate.  16 tokens: 2.8 to 3.1 us.)
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

__device__ __forceinline__ long long position(const tt_rotary_args& a, int token) {
    return a.position_bits == 64 ? static_cast<const long long*>(a.positions)[token] : (long long)static_cast<const int*>(a.positions)[token];
}

// 16 bytes of pairs side by side, or of their first and of their second values.
template <int TYPE, bool INTERLEAVED, int PAIRS>
__device__ __forceinline__ void turn_piece(uint4* w, const float (&c)[PAIRS], const float (&s)[PAIRS]) {
    const auto word = [&](int part, int i) -> uint32_t& { return i == 0 ? w[part].x : i == 1 ? w[part].y : i == 2 ? w[part].z : w[part].w; };
    if constexpr (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            if constexpr (TYPE == TT_TYPE_F32) {
                const float a = __uint_as_float(word(0, 2 * i)), b = __uint_as_float(word(0, 2 * i + 1));
                word(0, 2 * i) = __float_as_uint(a * c[i] - b * s[i]);
                word(0, 2 * i + 1) = __float_as_uint(b * c[i] + a * s[i]);
            } else {
                const float2 v = up2<TYPE>(word(0, i));
                word(0, i) = down2<TYPE>(v.x * c[i] - v.y * s[i], v.y * c[i] + v.x * s[i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == TT_TYPE_F32) {
                const float a = __uint_as_float(word(0, i)), b = __uint_as_float(word(1, i));
                word(0, i) = __float_as_uint(a * c[i] - b * s[i]);
                word(1, i) = __float_as_uint(b * c[i] + a * s[i]);
            } else {
                const float2 a = up2<TYPE>(word(0, i)), b = up2<TYPE>(word(1, i));
                word(0, i) = down2<TYPE>(a.x * c[2 * i] - b.x * s[2 * i], a.y * c[2 * i + 1] - b.y * s[2 * i + 1]);
                word(1, i) = down2<TYPE>(b.x * c[2 * i] + a.x * s[2 * i], b.y * c[2 * i + 1] + a.y * s[2 * i + 1]);
            }
        }
    }
}

// V values a piece: 16 bytes, or one (one pair, where values lie at no better than their own size).
template <int TYPE, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(128) tt_rotary_kernel(const Rotary g) {
    pdl_allow_next();
    pdl_wait_prev();
    typedef typename Element<TYPE>::type T;
    constexpr int kPairs = V == 1 ? 1 : INTERLEAVED ? V / 2 : V;       // pairs of a piece
    const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= g.threads) return;
    const int unit = (int)(t % g.units);
    const long long rest = t / g.units;
    const int h0 = (int)(rest % g.head_step), token = (int)(rest / g.head_step), half = g.a.rot >> 1;
    const bool turned = unit < g.rot_units;
    const int all = g.a.heads[0] + g.a.heads[1];
    // of head h, the piece's first value; in halves, the second part's are `half` further on
    const int at = !turned ? g.a.rot + (unit - g.rot_units) * V : INTERLEAVED ? unit * 2 * kPairs : unit * kPairs;
    const auto from = [&](int h) {
        const int w = h >= g.a.heads[0] ? 1 : 0;
        return static_cast<const T*>(g.a.x[w]) + ((long long)token * g.a.x_token[w] + (long long)(h - (w ? g.a.heads[0] : 0)) * g.a.x_head[w] + at);
    };
    const auto to = [&](int h) {
        const int w = h >= g.a.heads[0] ? 1 : 0;
        return static_cast<T*>(g.a.y[w]) + ((long long)token * g.a.y_token[w] + (long long)(h - (w ? g.a.heads[0] : 0)) * g.a.y_head[w] + at);
    };
    if constexpr (V == 1) {
        float c[1], s[1];
        if (turned) rotary_turn(position(g.a, token), g.a.turns[unit], g.a.factor, g.a.inverse != 0, c[0], s[0]);
        for (int h = h0; h < all; h += g.head_step) {
            const T* x = from(h);
            T* y = to(h);
            if (turned) {
                const int other = INTERLEAVED ? 1 : half;
                const float a = Element<TYPE>::up(x[0]), b = Element<TYPE>::up(x[other]);
                y[0] = Element<TYPE>::down(a * c[0] - b * s[0]);
                y[other] = Element<TYPE>::down(b * c[0] + a * s[0]);
            } else *y = *x;
        }
    } else {
        // kBatch heads are under way at a time, the first ones while the sines are taken
        constexpr int kParts = INTERLEAVED ? 1 : 2, kBatch = INTERLEAVED ? 4 : 2;
        uint4 v[kBatch][kParts];
        const auto load = [&](int h) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i, h += g.head_step) {
                if (h >= all) break;
                const T* x = from(h);
                v[i][0] = *reinterpret_cast<const uint4*>(x);
                if (kParts == 2 && turned) v[i][kParts - 1] = *reinterpret_cast<const uint4*>(x + half);
            }
        };
        load(h0);
        float c[kPairs], s[kPairs];
        if (turned) {
            const long long p = position(g.a, token);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) rotary_turn(p, g.a.turns[unit * kPairs + i], g.a.factor, g.a.inverse != 0, c[i], s[i]);
        }
        for (int h = h0; h < all;) {
            const int first = h;
            uint4 w[kBatch][kParts];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
#pragma unroll
                for (int j = 0; j < kParts; ++j) w[i][j] = v[i][j];
            h += kBatch * g.head_step;
            load(h);
            if (turned) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) turn_piece<TYPE, INTERLEAVED, kPairs>(w[i], c, s);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int hh = first + i * g.head_step;
                if (hh >= all) break;
                T* y = to(hh);
                *reinterpret_cast<uint4*>(y) = w[i][0];
                if (kParts == 2 && turned) *reinterpret_cast<uint4*>(y + half) = w[i][kParts - 1];
            }
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
