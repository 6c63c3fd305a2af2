// e4m3 and 16-bit values: conversions and loads shared by the 8-bit kernels.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "tt.h"

namespace tt {

constexpr int kF8Block = 128;           // columns of a block with a scale of its own

__host__ __device__ constexpr int type_bytes(int type) { return type == TT_TYPE_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == TT_TYPE_F32 || type == TT_TYPE_F16 || type == TT_TYPE_BF16; }

// The element types of the 8-bit operators, by their tt_type.
template <int TYPE> struct Element;
template <> struct Element<TT_TYPE_F32> {
    typedef float type;
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
template <> struct Element<TT_TYPE_F16> {
    typedef __half type;
    static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
};
template <> struct Element<TT_TYPE_BF16> {
    typedef __nv_bfloat16 type;
    static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
};

// Two values of a 16-bit type in one word, the first in the low half.
template <int TYPE>
__device__ __forceinline__ float2 up2(uint32_t w) {
    if constexpr (TYPE == TT_TYPE_F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    else return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <int TYPE>
__device__ __forceinline__ uint32_t down2(float a, float b) {
    if constexpr (TYPE == TT_TYPE_F16) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}

// N values from p, 16 bytes at a time (p on 16 bytes; N * bytes of the type a multiple of 16).
template <int TYPE, int N>
__device__ __forceinline__ void load_wide(const void* p, float (&v)[N]) {
    if constexpr (TYPE == TT_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 f = static_cast<const float4*>(p)[i];
            v[4 * i] = f.x; v[4 * i + 1] = f.y; v[4 * i + 2] = f.z; v[4 * i + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const uint4 u = static_cast<const uint4*>(p)[i];
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = up2<TYPE>(w[j]);
                v[8 * i + 2 * j] = f.x; v[8 * i + 2 * j + 1] = f.y;
            }
        }
    }
}
template <int TYPE, int N>
__device__ __forceinline__ void store_wide(void* p, const float (&v)[N]) {
    if constexpr (TYPE == TT_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) static_cast<float4*>(p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i)
            static_cast<uint4*>(p)[i] = make_uint4(down2<TYPE>(v[8 * i], v[8 * i + 1]), down2<TYPE>(v[8 * i + 2], v[8 * i + 3]),
                                                   down2<TYPE>(v[8 * i + 4], v[8 * i + 5]), down2<TYPE>(v[8 * i + 6], v[8 * i + 7]));
    }
}
// One value of a type known at run time.
__device__ __forceinline__ void store_one(void* p, long long i, int type, float v) {
    if (type == TT_TYPE_F32) static_cast<float*>(p)[i] = v;
    else if (type == TT_TYPE_F16) static_cast<__half*>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

// The largest magnitude so far and that of v; what is no number or not finite does not count.
__device__ __forceinline__ float finite_max(float most, float v) {
    const float a = fabsf(v);
    return a < INFINITY ? fmaxf(most, a) : most;
}
// The smallest power of two s, 2^-126 at least, with most <= 448 s = 1.75 * 2^8 s.
__device__ __forceinline__ float power_scale(float most) {
    const int bits = __float_as_int(most);
    const int e = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return __int_as_float(max(e, 1) << 23);
}
// 1 / s of such a power, which is exact (s is at most 2^120).
__device__ __forceinline__ float power_inverse(float s) { return __int_as_float((254 << 23) - __float_as_int(s)); }

// Four finite values -> four e4m3 bytes, the first in the low byte.
__device__ __forceinline__ uint32_t finite_to_e4m3x4(float a, float b, float c, float d) {
    uint32_t w;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(w) : "f"(a), "f"(b), "f"(c), "f"(d));
    return w;
}
// The same of any values: infinities, which the conversion would bring to 448, become NaN.
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
    const auto fine = [](float v) { return fabsf(v) < INFINITY ? v : __int_as_float(0x7fffffff); };
    return finite_to_e4m3x4(fine(a), fine(b), fine(c), fine(d));
}
// N times eight values as they lie in memory.  Magnitudes of 16-bit types are compared as integers, in pairs; values that are all finite, as they
// nearly always are, need no look at each.
template <int TYPE, int N>
struct Eights {
    uint4 raw[N * (TYPE == TT_TYPE_F32 ? 2 : 1)];

    // Values c .. c + 7, c + step .. c + step + 7, ... of a row of n (zeros behind it).
    __device__ __forceinline__ void load(const typename Element<TYPE>::type* x, int c, int step, int n, bool wide) {
        constexpr int kPer = 16 / type_bytes(TYPE);
#pragma unroll
        for (int h = 0; h < N; ++h)
#pragma unroll
            for (int q = 0; q < 8 / kPer; ++q) {
                const int at = c + step * h + q * kPer;
                uint4& w = raw[h * (8 / kPer) + q];
                if (wide && at + kPer <= n) w = *reinterpret_cast<const uint4*>(x + at);
                else {
                    uint32_t u[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        if (at + i >= n) continue;
                        if constexpr (TYPE == TT_TYPE_F32) u[i] = __float_as_uint(x[at + i]);
                        else u[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(x)[at + i] << (16 * (i & 1));
                    }
                    w = make_uint4(u[0], u[1], u[2], u[3]);
                }
            }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (uint4& w : raw) w = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ float2 pair(int i) const {                  // values 2 i, 2 i + 1
        if constexpr (TYPE == TT_TYPE_F32) {
            const uint4& w = raw[i >> 1];
            return i & 1 ? make_float2(__uint_as_float(w.z), __uint_as_float(w.w)) : make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
        } else {
            const uint4& w = raw[i >> 2];
            return up2<TYPE>((i & 3) == 0 ? w.x : (i & 3) == 1 ? w.y : (i & 3) == 2 ? w.z : w.w);
        }
    }
    // The largest magnitude, infinities and NaN included.
    __device__ __forceinline__ float most() const {
        if constexpr (TYPE == TT_TYPE_F32) {
            uint32_t m = 0u;
#pragma unroll
            for (const uint4& w : raw) m = max(max(m, max(w.x & 0x7fffffffu, w.y & 0x7fffffffu)), max(w.z & 0x7fffffffu, w.w & 0x7fffffffu));
            return __uint_as_float(m);
        } else {
            uint32_t m = 0u;
#pragma unroll
            for (const uint4& w : raw) m = __vmaxu2(__vmaxu2(__vmaxu2(m, w.x & 0x7fff7fffu), w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
            const uint32_t one = max(m & 0xffffu, m >> 16);
            return up2<TYPE>(one).x;
        }
    }
    __device__ __forceinline__ float finite_most() const {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) { const float2 v = pair(i); m = finite_max(finite_max(m, v.x), v.y); }
        return m;
    }
    // The bytes of eight h, times inv.
    template <bool FINITE>
    __device__ __forceinline__ uint2 bytes(int h, float inv) const {
        uint32_t w[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float2 a = pair(4 * h + 2 * q), b = pair(4 * h + 2 * q + 1);
            w[q] = FINITE ? finite_to_e4m3x4(a.x * inv, a.y * inv, b.x * inv, b.y * inv) : to_e4m3x4(a.x * inv, a.y * inv, b.x * inv, b.y * inv);
        }
        return make_uint2(w[0], w[1]);
    }
};

// Two e4m3 bytes (of the low half word) -> two values in one word of 16-bit floating point, which holds every e4m3 value.
__device__ __forceinline__ uint32_t f16x2_of_e4m3(uint32_t two) {
    uint32_t h;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(h) : "r"(two));
    return h;
}
// ... and those of a whole word, two pairs.
__device__ __forceinline__ void f16_pairs_of_e4m3(uint32_t four, uint32_t& first, uint32_t& second) {
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}" : "=r"(first), "=r"(second) : "r"(four));
}
__device__ __forceinline__ float float_of_e4m3(uint32_t byte) {
    const uint32_t h = f16x2_of_e4m3(byte & 0xffu);
    return __half2float(__ushort_as_half((unsigned short)(h & 0xffffu)));
}

// ---- host side: what the calls' entry points share ----
inline bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline tt_status status_of(cudaError_t e) {
    if (e == cudaSuccess) return TT_OK;
    cudaGetLastError();
    return TT_ERR_CUDA;
}

template <typename... Params, typename... Args>
cudaError_t launch(void (*kern)(Params...), dim3 grid, int threads, size_t smem, int cluster, void* stream, Args... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem; cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = 1; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = (unsigned)cluster;
        cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace tt
