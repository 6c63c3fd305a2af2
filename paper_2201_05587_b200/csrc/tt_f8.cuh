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
__device__ __forceinline__ float load_one(const void* p, long long i, int type) {
    return type == TT_TYPE_F32 ? static_cast<const float*>(p)[i] : type == TT_TYPE_F16 ? __half2float(static_cast<const __half*>(p)[i])
                                                                                       : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
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

// Four values -> four e4m3 bytes, the first in the low byte.  Infinities, which the conversion would bring to 448, become NaN.
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
    const auto fine = [](float v) { return fabsf(v) < INFINITY ? v : __int_as_float(0x7fffffff); };
    uint32_t w;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(w) : "f"(fine(a)), "f"(fine(b)), "f"(fine(c)), "f"(fine(d)));
    return w;
}
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
