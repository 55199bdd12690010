// Matrices in microscaled 4-bit floating point: layout and conversions that the kernels share.
#pragma once

#include "internal.h"

namespace ghd {
namespace mx4 {

constexpr int TILE = 128;                       // rows and columns of a tile
constexpr int TILE_CODES = TILE * TILE / 2, TILE_SCALES = TILE * TILE / 32;

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// where the scale byte of (row, 32 elements j) lies in a tile
__host__ __device__ constexpr int scale_at(int row, int j) { return (row % 32) * 16 + row / 32 * 4 + j; }

__device__ __forceinline__ float pow2_of(uint32_t byte) {            // 2^(byte - 127), NaN for 255
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// 8 values -> 8 codes, the first in the low half of the low byte: nearest, ties to the even code, held within +-6
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return r;
}
__device__ __forceinline__ void levels_of(uint32_t codes, float (&x)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

// 8 elements of a row from column c0, zeros past its end.  wide: the 8 lie on a 16-byte boundary.
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ row, int c0, int k, bool wide, float (&x)[8]) {
    if (wide && c0 + 8 <= k) {
        uint4 u[sizeof(T) / 2];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) u[i] = __ldg(reinterpret_cast<const uint4*>(row + c0) + i);
        const T* t = reinterpret_cast<const T*>(u);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_f<T>(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c0 + i < k ? to_f<T>(row[c0 + i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* row, int c0, int k, bool wide, const float (&x)[8]) {
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = from_f<T>(x[i]);
    if (wide && c0 + 8 <= k) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(row + c0)[i] = reinterpret_cast<const uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c0 + i < k) row[c0 + i] = t[i];
    }
}

}  // namespace mx4

// mx4_gemm.cu: y float [n][w.m] = x w^T, or (w2 given) u T [n][w.m] = SiLU(x w^T) * (x w2^T); x T rows ld elements apart
ghd_status launch_mx4_product(ghd_ctx* c, const void* x, int64_t ld, bool wide, const ghd_mx4* w, const ghd_mx4* w2, int n, void* out);
size_t mx4_terms_bytes(const ghd_model_cfg& m);      // workspace: the terms that rows of x are split into, and their scales

}  // namespace ghd
