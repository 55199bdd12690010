// Matrices in microscaled 4-bit floating point: quantise, read back, product.
#include <cstdio>

#include "internal.h"

namespace ghd {

namespace {

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

// ---------------------------------------------------------------- quantise, read back
// A warp takes 256 columns of a row at a time, 8 to a lane, so that four lanes have the 32 elements of a scale.
constexpr int ROWS_PER_CTA = 32;

template <typename T>
__global__ void __launch_bounds__(256) k_mx4_quantize(const T* __restrict__ x, int64_t ld, int m, int k, bool wide, uint32_t* __restrict__ codes, uint32_t* __restrict__ scales) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kt = (k + TILE - 1) / TILE;
    const int c0 = blockIdx.x * 256 + lane * 8, tile_k = c0 / TILE;
    if (c0 - lane * 8 + (lane & 16) * 8 >= kt * TILE) return;      // (16 lanes to a tile: they leave together)
    for (int i = warp; i < ROWS_PER_CTA; i += 8) {
        const int row = blockIdx.y * ROWS_PER_CTA + i;
        float v[8];
        if (row < m) load8(x + row * ld, c0, k, wide, v);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
        }
        const uint32_t mask = 0xffffu << (lane & 16);
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max_nan(top, fabsf(v[e]));
        top = max_nan(top, __shfl_xor_sync(mask, top, 1));
        top = max_nan(top, __shfl_xor_sync(mask, top, 2));
        // exponent field of the largest magnitude less 2: floor(log2) - 2 + 127, and 255 for infinity and NaN
        const uint32_t field = (__float_as_uint(top) >> 23) & 255u;
        const uint32_t byte = field == 255u ? 255u : field > 2u ? field - 2u : 0u;
        const float inv = __uint_as_float((254u - byte) << 23);     // 2^(127 - byte): at most 2^127, and 2^-125 at least
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = byte == 255u ? 0.f : v[e] * inv;
        const size_t tile = (size_t)(row / TILE) * kt + tile_k;
        codes[tile * (TILE_CODES / 4) + (row % TILE) * (TILE / 8) + (lane & 15)] = codes_of(v);
        uint32_t s = byte << (8 * ((lane >> 2) & 3));
        s |= __shfl_xor_sync(mask, s, 4);
        s |= __shfl_xor_sync(mask, s, 8);
        if ((lane & 15) == 0) scales[tile * (TILE_SCALES / 4) + scale_at(row % TILE, 0) / 4] = s;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_mx4_read(const uint32_t* __restrict__ codes, const uint32_t* __restrict__ scales, int m, int k, T* __restrict__ out, int64_t ld, bool wide) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kt = (k + TILE - 1) / TILE;
    const int c0 = blockIdx.x * 256 + lane * 8;
    if (c0 >= k) return;
    for (int i = warp; i < ROWS_PER_CTA; i += 8) {
        const int row = blockIdx.y * ROWS_PER_CTA + i;
        if (row >= m) return;
        const size_t tile = (size_t)(row / TILE) * kt + c0 / TILE;
        float v[8];
        levels_of(__ldg(codes + tile * (TILE_CODES / 4) + (row % TILE) * (TILE / 8) + (lane & 15)), v);
        const float s = pow2_of(__ldg(scales + tile * (TILE_SCALES / 4) + scale_at(row % TILE, 0) / 4) >> (8 * ((lane >> 2) & 3)) & 255u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= s;
        store8(out + row * ld, c0, k, wide, v);
    }
}

// ---------------------------------------------------------------- product
// A warp to a row of the matrix and NB rows of x.
constexpr int NB = 4;

template <typename T, bool GATE>
__global__ void __launch_bounds__(256) k_mx4_product(const T* __restrict__ x, int64_t ld, int n, int k, bool wide, const uint32_t* __restrict__ c0p, const uint32_t* __restrict__ s0p,
                                                     const uint32_t* __restrict__ c1p, const uint32_t* __restrict__ s1p, int m, float* __restrict__ y, T* __restrict__ u) {
    const int lane = threadIdx.x & 31, row = blockIdx.x * 8 + (threadIdx.x >> 5), kt = (k + TILE - 1) / TILE, n0 = blockIdx.y * NB;
    if (row >= m) return;
    float acc[GATE ? 2 : 1][NB] = {};
    for (int c = lane * 8; c < k; c += 256) {
        const size_t tile = (size_t)(row / TILE) * kt + c / TILE;
        const size_t ca = tile * (TILE_CODES / 4) + (row % TILE) * (TILE / 8) + (lane & 15), sa = tile * (TILE_SCALES / 4) + scale_at(row % TILE, 0) / 4;
        float w[2][8];
        for (int g = 0; g < (GATE ? 2 : 1); ++g) {
            levels_of(__ldg((g ? c1p : c0p) + ca), w[g]);
            const float s = pow2_of(__ldg((g ? s1p : s0p) + sa) >> (8 * ((lane >> 2) & 3)) & 255u);
            for (int e = 0; e < 8; ++e) w[g][e] *= s;
        }
        for (int i = 0; i < NB; ++i) {
            if (n0 + i >= n) break;
            float v[8];
            load8(x + (n0 + i) * ld, c, k, wide, v);
            for (int g = 0; g < (GATE ? 2 : 1); ++g)
                for (int e = 0; e < 8; ++e) acc[g][i] = fmaf(v[e], w[g][e], acc[g][i]);
        }
    }
    for (int i = 0; i < NB; ++i) {
        if (n0 + i >= n) break;
        for (int g = 0; g < (GATE ? 2 : 1); ++g)
            for (int o = 16; o; o >>= 1) acc[g][i] += __shfl_xor_sync(0xffffffffu, acc[g][i], o);
        if (lane == 0) {
            if (GATE) u[(size_t)(n0 + i) * m + row] = from_f<T>(acc[0][i] / (1.f + expf(-acc[0][i])) * acc[1][i]);
            else y[(size_t)(n0 + i) * m + row] = acc[0][i];
        }
    }
}

size_t es_of(const ghd_ctx* c) { return c->cfg.dtype == GHD_F32 ? 4 : 2; }

ghd_status check_matrix(ghd_ctx* c, const ghd_mx4* w) {
    if (!w || !w->codes || !w->scales) return fail(c, GHD_EINVAL, "mx4: null pointer");
    if (w->m < 1 || w->k < 1) return fail(c, GHD_EINVAL, "mx4: a matrix without rows or columns");
    if (ghd_mx4_code_bytes(w->m, w->k) == 0) return fail(c, GHD_ESHAPE, "mx4: more than 2^34 elements, or more than 2^20 rows or columns");
    if (((uintptr_t)w->codes & 31) || ((uintptr_t)w->scales & 15)) return fail(c, GHD_EINVAL, "mx4: codes must be 32-byte aligned, scales 16-byte aligned");
    return GHD_OK;
}

// rows of k elements, ld apart: a leading dimension of 0 is k
ghd_status check_rows(ghd_ctx* c, const void* p, int64_t* ld, int k, const char* what) {
    if (!p) return fail(c, GHD_EINVAL, what);
    if (*ld == 0) *ld = k;
    if (*ld < k || *ld > (int64_t)1 << 31) return fail(c, GHD_EINVAL, "mx4: a leading dimension below k or above 2^31");
    if ((uintptr_t)p & (es_of(c) - 1)) return fail(c, GHD_EINVAL, "mx4: rows are not aligned to their type");
    return GHD_OK;
}
bool wide_rows(const ghd_ctx* c, const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * es_of(c) % 16 == 0; }

ghd_status product(ghd_ctx* c, const void* x, int64_t ld, const ghd_mx4* w, const ghd_mx4* w2, int n, void* y) {
    if (!c) return GHD_EINVAL;
    if (n < 1) return fail(c, GHD_EINVAL, "mx4: n < 1");
    ghd_status s;
    if ((s = check_matrix(c, w)) != GHD_OK || (w2 && (s = check_matrix(c, w2)) != GHD_OK)) return s;
    if ((s = check_rows(c, x, &ld, w->k, "mx4: null x")) != GHD_OK) return s;
    if (!y || ((uintptr_t)y & (w2 ? es_of(c) - 1 : 3))) return fail(c, GHD_EINVAL, "mx4: null or unaligned output");
    if (w2 && (w2->m != w->m || w2->k != w->k)) return fail(c, GHD_ESHAPE, "mx4_gate_up: the two matrices differ in shape");
    if (n > c->cfg.max_nodes) return fail(c, GHD_ENOSPACE, "mx4: n > max_nodes");
    if (w->k > c->cfg.d_model && w->k > c->cfg.d_ffn) return fail(c, GHD_ENOSPACE, "mx4: k above both d_model and d_ffn");
    if (!c->ws) return fail(c, GHD_ENOSPACE, "no workspace set");
    const dim3 grid((w->m + 7) / 8, (n + NB - 1) / NB);
    const bool wide = wide_rows(c, x, ld);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (w2) launch_k(c, false, k_mx4_product<T, true>, grid, 256, 0, (const T*)x, ld, n, w->k, wide, (const uint32_t*)w->codes, (const uint32_t*)w->scales,
                         (const uint32_t*)w2->codes, (const uint32_t*)w2->scales, w->m, (float*)nullptr, (T*)y);
        else launch_k(c, false, k_mx4_product<T, false>, grid, 256, 0, (const T*)x, ld, n, w->k, wide, (const uint32_t*)w->codes, (const uint32_t*)w->scales,
                      (const uint32_t*)nullptr, (const uint32_t*)nullptr, w->m, (float*)y, (T*)nullptr);
    };
    if (c->cfg.dtype == GHD_F32) go(0.f);
    else go(__half());
    return check_cuda(c, w2 ? "mx4_gate_up" : "mx4_linear");
}

}  // namespace

}  // namespace ghd

using namespace ghd;

extern "C" {

size_t ghd_mx4_code_bytes(int32_t m, int32_t k) {
    if (m < 1 || k < 1 || m > (1 << 20) || k > (1 << 20)) return 0;
    const size_t tiles = (size_t)((m + TILE - 1) / TILE) * ((k + TILE - 1) / TILE);
    return tiles > (size_t)1 << 20 ? 0 : tiles * TILE_CODES;
}

size_t ghd_mx4_scale_bytes(int32_t m, int32_t k) { return ghd_mx4_code_bytes(m, k) / TILE_CODES * TILE_SCALES; }

ghd_status ghd_mx4_quantize(ghd_ctx* c, const void* x, int64_t ld, const ghd_mx4* w) {
    if (!c) return GHD_EINVAL;
    ghd_status s;
    if ((s = check_matrix(c, w)) != GHD_OK || (s = check_rows(c, x, &ld, w->k, "mx4_quantize: null x")) != GHD_OK) return s;
    const dim3 grid((w->k + 255) / 256, (w->m + TILE - 1) / TILE * (TILE / ROWS_PER_CTA));
    const bool wide = wide_rows(c, x, ld);
    if (c->cfg.dtype == GHD_F32) launch_k(c, false, k_mx4_quantize<float>, grid, 256, 0, (const float*)x, ld, w->m, w->k, wide, (uint32_t*)w->codes, (uint32_t*)w->scales);
    else launch_k(c, false, k_mx4_quantize<__half>, grid, 256, 0, (const __half*)x, ld, w->m, w->k, wide, (uint32_t*)w->codes, (uint32_t*)w->scales);
    return check_cuda(c, "mx4_quantize");
}

ghd_status ghd_mx4_read(ghd_ctx* c, const ghd_mx4* w, void* out, int64_t ld) {
    if (!c) return GHD_EINVAL;
    ghd_status s;
    if ((s = check_matrix(c, w)) != GHD_OK || (s = check_rows(c, out, &ld, w->k, "mx4_read: null out")) != GHD_OK) return s;
    const dim3 grid((w->k + 255) / 256, (w->m + ROWS_PER_CTA - 1) / ROWS_PER_CTA);
    const bool wide = wide_rows(c, out, ld);
    if (c->cfg.dtype == GHD_F32) launch_k(c, false, k_mx4_read<float>, grid, 256, 0, (const uint32_t*)w->codes, (const uint32_t*)w->scales, w->m, w->k, (float*)out, ld, wide);
    else launch_k(c, false, k_mx4_read<__half>, grid, 256, 0, (const uint32_t*)w->codes, (const uint32_t*)w->scales, w->m, w->k, (__half*)out, ld, wide);
    return check_cuda(c, "mx4_read");
}

ghd_status ghd_mx4_linear(ghd_ctx* c, const void* x, int64_t x_ld, const ghd_mx4* w, int32_t n, float* y) { return product(c, x, x_ld, w, nullptr, n, y); }

ghd_status ghd_mx4_gate_up(ghd_ctx* c, const void* h, int64_t h_ld, const ghd_mx4* w_gate, const ghd_mx4* w_up, int32_t n, void* u) {
    if (c && !w_up) return fail(c, GHD_EINVAL, "mx4_gate_up: null matrix");
    return product(c, h, h_ld, w_gate, w_up, n, u);
}

}  // extern "C"
