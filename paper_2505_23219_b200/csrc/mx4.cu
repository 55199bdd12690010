// Matrices in microscaled 4-bit floating point: quantise, read back, product.
#include <cstdio>

#include "mx4.cuh"

namespace ghd {

namespace {

using namespace mx4;

// ---------------------------------------------------------------- quantise, read back
// Both are bound by memory (27648 x 5120 halves: quantise 54 us, 6.6 TB/s; read back 59 us, 6.0).  A lane has eight elements of a row to read, sixteen to
// quantise (two lanes to a scale: instructions, shuffles above all, are as many for eight elements as for sixteen, and eight of them and one
// row's load at a time took 95 us), and the loads of ROWS neighbouring rows go out together.
constexpr int ROWS = 4, ROWS_PER_CTA = 8 * ROWS;      // rows of a warp

// largest magnitude of sixteen elements, NaN if one is
template <typename T> __device__ __forceinline__ float top_of(const T (&t)[16]);
template <> __device__ __forceinline__ float top_of<float>(const float (&t)[16]) {
    float a = fabsf(t[0]);
#pragma unroll
    for (int e = 1; e < 16; ++e) a = max_nan(a, fabsf(t[e]));
    return a;
}
template <> __device__ __forceinline__ float top_of<__half>(const __half (&t)[16]) {
    const __half2* h = reinterpret_cast<const __half2*>(t);
    __half2 a = __habs2(h[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) a = __hmax2_nan(a, __habs2(h[e]));
    return max_nan(__low2float(a), __high2float(a));
}

template <typename T>
__global__ void __launch_bounds__(256) k_mx4_quantize(const T* __restrict__ x, int64_t ld, int m, int k, bool wide, uint2* __restrict__ codes, uint32_t* __restrict__ scales) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kt = (k + TILE - 1) / TILE;
    const int c0 = blockIdx.x * 512 + lane * 16, tile_k = c0 / TILE;
    if (tile_k >= kt) return;                                      // (8 lanes to a tile: they leave together)
    const uint32_t mask = 0xffu << (lane & 24);
    const int row0 = blockIdx.y * ROWS_PER_CTA + warp * ROWS;
    alignas(16) T t[ROWS][16];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const T* row = x + (row0 + i) * ld;
        if (row0 + i < m && wide && c0 + 16 <= k) {
#pragma unroll
            for (int j = 0; j < (int)sizeof(T); ++j) reinterpret_cast<uint4*>(t[i])[j] = __ldg(reinterpret_cast<const uint4*>(row + c0) + j);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) t[i][e] = row0 + i < m && c0 + e < k ? row[c0 + e] : T(0.f);
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        float top = top_of<T>(t[i]);
        top = max_nan(top, __shfl_xor_sync(mask, top, 1));
        // exponent field of the largest magnitude less 2: floor(log2) - 2 + 127, and 255 for infinity and NaN
        const uint32_t field = (__float_as_uint(top) >> 23) & 255u;
        const uint32_t byte = field == 255u ? 255u : field > 2u ? field - 2u : 0u;
        const float inv = byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);     // 2^(127 - byte): at most 2^127, and 2^-125 at least
        float v[2][8];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e / 8][e % 8] = to_f<T>(t[i][e]) * inv;
        uint2 c = make_uint2(codes_of(v[0]), codes_of(v[1]));
        if (byte == 255u) c = make_uint2(0u, 0u);
        const int row = row0 + i;
        const size_t tile = (size_t)(row / TILE) * kt + tile_k;
        codes[tile * (TILE_CODES / 8) + (row % TILE) * (TILE / 16) + (lane & 7)] = c;
        uint32_t s = byte << (8 * ((lane >> 1) & 3));
        s |= __shfl_xor_sync(mask, s, 2);
        s |= __shfl_xor_sync(mask, s, 4);
        if ((lane & 7) == 0) scales[tile * (TILE_SCALES / 4) + scale_at(row % TILE, 0) / 4] = s;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_mx4_read(const uint32_t* __restrict__ codes, const uint32_t* __restrict__ scales, int m, int k, T* __restrict__ out, int64_t ld, bool wide) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kt = (k + TILE - 1) / TILE;
    const int c0 = blockIdx.x * 256 + lane * 8;
    if (c0 >= k) return;
    uint32_t codes8[ROWS], words[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = min((int)blockIdx.y * ROWS_PER_CTA + warp * ROWS + i, m - 1);
        const size_t tile = (size_t)(row / TILE) * kt + c0 / TILE;
        codes8[i] = __ldg(codes + tile * (TILE_CODES / 4) + (row % TILE) * (TILE / 8) + (lane & 15));
        words[i] = __ldg(scales + tile * (TILE_SCALES / 4) + scale_at(row % TILE, 0) / 4);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = blockIdx.y * ROWS_PER_CTA + warp * ROWS + i;
        if (row >= m) return;
        float v[8];
        levels_of(codes8[i], v);
        const float s = pow2_of(words[i] >> (8 * ((lane >> 2) & 3)) & 255u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= s;
        store8(out + row * ld, c0, k, wide, v);
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
    OnDevice dev(c);
    if ((s = launch_mx4_product(c, x, ld, wide_rows(c, x, ld), w, w2, n, y)) != GHD_OK) return s;
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
    OnDevice dev(c);
    const dim3 grid((w->k + 511) / 512, (w->m + TILE - 1) / TILE * (TILE / ROWS_PER_CTA));
    const bool wide = wide_rows(c, x, ld);
    if (c->cfg.dtype == GHD_F32) launch_k(c, false, k_mx4_quantize<float>, grid, 256, 0, (const float*)x, ld, w->m, w->k, wide, (uint2*)w->codes, (uint32_t*)w->scales);
    else launch_k(c, false, k_mx4_quantize<__half>, grid, 256, 0, (const __half*)x, ld, w->m, w->k, wide, (uint2*)w->codes, (uint32_t*)w->scales);
    return check_cuda(c, "mx4_quantize");
}

ghd_status ghd_mx4_read(ghd_ctx* c, const ghd_mx4* w, void* out, int64_t ld) {
    if (!c) return GHD_EINVAL;
    ghd_status s;
    if ((s = check_matrix(c, w)) != GHD_OK || (s = check_rows(c, out, &ld, w->k, "mx4_read: null out")) != GHD_OK) return s;
    OnDevice dev(c);
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
