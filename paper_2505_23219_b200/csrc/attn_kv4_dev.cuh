// What the attention kernels over the paged 4-bit cache share: parameters, the run of units of a CTA, small numerics.
#pragma once

#include "kv4.cuh"

namespace ghd {

struct Kv4AttnParams {
    Kv4View w;
    const uint8_t* pool;
    const void* q;
    void* out;
    const uint64_t* mask;
    int mask_words, q_heads, group, ctas;
    float scale;                 // 1 / sqrt(d_head)
    float* part;                 // [ctas][2] slots of [tile rows][d_head] sums, then [tile rows][2] (reference, sum of weights)
    int* counters;               // [ctas], zero between launches
};

constexpr float KV4_LOG2E = 1.4426950408889634f;

// attn_kv4_tc.cu: tiles of many query rows on the tcgen05 tensor cores (GHD_F16)
ghd_status launch_attn_kv4_tc(ghd_ctx* c, Kv4AttnParams& p, int tile_rows);

#ifdef __CUDACC__
namespace kv4 {

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ float2 load_params(const uint8_t* p);        // (scale, min)
template <> __device__ __forceinline__ float2 load_params<__half>(const uint8_t* p) { return __half22float2(__ldg(reinterpret_cast<const __half2*>(p))); }
template <> __device__ __forceinline__ float2 load_params<float>(const uint8_t* p) { return __ldg(reinterpret_cast<const float2*>(p)); }

template <typename T> __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d);
template <> __device__ __forceinline__ void store4<float>(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
template <> __device__ __forceinline__ void store4<__half>(__half* p, float a, float b, float c, float d) {
    const __half2 lo = __floats2half2_rn(a, b), hi = __floats2half2_rn(c, d);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

// Whether new row i of a sequence sees the new row j >= 0 (j <= i, and the mask's bit when there is a mask).
__device__ __forceinline__ bool sees_new(const Kv4AttnParams& p, const Kv4Seq& q, int i, int j) {
    if (j > i || j >= q.n_new || i >= q.n) return false;
    if (!p.mask) return true;
    return (j >> 6) < p.mask_words && ((__ldg(p.mask + (size_t)(q.row0 + i) * p.mask_words + (j >> 6)) >> (j & 63)) & 1ull);
}

// Codes of half type, less 8, for the two nibbles at bits SH .. SH + 3 of the half words of w: (w & mask) | exponent is
// 1024 + c or 64 + c.
template <int SH> __device__ __forceinline__ uint32_t centred_half(uint32_t w) {
    constexpr uint32_t m = SH == 0 ? 0x000f000fu : 0x00f000f0u, e = SH == 0 ? 0x64006400u : 0x54005400u;
    const uint32_t x = (w & m) | e;
    const __half2 off = SH == 0 ? __floats2half2_rn(-1032.f, -1032.f) : __floats2half2_rn(-72.f, -72.f);
    const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&x), off);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Exclusive sums of the sequences' units in shared memory; -> all units.  Called by every thread of the block.
__device__ __forceinline__ int64_t unit_sums(const Kv4View& w, const Kv4Tiling& t, int64_t* sums /* [n_seqs + 1] */, int64_t* scratch /* [32] */) {
    const int nt = blockDim.x, each = (w.n_seqs + nt - 1) / nt, s0 = threadIdx.x * each;
    int64_t mine = 0;
    for (int s = s0; s < s0 + each && s < w.n_seqs; ++s) {
        const Kv4Seq q = kv4_load_seq(w, s);
        if (q.bad) atomicCAS(w.status, DEV_OK, DEV_KV4_ROWS);
        const int64_t u = (int64_t)t.heads * kv4_head_units(t, q);
        sums[s] = u;
        mine += u;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t run = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
    }
    if (lane == 31) scratch[warp] = run;
    __syncthreads();
    int64_t base = run - mine;
    for (int i = 0; i < warp; ++i) base += scratch[i];
    for (int s = s0; s < s0 + each && s < w.n_seqs; ++s) {
        const int64_t u = sums[s];
        sums[s] = base;
        base += u;
    }
    if (s0 < w.n_seqs && s0 + each >= w.n_seqs) sums[w.n_seqs] = base;
    __syncthreads();
    return sums[w.n_seqs];
}

// Adds the partial sums that CTAs c0 .. c1 left of one item, in that order, and writes its rows.  NT threads take part.
template <typename T, int D>
__device__ __forceinline__ void merge_item(const Kv4AttnParams& p, const Kv4Item& it, int tile_rows, int rows, int64_t c0, int64_t c1, int tid, int nt) {
    const size_t slot = (size_t)tile_rows * (D + 2);
    for (int x = tid; x < rows * (D / 4); x += nt) {
        const int rl = x / (D / 4), c = 4 * (x % (D / 4));
        float m = -INFINITY, lsum = 0.f;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int64_t k = c0; k <= c1; ++k) {
            const float* sl = p.part + ((size_t)k * 2 + (k == c0 ? 1 : 0)) * slot;
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(sl + (size_t)tile_rows * D + 2 * rl));
            const float4 b = __ldcg(reinterpret_cast<const float4*>(sl + (size_t)rl * D + c));
            if (ml.x == -INFINITY && ml.y == 0.f) continue;      // saw nothing (a NaN goes on)
            const float mn = fmaxf(m, ml.x), fa = m == -INFINITY ? 0.f : ex2(m - mn), fb = ex2(ml.x - mn);
            a.x = a.x * fa + b.x * fb; a.y = a.y * fa + b.y * fb; a.z = a.z * fa + b.z * fb; a.w = a.w * fa + b.w * fb;
            lsum = lsum * fa + ml.y * fb;
            m = mn;
        }
        const int rr = it.tile * tile_rows + rl;
        const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
        T* dst = (T*)p.out + ((size_t)(it.q.row0 + rr / p.group) * p.q_heads + it.head * p.group + rr % p.group) * D + c;
        store4<T>(dst, a.x * inv, a.y * inv, a.z * inv, a.w * inv);
    }
}

}  // namespace kv4
#endif

}  // namespace ghd
