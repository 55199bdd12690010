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
ghd_status launch_attn_kv4_tc(ghd_ctx* c, Kv4AttnParams& p);

#ifdef __CUDACC__
namespace kv4 {

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a scale of V adds, in powers of two, to the operand of the second product: its logarithm, held at that of half's smallest number.
// A scale that is no finite half makes its rows NaN whatever the reference, and has no say in it.
__device__ __forceinline__ float scale_bits(float s) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
    return s <= 65504.f ? fmaxf(y, -24.f) : -24.f;
}

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d);
template <> __device__ __forceinline__ void store4<float>(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
template <> __device__ __forceinline__ void store4<__half>(__half* p, float a, float b, float c, float d) {
    const __half2 lo = __floats2half2_rn(a, b), hi = __floats2half2_rn(c, d);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

template <typename T> __device__ __forceinline__ void store2(T* p, float a, float b);
template <> __device__ __forceinline__ void store2<float>(float* p, float a, float b) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }
template <> __device__ __forceinline__ void store2<__half>(__half* p, float a, float b) { *reinterpret_cast<__half2*>(p) = __floats2half2_rn(a, b); }

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) {     // 16 bytes, or zeros when they are not there
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Which of the keys j0 .. j0 + 31 (numbers among the sequence's new rows; below 0: cache rows) new row i sees: bit d for
// j0 + d.  Cache rows are seen; new rows up to i itself, where the mask's bit is set (without a mask: all of them).
// No branch depends on a load, so that the words of many rows are fetched together.
__device__ __forceinline__ uint32_t sees(const Kv4AttnParams& p, const Kv4Seq& q, int i, int j0) {
    auto low = [](int n) -> uint32_t { return n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u); };
    uint32_t w = 0xffffffffu;
    if (p.mask) {
        const int at = j0 >> 6, sh = j0 & 63;                    // floor: -1 and below are cache rows
        const uint64_t* row = p.mask + (size_t)(q.row0 + min(i, q.n - 1)) * p.mask_words;
        const uint64_t a = at >= 0 && at < p.mask_words ? __ldg(row + at) : 0ull, b = at + 1 >= 0 && at + 1 < p.mask_words ? __ldg(row + at + 1) : 0ull;
        w = (uint32_t)(sh ? (a >> sh) | (b << (64 - sh)) : a);
    }
    return low(-j0) | (w & low(min(i, q.n_new - 1) + 1 - j0));
}

// Codes of half type, less 8, for the two nibbles at bits SH .. SH + 3 of the half words of w: (w & mask) | exponent is
// 1024 + c or 64 + c.  The exponents come in registers the compiler does not see through, so that the two operations
// stay one instruction.
struct HalfMagic {
    uint32_t e0, e4;
    __device__ __forceinline__ HalfMagic() : e0(0x64006400u), e4(0x54005400u) { asm volatile("" : "+r"(e0), "+r"(e4)); }
};
template <int SH> __device__ __forceinline__ uint32_t centred_half(uint32_t w, const HalfMagic& m) {
    uint32_t x;
    if constexpr (SH == 0) asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(x) : "r"(w), "r"(m.e0));
    else asm("lop3.b32 %0, %1, 0x00f000f0, %2, 0xea;" : "=r"(x) : "r"(w), "r"(m.e4));
    const __half2 off = SH == 0 ? __floats2half2_rn(-1032.f, -1032.f) : __floats2half2_rn(-72.f, -72.f);
    const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&x), off);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Exclusive sums of the sequences' units in shared memory; -> all units.  Called by every thread of the block.
__device__ __forceinline__ int64_t unit_sums(const Kv4View& w, const Kv4Tiling& t, int64_t* sums /* [n_seqs + 1] */, int64_t* scratch /* [32] */) {
    const int nt = blockDim.x, each = (w.n_seqs + nt - 1) / nt, s0 = threadIdx.x * each;
    int64_t mine = 0;
#pragma unroll 1
    for (int s = s0; s < s0 + each && s < w.n_seqs; ++s) {
        const Kv4Seq q = kv4_load_seq(w, s);
        if (q.bad) atomicCAS(w.input_status, DEV_OK, DEV_KV4_ROWS);
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
#pragma unroll 1
    for (int i = 0; i < warp; ++i) base += scratch[i];
#pragma unroll 1
    for (int s = s0; s < s0 + each && s < w.n_seqs; ++s) {
        const int64_t u = sums[s];
        sums[s] = base;
        base += u;
    }
    if (s0 < w.n_seqs && s0 + each >= w.n_seqs) sums[w.n_seqs] = base;
    __syncthreads();
    return sums[w.n_seqs];
}

// An item in shared memory becomes the one behind it, by one thread.  Out of line: it is called from several places, and
// instruction fetch is what short calls wait for.
template <int TILE_ROWS, int CHUNK, int LEAD>
__device__ __noinline__ void advance_item(const Kv4View* w, int group, Kv4Item* it, int64_t u_end) {
    const Kv4Tiling t{w->heads, group, TILE_ROWS, CHUNK, LEAD};
    Kv4Item x = *it;
    kv4_next_item(t, [&](int s) { return kv4_load_seq(*w, s); }, x, u_end);
    x.keys = kv4_tile_keys(t, x.q, x.tile);
    *it = x;
}

// Counts a CTA in, after a barrier of its threads: what they wrote before goes before the count, and who finds all counted sees
// what the others wrote.
__device__ __forceinline__ int arrive_at(int* counter) {
    int old;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
    return old;
}

// Adds the partial sums that CTAs c0 .. c1 left of one item, in that order, and writes its rows.  A warp takes RB rows at a
// time (the lanes hold D / 32 channels each) and KB contributors of each: what the merge costs is the latency of its loads
// and, in short calls, the fetch of its instructions (KB = 16 for RB = 1: 11.8 us instead of 11.5 for one token).  With few rows several warps share the contributors and meet in `xch`,
// floats [warps][D + 2].  `sync` is a barrier of the NW warps that take part.
template <typename T, int D, int RB, typename Sync>
__device__ __forceinline__ void merge_item(const Kv4AttnParams& p, const Kv4Item& it, int tile_rows, int rows, int64_t c0, int64_t c1, int warp, int nw, float* xch, Sync sync) {
    constexpr int VL = D / 32, KB = RB == 1 ? 8 : 16 / RB;
    const size_t slot = (size_t)tile_rows * (D + 2);
    const int lane = threadIdx.x & 31, n = (int)(c1 - c0) + 1;
    int share = 1;                                               // warps a row: a power of two (only where a warp takes one row at a time)
    if (RB == 1) {
#pragma unroll 1
        while (share * 2 * rows <= nw && share * KB < n) share *= 2;
    }
    const int sub = warp & (share - 1), team = warp / share, teams = nw / share;
    const int k_beg = n * sub / share, k_end = n * (sub + 1) / share;
    // contributor 0 has begun the item (its second slot), the others have gone on with it (their first)
    const float* first = p.part + ((size_t)c0 * 2 + 1) * slot;
    const float* rest = p.part + (size_t)c0 * 2 * slot;
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += teams * RB) {
        float m[RB], lsum[RB], a[RB][VL];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            m[r] = -INFINITY;
            lsum[r] = 0.f;
#pragma unroll
            for (int e = 0; e < VL; ++e) a[r][e] = 0.f;
        }
#pragma unroll 1
        for (int kb = k_beg; kb < k_end; kb += KB) {
            float2 ml[KB][RB];
            float v[KB][RB][VL];
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                const float* sl = kb + k == 0 ? first : rest + (size_t)(kb + k) * 2 * slot;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const int rl = r0 + team * RB + r;
                    ml[k][r] = make_float2(-INFINITY, 0.f);
#pragma unroll
                    for (int e = 0; e < VL; ++e) v[k][r][e] = 0.f;
                    if (kb + k < k_end && rl < rows) {
                        ml[k][r] = __ldcg(reinterpret_cast<const float2*>(sl + tile_rows * D + 2 * rl));
                        const float* src = sl + rl * D + VL * lane;
                        if constexpr (VL == 4) { const float4 x = __ldcg(reinterpret_cast<const float4*>(src)); v[k][r][0] = x.x; v[k][r][1] = x.y; v[k][r][2] = x.z; v[k][r][3] = x.w; }
                        else { const float2 x = __ldcg(reinterpret_cast<const float2*>(src)); v[k][r][0] = x.x; v[k][r][1] = x.y; }
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                float mn = m[r];
#pragma unroll
                for (int k = 0; k < KB; ++k) mn = fmaxf(mn, ml[k][r].x);
                const float f = m[r] == -INFINITY ? (lsum[r] == 0.f ? 0.f : 1.f) : ex2(m[r] - mn);      // keeps a NaN
                lsum[r] *= f;
#pragma unroll
                for (int e = 0; e < VL; ++e) a[r][e] *= f;
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    // (not there, or saw nothing: weight 0; a NaN goes on)
                    const float g = ml[k][r].x == -INFINITY && ml[k][r].y == 0.f ? 0.f : ex2(ml[k][r].x - mn);
                    lsum[r] = fmaf(ml[k][r].y, g, lsum[r]);
#pragma unroll
                    for (int e = 0; e < VL; ++e) a[r][e] = fmaf(v[k][r][e], g, a[r][e]);
                }
                m[r] = mn;
            }
        }
        if (RB == 1 && share > 1) {
            float* mine = xch + warp * (D + 2);
#pragma unroll
            for (int e = 0; e < VL; ++e) mine[VL * lane + e] = a[0][e];
            if (lane == 0) { mine[D] = m[0]; mine[D + 1] = lsum[0]; }
            sync();
            if (sub == 0) {
                float mn = m[0];
#pragma unroll 1
                for (int k = 1; k < share; ++k) mn = fmaxf(mn, mine[k * (D + 2) + D]);
                lsum[0] = 0.f;
#pragma unroll
                for (int e = 0; e < VL; ++e) a[0][e] = 0.f;
#pragma unroll 1
                for (int k = 0; k < share; ++k) {
                    const float* x = mine + k * (D + 2);
                    if (x[D] == -INFINITY && x[D + 1] == 0.f) continue;
                    const float g = ex2(x[D] - mn);
                    lsum[0] = fmaf(x[D + 1], g, lsum[0]);
#pragma unroll
                    for (int e = 0; e < VL; ++e) a[0][e] = fmaf(x[VL * lane + e], g, a[0][e]);
                }
            }
            sync();                                              // xch is written again
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int rl = r0 + team * RB + r;
            if (rl >= rows || sub != 0) continue;
            const int rr = it.tile * tile_rows + rl;
            const float inv = lsum[r] == 0.f ? 0.f : 1.f / lsum[r];
            T* dst = (T*)p.out + ((size_t)(it.q.row0 + rr / p.group) * p.q_heads + it.head * p.group + rr % p.group) * D + VL * lane;
            if constexpr (VL == 4) store4<T>(dst, a[r][0] * inv, a[r][1] * inv, a[r][2] * inv, a[r][3] * inv);
            else store2<T>(dst, a[r][0] * inv, a[r][1] * inv);
        }
    }
}

}  // namespace kv4
#endif

}  // namespace ghd
