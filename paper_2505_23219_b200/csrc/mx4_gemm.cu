// Product with matrices in microscaled 4-bit floating point on the 5th-generation tensor cores (sm_100a): y[n][m] = x[n][k] w[m][k]^T.
//
// tcgen05.mma of kind::mxf8f6f4 multiplies 4-bit elements with 8-bit ones as they are, each 32 along k with a power-of-two scale
// on either side.  x has 16 or 32 bits, so 32 elements of it are split into TERMS sums of e4m3 numbers: with 2^e <= largest < 2^(e+1)
// the first term is x / 2^(e-7) rounded to e4m3 (4 significant bits, at most 256), the next 2^5 times what is left, and so on.  A term
// leaves at most 2^-4 of its element, so three of them hold the 11 bits of a half and five the 24 of a float, exactly but for what is
// below 2^-27 (2^-37) of the largest of the 32.  The terms of a row are neighbouring columns of one MMA (N = TERMS * rows), so
// that a weight is read once for all; the epilogue adds them.
//
// As in the half-precision projection, 128 rows of w are the M of an MMA, the columns of x its N; a unit is one tile of 128 rows (MT = 1)
// or two (MT = 2: two neighbours that share the loads of x, or a gate tile with its up tile; which: at the launch below).  Where there are fewer than half as many
// units as SMs, a cluster of CTAs shares each, a part of k to every CTA, and adds up through distributed shared memory.
// Otherwise the flattened (unit, k-step) space is cut into equal ranges, one per CTA: whoever has the first k-step of a unit finishes
// it, with its own sums in registers, as the last of its range; the others have come to it first and left their sums in the workspace (a
// bounded wait makes sure; they have started before it).  Both add in the order of k.
//
// The tensor cores cut off a little of each sum they add to, so that long sums of one sign lose more than rounded ones, the more the longer: accumulators
// are taken out every CHUNK k-steps and added up in registers with rounding.  Relative error of the norm, sums of 4096 to 14336 elements of one sign, for
// CHUNK 8 / 16 / 32 / 64: 5e-8 / 7e-8 / 1.4e-7 / 1.4e-7 to 3.8e-7; of both signs 4e-8 to 7e-8 with each; a plain float product 5e-7 to 1.6e-6.
// Time: gate and up of 256 rows by 13824 x 5120 97 / 93 / 91 / 90 us (floats 157 / 151 / 147 / 145), of 64 rows by 11008 x 4096
// 26.6 / 25.6 / 24.6 / 24.6 (31.5 / 30.1 / 29.4 / 29.4).  16 where five terms hold a float's 24 bits, 32 for halves.
//
// What bounds it: with up to 16 rows the memory (16 rows by 32000 x 4096: 20 us of which 11 are streaming at 345 cycles a k-step, the rest
// set-up and the last unit's end; 68 MB of weights), with 64 and more the MMAs (a stage of eight of 128 x 192 x 32 takes 806 cycles of 768: gate and up of
// 256 rows by 13824 x 5120 twice, 91 us, 2.4 PFLOP/s of e4m3 products under the power cap).  One row by 4096 x 4096: 7.4 us, half of it in the two launches.
// cta_group::2 would halve x's share of the loads, which do not bound it; kind::f16 with unpacked weights would need twice the
// shared memory's bandwidth for them.
#include <cuda.h>
#include <cuda_fp8.h>

#include <cstdio>

#include "mx4.cuh"
#include "tc_common.cuh"

namespace ghd {

namespace {

using namespace mx4;
using namespace tc;

constexpr int THREADS = 384;            // weights' loads, MMAs, eight epilogue warps, x's loads, weights to the L2
constexpr int AHEAD = 32 * 1024;        // bytes of weights that a CTA has asked the L2 for beyond its loads (192 KB: 2 us more for 16 rows of an lm_head, whose first loads wait)
constexpr int MAX_STAGES = 10;
constexpr int MAX_WORKERS = 1024;       // CTAs at most: each has an arrival counter
constexpr int MAX_SPLIT = 8;            // CTAs of a cluster
constexpr int A_BYTES = TILE * TILE;    // a tile of 4-bit elements in shared memory, a byte each
constexpr int SF_BYTES = 512;           // scales of 128 rows and 128 columns

struct Mx4Params {
    int n, m, kt;                       // rows of x, rows of w, k-steps (tiles along k)
    int tiles;                          // tiles of 128 rows of w
    int per_group, groups, cols;        // rows of x are worked on in groups of per_group: cols = TERMS * per_group, up to a multiple of 16
    int sf_atoms;                       // ceil(cols / 128)
    int units, stages;                  // units: row units * groups, groups of one row unit behind one another
    int split;                          // CTAs (a cluster) to a unit; 1: ranges of the flattened space
    long long total;                    // units * kt
    const uint8_t *codes, *codes2;      // of w, of the second matrix
    const uint8_t *scales, *scales2;
    const uint8_t* x_scales;
    float* part;                        // [CTA][MT * per_group][128]: sums of its first unit, if that began in another CTA's range
    int* counters;
    int* status;
    void* out;
};

// one k-step and, behind it, ks of them in one box: of w, of the second matrix, of the terms of x
struct Mx4Maps { CUtensorMap w[2], w2[2], x[2]; };

struct Smem {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES];
    uint64_t acc_full, acc_empty, drain;
    uint32_t tmem_base;
    int abort_flag;
    volatile int loaded;                // k-steps whose loads have been started
    volatile int others_in;             // the other CTAs' sums of the unit that this one finishes are in the workspace
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(policy) : "memory");
}

__device__ __forceinline__ void prefetch_l2(const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

// scales of 128 rows: 32 rows of 16 bytes, 8 of them 128 bytes apart, no swizzle
__device__ __forceinline__ uint64_t smem_desc_scales(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {       // to four columns, the same in all four quarters of the lanes
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// kind::mxf8f6f4: A e2m1 (5), B e4m3 (0), scales e8m0, D float, M = 128; byte q of the scale words belongs to the q-th 32 of 128 columns
__device__ __forceinline__ uint32_t instr_desc_mx(int cols, int q) {
    return 5u << 7 | (uint32_t)(cols >> 3) << 17 | 1u << 23 | (uint32_t)(TILE >> 4) << 24 | (uint32_t)q << 29 | (uint32_t)q << 4;
}
// the four MMAs of a k-step (32 columns of 128 each), in one statement so that their operands differ by constants only
__device__ __forceinline__ void mma_step(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, t;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t.reg .b32 i1, i2, i3;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "setp.ne.b32 t, 1, 0;\n\t"
        "add.s64 a1, %1, 2;\n\tadd.s64 a2, %1, 4;\n\tadd.s64 a3, %1, 6;\n\t"
        "add.s64 b1, %2, 2;\n\tadd.s64 b2, %2, 4;\n\tadd.s64 b3, %2, 6;\n\t"
        "add.u32 i1, %3, 0x20000010;\n\tadd.u32 i2, %3, 0x40000020;\n\tadd.u32 i3, %3, 0x60000030;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, i1, [%4], [%5], t;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, i2, [%4], [%5], t;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, i3, [%4], [%5], t;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void ld8(uint32_t taddr, uint32_t* r) {                // 8 columns of this warp's 32 lanes; not there until ld_wait
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ld_wait8(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])::"memory");
}
// barrier of the epilogue warps that tells whether all of them are well: they take the same way out
__device__ __forceinline__ bool epi_all(bool ok) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)ok) : "memory");
    return r != 0;
}

__device__ __forceinline__ float4 ld_cluster(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// SiLU(g) * up = g s^2 up / (1 + s^2) with s = e^(g/2) for g < 0, g up / (1 + s^2) with s = e^(-g/2) otherwise.  Both sums can have any exponent, so nothing
// on the way may leave the type's range where the result does not: g * up may, and so may e^-g.  Halves (11 bits) take the faster exponential.
// Floats take the plain form, rounded four times, down to DEEP, where 1 + e^-g is e^-g to the last bit; below it up is multiplied by e^(g/4)
// four times (s itself would run out of bits at -174).
// (g * up / (1 + e^-g) before: 64 rows by 11008 x 4096 23.9 us against 24.4 in halves, 28.7 against 29.4 in floats.)
constexpr float DEEP = -80.f;
template <typename T> __device__ __forceinline__ float silu_times(float g, float up);
template <> __device__ __forceinline__ float silu_times<__half>(float g, float up) {
    const float s = __expf(-0.5f * fabsf(g)), c = g < 0.f ? s : 1.f;
    return g * c * up * __fdividef(c, fmaf(s, s, 1.f));
}
template <> __device__ __forceinline__ float silu_times<float>(float g, float up) { return __fdividef(g, 1.f + expf(-g)) * up; }
__device__ __forceinline__ float silu_times_deep(float g, float up) {
    const float t = expf(0.25f * g);
    return g * t * up * t * t * t;
}

// ---------------------------------------------------------------- x -> terms
template <typename T> constexpr int TERMS = sizeof(T) == 2 ? 3 : 5;
template <int P> constexpr int CHUNK = P == 3 ? 32 : 16;                          // k-steps of 128 that one accumulator takes
template <typename T> constexpr int GROUP = sizeof(T) == 2 ? 64 : 32;             // rows of x that one pass over w takes at most

template <typename T>
__global__ void __launch_bounds__(256) k_mx4_terms(const T* __restrict__ x, int64_t ld, int n, int k, bool wide, int kt, int per_group, int cols, int sf_atoms,
                                                   uint2* __restrict__ terms, uint32_t* __restrict__ scales) {
    constexpr int P = TERMS<T>;
    pdl_trigger();
    const int lane = threadIdx.x & 31, w = blockIdx.x * 8 + (threadIdx.x >> 5), per_row = (kt + 1) / 2;
    const int i = w / per_row, c0 = (w - i * per_row) * 256 + lane * 8, tk = c0 / TILE;
    if (i >= n || tk >= kt) return;                              // (16 lanes to a k-step: they leave together)
    const uint32_t mask = 0xffffu << (lane & 16);
    float v[8];
    load8(x + i * ld, c0, k, wide, v);
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max_nan(top, fabsf(v[e]));
    top = max_nan(top, __shfl_xor_sync(mask, top, 1));
    top = max_nan(top, __shfl_xor_sync(mask, top, 2));
    uint32_t field = (__float_as_uint(top) >> 23) & 255u;
    const bool none = field == 255u;
    field = max(field, 7u + 5u * (P - 1));                       // (so that the last term's scale is one)
    const float unit = __uint_as_float((261u - field) << 23);    // 2^(7 - e)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = none ? 0.f : v[e] * unit;
    // Floats from 1.9375 x 2^127 up would round to 2^128: their first term stays at 240 and leaves up to 16, so the next one's factor is 2^4.
    const bool high = sizeof(T) == 4 && field == 254u;
    const int g = i / per_group, col0 = (i - g * per_group) * P;
    const size_t step = (size_t)g * kt + tk;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        uint32_t r[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float most = p == 0 && high ? 240.f : 448.f;
            float h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = fminf(fmaxf(v[4 * q + e], -most), most);
            const __nv_fp8x2_storage_t a = __nv_cvt_float2_to_fp8x2(make_float2(h[0], h[1]), __NV_SATFINITE, __NV_E4M3);
            const __nv_fp8x2_storage_t b = __nv_cvt_float2_to_fp8x2(make_float2(h[2], h[3]), __NV_SATFINITE, __NV_E4M3);
            r[q] = (uint32_t)a | (uint32_t)b << 16;
            const float2 f0 = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(a, __NV_E4M3))), f1 = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(b, __NV_E4M3)));
            const float f[4] = {f0.x, f0.y, f1.x, f1.y};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = (v[4 * q + e] - f[e]) * (p == 0 && high ? 16.f : 32.f);
        }
        const int col = col0 + p;
        terms[(step * cols + col) * 16 + (lane & 15)] = make_uint2(r[0], r[1]);
        uint32_t s = (none ? 255u : field - 7u - 5u * p + (high && p ? 1u : 0u)) << (8 * ((lane >> 2) & 3));
        s |= __shfl_xor_sync(mask, s, 4);
        s |= __shfl_xor_sync(mask, s, 8);
        if ((lane & 15) == 0) scales[(step * sf_atoms + col / TILE) * (SF_BYTES / 4) + scale_at(col % TILE, 0) / 4] = s;
    }
}

// ---------------------------------------------------------------- product
template <int P, int MT, bool GATE, int KS>
__global__ void __launch_bounds__(THREADS, 1)
k_mx4_gemm(const __grid_constant__ Mx4Maps maps, const Mx4Params p) {
    static_assert(!GATE || MT == 2, "a gate tile and its up tile");
    // KS: k-steps of a stage at most (fewer at the end of a range or a unit)
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    uint8_t* tiles = smem_raw + ((1024u - (raw_addr & 1023u)) & 1023u);
    const uint32_t tiles_addr = smem_u32(tiles);
    // a stage: weight tiles [MT][ks] | columns of x [ks] | scales of the tiles [MT][ks] | scales of x [ks]
    const uint32_t x_tile = (uint32_t)p.cols * TILE, x_sf = (uint32_t)p.sf_atoms * SF_BYTES;
    const uint32_t b_off = MT * KS * A_BYTES, sa_off = b_off + KS * x_tile, sb_off = sa_off + MT * KS * SF_BYTES;
    const uint32_t stage_bytes = (sb_off + KS * x_sf + 1023u) & ~1023u;
    Smem* sm = reinterpret_cast<Smem*>(tiles + (size_t)p.stages * stage_bytes);

    // Ranges are dealt from the last one on: a CTA waits for those with the ranges behind its own, which then have started before it, also where a kernel of
    // another stream holds SMs back.
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ctas = gridDim.x, cta = p.split > 1 ? (int)blockIdx.x : ctas - 1 - (int)blockIdx.x;
    int unit0, kc0, my_iters;
    if (p.split > 1) {
        const int rank = cta % p.split;
        unit0 = cta / p.split;
        kc0 = p.kt * rank / p.split;
        my_iters = p.kt * (rank + 1) / p.split - kc0;
    } else {
        const long long beg = p.total * cta / ctas;
        unit0 = (int)(beg / p.kt);
        kc0 = (int)(beg - (long long)unit0 * p.kt);
        my_iters = (int)(p.total * (cta + 1) / ctas - beg);
    }
    // tiles of a unit: the two of a pair, or one behind which there is none
    auto tiles_of = [&](int ru) { return GATE || MT == 1 ? MT : ru * MT + 1 < p.tiles ? 2 : 1; };
    // Walks the stages of this CTA (divisions once a unit: they cost a loading thread as much as the loads of a stage).
    struct Cursor { int unit, kc, left, take, nt, xstep; long long tile; };
    auto enter = [&](Cursor& c) {
        const int ru = c.unit / p.groups;
        c.nt = tiles_of(ru);
        c.tile = (long long)(GATE ? ru : ru * MT) * p.kt + c.kc;
        c.xstep = (c.unit - ru * p.groups) * p.kt + c.kc;
    };
    auto size = [&](Cursor& c) { c.take = min(KS, min(p.kt - c.kc, c.left)); };
    auto begin = [&] {
        Cursor c{unit0, kc0, my_iters};
        enter(c);
        size(c);
        return c;
    };
    auto step = [&](Cursor& c) {
        c.tile += c.take;
        c.xstep += c.take;
        c.left -= c.take;
        if ((c.kc += c.take) == p.kt) { c.kc = 0; ++c.unit; enter(c); }
        size(c);
    };
    auto load_w = [&](uint32_t stage, const Cursor& c, uint64_t pol) {
        const uint32_t at = tiles_addr + stage * stage_bytes, bar = smem_u32(&sm->full[stage]);
        mbar_expect_tx(bar, (uint32_t)c.take * ((uint32_t)c.nt * (TILE_CODES + SF_BYTES) + x_tile + x_sf));     // (the 4-bit tiles count as they lie in memory)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (t >= c.nt) break;
            const long long tile = c.tile + (GATE ? 0 : t * p.kt);
            tma_load_2d(at + t * KS * A_BYTES, GATE && t ? &maps.w2[c.take - 1] : &maps.w[c.take - 1], 0, (int)(tile * TILE), bar, pol);
        }
    };
    auto load_x = [&](uint32_t stage, const Cursor& c, uint64_t pol) {
        const uint32_t at = tiles_addr + stage * stage_bytes, bar = smem_u32(&sm->full[stage]);
        tma_load_2d(at + b_off, &maps.x[c.take - 1], 0, c.xstep * p.cols, bar, pol);
        bulk_load(at + sb_off, p.x_scales + (size_t)c.xstep * x_sf, c.take * x_sf, bar, pol);
    };
    auto load_scales = [&](uint32_t stage, const Cursor& c, uint64_t pol) {
        const uint32_t at = tiles_addr + stage * stage_bytes, bar = smem_u32(&sm->full[stage]);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (t >= c.nt) break;
            const long long tile = c.tile + (GATE ? 0 : t * p.kt);
            bulk_load(at + sa_off + t * KS * SF_BYTES, (GATE && t ? p.scales2 : p.scales) + tile * TILE_SCALES, c.take * SF_BYTES, bar, pol);
        }
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(smem_u32(&sm->full[s]), 1); mbar_init(smem_u32(&sm->empty[s]), 1); }
        mbar_init(smem_u32(&sm->acc_full), 1);
        mbar_init(smem_u32(&sm->acc_empty), 8);
        mbar_init(smem_u32(&sm->drain), 1);
        sm->abort_flag = 0;
        sm->loaded = 0;
        sm->others_in = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm->tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;
    volatile int* abort_flag = &sm->abort_flag;
    float* sums = reinterpret_cast<float*>(tiles);              // a CTA's sums of a unit that a cluster shares

    if (warp == 0) {
        // Weights do not depend on the kernel before: the ring's first ones are under way before the terms of x are there.
        if (lane == 0) {
            uint64_t pol;
            asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
            if (p.groups > 1) asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol));     // read again by the next group
            uint32_t stage = 0, phase = 0;
            int issued = 0;
            bool ok = true;
            for (Cursor c = begin(); c.left > 0; step(c)) {
                if (issued >= p.stages) ok = mbar_wait(smem_u32(&sm->empty[stage]), phase ^ 1, abort_flag, p.status, DEV_TIMEOUT_TMA);
                if (!ok) break;
                load_w(stage, c, pol);
                sm->loaded = my_iters - c.left + c.take;
                ++issued;
                if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1; }
            }
            if (!ok) {                                         // nothing may be in flight when the CTA ends
                const int inflight = issued < p.stages ? issued : p.stages;
                for (int q = 0; q < inflight; ++q) {
                    if (stage == 0) { stage = p.stages - 1; phase ^= 1; } else --stage;
                    for (uint32_t spin = 0; spin < SPIN_LIMIT && !mbar_try(smem_u32(&sm->full[stage]), phase); ++spin) __nanosleep(64);
                }
            }
        }
    } else if (warp == 10) {
        // A thread takes 65 ns to start a copy, so that one could not keep up with the memory: this one starts the other half of them.
        if (lane == 0) {
            uint64_t pol, pol_keep;
            asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
            if (p.groups > 1) asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol));
            asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol_keep));
            uint32_t stage = 0, phase = 0;
            int issued = 0;
            bool ok = true;
            pdl_wait();                                        // x's terms belong to the kernel before until now
            for (Cursor c = begin(); c.left > 0; step(c)) {
                if (issued >= p.stages) ok = mbar_wait(smem_u32(&sm->empty[stage]), phase ^ 1, abort_flag, p.status, DEV_TIMEOUT_TMA);
                if (!ok) break;
                load_x(stage, c, pol_keep);
                load_scales(stage, c, pol);
                ++issued;
                if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1; }
            }
            // All is on its way: this thread looks out for the others' sums, so that the epilogue need not ask the memory.
            const long long end = (long long)unit0 * p.kt + kc0 + my_iters, first = (end - 1) / p.kt * p.kt;
            if (ok && p.split == 1 && end < first + p.kt && first >= end - my_iters) {
                const int others = (int)(((first + p.kt) * ctas - 1) / p.total) - cta;
                uint32_t spin = 0;
                while (ld_acquire_gpu(p.counters + cta) != others) {
                    if (++spin >= SPIN_LIMIT || *abort_flag) { *abort_flag = 1; atomicCAS(p.status, DEV_OK, DEV_TIMEOUT_GRID); break; }
                    __nanosleep(spin > 64 ? 64 : 20);
                }
                p.counters[cta] = 0;                             // ready for the next launch
                __threadfence_block();
                sm->others_in = 1;
            }
        }
    } else if (warp == 11) {
        // Memory answers after 1.5 us, in which the ring (4-bit elements take a byte in it) holds too little: the weights are brought to
        // the L2 first, AHEAD bytes before their loads.
        if (lane == 0) {
            constexpr int STEPS = AHEAD / (MT * TILE_CODES);
            int asked = 0;
            for (Cursor c = begin(); c.left > 0; step(c)) {
                while (asked - sm->loaded > STEPS && !*abort_flag) __nanosleep(100);
                if (*abort_flag) break;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    if (t >= c.nt) break;
                    const long long tile = c.tile + (GATE ? 0 : t * p.kt);
                    prefetch_l2((GATE && t ? p.codes2 : p.codes) + tile * TILE_CODES, c.take * TILE_CODES);
                    prefetch_l2((GATE && t ? p.scales2 : p.scales) + tile * TILE_SCALES, c.take * TILE_SCALES);
                }
                asked += c.take;
            }
        }
    } else if (warp == 1) {
        // The whole warp walks along, one lane issues: values that all lanes share sit in uniform registers, where the instructions take
        // their operands (from one lane's registers each MMA took 200 cycles to issue, N = 48 needs 46).  What lies between two stages' MMAs
        // is idle time of the tensor cores, so there is little.
        // Columns of tensor memory: the accumulators, then the scales of every stage (written again only after the MMAs of the stage's last
        // use are through, which the ring makes sure of).
        const uint32_t leader = elect_one();
        const uint32_t sf_step = 4u * (MT + p.sf_atoms), sf0 = tmem + (uint32_t)(MT * p.cols), idesc = instr_desc_mx(p.cols, 0);
        const uint64_t a0 = smem_desc_sw128(tiles_addr), b0 = smem_desc_sw128(tiles_addr + b_off);
        const uint64_t sa0 = smem_desc_scales(tiles_addr + sa_off), sb0 = smem_desc_scales(tiles_addr + sb_off);
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        auto wait = [&](uint32_t bar, uint32_t parity, int code) {
            if (!__all_sync(0xffffffffu, mbar_try(bar, parity))) ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.status, code));
            return ok;
        };
        for (int left = my_iters, kc = kc0, chunk = 0; left > 0; ++chunk) {
            const int take = min(min(p.kt - kc, left), CHUNK<P>);
            if (chunk > 0 && !wait(smem_u32(&sm->acc_empty), (chunk - 1) & 1, DEV_TIMEOUT_TMEM)) break;
            for (int k = take; k > 0; k -= KS) {
                if (!wait(smem_u32(&sm->full[stage]), phase, DEV_TIMEOUT_MMA)) break;
                tc_fence_after();
                if (leader) {
                    const uint64_t at = stage * (stage_bytes >> 4);
                    const uint32_t sf = sf0 + stage * (KS * sf_step);
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        if (s > 0 && s >= k) break;
                        const uint32_t sfa = sf + s * sf_step, sfb = sfa + 4 * MT, acc = s > 0 ? 1u : (uint32_t)(k < take);
                        copy_scales(sfa, sa0 + at + s * (SF_BYTES >> 4));
                        if (MT == 2) copy_scales(sfa + 4, sa0 + at + ((KS + s) * SF_BYTES >> 4));      // (of a tile that is not there: what the ring holds)
                        copy_scales(sfb, sb0 + at + s * (x_sf >> 4));
                        if (p.sf_atoms == 2) copy_scales(sfb + 4, sb0 + at + s * (x_sf >> 4) + (SF_BYTES >> 4));
                        mma_step(tmem, a0 + at + s * (A_BYTES >> 4), b0 + at + s * (x_tile >> 4), idesc, sfa, sfb, acc);
                        if (MT == 2) mma_step(tmem + p.cols, a0 + at + ((KS + s) * A_BYTES >> 4), b0 + at + s * (x_tile >> 4), idesc, sfa + 4, sfb, acc);
                    }
                    tc_commit(smem_u32(&sm->empty[stage]));
                }
                __syncwarp();
                if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1; }
            }
            if (!ok) break;
            if (leader) tc_commit(smem_u32(&sm->acc_full));
            __syncwarp();
            left -= take;
            if ((kc += take) == p.kt) kc = 0;
        }
        if (!ok && leader) {                                   // no MMA may run when the tensor memory goes
            tc_commit(smem_u32(&sm->drain));
            for (uint32_t spin = 0; spin < SPIN_LIMIT && !mbar_try(smem_u32(&sm->drain), 0); ++spin) __nanosleep(64);
        }
        __syncwarp();
    } else {
        // Epilogue warps 2 .. 9: the lanes of a warp are 32 rows of w; the first four warps take the first half of the rows of x, the others
        // the second, in eights.
        constexpr int NODES = (P == 3 ? 64 : 32) / 2;
        const int quad = warp & 3, grp = (warp - 2) >> 2, row = quad * 32 + lane, et = threadIdx.x - 64;
        const size_t slot = (size_t)MT * p.per_group * TILE;
        const int half = ((p.per_group + 15) / 16) * 8, j0 = grp * half;
        float acc[MT][NODES];
        uint32_t chunks = 0;
        bool ok = true, waited = false;
        int unit = unit0, kc = kc0;
        float* y = (float*)p.out;
        using T = typename std::conditional<P == 3, __half, float>::type;
        T* u = (T*)p.out;
        for (int i = 0; i < my_iters && ok;) {
            const int first = kc, end = min(p.kt, kc + my_iters - i), g = unit % p.groups, ru = unit / p.groups;
            const int rows_here = min(p.per_group, p.n - g * p.per_group), mine = max(0, min(half, rows_here - j0));
            for (int c = first; c < end && ok; c += CHUNK<P>) {
                const bool fresh = c == first;
                // (one warp asks the barrier: eight of them asking took a third of the MMA warp's issue slots)
                ok = epi_all(warp != 2 || mbar_wait(smem_u32(&sm->acc_full), chunks & 1, abort_flag, p.status, DEV_TIMEOUT_EPI));
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < NODES; e += 8)
                        if (e < mine) {
                            uint32_t r[8 * P];
                            const uint32_t at = tmem + t * p.cols + P * (j0 + e) + ((uint32_t)(quad * 32) << 16);
#pragma unroll
                            for (int q = 0; q < P; ++q) ld8(at + 8 * q, r + 8 * q);
#pragma unroll
                            for (int q = 0; q < P; ++q) ld_wait8(r + 8 * q);
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                float v = __uint_as_float(r[P * j + P - 1]);
#pragma unroll
                                for (int q = P - 2; q >= 0; --q) v += __uint_as_float(r[P * j + q]);
                                acc[t][e + j] = fresh ? v : acc[t][e + j] + v;
                            }
                        }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm->acc_empty));
                ++chunks;
            }
            if (!ok) break;
            if (!waited) { pdl_wait(); waited = true; }        // outputs and partial sums belong to the kernel before until now
            const bool whole = first == 0 && end == p.kt;
            if (!whole && p.split > 1) {
                // everything that was loaded has been read: the ring's memory takes the sums
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < NODES; ++e)
                        if (e < mine) sums[(t * p.per_group + j0 + e) * TILE + row] = acc[t][e];
            } else if (first != 0) {
                float* at = p.part + (size_t)cta * slot + row;
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < NODES; ++e)
                        if (e < mine) __stcg(at + (t * p.per_group + j0 + e) * TILE, acc[t][e]);
                epi_all(true);
                if (et == 0) atom_add_acq_rel_gpu(p.counters + (int)((((long long)unit * p.kt + 1) * ctas - 1) / p.total), 1);
            } else {
                if (!whole) {
                    // the ones behind this CTA: those whose ranges reach into the unit
                    const int others = (int)((((long long)unit * p.kt + p.kt) * ctas - 1) / p.total) - cta;
                    if (et == 0) {
                        while (!sm->others_in && !*abort_flag) __nanosleep(20);       // (the loading thread's wait is bounded, or it has given up)
                        ok = !*abort_flag;
                        __threadfence_block();
                    }
                    ok = epi_all(ok);
                    if (!ok) break;
                    for (int o = 1; o <= others; ++o) {
                        const float* at = p.part + (size_t)(cta + o) * slot + row;
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            float v[NODES];                      // all of a tile's are on their way together
#pragma unroll
                            for (int e = 0; e < NODES; ++e) v[e] = e < mine ? __ldcg(at + (t * p.per_group + j0 + e) * TILE) : 0.f;
#pragma unroll
                            for (int e = 0; e < NODES; ++e) acc[t][e] += v[e];
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < (GATE ? 1 : MT); ++t) {
                    const int f = (GATE ? ru : ru * MT + t) * TILE + row;
#pragma unroll
                    for (int e = 0; e < NODES; ++e)
                        if (e < mine && f < p.m) {
                            const size_t at = (size_t)(g * p.per_group + j0 + e) * p.m + f;
                            if constexpr (GATE) u[at] = from_f<T>(silu_times<T>(acc[0][e], acc[1][e]));
                            else y[at] = acc[t][e];
                        }
                }
                if constexpr (GATE && P == 5) {
                    // (apart, and hardly ever run)
                    bool deep = false;
#pragma unroll
                    for (int e = 0; e < NODES; ++e) deep |= e < mine && acc[0][e] < DEEP;
                    const int f = ru * TILE + row;
                    if (deep && f < p.m)
#pragma unroll
                        for (int e = 0; e < NODES; ++e)
                            if (e < mine && acc[0][e] < DEEP) u[(size_t)(g * p.per_group + j0 + e) * p.m + f] = from_f<T>(silu_times_deep(acc[0][e], acc[1][e]));
                }
            }
            i += end - first;
            kc = end;
            if (kc == p.kt) { kc = 0; ++unit; }
        }
    }
    if (p.split > 1) {
        // Every CTA of the cluster finishes a slice of the unit's sums; one that gave up takes part in the barriers only.
        __syncwarp();
        cluster_sync_all();
        using T = typename std::conditional<P == 3, __half, float>::type;
        const int rank = cta % p.split, ru = unit0 / p.groups, g = unit0 - ru * p.groups, nt = tiles_of(ru);
        const int rows_here = min(p.per_group, p.n - g * p.per_group), vecs = (GATE ? 1 : nt) * rows_here * (TILE / 4);
        const int lo = vecs * rank / p.split, hi = *abort_flag ? 0 : vecs * (rank + 1) / p.split;
        const uint32_t base = smem_u32(sums);
        for (int v = lo + (int)threadIdx.x; v < hi; v += THREADS) {
            const int r4 = (v % (TILE / 4)) * 4, col = v / (TILE / 4), t = !GATE && MT == 2 && col >= rows_here ? 1 : 0, j = col - t * rows_here;
            float4 sum[GATE ? 2 : 1];
#pragma unroll
            for (int h = 0; h < (GATE ? 2 : 1); ++h) {
                const uint32_t off = base + (uint32_t)(((t + h) * p.per_group + j) * TILE + r4) * 4;
                float4 b[MAX_SPLIT];
#pragma unroll
                for (int d = 0; d < MAX_SPLIT; ++d)
                    if (d < p.split) b[d] = ld_cluster(mapa_shared(off, d));
                float4 a = b[0];
#pragma unroll
                for (int d = 1; d < MAX_SPLIT; ++d)
                    if (d < p.split) { a.x += b[d].x; a.y += b[d].y; a.z += b[d].z; a.w += b[d].w; }
                sum[h] = a;
            }
            const float s[4] = {sum[0].x, sum[0].y, sum[0].z, sum[0].w};
            const int f = (GATE ? ru : ru * MT + t) * TILE + r4;
            const size_t at = (size_t)(g * p.per_group + j) * p.m + f;
            if constexpr (GATE) {
                const float up[4] = {sum[GATE ? 1 : 0].x, sum[GATE ? 1 : 0].y, sum[GATE ? 1 : 0].z, sum[GATE ? 1 : 0].w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (f + e < p.m) ((T*)p.out)[at + e] = from_f<T>(P == 5 && s[e] < DEEP ? silu_times_deep(s[e], up[e]) : silu_times<T>(s[e], up[e]));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (f + e < p.m) ((float*)p.out)[at + e] = s[e];
            }
        }
        cluster_sync_all();                                      // nobody leaves while its sums are being read
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// ---------------------------------------------------------------- host side
struct Groups { int per, groups, cols, atoms; };
Groups groups_of(int n, int terms, int most) {
    Groups g;
    g.groups = (n + most - 1) / most;
    g.per = (n + g.groups - 1) / g.groups;
    g.groups = (n + g.per - 1) / g.per;
    g.cols = (terms * g.per + 15) / 16 * 16;
    g.atoms = (g.cols + TILE - 1) / TILE;
    return g;
}

// Raises the kernels' limits of shared memory and finds out how many clusters the device holds, once a context.
template <int P>
ghd_status prepare(ghd_ctx* c) {
    if (c->attr_mx4) return GHD_OK;
    const void* kernels[] = {(const void*)k_mx4_gemm<P, 1, false, 2>, (const void*)k_mx4_gemm<P, 1, false, 1>, (const void*)k_mx4_gemm<P, 2, false, 1>,
                             (const void*)k_mx4_gemm<P, 2, true, 1>};       // (a context has one type)
    for (const void* f : kernels)
        if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) return check_cuda(c, "mx4: shared memory");
    // clusters that the device holds at a time (they do not straddle its groups of SMs): fewer than SMs / size for the larger ones
    for (int k = 2; k <= MAX_SPLIT; ++k) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(k);
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = 227 * 1024;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)k;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&c->mx4_clusters[k], k_mx4_gemm<P, 1, false, 2>, &cfg) != cudaSuccess) return check_cuda(c, "mx4: clusters");
    }
    c->attr_mx4 = true;
    return GHD_OK;
}

// CTAs (a cluster) that share a unit where there are fewer than half as many units as SMs; else 1
int split_of(const ghd_ctx* c, int units, int kt, int sms) {
    int split = 1;
    if (units * 2 <= sms)
        for (int k = 2; k <= MAX_SPLIT && k <= kt; ++k)
            if (c->mx4_clusters[k] >= units) split = k;
    return split;
}

template <typename T>
ghd_status go(ghd_ctx* c, const T* x, int64_t ld, bool wide, const ghd_mx4* w, const ghd_mx4* w2, int n, void* out) {
    constexpr int P = TERMS<T>;
    const Groups g = groups_of(n, P, GROUP<T>);
    Mx4Params p{};
    p.n = n; p.m = w->m;
    p.kt = (w->k + TILE - 1) / TILE;
    p.tiles = (w->m + TILE - 1) / TILE;
    p.per_group = g.per; p.groups = g.groups; p.cols = g.cols; p.sf_atoms = g.atoms;
    const ghd_status ready = prepare<P>(c);
    if (ready != GHD_OK) return ready;
    int ctas = c->sm_count < MAX_WORKERS ? c->sm_count : MAX_WORKERS;
    // Two tiles share the columns of x as soon as these are more bytes than a tile (64 a row).  Single ones have half as many sums to exchange at
    // the end, but load x twice as often, which costs 0.1 us a k-step: they are taken where clusters share few k-steps, or where clusters of pairs
    // would leave many SMs without work.  Kernel us, pairs / single: 64 rows by 1024 x 1024 9.6 / 7.3, 4096 x 4096 13.3 / 10.4, 4096 x 11008 18.1 / 15.9;
    // not taken: 96 rows by 4096 x 11008 20.8 / 23.3, 24 rows by 5120 x 13824 16.1 / 18.3, 24 rows of floats by 8192 x 4096 11.1 / 12.0.
    int mt = w2 || g.cols > 64 ? 2 : 1;
    if (mt == 2 && !w2) {
        const int one = split_of(c, p.tiles * g.groups, p.kt, ctas), two = split_of(c, (p.tiles + 1) / 2 * g.groups, p.kt, ctas);
        const int steps = (p.kt + one - 1) / one, pair_steps = (p.kt + two - 1) / two;
        if (p.tiles * g.groups * 2 <= ctas && (steps * P <= 48 || 2 * steps <= 3 * pair_steps)) mt = 1;
    }
    p.units = (w2 ? p.tiles : (p.tiles + mt - 1) / mt) * g.groups;
    p.total = (long long)p.units * p.kt;
    const int ks = mt == 1 && g.cols <= 64 ? 2 : 1;              // (ks * cols rows of x are one box)
    const size_t stage = (ks * ((size_t)mt * (A_BYTES + SF_BYTES) + (size_t)g.cols * TILE + (size_t)g.atoms * SF_BYTES) + 1023) / 1024 * 1024;
    p.stages = (int)((227 * 1024 - 1024 - sizeof(Smem)) / stage);
    if (p.stages > MAX_STAGES) p.stages = MAX_STAGES;
    const int sf_room = (512 - mt * g.cols) / (4 * ks * (mt + g.atoms));
    if (p.stages > sf_room) p.stages = sf_room;
    p.codes = (const uint8_t*)w->codes;
    p.codes2 = w2 ? (const uint8_t*)w2->codes : nullptr;
    p.scales = (const uint8_t*)w->scales;
    p.scales2 = w2 ? (const uint8_t*)w2->scales : nullptr;
    uint8_t* terms = c->mx4_terms;
    uint8_t* x_scales = terms + (size_t)g.groups * p.kt * g.cols * TILE;
    p.x_scales = x_scales;
    p.part = c->gemm_part;
    p.counters = c->counters;
    p.status = c->status;
    p.out = out;
    Mx4Maps maps;
    const uint64_t rows = (uint64_t)p.tiles * p.kt * TILE;
    for (int q = 0; q < ks; ++q)
        if (!tmap_bytes(c, w->codes, rows, TILE * (q + 1), true, &maps.w[q]) || !tmap_bytes(c, (w2 ? w2 : w)->codes, rows, TILE * (q + 1), true, &maps.w2[q]) ||
            !tmap_bytes(c, terms, (uint64_t)g.groups * p.kt * g.cols, (uint32_t)(g.cols * (q + 1)), false, &maps.x[q]))
            return fail(c, GHD_ECUDA, "mx4: tensor map encoding failed");
    for (int q = ks; q < 2; ++q) { maps.w[q] = maps.w[0]; maps.w2[q] = maps.w2[0]; maps.x[q] = maps.x[0]; }
    const int warps = n * ((p.kt + 1) / 2);
    launch_k(c, false, k_mx4_terms<T>, (warps + 7) / 8, 256, 0, x, ld, n, (int)w->k, wide, p.kt, g.per, g.cols, g.atoms, (uint2*)terms, (uint32_t*)x_scales);
    p.split = split_of(c, p.units, p.kt, ctas);
    if (p.units * 2 <= ctas) {
        ctas = p.units * p.split;
    } else if (p.units < ctas) {
        // ranges of (q - 1) / q of a unit: each holds the border between two units, and nobody's range lies within one
        for (int q = 2; q <= 64; ++q)
            if ((long long)p.units * q % (q - 1) == 0 && (long long)p.units * q / (q - 1) <= ctas) { ctas = p.units * q / (q - 1); break; }
    }
    if (ctas > p.total) ctas = (int)p.total;
    const size_t smem = 1024 + p.stages * stage + sizeof(Smem);
    if (p.stages < 2 || p.stages * stage < (size_t)mt * g.per * TILE * sizeof(float)) return fail(c, GHD_EUNSUPPORTED, "mx4: no room for a ring of stages");
    if (w2) launch_kc(c, true, p.split, k_mx4_gemm<P, 2, true, 1>, ctas, THREADS, smem, maps, p);
    else if (mt == 2) launch_kc(c, true, p.split, k_mx4_gemm<P, 2, false, 1>, ctas, THREADS, smem, maps, p);
    else if (ks == 1) launch_kc(c, true, p.split, k_mx4_gemm<P, 1, false, 1>, ctas, THREADS, smem, maps, p);
    else launch_kc(c, true, p.split, k_mx4_gemm<P, 1, false, 2>, ctas, THREADS, smem, maps, p);
    return GHD_OK;
}

}  // namespace

size_t mx4_terms_bytes(const ghd_model_cfg& m) {
    const int terms = m.dtype == GHD_F32 ? TERMS<float> : TERMS<__half>, most = m.dtype == GHD_F32 ? GROUP<float> : GROUP<__half>;
    const size_t kt = ((m.d_model > m.d_ffn ? m.d_model : m.d_ffn) + TILE - 1) / TILE;
    size_t best = 0;                                             // (n rows can take more than n + 1)
    for (int n = 1; n <= m.max_nodes; ++n) {
        const Groups g = groups_of(n, terms, most);
        const size_t b = (size_t)g.groups * kt * ((size_t)g.cols * TILE + (size_t)g.atoms * SF_BYTES);
        if (b > best) best = b;
    }
    return best;
}

ghd_status launch_mx4_product(ghd_ctx* c, const void* x, int64_t ld, bool wide, const ghd_mx4* w, const ghd_mx4* w2, int n, void* out) {
    c->entry_fresh = 1;
    return c->cfg.dtype == GHD_F32 ? go(c, (const float*)x, ld, wide, w, w2, n, out) : go(c, (const __half*)x, ld, wide, w, w2, n, out);
}

}  // namespace ghd
