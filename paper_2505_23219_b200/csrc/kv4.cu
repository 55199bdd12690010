// The paged cache in 4 bits: append (rotation and quantisation on the way), read back, commit, and the C entry points.
#include <cstdio>
#include <cstring>
#include <type_traits>

#include "kv4.cuh"

namespace ghd {

namespace {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// theta^(-2 t / d) for every pair of channels, worked out on the host in 64 bits
struct RopeFreq { double f[64]; };

// Sine and cosine in 64 bits of |x| < 2^31: x less a whole number of quarter turns (pi / 2 in two parts, the second below
// 2^-53 of the first, so the remainder is off by about 2^-53), then the power series, whose first term left out is below 2^-54
// on [-pi / 4, pi / 4].  The library's function takes any argument and three times the instructions, and keeps a local array.
__device__ __forceinline__ void sincos_turns(double x, double& sn, double& cs) {
    constexpr double HALF_PI_HI = 1.57079632679489655800, HALF_PI_LO = 6.12323399573676603587e-17;
    const double n = rint(x * 0.63661977236758134308);
    double r = fma(-n, HALF_PI_HI, x);
    r = fma(-n, HALF_PI_LO, r);
    const double z = r * r;
    constexpr double F[7] = {1.0 / 6, 1.0 / 120, 1.0 / 5040, 1.0 / 362880, 1.0 / 39916800, 1.0 / 6227020800.0, 1.0 / 1307674368000.0};      // 1 / (2 k + 3)!
    constexpr double G[8] = {0.5, 1.0 / 24, 1.0 / 720, 1.0 / 40320, 1.0 / 3628800, 1.0 / 479001600, 1.0 / 87178291200.0, 1.0 / 20922789888000.0};   // 1 / (2 k + 2)!
    double a = F[6], b = G[7];
#pragma unroll
    for (int k = 5; k >= 0; --k) a = fma(-a, z, F[k]);
#pragma unroll
    for (int k = 6; k >= 0; --k) b = fma(-b, z, G[k]);
    a = fma(-a * z, r, r);               // r - r^3 / 6 + ...
    b = fma(-b, z, 1.0);                 // 1 - r^2 / 2 + ...
    const int quarter = (int)(long long)n & 3;
    const double u = quarter & 1 ? b : a, w = quarter & 1 ? a : b;
    sn = quarter & 2 ? -u : u;
    cs = (quarter == 1 || quarter == 2) ? -w : w;
}

// min and max that keep a NaN (fminf and fmaxf drop it)
__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// 8 consecutive values, 16-byte aligned, as they come and as floats
template <typename T> struct Raw8 { uint4 u[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Raw8<T> load8(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = reinterpret_cast<const uint4*>(p)[i];
    return r;
}
template <typename T> __device__ __forceinline__ void floats(const Raw8<T>& r, float (&x)[8]);
template <> __device__ __forceinline__ void floats<float>(const Raw8<float>& w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[4 * i] = __uint_as_float(w.u[i].x); x[4 * i + 1] = __uint_as_float(w.u[i].y);
        x[4 * i + 2] = __uint_as_float(w.u[i].z); x[4 * i + 3] = __uint_as_float(w.u[i].w);
    }
}
template <> __device__ __forceinline__ void floats<__half>(const Raw8<__half>& w, float (&x)[8]) {
    const uint32_t r[4] = {w.u[0].x, w.u[0].y, w.u[0].z, w.u[0].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r[e]));
        x[2 * e] = f.x;
        x[2 * e + 1] = f.y;
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&x)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
template <> __device__ __forceinline__ void store8<__half>(__half* p, const float (&x)[8]) {
    uint32_t r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __half2 h = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
        r[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}
// Codes of 16 values, x[0 .. 7] in c[0] from the low end.  The quotient decides between two codes, so it is taken in 64 bits
// where 32 could fall on the other side of a half: the difference, 15 scale, its reciprocal and the product, rounded once each, are
// off by less than 2^-22 of the quotient, which is held in [0, 15] (as 15 times a number that the product clamps to [0, 1]), so
// values within 2^-18 of a half are done again, and all of them where the reciprocal is none or the differences could leave the
// range of 32 bits.  Such values are common: differences of halves lie on a grid and many are ties.  Adding 1.5 * 2^23 rounds
// to a whole number, ties to even, and leaves it in the low bits.
__device__ __forceinline__ void codes_of(const float (&x)[16], float mn, float scale, uint32_t (&c)[2]) {
    constexpr float MAGIC = 12582912.f, NEAR = 0.5f - 0x1p-18f;
    constexpr uint32_t BITS = 0x4b400000u * 0x11111111u;            // MAGIC's bits, shifted and added up as the codes are
    const float inv = scale == 0.f ? 0.f : 1.f / (15.f * scale);
    auto share = [&](int i) { return __saturatef((x[i] - mn) * inv); };
    auto off = [&](float t, float r) { return fabsf(fmaf(t, 15.f, MAGIC - r)); };
    float far = 0.f;
    c[0] = c[1] = 0u - BITS;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float t = share(i), r = fmaf(t, 15.f, MAGIC);
        far = fmaxf(far, off(t, r));
        c[i >> 3] += __float_as_uint(r) << (4 * (i & 7));
    }
    uint32_t again = 0;
    if (far > NEAR) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float t = share(i);
            again |= (uint32_t)(off(t, fmaf(t, 15.f, MAGIC)) > NEAR) << i;
        }
    }
    if (!(inv < INFINITY) || scale > 0x1p121f) again = 0xffffu;
    while (again) {
        const int i = __ffs(again) - 1;
        again &= again - 1;
        float y = x[0];
#pragma unroll
        for (int k = 1; k < 16; ++k) if (k == i) y = x[k];
        const float r = fminf(fmaxf((float)rint(((double)y - (double)mn) / (double)scale), 0.f), 15.f);
        const int at = 4 * (i & 7);
        if (i < 8) c[0] = (c[0] & ~(15u << at)) | (uint32_t)r << at;
        else c[1] = (c[1] & ~(15u << at)) | (uint32_t)r << at;
    }
}

// Rows of the call that one warp works through, and their sequence: found by the lanes together when a row leaves the
// sequence of the one before.
struct RowOwner {
    int seq, end;       // -1: nobody's; rows up to `end` (excluded) have the same answer
    Kv4Seq q;
};
__device__ __forceinline__ void find_owner(const Kv4View& w, int row, bool lengths, RowOwner& o) {      // lengths: the rows go behind kv_len
    const int lane = threadIdx.x & 31;
    int seq = -1;
    for (int s0 = 0; s0 < w.n_seqs && seq < 0; s0 += 32) {
        const int s = s0 + lane;
        const bool mine = s < w.n_seqs && __ldg(w.row_start + s) <= row && row < __ldg(w.row_start + s + 1);
        const uint32_t b = __ballot_sync(0xffffffffu, mine);
        if (b) seq = s0 + __ffs(b) - 1;
    }
    o.seq = seq;
    o.end = row + 1;
    if (seq >= 0) {
        o.q = lengths ? kv4_load_seq(w, seq) : kv4_seq(__ldg(w.row_start + seq), __ldg(w.row_start + seq + 1), w.n_rows, 0, 0x7fffffffll);
        if (o.q.bad && lane == 0) atomicCAS(w.input_status, DEV_OK, DEV_KV4_ROWS);
        if (row < o.q.row0 || row >= o.q.row0 + o.q.n) o.seq = -1;      // starts out of order
        else o.end = o.q.row0 + o.q.n;
    }
}

constexpr int ROW_WARPS = 4;       // warps of a block; each has rows of its own
constexpr int APPEND_RESIDENT = 16;     // warps of k_kv4_append on an SM at a time

// Rotates the queries and appends keys and values; in a grid of two rows blockIdx.y 0 does the latter and 1 the former.  A warp
// takes a row and every `slices`-th of its jobs: a job is the K, V or q rows of HPW heads, D / 16 lanes each.  Lane j of a head holds
// the pairs t = 8 j .. 8 j + 7 with both halves (K, q), so the rotation needs no exchange and its codes are two words; of V the 16
// channels from 16 j on.  What the next two jobs read is asked for ahead.  The row's angles (64-bit sincos, D / 2 of them) are
// shared out over the lanes and passed round by shuffles.
// One row of 32 heads takes 4.6 us, a launch and a chain of loads; 2048 rows, 32 heads on 8 (44 MB), 15.6 from DRAM, 12.6 from the L2.
// 8 ragged prompts of up to 2048 rows (q in and out, k and v in, codes out: 298 MB) take 74 us, 4.0 TB/s; k and v alone 39; 16 warps an
// SM (126 registers) wait for loads and for one another's results.  More warps with spills: 79 us when this took 85, but one row 5.2
// instead of 4.3; quotients in paired instructions: slower.  32 bits instead of 64 for the keys' rotation or the angles would save 2 us.
// Float (582 MB): 107 us, 5.4 TB/s.
template <typename T, int D>
__global__ void __launch_bounds__(ROW_WARPS * 32, APPEND_RESIDENT / ROW_WARPS) k_kv4_append(const __grid_constant__ Kv4View w, const __grid_constant__ RopeFreq fr, uint8_t* __restrict__ pool,
                                                               const int32_t* __restrict__ pos, const T* q, int64_t q_ld, const T* __restrict__ k,
                                                               const T* __restrict__ v, int64_t kv_ld, T* q_out, int q_heads, int slices, int rows_each) {
    constexpr int R2 = D / 2, LPH = D / 16, HPW = 32 / LPH, ANG = R2 / 32, es = (int)sizeof(T);
    const int lane = threadIdx.x & 31, j = lane % LPH, sub = lane / LPH;
    const int wid = blockIdx.x * ROW_WARPS + (threadIdx.x >> 5), slice = wid % slices;
    const int R = 1 << w.shift, kv_jobs = (w.heads + HPW - 1) / HPW, q_jobs = (q_heads + HPW - 1) / HPW;
    const bool do_q = q && (gridDim.y == 1 || blockIdx.y != 0), do_kv = blockIdx.y == 0;
    struct Pair { Raw8<T> a, b; };
    RowOwner o;
    o.end = -1;
    const int64_t first = (int64_t)(wid / slices) * rows_each;
#pragma unroll 1
    for (int64_t row_ = first; row_ < first + rows_each && row_ < w.n_rows; ++row_) {
        const int row = (int)row_;
        if (row >= o.end) find_owner(w, row, true, o);
        if (o.seq < 0) continue;
        const int slot = o.q.len + (row - o.q.row0);
        const int p0 = pos ? __ldg(pos + row) : slot;
        // 16 values a lane of a job; which: 0 K, 1 V, 2 q
        auto ask = [&](int job, bool queries) {
            Pair x{};
            const int which = queries ? 2 : job >= kv_jobs, h = (which == 1 ? job - kv_jobs : job) * HPW + sub;
            if (job < (queries ? q_jobs : 2 * kv_jobs) && h < (queries ? q_heads : w.heads)) {
                const T* src = (which == 2 ? q + (int64_t)row * q_ld : (which ? v : k) + (int64_t)row * kv_ld) + (int64_t)h * D + (which == 1 ? 16 : 8) * j;
                x.a = load8<T>(src);
                x.b = load8<T>(src + (which == 1 ? 8 : R2));
            }
            return x;
        };
        Pair next = ask(slice, do_q), after = ask(slice + slices, do_q);
        double mc[ANG], msn[ANG];                                   // angles ANG lane + i
#pragma unroll
        for (int i = 0; i < ANG; ++i) sincos_turns((double)p0 * fr.f[ANG * lane + i], msn[i], mc[i]);
        if (do_q) {
            // Rotated and rounded once: float in 64 bits (8 prompts of up to 2048 rows 107 us; 103 in 32, and a third less exact), half in
            // 32 with sine and cosine rounded to them, off by 2^-22 of the pair's size at most where half's own rounding is 2^-11.
            typedef std::conditional_t<es == 4, double, float> Rot;
            Rot cs[8], sn[8];                                       // angles 8 j + i
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                cs[i] = __shfl_sync(0xffffffffu, (Rot)mc[i % ANG], (8 * j + i) / ANG);
                sn[i] = __shfl_sync(0xffffffffu, (Rot)msn[i % ANG], (8 * j + i) / ANG);
            }
#pragma unroll 1
            for (int job = slice; job < q_jobs; job += slices) {
                const Pair now = next;
                next = after;
                after = ask(job + 2 * slices, true);
                float a[8], b[8], c[8], d[8];
                floats<T>(now.a, a);
                floats<T>(now.b, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    c[i] = (float)((Rot)a[i] * cs[i] - (Rot)b[i] * sn[i]);
                    d[i] = (float)((Rot)b[i] * cs[i] + (Rot)a[i] * sn[i]);
                }
                const int h = job * HPW + sub;
                if (h < q_heads) {
                    T* y = q_out + ((int64_t)row * q_heads + h) * D + 8 * j;
                    store8<T>(y, c);
                    store8<T>(y + R2, d);
                }
            }
            if (!do_kv) continue;
            next = ask(slice, false);
            after = ask(slice + slices, false);
        }
        const int page = row - o.q.row0 < o.q.n_new ? kv4_page(w, o.seq, slot) : -1;
        if (page < 0) continue;
        const int r = slot & (R - 1);
        double cs[8], sn[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            cs[i] = __shfl_sync(0xffffffffu, mc[i % ANG], (8 * j + i) / ANG);
            sn[i] = __shfl_sync(0xffffffffu, msn[i % ANG], (8 * j + i) / ANG);
        }
#pragma unroll 1
        for (int job = slice; job < 2 * kv_jobs; job += slices) {
            const Pair now = next;
            next = after;
            after = ask(job + 2 * slices, false);
            const int which = job >= kv_jobs, h = (which ? job - kv_jobs : job) * HPW + sub;
            float a[8], b[8], x[16];
            floats<T>(now.a, a);
            floats<T>(now.b, b);
            if (which) {
#pragma unroll
                for (int i = 0; i < 8; ++i) { x[i] = a[i]; x[8 + i] = b[i]; }
            } else {                                                // rotated in 64 bits, then rounded to 32
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = (float)((double)a[i] * cs[i] - (double)b[i] * sn[i]);
                    x[8 + i] = (float)((double)b[i] * cs[i] + (double)a[i] * sn[i]);
                }
            }
            float lo = x[0], hi = x[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) { lo = min_nan(lo, x[i]); hi = max_nan(hi, x[i]); }
#pragma unroll
            for (int s = 1; s < LPH; s <<= 1) {
                lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, s));
                hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, s));
            }
            const T mn = from_f<T>(lo), scale = from_f<T>((float)(((double)hi - (double)lo) / 15.0));
            uint32_t c[2];
            codes_of(x, to_f<T>(mn), to_f<T>(scale), c);
            if (h >= w.heads) continue;
            uint8_t* blk = pool + kv4_block_at(w, page, h);
            uint8_t* codes = blk + kv4_code_at(R, D, which, r);
            if (which) {
                *reinterpret_cast<uint2*>(codes + 8 * j) = make_uint2(c[0], c[1]);
            } else {
                *reinterpret_cast<uint32_t*>(codes + 4 * j) = c[0];
                *reinterpret_cast<uint32_t*>(codes + D / 4 + 4 * j) = c[1];
            }
            if (j == 0) {
                T* par = reinterpret_cast<T*>(blk + kv4_param_at(R, D, es, which, r));
                par[0] = scale;
                par[1] = mn;
            }
        }
    }
}

// min + scale * code of 8 channels, rounded once, and stored.  fp16: a byte of two codes goes to both halves of a register under
// the exponent of 1024 (1024 + c and 1024 + 16 c), one fma makes both c exactly and one more is the value: a fused product and
// sum of halves rounds once.
template <typename T> struct RowPar;
template <> struct RowPar<float> { float2 v; };
template <> struct RowPar<__half> { __half2 v; };
__device__ __forceinline__ void decode8(uint32_t c, RowPar<float> f, float* y) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(f.v.x, (float)((c >> (4 * i)) & 15u), f.v.y);
    store8<float>(y, x);
}
__device__ __forceinline__ void decode8(uint32_t c, RowPar<__half> f, __half* y) {
    const __half2 one = __floats2half2_rn(1.f, 0.0625f), off = __floats2half2_rn(-1024.f, -64.f);
    const __half2 scale = __low2half2(f.v), mn = __high2half2(f.v);
    uint32_t r[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const uint32_t w = (__byte_perm(c, 0u, b | b << 8) & 0x00f0000fu) | 0x64006400u;
        const __half2 v = __hfma2(scale, __hfma2(*reinterpret_cast<const __half2*>(&w), one, off), mn);
        r[b] = *reinterpret_cast<const uint32_t*>(&v);
    }
    *reinterpret_cast<uint4*>(y) = make_uint4(r[0], r[1], r[2], r[3]);
}

// A warp takes a row and every `slices`-th of its jobs: K and V of HPW heads, D / 8 lanes each; a lane decodes eight channels of
// both (4 bytes in, 16 or 32 out).  AHEAD jobs' loads are under way together.  The bytes written bound it when there are many rows:
// 8 sequences of up to 2048 rows, 32 heads (177 MB): 37 us, 4.8 TB/s (59 us with codes converted to 32 bits one by one); float (319 MB)
// 86 us, 3.7 TB/s.  13 rows: 2.7 us.
template <typename T, int D>
__global__ void __launch_bounds__(ROW_WARPS * 32) k_kv4_read(const __grid_constant__ Kv4View w, const uint8_t* __restrict__ pool, const int32_t* __restrict__ first,
                                                             T* __restrict__ k_out, T* __restrict__ v_out, int slices, int rows_each) {
    constexpr int LPH = D / 8, HPW = 32 / LPH, AHEAD = 4, es = (int)sizeof(T);
    const int lane = threadIdx.x & 31, j = lane % LPH, sub = lane / LPH;
    const int wid = blockIdx.x * ROW_WARPS + (threadIdx.x >> 5), slice = wid % slices;
    const int R = 1 << w.shift;
    RowOwner o;
    o.end = -1;
    const int64_t begin = (int64_t)(wid / slices) * rows_each;
    for (int64_t row_ = begin; row_ < begin + rows_each && row_ < w.n_rows; ++row_) {
        const int row = (int)row_;
        if (row >= o.end) find_owner(w, row, !first, o);
        if (o.seq < 0) continue;
        const int64_t slot = (int64_t)(first ? __ldg(first + o.seq) : o.q.len) + (row - o.q.row0);
        if (slot < 0 || slot >= kv4_capacity(w)) {
            if (lane == 0) atomicCAS(w.input_status, DEV_OK, DEV_KV4_ROWS);
            continue;
        }
        const int page = kv4_page(w, o.seq, (int)slot);
        if (page < 0) continue;
        const int r = (int)slot & (R - 1);
        const uint8_t* codes = pool + kv4_block_at(w, page, 0) + kv4_code_at(R, D, 0, r) + 4 * j;
        const uint8_t* pars = pool + kv4_block_at(w, page, 0) + kv4_param_at(R, D, es, 0, r);
        const size_t codes_v = kv4_code_at(R, D, 1, 0) - kv4_code_at(R, D, 0, 0), pars_v = kv4_param_at(R, D, es, 1, 0) - kv4_param_at(R, D, es, 0, 0);
        const int64_t out = (int64_t)row * w.heads * D + 8 * j;
#pragma unroll 1
        for (int h0 = slice * HPW + sub; h0 - sub < w.heads; h0 += AHEAD * slices * HPW) {
            uint32_t c[AHEAD][2];
            RowPar<T> f[AHEAD][2];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int h = h0 + a * slices * HPW;
                if (h < w.heads) {
                    const uint8_t *pc = codes + (size_t)h * w.block, *pp = pars + (size_t)h * w.block;
                    c[a][0] = __ldg(reinterpret_cast<const uint32_t*>(pc));
                    c[a][1] = __ldg(reinterpret_cast<const uint32_t*>(pc + codes_v));
                    f[a][0] = *reinterpret_cast<const RowPar<T>*>(pp);
                    f[a][1] = *reinterpret_cast<const RowPar<T>*>(pp + pars_v);
                }
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int h = h0 + a * slices * HPW;
                if (h >= w.heads) break;
                if (k_out) decode8(c[a][0], f[a][0], k_out + out + (int64_t)h * D);
                if (v_out) decode8(c[a][1], f[a][1], v_out + out + (int64_t)h * D);
            }
        }
    }
}

// Block = one (pool, sequence, head); a lane owns one piece of a row: 16 bytes of K or V codes, or the scale and minimum
// of K or V.  Lanes own disjoint pieces: no synchronisation.  Eight rows of the path are read together and then written: what a
// call costs is the latency of node, page and piece, one behind the other (16 sequences, paths of 5, 8 layers, both launches:
// 6.2 us row by row, 5.1 so; 32 layers of 16 sequences 7.2).  Accepted nodes rise and nodes[j] >= j, so no row is written before it has been read.
constexpr int COMMIT_POOLS = 64, COMMIT_ROWS = 8;
struct CommitPools { uint8_t* p[COMMIT_POOLS]; };

__global__ void __launch_bounds__(32) k_kv4_commit(const __grid_constant__ Kv4View w, const __grid_constant__ CommitPools pools, int es, const ghd_accept_result* __restrict__ results) {
    const int s = blockIdx.y, head = blockIdx.x % w.heads, layer = blockIdx.x / w.heads, lane = threadIdx.x;
    const Kv4Seq sq = kv4_load_seq(w, s);
    if (sq.n <= 0) return;
    const ghd_accept_result* res = results + s;
    int m = res->n_matched;
    if (m > GHD_MAX_NODES - 1) m = GHD_MAX_NODES - 1;
    const int R = 1 << w.shift, D = w.d_head, half = D / 32;         // 16-byte pieces of a row's codes
    if (lane >= 2 * half + 2) return;
    uint8_t* pool = pools.p[layer];
    const int which = lane < half ? 0 : (lane < 2 * half ? 1 : lane - 2 * half), bytes = lane < 2 * half ? 16 : 2 * es;
    auto piece = [&](int page, int row) {
        return pool + kv4_block_at(w, page, head) + (bytes == 16 ? kv4_code_at(R, D, which, row) + 16 * (lane - which * half) : kv4_param_at(R, D, es, which, row));
    };
#pragma unroll 1
    for (int j0 = 1; j0 <= m; j0 += COMMIT_ROWS) {
        uint4 v[COMMIT_ROWS];
        int src[COMMIT_ROWS], pf[COMMIT_ROWS], pt[COMMIT_ROWS];
#pragma unroll
        for (int k = 0; k < COMMIT_ROWS; ++k) src[k] = j0 + k <= m ? res->nodes[j0 + k] : j0 + k;
#pragma unroll
        for (int k = 0; k < COMMIT_ROWS; ++k) {
            const int j = j0 + k;
            const bool moves = src[k] > j && src[k] < sq.n_new;
            if (src[k] != j && !moves) atomicCAS(w.input_status, DEV_OK, DEV_KV4_ROWS);
            pf[k] = moves ? kv4_page(w, s, sq.len + src[k]) : -1;
            pt[k] = moves ? kv4_page(w, s, sq.len + j) : -1;
        }
#pragma unroll
        for (int k = 0; k < COMMIT_ROWS; ++k) {
            v[k] = make_uint4(0, 0, 0, 0);
            if (pf[k] < 0 || pt[k] < 0) continue;
            const uint8_t* a = piece(pf[k], (sq.len + src[k]) & (R - 1));
            if (bytes == 16) v[k] = *reinterpret_cast<const uint4*>(a);
            else if (bytes == 8) { const uint2 x = *reinterpret_cast<const uint2*>(a); v[k].x = x.x; v[k].y = x.y; }
            else v[k].x = *reinterpret_cast<const uint32_t*>(a);
        }
#pragma unroll
        for (int k = 0; k < COMMIT_ROWS; ++k) {
            if (pf[k] < 0 || pt[k] < 0) continue;
            uint8_t* b = piece(pt[k], (sq.len + j0 + k) & (R - 1));
            if (bytes == 16) *reinterpret_cast<uint4*>(b) = v[k];
            else if (bytes == 8) *reinterpret_cast<uint2*>(b) = make_uint2(v[k].x, v[k].y);
            else *reinterpret_cast<uint32_t*>(b) = v[k].x;
        }
    }
}

// The lengths grow behind the moves: by the accepted path, or by all new rows.
__global__ void k_kv4_advance(Kv4View w, int32_t* kv_len, const ghd_accept_result* __restrict__ results) {
    const int s = blockIdx.x * blockDim.x + threadIdx.x;
    if (s >= w.n_seqs) return;
    const Kv4Seq sq = kv4_seq(w.row_start[s], w.row_start[s + 1], w.n_rows, kv_len[s], kv4_capacity(w));
    if (sq.bad) atomicCAS(w.input_status, DEV_OK, DEV_KV4_ROWS);
    if (sq.n <= 0) return;
    int add = sq.n_new;
    if (results) {
        int m = results[s].n_matched;
        if (m < 0) m = 0;
        if (m > GHD_MAX_NODES - 1) m = GHD_MAX_NODES - 1;
        if (m + 1 > sq.n_new) atomicCAS(w.input_status, DEV_OK, DEV_KV4_ROWS);
        else add = m + 1;
    }
    kv_len[s] = sq.len + add;
}

// Warps of a call over rows; `resident`: those that an SM holds at a time.  Few rows: their jobs are dealt to several warps
// (slices) until the device is full once, and no further, since every warp of a row works out its angles (append with four
// times as many: 512 / 1024 / 2048 rows of 32 heads on 8 took 11.6 / 20.0 / 23.1 us where they take 6.6 / 8.4 / 12.6).  Many rows: a warp takes
// several in turn, whose sequence it then looks up once.
struct RowGrid { int slices, rows_each, blocks; };
RowGrid row_grid(const ghd_ctx* c, int n_rows, int jobs, int resident) {
    const int64_t want = (int64_t)c->sm_count * resident;
    RowGrid g;
    int64_t s = want / n_rows;
    g.slices = (int)(s < 1 ? 1 : (s > jobs ? jobs : s));
    g.rows_each = (int)((n_rows + want - 1) / want);
    const int64_t warps = ((int64_t)n_rows + g.rows_each - 1) / g.rows_each * g.slices;
    g.blocks = (int)((warps + ROW_WARPS - 1) / ROW_WARPS);
    return g;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// What is wrong with the sizes of a cache: a status and a reason.
struct Kv4Fault {
    ghd_status status;
    const char* what;
};
Kv4Fault size_fault(const ghd_ctx* c, const ghd_kv4* kv) {
    if (kv->n_seqs < 1 || kv->n_seqs > GHD_MAX_SEQS) return {GHD_EINVAL, "kv4: n_seqs outside [1, GHD_MAX_SEQS]"};
    if (kv->page_rows != 16 && kv->page_rows != 32 && kv->page_rows != 64 && kv->page_rows != 128) return {GHD_EINVAL, "kv4: page_rows is not 16, 32, 64 or 128"};
    if (kv->n_pages < 1 || kv->max_pages < 1 || (int64_t)kv->max_pages * kv->page_rows > (1ll << 30)) return {GHD_EINVAL, "kv4: bad page counts"};
    if (kv->n_kv_heads < 1 || c->cfg.n_heads % kv->n_kv_heads) return {GHD_ESHAPE, "kv4: n_kv_heads does not divide n_heads"};
    return {GHD_OK, ""};
}

ghd_status check_kv4(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows) {
    if (!kv || !rows) return fail(c, GHD_EINVAL, "kv4: null description");
    const Kv4Fault f = size_fault(c, kv);
    if (f.status != GHD_OK) return fail(c, f.status, f.what);
    if (!kv->page_table || !kv->kv_len || !rows->row_start) return fail(c, GHD_EINVAL, "kv4: null page table, lengths or row starts");
    if ((((uintptr_t)kv->page_table | (uintptr_t)kv->kv_len | (uintptr_t)rows->row_start | (uintptr_t)rows->pos) & 3) || ((uintptr_t)rows->mask & 7))
        return fail(c, GHD_EINVAL, "kv4: a table, length, row start, position or mask that is not aligned to its type");
    if (rows->n_rows < 0) return fail(c, GHD_EINVAL, "kv4: negative n_rows");
    if (rows->mask && rows->mask_words < 1) return fail(c, GHD_EINVAL, "kv4: a mask needs mask_words >= 1");
    if (!c->ws) return fail(c, GHD_ENOSPACE, "no workspace set");
    return GHD_OK;
}

}  // namespace

Kv4View kv4_view(const ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows) {
    Kv4View w{};
    w.table = kv->page_table; w.kv_len = kv->kv_len; w.row_start = rows->row_start;
    w.n_seqs = kv->n_seqs; w.n_pages = kv->n_pages; w.max_pages = kv->max_pages; w.n_rows = rows->n_rows;
    w.shift = kv->page_rows == 16 ? 4 : kv->page_rows == 32 ? 5 : kv->page_rows == 64 ? 6 : 7;
    w.heads = kv->n_kv_heads; w.d_head = c->cfg.d_head;
    w.block = kv4_block_bytes(kv->page_rows, c->cfg.d_head, c->cfg.dtype == GHD_F32 ? 4 : 2);
    w.status = c->status; w.input_status = c->input_status;
    return w;
}

}  // namespace ghd

using namespace ghd;

extern "C" {

size_t ghd_kv4_pool_bytes(const ghd_ctx* c, const ghd_kv4* kv) {
    if (!c || !kv || size_fault(c, kv).status != GHD_OK) return 0;
    return (size_t)kv->n_pages * kv->n_kv_heads * kv4_block_bytes(kv->page_rows, c->cfg.d_head, c->cfg.dtype == GHD_F32 ? 4 : 2);
}

ghd_status ghd_kv4_append(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows, void* pool, const void* q, int64_t q_ld, const void* k,
                          const void* v, int64_t kv_ld, void* q_out) {
    if (!c) return GHD_EINVAL;
    ghd_status st = check_kv4(c, kv, rows);
    if (st != GHD_OK || rows->n_rows == 0) return st;               // (no rows: their buffers may be null)
    const ghd_model_cfg& m = c->cfg;
    const int D = m.d_head;
    if (!pool || !k || !v || (!q != !q_out)) return fail(c, GHD_EINVAL, "kv4_append: null pool, k or v, or only one of q and q_out");
    if (q_ld == 0) q_ld = (int64_t)m.n_heads * D;
    if (kv_ld == 0) kv_ld = (int64_t)kv->n_kv_heads * D;
    if (q_ld < (int64_t)m.n_heads * D || kv_ld < (int64_t)kv->n_kv_heads * D || q_ld % 8 || kv_ld % 8)
        return fail(c, GHD_EINVAL, "kv4_append: a leading dimension below the row's width, or not a multiple of 8");
    if (!aligned16(pool) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out)) return fail(c, GHD_EINVAL, "kv4_append: pointers must be 16-byte aligned");
    if (q == q_out && q && q_ld != (int64_t)m.n_heads * D) return fail(c, GHD_EINVAL, "kv4_append: q_out may be q only when q is contiguous");
    OnDevice dev(c);
    RopeFreq fr;
    memcpy(fr.f, c->rope_freq, sizeof(fr.f));
    const Kv4View w = kv4_view(c, kv, rows);
    const int hpw = 32 / (D / 16);
    const int q_jobs = (m.n_heads + hpw - 1) / hpw, kv_jobs = 2 * ((kv->n_kv_heads + hpw - 1) / hpw);
    const RowGrid g = row_grid(c, rows->n_rows, q ? q_jobs : kv_jobs, APPEND_RESIDENT);
    // Blocks of their own for the queries while all fit the device at once (one row 4.6 us, 64 rows 4.5); else a warp does both, with
    // one set of angles (512 / 1024 rows of 32 heads on 8: 8.2 / 9.9 us apart, 6.6 / 8.4 together).
    const bool apart = q && 2 * (int64_t)rows->n_rows * q_jobs <= (int64_t)c->sm_count * APPEND_RESIDENT;
    const dim3 grid(g.blocks, apart ? 2 : 1);
#define GHD_APPEND(T, DH) k_kv4_append<T, DH><<<grid, ROW_WARPS * 32, 0, c->cur>>>(w, fr, (uint8_t*)pool, rows->pos, (const T*)q, q_ld, (const T*)k, (const T*)v, kv_ld, (T*)q_out, m.n_heads, g.slices, g.rows_each)
    if (m.dtype == GHD_F32) { if (D == 64) GHD_APPEND(float, 64); else GHD_APPEND(float, 128); }
    else { if (D == 64) GHD_APPEND(__half, 64); else GHD_APPEND(__half, 128); }
#undef GHD_APPEND
    c->launches++;
    return check_cuda(c, "kv4_append");
}

ghd_status ghd_kv4_attention(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows, const void* pool, const void* q, void* out) {
    if (!c) return GHD_EINVAL;
    ghd_status st = check_kv4(c, kv, rows);
    if (st != GHD_OK || rows->n_rows == 0) return st;               // (no rows: their buffers may be null)
    if (!pool || !q || !out) return fail(c, GHD_EINVAL, "kv4_attention: null pool, q or out");
    if (!aligned16(pool) || !aligned16(q) || !aligned16(out)) return fail(c, GHD_EINVAL, "kv4_attention: pointers must be 16-byte aligned");
    if (q == out) return fail(c, GHD_EINVAL, "kv4_attention: out may not be q");
    OnDevice dev(c);
    c->entry_fresh = c->opt_chain_calls ? 0 : 1;
    st = launch_attn_kv4(c, kv4_view(c, kv, rows), rows, pool, q, out);
    return st != GHD_OK ? st : check_cuda(c, "kv4_attention");
}

ghd_status ghd_kv4_read(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows, const void* pool, const int32_t* first, void* k_out, void* v_out) {
    if (!c) return GHD_EINVAL;
    ghd_status st = check_kv4(c, kv, rows);
    if (st != GHD_OK || rows->n_rows == 0) return st;               // (no rows: their buffers may be null)
    if (!pool || (!k_out && !v_out)) return fail(c, GHD_EINVAL, "kv4_read: null pool, or neither output");
    if (!aligned16(pool) || !aligned16(k_out) || !aligned16(v_out) || ((uintptr_t)first & 3)) return fail(c, GHD_EINVAL, "kv4_read: pointers must be 16-byte aligned (first: 4)");
    if (k_out == v_out) return fail(c, GHD_EINVAL, "kv4_read: k_out and v_out are the same");
    OnDevice dev(c);
    const Kv4View w = kv4_view(c, kv, rows);
    const int hpw = 32 / (c->cfg.d_head / 8);
    const RowGrid g = row_grid(c, rows->n_rows, (kv->n_kv_heads + hpw - 1) / hpw, 64);
#define GHD_READ(T, DH) k_kv4_read<T, DH><<<g.blocks, ROW_WARPS * 32, 0, c->cur>>>(w, (const uint8_t*)pool, first, (T*)k_out, (T*)v_out, g.slices, g.rows_each)
    if (c->cfg.dtype == GHD_F32) { if (c->cfg.d_head == 64) GHD_READ(float, 64); else GHD_READ(float, 128); }
    else { if (c->cfg.d_head == 64) GHD_READ(__half, 64); else GHD_READ(__half, 128); }
#undef GHD_READ
    c->launches++;
    return check_cuda(c, "kv4_read");
}

ghd_status ghd_kv4_commit(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows, void* const* pools, int32_t n_layers, const ghd_accept_result* results) {
    if (!c) return GHD_EINVAL;
    ghd_status st = check_kv4(c, kv, rows);
    if (st != GHD_OK) return st;
    if ((uintptr_t)results & 3) return fail(c, GHD_EINVAL, "kv4_commit: results are not aligned");
    if (n_layers < 0 || (results && (n_layers < 1 || !pools))) return fail(c, GHD_EINVAL, "kv4_commit: no pools");
    for (int l = 0; results && l < n_layers; ++l)
        if (!pools[l] || !aligned16(pools[l])) return fail(c, GHD_EINVAL, "kv4_commit: a pool is null or not 16-byte aligned");
    for (int l = 1; results && l < n_layers; ++l)
        for (int e = 0; e < l; ++e)
            if (pools[e] == pools[l]) return fail(c, GHD_EINVAL, "kv4_commit: the same pool twice");
    if (rows->n_rows == 0) return GHD_OK;
    OnDevice dev(c);
    const Kv4View w = kv4_view(c, kv, rows);
    for (int l0 = 0; results && l0 < n_layers; l0 += COMMIT_POOLS) {
        CommitPools cp{};
        const int cnt = n_layers - l0 < COMMIT_POOLS ? n_layers - l0 : COMMIT_POOLS;
        for (int l = 0; l < cnt; ++l) cp.p[l] = (uint8_t*)pools[l0 + l];
        k_kv4_commit<<<dim3(cnt * w.heads, w.n_seqs), 32, 0, c->cur>>>(w, cp, c->cfg.dtype == GHD_F32 ? 4 : 2, results);
        c->launches++;
    }
    k_kv4_advance<<<(w.n_seqs + 127) / 128, 128, 0, c->cur>>>(w, kv->kv_len, results);
    c->launches++;
    return check_cuda(c, "kv4_commit");
}

}  // extern "C"
