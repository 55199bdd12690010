// Attention of new rows (single tokens, draft trees, prompt pieces) over the paged 4-bit cache.
//
// The scales stay out of the matrix products.  With value = min + scale * code,
//   q . k_j = scale_j (q . c_j) + min_j sum(q),      o = sum_j (p_j scale_j) (c_j - 8) + sum_j p_j (min_j + 8 scale_j),
// so the tensor cores multiply by small whole numbers (exact in half and in bfloat16), a key's scale and minimum enter
// once per score, and what a key holds can only reach the rows that see it (a masked NaN has weight zero by selection,
// not by multiplication).
//
// Keys are the M side of both products: S^T [16 keys x 8 rows] = K Q^T and O^T [16 channels x 8 rows] = V^T P^T
// (mma.sync m16n8k16), so one to eight rows cost one n-tile.  The lanes' channels are permuted so that a lane's codes are
// consecutive bytes of a row; nibbles become operands in registers.  A warp takes 16 keys of every chunk of 64 and keeps
// its own running reference (raised when a score exceeds it by 2^2: p * scale then fits half for every scale) and sums;
// the warps meet in shared memory.
//
// Work is dealt by device-side lengths: all chunks of all (sequence, head, row tile) items are numbered and each CTA takes
// an equal run of them (kv4_layout.h), so ragged batches and single long sequences fill the device alike.  An item cut by
// a run's border leaves partial sums; the last of its CTAs to arrive adds them in CTA order (the result does not
// depend on who was last).  Float contexts split q and p * scale into three bfloat16 terms (24 bits).
#include "attn_kv4_dev.cuh"

#include <cuda_bf16.h>

#include <cstdio>

namespace ghd {

namespace {

constexpr int WARPS = 4, CHUNK = 16 * WARPS;
constexpr float RAISE = 2.f;

using namespace kv4;

// ---------------------------------------------------------------- operands of the two storage types
template <typename T> struct Op;
template <> struct Op<__half> {
    static constexpr int TERMS = 1;
    static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
    // two codes (at bits SH .. SH + 3 of each half word) less 8
    template <int SH> static __device__ __forceinline__ uint32_t centred(uint32_t w) { return centred_half<SH>(w); }
    // (a, b) as TERMS packed pairs whose sum is (a, b) to 11 bits
    static __device__ __forceinline__ void split(float a, float b, uint32_t (&t)[1]) {
        const __half2 h = __floats2half2_rn(a, b);
        t[0] = *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <> struct Op<float> {
    static constexpr int TERMS = 3;
    static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
    template <int SH> static __device__ __forceinline__ uint32_t centred(uint32_t w) {
        const uint32_t x = ((w >> SH) & 0x000f000fu) | 0x43004300u;                  // 128 + c
        const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), __floats2bfloat162_rn(136.f, 136.f));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    // (a, b) to 24 bits: each term is what the ones before left over
    static __device__ __forceinline__ void split(float a, float b, uint32_t (&t)[3]) {
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
            t[i] = *reinterpret_cast<const uint32_t*>(&h);
            a -= __bfloat162float(h.x);
            b -= __bfloat162float(h.y);
        }
    }
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <int N> struct Words { uint32_t w[N]; };
template <int N> __device__ __forceinline__ Words<N> load_words(const uint8_t* p) {
    Words<N> r;
    if constexpr (N == 4) { const uint4 v = __ldg(reinterpret_cast<const uint4*>(p)); r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w; }
    else if constexpr (N == 2) { const uint2 v = __ldg(reinterpret_cast<const uint2*>(p)); r.w[0] = v.x; r.w[1] = v.y; }
    else r.w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
    return r;
}

template <typename T, int D, int NT>
struct Narrow {
    static constexpr int RT = 8 * NT;                          // query rows of a tile
    static constexpr int KW = D / 32, VW = D / 64;             // 32-bit words of codes a lane holds of a K row, of a V row
    static constexpr int KS = D / 16;                          // k-steps of S^T
    static constexpr int MT = D / 16;                          // m-tiles of O^T
    static constexpr size_t SLOT = (size_t)RT * (D + 2);       // floats of a partial
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(WARPS * 32, NT == 1 && sizeof(T) == 2 ? 4 : 2) k_attn_kv4(const Kv4AttnParams p) {
    using N = Narrow<T, D, NT>;
    using O_ = Op<T>;
    constexpr int RT = N::RT, KW = N::KW, VW = N::VW, KS = N::KS, MT = N::MT, TERMS = O_::TERMS;
    __shared__ int64_t sums[GHD_MAX_SEQS + 1];
    __shared__ int64_t scratch[32];
    __shared__ __align__(16) float xo[WARPS][RT][D + 4];
    __shared__ float xm[WARPS][RT], xl[WARPS][RT], xs[WARPS][RT];
    __shared__ int arrived;

    const Kv4View& w = p.w;
    const Kv4Tiling til{w.heads, p.group, RT, CHUNK};
    const int64_t units = unit_sums(w, til, sums, scratch);
    const int64_t per = kv4_units_per_cta(units, p.ctas);
    int64_t u = per * blockIdx.x;
    const int64_t u_end = u + per < units ? u + per : units;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int R = 1 << w.shift;
    constexpr int es = (int)sizeof(T);
    const float sl2 = p.scale * KV4_LOG2E;

    while (u < u_end) {
        const Kv4Item it = kv4_find_item(til, sums, w.n_seqs, [&](int s_) { return kv4_load_seq(w, s_); }, u, u_end);
        const int rows = min(RT, it.q.n * p.group - it.tile * RT);      // query rows of this tile
        const int keys = kv4_tile_keys(til, it.q, it.tile);

        // ---- queries: lane (g, t) holds row 8 nt + g, channels [t D/4, (t + 1) D/4), pairs in the order the codes come in
        uint32_t bq[NT][KS][TERMS][2];
        float qs[NT][2];                                                // sums of the queries of rows 8 nt + 2 t, + 1
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int rl = nt * 8 + g, rr = it.tile * RT + rl;
            float x[D / 4];
#pragma unroll
            for (int c = 0; c < D / 4; ++c) x[c] = 0.f;
            if (rl < rows) {
                const T* src = (const T*)p.q + ((size_t)(it.q.row0 + rr / p.group) * p.q_heads + it.head * p.group + rr % p.group) * D + t * (D / 4);
#pragma unroll
                for (int c = 0; c < D / 4; ++c) x[c] = to_f<T>(src[c]);
            }
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < D / 4; ++c) sum += x[c];
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            qs[nt][0] = __shfl_sync(0xffffffffu, sum, 8 * t);
            qs[nt][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {                           // word ks / 2: code pairs (0, 4) (1, 5) or (2, 6) (3, 7)
                const int c = 8 * (ks >> 1) + 2 * (ks & 1);
                uint32_t a[TERMS], b[TERMS];
                O_::split(x[c], x[c + 4], a);
                O_::split(x[c + 1], x[c + 5], b);
#pragma unroll
                for (int e = 0; e < TERMS; ++e) { bq[nt][ks][e][0] = a[e]; bq[nt][ks][e][1] = b[e]; }
            }
        }
        int node[NT][2];                                                // new row of score columns 2 t, 2 t + 1
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) node[nt][e] = (it.tile * RT + nt * 8 + 2 * t + e) / p.group;

        float o[MT][NT][4];
        float ref[NT][2], l[NT][2], ms[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { ref[nt][e] = -INFINITY; l[nt][e] = 0.f; ms[nt][e] = 0.f; }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mt][nt][e] = 0.f;
        }

        for (int ch = it.chunk0; ch < it.chunk0 + it.take; ++ch) {
            const int key0 = ch * CHUNK + warp * 16;
            if (key0 >= keys) continue;
            const int page = kv4_page(w, it.seq, key0);
            if (page < 0) continue;                                     // such keys are not visible
            const uint8_t* blk = p.pool + kv4_block_at(w, page, it.head);
            const int r0 = key0 & (R - 1);
            // A-operand rows g and g + 8 are keys r0 + g and r0 + g + 8; a lane's channels [t D/4, (t + 1) D/4)
            const Words<KW> k0 = load_words<KW>(blk + kv4_code_at(R, D, 0, r0 + g) + t * (D / 8));
            const Words<KW> k1 = load_words<KW>(blk + kv4_code_at(R, D, 0, r0 + g + 8) + t * (D / 8));
            float2 kp0 = load_params<T>(blk + kv4_param_at(R, D, es, 0, r0 + g)), kp1 = load_params<T>(blk + kv4_param_at(R, D, es, 0, r0 + g + 8));
            float2 vp0 = load_params<T>(blk + kv4_param_at(R, D, es, 1, r0 + g)), vp1 = load_params<T>(blk + kv4_param_at(R, D, es, 1, r0 + g + 8));
            // V: keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9, a lane's channels [g D/8, (g + 1) D/8)
            Words<VW> v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = load_words<VW>(blk + kv4_code_at(R, D, 1, r0 + 2 * t + (e & 1) + 8 * (e >> 1)) + g * (D / 16));

            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
            for (int i = 0; i < KW; ++i) {
#pragma unroll
                for (int hlf = 0; hlf < 2; ++hlf) {
                    const uint32_t wa = k0.w[i] >> (8 * hlf), wb = k1.w[i] >> (8 * hlf);
                    const uint32_t a0 = O_::template centred<0>(wa), a1 = O_::template centred<0>(wb);
                    const uint32_t a2 = O_::template centred<4>(wa), a3 = O_::template centred<4>(wb);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < TERMS; ++e) O_::mma(s[nt], a0, a1, a2, a3, bq[nt][2 * i + hlf][e][0], bq[nt][2 * i + hlf][e][1]);
                }
            }
            const float ks0 = kp0.x * sl2, ks1 = kp1.x * sl2;
            const float km0 = fmaf(8.f, kp0.x, kp0.y) * sl2, km1 = fmaf(8.f, kp1.x, kp1.y) * sl2;
            bool vis[NT][4];
            const bool all = key0 + 16 <= it.q.len;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[nt][e] = (e < 2) ? fmaf(ks0, s[nt][e], km0 * qs[nt][e & 1]) : fmaf(ks1, s[nt][e], km1 * qs[nt][e & 1]);
                    vis[nt][e] = true;
                }
            if (!all) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = key0 + g + 8 * (e >> 1) - it.q.len;
                        const bool ok = j < 0 || sees_new(p, it.q, node[nt][e & 1], j);
                        vis[nt][e] = ok;
                        if (!ok) s[nt][e] = -INFINITY;
                    }
            }
            bool over = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) over = over || (s[nt][e] - ref[nt][e & 1] > RAISE);
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(s[nt][e], s[nt][e + 2]);
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        if (mx > ref[nt][e]) {
                            const float f = ex2(ref[nt][e] - mx);       // 0 from a reference of -infinity
                            ref[nt][e] = mx;
                            l[nt][e] *= f;
                            ms[nt][e] *= f;
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) { o[mt][nt][e] *= f; o[mt][nt][e + 2] *= f; }
                        }
                    }
            }
            uint32_t bp[NT][TERMS][2];
            const float vm0 = fmaf(8.f, vp0.x, vp0.y), vm1 = fmaf(8.f, vp1.x, vp1.y);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float ps[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float rf = ref[nt][e & 1];
                    float pe = ex2(s[nt][e] - (rf == -INFINITY ? 0.f : rf));
                    float a = pe * (e < 2 ? vp0.x : vp1.x), b = pe * (e < 2 ? vm0 : vm1);
                    if (!all && !vis[nt][e]) pe = a = b = 0.f;
                    l[nt][e & 1] += pe;
                    ms[nt][e & 1] += b;
                    ps[e] = a;
                }
                uint32_t x[TERMS], y[TERMS];
                O_::split(ps[0], ps[1], x);
                O_::split(ps[2], ps[3], y);
#pragma unroll
                for (int e = 0; e < TERMS; ++e) { bp[nt][e][0] = transpose8x8(x[e]); bp[nt][e][1] = transpose8x8(y[e]); }
            }
            // O^T: m-tile mt holds the lane's channels 2 mt (operand row g) and 2 mt + 1 (row g + 8)
#pragma unroll
            for (int i = 0; i < VW; ++i)
#pragma unroll
                for (int z = 0; z < 2; ++z) {                           // half words of the two keys of a pair side by side
                    const uint32_t x = __byte_perm(v[0].w[i], v[1].w[i], z ? 0x7632 : 0x5410), y = __byte_perm(v[2].w[i], v[3].w[i], z ? 0x7632 : 0x5410);
#pragma unroll
                    for (int hlf = 0; hlf < 2; ++hlf) {
                        const uint32_t xs_ = x >> (8 * hlf), ys_ = y >> (8 * hlf);
                        const uint32_t a0 = O_::template centred<0>(xs_), a1 = O_::template centred<4>(xs_);
                        const uint32_t a2 = O_::template centred<0>(ys_), a3 = O_::template centred<4>(ys_);
                        const int mt = 4 * i + 2 * z + hlf;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < TERMS; ++e) O_::mma(o[mt][nt], a0, a1, a2, a3, bp[nt][e][0], bp[nt][e][1]);
                    }
                }
        }

        // ---- the warps' sums meet
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float a = l[nt][e], b = ms[nt][e];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) { a += __shfl_xor_sync(0xffffffffu, a, x); b += __shfl_xor_sync(0xffffffffu, b, x); }
                const int rl = nt * 8 + 2 * t + e;
                if (g == 0) { xm[warp][rl] = ref[nt][e]; xl[warp][rl] = a; xs[warp][rl] = b; }
#pragma unroll
                for (int mt = 0; mt < MT; mt += 2)
                    *reinterpret_cast<float4*>(&xo[warp][rl][g * (D / 8) + 2 * mt]) = make_float4(o[mt][nt][e], o[mt][nt][e + 2], o[mt + 1][nt][e], o[mt + 1][nt][e + 2]);
            }
        __syncthreads();
        const int64_t c0 = it.first / per, c1 = (it.first + it.chunks - 1) / per;      // CTAs that share the item
        const bool whole = c0 == c1;
        float* slot = p.part + ((size_t)blockIdx.x * 2 + ((int64_t)blockIdx.x == c0 ? 1 : 0)) * N::SLOT;
        for (int x = threadIdx.x; x < rows * (D / 4); x += WARPS * 32) {
            const int rl = x / (D / 4), c = 4 * (x % (D / 4));
            float m = xm[0][rl];
#pragma unroll
            for (int k = 1; k < WARPS; ++k) m = fmaxf(m, xm[k][rl]);
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
            float lsum = 0.f;
#pragma unroll
            for (int k = 0; k < WARPS; ++k) {
                if (xm[k][rl] == -INFINITY && xl[k][rl] == 0.f) continue;   // a warp that saw nothing (a NaN goes on)
                const float f = ex2(xm[k][rl] - m);
                const float4 b = *reinterpret_cast<const float4*>(&xo[k][rl][c]);
                const float mm = xs[k][rl];
                a.x += f * (b.x + mm); a.y += f * (b.y + mm); a.z += f * (b.z + mm); a.w += f * (b.w + mm);
                lsum += f * xl[k][rl];
            }
            if (whole) {
                const int rr = it.tile * RT + rl;
                const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
                T* dst = (T*)p.out + ((size_t)(it.q.row0 + rr / p.group) * p.q_heads + it.head * p.group + rr % p.group) * D + c;
                store4<T>(dst, a.x * inv, a.y * inv, a.z * inv, a.w * inv);
            } else {
                __stcg(reinterpret_cast<float4*>(slot + (size_t)rl * D + c), a);
                if (c == 0) __stcg(reinterpret_cast<float2*>(slot + (size_t)RT * D + 2 * rl), make_float2(m, lsum));
            }
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                const int want = (int)(c1 - c0), old = atomicAdd(p.counters + c0, 1);
                if (old == want) p.counters[c0] = 0;                     // everybody has arrived: ready for the next launch
                arrived = old == want;
                __threadfence();
            }
            __syncthreads();
            if (arrived) {
                merge_item<T, D>(p, it, RT, rows, c0, c1, threadIdx.x, WARPS * 32);
            }
        }
        __syncthreads();                                                 // the exchange buffers are written again
        u += it.take;
    }
}

template <typename T, int D, int NT>
ghd_status launch_narrow(ghd_ctx* c, Kv4AttnParams& p) {
    p.ctas = c->sm_count * (NT == 1 && sizeof(T) == 2 ? 4 : 2);
    const size_t have = (size_t)c->sm_count * 2 * 256 * 128;             // floats of the tile scratch (carve_workspace)
    if ((size_t)p.ctas * 2 * Narrow<T, D, NT>::SLOT > have || p.ctas > 4096) return fail(c, GHD_ENOSPACE, "kv4_attention: workspace too small");
    launch_k(c, false, k_attn_kv4<T, D, NT>, dim3(p.ctas), dim3(WARPS * 32), 0, p);
    return GHD_OK;
}

}  // namespace

ghd_status launch_attn_kv4(ghd_ctx* c, const Kv4View& w, const ghd_kv4_rows* rows, const void* pool, const void* q, void* out) {
    const ghd_model_cfg& m = c->cfg;
    Kv4AttnParams p{};
    p.w = w;
    p.pool = (const uint8_t*)pool; p.q = q; p.out = out;
    p.mask = rows->mask; p.mask_words = rows->mask_words;
    p.q_heads = m.n_heads; p.group = m.n_heads / w.heads;
    p.scale = 1.0f / sqrtf((float)m.d_head);
    p.part = c->gemm_part; p.counters = c->counters;
    const int64_t avg = ((int64_t)rows->n_rows * p.group + w.n_seqs - 1) / w.n_seqs;      // query rows of a sequence and head, on average
    if (m.dtype == GHD_F32) return m.d_head == 64 ? launch_narrow<float, 64, 1>(c, p) : launch_narrow<float, 128, 1>(c, p);
    if (avg > 16) return launch_attn_kv4_tc(c, p, avg > 64 ? 128 : 64);
    if (m.d_head == 64) return avg <= 8 ? launch_narrow<__half, 64, 1>(c, p) : launch_narrow<__half, 64, 2>(c, p);
    return avg <= 8 ? launch_narrow<__half, 128, 1>(c, p) : launch_narrow<__half, 128, 2>(c, p);
}

}  // namespace ghd
