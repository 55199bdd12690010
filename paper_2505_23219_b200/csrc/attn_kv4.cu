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
// consecutive bytes of a row; nibbles become operands in registers.  A warp takes 32 keys of every chunk of 128 and keeps
// its own running reference and sums; the warps meet in shared memory.
//
// Half range: p * scale is the operand of the second product, rounded to half's 11 bits.  So a row's reference goes by score + log2(scale) of
// the keys that it sees: it is raised when that passes 2^15 of it, and then lies 2^10 below the largest product, so products
// down to 2^-24 of the largest keep all bits, whatever the values' size, and no key has a say in rows that do not see it.  p itself
// stays below 2^40, within 32 bits.  (With references by the scores alone, p * scale of small values and of keys far below the
// top fell below half's normal range.)  Float: by the scores alone, raised by more than 2^2.
//
// Work is dealt by device-side lengths: all chunks of all (sequence, head, row tile) items are numbered and each CTA takes
// an equal run of them (kv4_layout.h), so ragged batches and single long sequences fill the device alike.  An item cut by
// a run's border leaves partial sums; the last of its CTAs to arrive adds them in CTA order (the result does not
// depend on who was last).  Float contexts split q and p * scale into three bfloat16 terms (24 bits).
//
// What it costs.  One token over 2048 rows of 32 heads (8.9 MB): 11.5 us, a chain of latencies (in clocks, of 21000: lengths and prefix
// sums 2300, item 2000, page ids and first rows 2200, queries 1200, two chunks 4000, sums 1500, arrival 2000, merge 2500); over 16384 rows
// 27 us, 2.6 TB/s.  One token each of 32 ragged sequences of up to 8192 rows, 32 heads on 8 (174.5 MB): 54 us, 3.2 TB/s.  That is
// instructions: 700 a warp for 32 keys, all included (9 for a word of eight codes, 32 words a lane; the products are 32), 2.2 an SM a clock out of 12 warps (161 registers a thread).  Four CTAs an SM spill, deeper rings take CTAs away.
//
// Rounding.  Scores, exponentials (ex2.approx: 2 units of 2^-23), weights, sums and the middles' sums are 32 bits.  Half: the weight
// times scale has 11 bits in the second product, so that a key costs one product and not two; it adds about 1e-4 of the output's size
// to the 2e-4 of its rounding to half.  Float: q and the weights are three bfloat16 terms.
#include "attn_kv4_dev.cuh"

#include <cuda_bf16.h>

#include <cstdio>
#include <type_traits>

namespace ghd {

namespace {

constexpr int WARPS = 4, WKEYS = 32, CHUNK = WKEYS * WARPS;      // a warp takes 32 keys of every chunk
constexpr int LEAD = 4;          // an item's fixed cost in chunks (one token of 32 heads over 2048 and 16384 rows: 2: 11.1 and 28.8 us, 3: 11.0 and 28.0, 4: 11.5 and 27.1)

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
    typedef HalfMagic Magic;
    template <int SH> static __device__ __forceinline__ uint32_t centred(uint32_t w, const Magic& m) { return centred_half<SH>(w, m); }
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
    struct Magic {
        uint32_t e;
        __device__ __forceinline__ Magic() : e(0x43004300u) { asm volatile("" : "+r"(e)); }
    };
    template <int SH> static __device__ __forceinline__ uint32_t centred(uint32_t w, const Magic& m) {
        uint32_t x;                                                                  // 128 + c
        asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(x) : "r"(w >> SH), "r"(m.e));
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

template <typename T> __device__ __forceinline__ float2 param_of(const uint8_t* p, int key);
template <> __device__ __forceinline__ float2 param_of<__half>(const uint8_t* p, int key) { return __half22float2(reinterpret_cast<const __half2*>(p)[key]); }
template <> __device__ __forceinline__ float2 param_of<float>(const uint8_t* p, int key) { return reinterpret_cast<const float2*>(p)[key]; }
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// N consecutive values of a row in 16-byte loads (zeros for no row)
template <typename T, int N>
__device__ __forceinline__ void load_row(const T* src, float (&x)[N]) {
    constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
    for (int c = 0; c < N; c += E) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (src) v = __ldg(reinterpret_cast<const uint4*>(src + c));
        const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
        for (int k = 0; k < E; ++k) x[c + k] = to_f<T>(e[k]);
    }
}

// Key rows of a block of 16 in operand order: operand rows 2 t and 2 t + 1 (and + 8) are keys 2 t + (t & 1) and the other of
// the pair, so that eight lanes reading K and sixteen reading V from shared memory meet different banks.
__device__ __forceinline__ int key_of(int k) { return (k & ~1) | ((k ^ (k >> 1)) & 1); }

template <typename T, int D, int NT>
struct Narrow {
    static constexpr int RT = 8 * NT;                          // query rows of a tile
    static constexpr int KW = D / 32, VW = D / 64;             // 32-bit words of codes a lane holds of a K row, of a V row
    static constexpr int KS = D / 16;                          // k-steps of S^T
    static constexpr int MT = D / 16;                          // m-tiles of O^T
    static constexpr size_t SLOT = (size_t)RT * (D + 2);       // floats of a partial
    static constexpr int ES = (int)sizeof(T), ROW = D / 2;     // bytes of a scale, of a packed row
    // a warp's stage: K rows, V rows, K and V (scale, min) of 32 keys, and which of the two groups of 16 have a page
    static constexpr int V_AT = WKEYS * ROW, P_AT = 2 * WKEYS * ROW, VP_AT = P_AT + 2 * WKEYS * ES, FLAG_AT = VP_AT + 2 * WKEYS * ES, STAGE = FLAG_AT + 16;
    static constexpr int STAGES = 2;                           // (32 ragged sequences: 54 us; three stages 56, four 81: fewer CTAs fit)
    static constexpr int XO = D + 4;                           // floats between rows of the exchange buffer
    static constexpr int SMEM = WARPS * STAGES * STAGE + WARPS * RT * (XO + 3) * 4 + WARPS * (D + 2) * 4;
    static constexpr int BLOCKS = NT == 1 && sizeof(T) == 2 ? (D == 64 ? 4 : 3) : 2;      // CTAs an SM
    // place of 16-byte piece c of packed row r
    static __device__ __forceinline__ int piece(int r, int c) { return D == 128 ? r * 64 + ((c ^ ((r >> 1) & 2)) << 4) : r * 32 + (c << 4); }
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(WARPS * 32, Narrow<T, D, NT>::BLOCKS) k_attn_kv4(const __grid_constant__ Kv4AttnParams p) {
    using N = Narrow<T, D, NT>;
    using O_ = Op<T>;
    constexpr bool HALF = sizeof(T) == 2;
    constexpr float RAISE = HALF ? 15.f : 2.f, TOP = HALF ? 10.f : 0.f;      // where a reference is raised, and what lies above a new one
    constexpr int RT = N::RT, KW = N::KW, VW = N::VW, KS = N::KS, MT = N::MT, TERMS = O_::TERMS, XO = N::XO, es = N::ES;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int64_t scratch[32];
    __shared__ int arrived;
    float* xo = reinterpret_cast<float*>(smem + WARPS * N::STAGES * N::STAGE);       // [WARPS][RT][XO]
    float* xm = xo + WARPS * RT * XO;                                                // reference, sum, middles' sum: [WARPS][RT] each
    float* xl = xm + WARPS * RT;
    float* xs = xl + WARPS * RT;
    float* xmerge = xs + WARPS * RT;                                                 // [WARPS][D + 2]
    int64_t* sums = reinterpret_cast<int64_t*>(smem + ((N::SMEM + 15) & ~15));       // [n_seqs + 1]

    const Kv4View& w = p.w;
    const Kv4Tiling til{w.heads, p.group, RT, CHUNK, LEAD};
    const int64_t units = unit_sums(w, til, sums, scratch);
    const int64_t per = kv4_units_per_cta(units, p.ctas);
    const int64_t u_beg = per * blockIdx.x, u_end = u_beg + per < units ? u_beg + per : units;
    if (u_beg >= u_end) return;                                                      // (the whole block)
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int R = 1 << w.shift;
    const float sl2 = p.scale * KV4_LOG2E;
    const typename O_::Magic magic;
    // the block's item, and by warp the one that it loads rows of
    __shared__ Kv4Item cur, ahead[WARPS];
    if (threadIdx.x == 0) {
        Kv4Item it = kv4_find_item(til, sums, w.n_seqs, [&](int s) { return kv4_load_seq(w, s); }, u_beg, u_end);
        it.keys = kv4_tile_keys(til, it.q, it.tile);
        cur = it;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) ahead[k] = it;
    }
    __syncthreads();

    // ---- this warp's ring: 32 keys a stage, STAGES - 1 units ahead, over the borders of items
    uint8_t* ring = smem + warp * N::STAGES * N::STAGE;
    const uint32_t ring_a = (uint32_t)__cvta_generic_to_shared(ring);
    int lch, lend, lkeys, lseq, lhead, pages = -1, pbase;
    bool lmore;
    auto look_ahead = [&]() {
        const Kv4Item& it = ahead[warp];
        lch = it.chunk0; lend = it.chunk0 + it.take; lkeys = it.keys; lseq = it.seq; lhead = it.head;
        lmore = it.next < u_end;
        pbase = lch - 16;
    };
    look_ahead();
    // 16 rows are contiguous: lane's piece of them, and its place; lane (which, group, piece) of the scales
    constexpr int PIECES = N::ROW / 16, PER = 32 / PIECES, PP = es * 2;              // pieces of a row, rows a warp-wide copy covers, pieces of 16 keys' scales
    const uint32_t put = N::piece(lane / PIECES, lane % PIECES);
    const int pwhich = lane / (2 * PP), pgrp = lane / PP & 1, pc = lane % PP;
    const uint32_t pput = (pwhich ? N::VP_AT : N::P_AT) + pgrp * 32 * es + 16 * pc;
    auto load_next = [&](int i) {
        if (lch >= lend && lmore) {
            __syncwarp();
            if (lane == 0) advance_item<RT, CHUNK, LEAD>(&w, p.group, &ahead[warp], u_end);
            __syncwarp();
            look_ahead();
        }
        if (lch < lend) {
            if (lch >= pbase + 16) {                                                 // page ids of sixteen units: lane 2 u + h has unit pbase + u, keys 16 h on
                const int key = (lch + (lane >> 1)) * CHUNK + warp * WKEYS + 16 * (lane & 1);
                pbase = lch;
                pages = lch + (lane >> 1) < lend && key < lkeys ? __ldg(w.table + (size_t)lseq * w.max_pages + (key >> w.shift)) : -1;
                if ((unsigned)pages >= (unsigned)w.n_pages) {
                    if (lch + (lane >> 1) < lend && key < lkeys) atomicCAS(w.input_status, DEV_OK, DEV_KV4_PAGE);
                    pages = -1;                                                      // such keys are not visible
                }
            }
            const int pg[2] = {__shfl_sync(0xffffffffu, pages, 2 * (lch - pbase)), __shfl_sync(0xffffffffu, pages, 2 * (lch - pbase) + 1)};
            const int r0 = (lch * CHUNK + warp * WKEYS) & (R - 1);
            const uint32_t st = ring_a + (uint32_t)(i % N::STAGES) * N::STAGE;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t* src = p.pool + kv4_block_at(w, pg[h] < 0 ? 0 : pg[h], lhead) + (((r0 + 16 * h) & (R - 1)) * N::ROW + 16 * lane);
#pragma unroll
                for (int which = 0; which < 2; ++which)
#pragma unroll
                    for (int j = 0; j < 16 / PER; ++j)
                        cp16(st + (which ? N::V_AT : 0) + h * 16 * N::ROW + j * 512 + put, src + which * R * N::ROW + j * 512, pg[h] >= 0);
            }
            if (lane < 4 * PP) {
                const int page = pgrp ? pg[1] : pg[0];
                cp16(st + pput, p.pool + kv4_block_at(w, page < 0 ? 0 : page, lhead) + kv4_param_at(R, D, es, pwhich, (r0 + 16 * pgrp) & (R - 1)) + 16 * pc, page >= 0);
            }
            if (lane == 0) *reinterpret_cast<int*>(ring + (i % N::STAGES) * N::STAGE + N::FLAG_AT) = (pg[0] >= 0 ? 1 : 0) | (pg[1] >= 0 ? 2 : 0);
            ++lch;
        }
        cp_commit();
    };
#pragma unroll 1
    for (int i = 0; i < N::STAGES - 1; ++i) load_next(i);

    const int ka = key_of(g);                                           // operand rows g and g + 8 of a block of 16 are its keys ka and ka + 8
    const uint32_t kat = D == 128 ? N::piece(ka, t) : ka * 32 + 8 * t;
    uint32_t vat[2];                                                    // of keys 2 t and 2 t + 1 in operand order; + 8 rows for the other two
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int r = key_of(2 * t + e);
        vat[e] = N::V_AT + (D == 128 ? N::piece(r, g >> 1) + 8 * (g & 1) : r * 32 + 4 * g);
    }
    int i = 0;                                                          // unit of this CTA
#pragma unroll 1
    for (;;) {
        const Kv4Item it = cur;
        if (it.take == 0) break;                                        // (the run ends before the item's first chunk)
        const int rows = min(RT, it.q.n * p.group - it.tile * RT);      // query rows of this tile

        // ---- queries: lane (g, t) holds row 8 nt + g, channels [t D/4, (t + 1) D/4), pairs in the order the codes come in
        uint32_t bq[NT][KS][TERMS][2];
        float qs[NT][2];                                                // sums of the queries of rows 8 nt + 2 t, + 1
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int rl = nt * 8 + g, rr = it.tile * RT + rl;
            float x[D / 4];
            load_row<T, D / 4>(rl < rows ? (const T*)p.q + ((size_t)(it.q.row0 + rr / p.group) * p.q_heads + it.head * p.group + rr % p.group) * D + t * (D / 4) : nullptr, x);
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

        // base: what a row's scores are taken against, its reference, or 0 while it has none (its bit of `none`)
        float o[MT][NT][4];
        float base[NT][2], l[NT][2], ms[NT][2];
        uint32_t none = (1u << 2 * NT) - 1u;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { base[nt][e] = 0.f; l[nt][e] = 0.f; ms[nt][e] = 0.f; }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mt][nt][e] = 0.f;
        }

#pragma unroll 1
        for (int ch = it.chunk0; ch < it.chunk0 + it.take; ++ch, ++i) {
            __syncwarp();                                               // everybody has read the stage that is filled next
            load_next(i + N::STAGES - 1);
            cp_wait<N::STAGES - 1>();
            __syncwarp();
            const uint8_t* st = ring + (i % N::STAGES) * N::STAGE;
            const int key0 = ch * CHUNK + warp * WKEYS;
            const int there = *reinterpret_cast<const int*>(st + N::FLAG_AT);
            if (there == 0) continue;
            const bool all = key0 + WKEYS <= it.q.len && there == 3;   // every key is visible to every row

            float s[2][NT][4];                                          // block z: key ka rows 2 t, 2 t + 1, then key ka + 8
#pragma unroll
            for (int z = 0; z < 2; ++z) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[z][nt][e] = 0.f;
                uint32_t k0[KW], k1[KW];
                const uint8_t* kp = st + z * 16 * N::ROW + kat;
                if constexpr (D == 128) {
                    const uint4 x = *reinterpret_cast<const uint4*>(kp), y = *reinterpret_cast<const uint4*>(kp + 8 * N::ROW);
                    k0[0] = x.x; k0[1] = x.y; k0[2] = x.z; k0[3] = x.w;
                    k1[0] = y.x; k1[1] = y.y; k1[2] = y.z; k1[3] = y.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(kp), y = *reinterpret_cast<const uint2*>(kp + 8 * N::ROW);
                    k0[0] = x.x; k0[1] = x.y;
                    k1[0] = y.x; k1[1] = y.y;
                }
#pragma unroll
                for (int j = 0; j < KW; ++j) {
#pragma unroll
                    for (int hlf = 0; hlf < 2; ++hlf) {
                        const uint32_t wa = k0[j] >> (8 * hlf), wb = k1[j] >> (8 * hlf);
                        const uint32_t a0 = O_::template centred<0>(wa, magic), a1 = O_::template centred<0>(wb, magic);
                        const uint32_t a2 = O_::template centred<4>(wa, magic), a3 = O_::template centred<4>(wb, magic);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < TERMS; ++e) O_::mma(s[z][nt], a0, a1, a2, a3, bq[nt][2 * j + hlf][e][0], bq[nt][2 * j + hlf][e][1]);
                    }
                }
            }
            // scores in powers of two, less the base
            float top = -INFINITY, vs[2][2], lv[2][2] = {};              // V's scales of keys (z, h), and what they add to a product
            auto product = [&](int z, int h, float v) { return HALF ? v + lv[z][h] : v; };
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    vs[z][h] = param_of<T>(st + N::VP_AT, 16 * z + ka + 8 * h).x;
                    lv[z][h] = HALF ? scale_bits(vs[z][h]) : 0.f;
                    const float2 kp = param_of<T>(st + N::P_AT, 16 * z + ka + 8 * h);
                    // km - km: 0, or NaN for a minimum that the rotation took to -inf (the key reads as -inf throughout, and a product of
                    // that with a query is no number; -inf times the queries' sum would drop the key, or not, by the sum's sign)
                    const float km = fmaf(8.f, kp.x, kp.y) * sl2, ks = fmaf(kp.x, sl2, HALF ? km - km : 0.f);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float& v = s[z][nt][2 * h + e];
                            v = fmaf(ks, v, fmaf(km, qs[nt][e], -base[nt][e]));
                            top = fmaxf(top, product(z, h, v));
                        }
                }
            bool over = none != 0u || top > RAISE;                      // (a row's first keys may have had no page)
            uint32_t vis = 0xffffffffu;                                 // bit 8 nt + 4 z + e: score s[z][nt][e] counts
            if (__builtin_expect(!all, 0)) {
                // a lane looks up the warp's 32 keys for one of the tile's rows; the others get the word by shuffle
                uint32_t word = sees(p, it.q, (it.tile * RT + min(lane, RT - 1)) / p.group, key0 - it.q.len);
                word &= (there & 1 ? 0x0000ffffu : 0u) | (there & 2 ? 0xffff0000u : 0u);
                vis = 0u;
                over = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t b = __shfl_sync(0xffffffffu, word, 8 * nt + 2 * t + e) >> ka;
#pragma unroll
                        for (int z = 0; z < 2; ++z)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float& v = s[z][nt][2 * h + e];
                                if ((b >> (16 * z + 8 * h)) & 1u) vis |= 1u << (8 * nt + 4 * z + 2 * h + e);
                                else v = -INFINITY;
                                over = over || product(z, h, v) > ((none >> (2 * nt + e)) & 1u ? -INFINITY : RAISE);
                            }
                    }
            }
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float up = fmaxf(fmaxf(product(0, 0, s[0][nt][e]), product(0, 1, s[0][nt][e + 2])), fmaxf(product(1, 0, s[1][nt][e]), product(1, 1, s[1][nt][e + 2])));
                        up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, 4));
                        up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, 8));
                        up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, 16));
                        up -= TOP;
                        const bool had = !((none >> (2 * nt + e)) & 1u);
                        if (up > (had ? 0.f : -INFINITY)) {             // the new reference is `up` above the base
                            const float f = had ? ex2(-up) : 0.f;
                            none &= ~(1u << (2 * nt + e));
                            base[nt][e] += up;
                            l[nt][e] *= f;
                            ms[nt][e] *= f;
#pragma unroll
                            for (int z = 0; z < 2; ++z) { s[z][nt][e] -= up; s[z][nt][e + 2] -= up; }
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) { o[mt][nt][e] *= f; o[mt][nt][e + 2] *= f; }
                        }
                    }
            }
            uint32_t bp[2][NT][TERMS][2];
            auto weights = [&](auto plain) {                            // (the common case in one run of instructions)
                constexpr bool PLAIN = decltype(plain)::value;
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const float2 vp0 = param_of<T>(st + N::VP_AT, 16 * z + ka), vp1 = param_of<T>(st + N::VP_AT, 16 * z + ka + 8);
                    const float vm0 = fmaf(8.f, vp0.x, vp0.y), vm1 = fmaf(8.f, vp1.x, vp1.y);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float ps[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float pe = ex2(s[z][nt][e]);
                            l[nt][e & 1] += pe;
                            ps[e] = pe * vs[z][e >> 1];
                            if (PLAIN || ((vis >> (8 * nt + 4 * z + e)) & 1u)) ms[nt][e & 1] = fmaf(pe, e < 2 ? vm0 : vm1, ms[nt][e & 1]);
                            else ps[e] = 0.f;                           // by selection: what a key holds stays out of rows that do not see it
                        }
                        uint32_t x[TERMS], y[TERMS];
                        O_::split(ps[0], ps[1], x);
                        O_::split(ps[2], ps[3], y);
#pragma unroll
                        for (int e = 0; e < TERMS; ++e) { bp[z][nt][e][0] = transpose8x8(x[e]); bp[z][nt][e][1] = transpose8x8(y[e]); }
                    }
                }
            };
            if (__builtin_expect(all, 1)) weights(std::true_type{});
            else weights(std::false_type{});
            // O^T: m-tile mt holds the lane's channels 2 mt (operand row g) and 2 mt + 1 (row g + 8) of the D/8 from g D/8 on
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                uint32_t v[4][VW];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint8_t* vp = st + z * 16 * N::ROW + vat[e & 1] + (e >> 1) * 8 * N::ROW;
                    if constexpr (D == 128) {
                        const uint2 x = *reinterpret_cast<const uint2*>(vp);
                        v[e][0] = x.x; v[e][1] = x.y;
                    } else {
                        v[e][0] = *reinterpret_cast<const uint32_t*>(vp);
                    }
                }
#pragma unroll
                for (int j = 0; j < VW; ++j)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {                       // half words of the two keys of a pair side by side
                        const uint32_t a = __byte_perm(v[0][j], v[1][j], y ? 0x7632 : 0x5410), b = __byte_perm(v[2][j], v[3][j], y ? 0x7632 : 0x5410);
#pragma unroll
                        for (int hlf = 0; hlf < 2; ++hlf) {
                            const uint32_t as = a >> (8 * hlf), bs = b >> (8 * hlf);
                            const uint32_t a0 = O_::template centred<0>(as, magic), a1 = O_::template centred<4>(as, magic);
                            const uint32_t a2 = O_::template centred<0>(bs, magic), a3 = O_::template centred<4>(bs, magic);
                            const int mt = 4 * j + 2 * y + hlf;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int e = 0; e < TERMS; ++e) O_::mma(o[mt][nt], a0, a1, a2, a3, bp[z][nt][e][0], bp[z][nt][e][1]);
                        }
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
                if (rl >= rows) continue;
                if (g == 0) { xm[warp * RT + rl] = (none >> (2 * nt + e)) & 1u ? -INFINITY : base[nt][e]; xl[warp * RT + rl] = a; xs[warp * RT + rl] = b; }
#pragma unroll
                for (int mt = 0; mt < MT; mt += 2)
                    *reinterpret_cast<float4*>(xo + (warp * RT + rl) * XO + g * (D / 8) + 2 * mt) = make_float4(o[mt][nt][e], o[mt][nt][e + 2], o[mt + 1][nt][e], o[mt + 1][nt][e + 2]);
            }
        __syncthreads();
        const int64_t c0 = kv4_cta_of(it.first, per), c1 = kv4_cta_of(it.first + it.chunks - 1, per);      // CTAs that share the item
        const bool whole = c0 == c1;
        float* slot = p.part + ((size_t)blockIdx.x * 2 + ((int64_t)blockIdx.x == c0 ? 1 : 0)) * N::SLOT;
#pragma unroll 1
        for (int x = threadIdx.x; x < rows * (D / 4); x += WARPS * 32) {
            const int rl = x / (D / 4), c = 4 * (x % (D / 4));
            float m = xm[rl];
#pragma unroll
            for (int k = 1; k < WARPS; ++k) m = fmaxf(m, xm[k * RT + rl]);
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
            float lsum = 0.f;
#pragma unroll
            for (int k = 0; k < WARPS; ++k) {
                const int at = k * RT + rl;
                const float f = xm[at] == -INFINITY && xl[at] == 0.f ? 0.f : ex2(xm[at] - m), mm = xs[at];      // (saw nothing: 0; a NaN goes on)
                const float4 b = *reinterpret_cast<const float4*>(xo + at * XO + c);
                a.x += f * (b.x + mm); a.y += f * (b.y + mm); a.z += f * (b.z + mm); a.w += f * (b.w + mm);
                lsum += f * xl[at];
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
            __syncthreads();
            if (threadIdx.x == 0) {
                const int want = (int)(c1 - c0), old = arrive_at(p.counters + c0);
                if (old == want) p.counters[c0] = 0;                     // everybody has arrived: ready for the next launch
                arrived = old == want;
            }
            __syncthreads();
            if (arrived) merge_item<T, D, 1>(p, it, RT, rows, c0, c1, warp, WARPS, xmerge, [] { __syncthreads(); });
        }
        if (it.next >= u_end) break;
        __syncthreads();                                                 // everybody has the item, and the exchange buffers are written again
        if (threadIdx.x == 0) advance_item<RT, CHUNK, LEAD>(&w, p.group, &cur, u_end);
        __syncthreads();
    }
    cp_wait<0>();
}

template <typename T, int D, int NT>
ghd_status launch_narrow(ghd_ctx* c, Kv4AttnParams& p) {
    using N = Narrow<T, D, NT>;
    constexpr int FIXED = (N::SMEM + 15) & ~15, VARIANT = (sizeof(T) == 2 ? 0 : 4) + (D == 64 ? 0 : 2) + NT - 1;
    const int smem = FIXED + (p.w.n_seqs + 1) * 8;
    if (!(c->attr_kv4 >> VARIANT & 1)) {                                 // once a context, for as many sequences as a call takes
        if (cudaFuncSetAttribute(k_attn_kv4<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, FIXED + (GHD_MAX_SEQS + 1) * 8) != cudaSuccess) {
            cudaGetLastError();
            return fail(c, GHD_ECUDA, "kv4_attention: cannot raise dynamic shared memory");
        }
        c->attr_kv4 |= 1u << VARIANT;
    }
    p.ctas = c->sm_count * N::BLOCKS;
    const size_t have = (size_t)c->sm_count * 2 * 256 * 128;             // floats of the tile scratch (carve_workspace)
    if ((size_t)p.ctas * 2 * N::SLOT > have || p.ctas > 4096) return fail(c, GHD_ENOSPACE, "kv4_attention: workspace too small");
    c->path_count[GHD_PATH_KV4_ROWS]++;
    launch_k(c, false, k_attn_kv4<T, D, NT>, dim3(p.ctas), dim3(WARPS * 32), smem, p);
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
    if (m.dtype == GHD_F32) {
        if (c->opt_attn_path == 2) return fail(c, GHD_EUNSUPPORTED, "kv4_attention: the tcgen05 kernel takes GHD_F16 only");
        // Two tiles of eight rows at a time unpack a key half as often and leave half as many items to deal: with more than 128 rows, or
        // more than 64 and tiles for two SMs of three.  1 and 5 sequences over 512 and 4096 keys, ones / twos in us: 28 heads on 4 of 128,
        // 112 rows 16 / 18, 26 / 30, 24 / 25, 59 / 53; up to 252 rows 24 / 23, 46 / 41, 36 / 32, 86 / 76; 32 heads, 80 rows 27 / 27, 81 / 72,
        // 55 / 53, 179 / 154; 8 heads of 64, 48 rows 12 / 13, 17 / 20, 17 / 17, 32 / 29.  Over 280 such calls (9 to 640 rows) 1 % above the
        // better of the two on average, 44 % at worst (65 rows of 32 heads over 512 keys: 18.5 / 26.7).
        const int64_t tiles = (avg + 15) / 16 * w.heads * w.n_seqs;
        if (avg > 128 || (avg > 64 && 3 * tiles > 2 * (int64_t)c->sm_count)) return m.d_head == 64 ? launch_narrow<float, 64, 2>(c, p) : launch_narrow<float, 128, 2>(c, p);
        return m.d_head == 64 ? launch_narrow<float, 64, 1>(c, p) : launch_narrow<float, 128, 1>(c, p);
    }
    // The tcgen05 kernel for tiles of many rows.  Up to 32 rows two tiles of this file's kernel start sooner and cost a key as much (8
    // sequences, 32 heads, 32 rows over 0 / 512 / 2048 / 8192 keys: 18 / 28 / 54 / 97 us here, 20 / 31 / 54 / 104 there).  Up to 64 rows
    // they do while its tiles leave half of the SMs free (32 tiles over 256 / 2048 keys: 15 / 18 us here, 18 / 25 there; but 128 tiles over
    // 1024 / 4096: 23 / 38 here, 22 / 33 there).  128 rows, 32 heads over 512 / 1024 / 2048 keys: 26 / 32 / 43 here, 24 / 27 / 34 there.
    // The rows of a sequence are known on the device alone, so all rules go by the average, rows behind the last sequence included.  Where
    // sequences are unlike, one call takes longer than one for each kind (32 heads on 8: a tree of 256 nodes beside 63 tokens over up to
    // 4096 rows 190 us, apart 74 + 56; a prompt of 2048 rows beside 31 tokens 353, apart 260 + 32).
    const int64_t tiles = (avg + 15) / 16 * w.heads * w.n_seqs;
    if (c->opt_attn_path == 2 || (c->opt_attn_path == 0 && avg > 32 && (avg > 64 || 2 * tiles > c->sm_count))) return launch_attn_kv4_tc(c, p);
    if (m.d_head == 64) return avg <= 8 ? launch_narrow<__half, 64, 1>(c, p) : launch_narrow<__half, 64, 2>(c, p);
    return avg <= 8 ? launch_narrow<__half, 128, 1>(c, p) : launch_narrow<__half, 128, 2>(c, p);
}

}  // namespace ghd
