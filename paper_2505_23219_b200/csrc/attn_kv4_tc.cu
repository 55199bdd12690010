// Attention over the paged 4-bit cache for tiles of many query rows (trees, groups of heads): tcgen05 on sm_100a.
//
// As in attn_kv4.cu the scales stay out of the products and keys are the M side: S^T [128 keys x rows] = K Q^T,
// O^T [d_head x rows] = V^T P^T.  With keys on the tensor-memory lanes a thread owns whole key rows:
//   K        four warps: one thread per key unpacks its 4-bit row in registers and stores it to tensor memory, from where
//            the first product takes its A operand - the unpacked keys never touch shared memory;
//   V        four warps unpack V rows into a swizzled shared-memory tile (A operand of the second product, M-major);
//   softmax  warps read S^T in the 16x256b fragment form: a thread holds 4 keys x 8 query rows, so a key's
//            scales and minima are a few registers and a row's running sums one each; weights times V's scale go to
//            shared memory by stmatrix as the B operand of the second product;
//   one warp each issues the first and the second product, and works out the CTA's items ahead of
//            everybody.
// O^T stays in tensor memory over all keys of an item.  Nibbles come out of a word in the order 0 4 1 5 2 6 3 7; the
// queries are stored in that order, and the output's lanes are read back through it.
//
// Half range: as in attn_kv4.cu a row's reference goes by score + log2(V's scale) of the keys that it sees, so that the operand (11 bits)
// stays below 2^15; it is raised when that passes 2^15 of it, and then lies 2^7 below the largest.  Raising rescales O^T in place
// (rare after the first unit); the 128 threads that share query rows agree on it by one barrier a unit.
//
// Work is dealt as in attn_kv4.cu, one CTA an SM.
//
// What it costs.  8 ragged trees of up to 64 nodes over up to 8192 rows, 32 heads (148 MB, 30 GFLOP): 122 us; one tree of 256 nodes over
// 4096 rows, 40 heads (22 GFLOP): 83 us.  A unit of 128 keys x 64 rows takes about 2700 clocks where its products take 900 and its
// exponentials 500: the softmax warps' chain (in clocks: scores 550, agreement on references 270, fetch of the next scores 700, wait
// for a P buffer 350 though it is free, weights 900, hand-over 250), at 2 instructions an SM a clock; K and V are two units ahead.  A unit
// with masked keys costs 2000 more, raising references 1700.  An item costs about 9000 besides (queries 3000, sums 900, sums out
// 2500, arrival and merge 2400 where it is split), a launch 11000 before the first scores.  Measured and dropped: 16 softmax warps on
// one unit, two groups of eight on units in turn (142 us against 132: 88 registers a thread spill), tiles of 128 rows.
#include <cstddef>
#include <cstdio>
#include <type_traits>

#include "attn_kv4_dev.cuh"
#include "tc_common.cuh"

namespace ghd {

namespace {

using namespace tc;
using namespace kv4;

constexpr int UNIT = 128;                      // keys of a unit (MMA M of S^T, MMA K of O^T)
constexpr int N = 64;                          // query rows of a tile; tiles of 128 rows unpack each key half as often and measured slower
                                               // (256 nodes, 13B shape, 4096 rows: 108 us against 90): their code does not fit the cache
constexpr int SOFT = 256, CONV = 256;          // threads of the softmax and of the unpacking warps
constexpr int PARTS = SOFT / 128;              // 128 threads (one a key of four) share query rows, as pairs of blocks of eight: pair part, part + PARTS, ...
constexpr int THREADS = SOFT + CONV + 128, SW = SOFT / 32, CW = SW + CONV / 32;      // first unpacking warp, first of the others
static_assert(N / 8 / PARTS == 4, "a lane of eight ends up with one of 4 + 4 blocks' sums");
// registers a thread after the split by warpgroups, within those launched with
constexpr int REGS_LAUNCH = 96, REGS_SOFT = 152, REGS_CONV = 56, REGS_ISSUE = 56;
static_assert(SOFT * REGS_SOFT + CONV * REGS_CONV + 128 * REGS_ISSUE <= THREADS * REGS_LAUNCH && THREADS * REGS_LAUNCH <= 65536, "register split");
constexpr float RAISE = 15.f, TOP = 7.f;       // where a reference is raised, and what lies above a new one
constexpr int LEAD = 4;                        // an item's fixed cost in units (8 ragged trees: 3: 124 us, 4: 120, 5: 120, 6: 122; one of 64 nodes over 512 rows: 20.5, 20.5, 21.9, 22.0)
// What the softmax warps need of a unit's keys is ready when its keys are.  The K warps are two units ahead of the first
// product, that is two ahead of the scores being fetched, and those one ahead of what the softmax warps work on: five in use.
constexpr int PAR_SLOTS = 8;
// The copies are asked for three units ahead of the unpacking.
constexpr int GROUP_SLOTS = 16;
constexpr uint32_t V_SLAB = UNIT * 128;        // [128 keys x 64 channels] half

template <int D>
struct Shape {
    static constexpr int STAGES = 4, SLABS = D / 64;
    static constexpr uint32_t Q_BYTES = SLABS * N * 128, V_BYTES = SLABS * V_SLAB, P_BYTES = UNIT * 128;
    static constexpr uint32_t ST_BYTES = UNIT * (D + 8);                 // codes of a unit, D / 2 bytes a row, K then V; then K's and V's (scale, min)
    static constexpr uint32_t V_AT = Q_BYTES, P_AT = V_AT + 2 * V_BYTES, ST_AT = P_AT + 2 * P_BYTES, CTRL_AT = ST_AT + STAGES * ST_BYTES;
    static constexpr uint32_t T_K = 0, T_S = 2 * (D / 2), T_O = T_S + 2 * N;      // tensor-memory columns
    static_assert(T_O + N <= 512, "tensor memory");
};

constexpr int ITEMS = 4;                       // items that the scheduler is ahead, at most

struct Ctrl {
    uint64_t item_full[ITEMS], item_empty[ITEMS];
    Kv4Item item[ITEMS], cur[3];     // cur: the softmax warps' items: the one being finished, the next, and a slot for who is behind
    uint64_t c_full[CONV / 32][4];   // packed rows of a unit, by unpacking warp and stage
    uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], s_empty[2], p_full[2], p_empty[2], drain, drain_pv;
    uint32_t tmem_base;
    uint32_t looks;                  // how often a wait looks before it gives up
    int arrived;
    alignas(16) float qs[N];       // sums of the tile's queries
    alignas(16) float fac[N];      // factors of a rescale, by row
    float4 tot[N];                   // a row's sum of weights, its inverse, sum of weighted middles
    alignas(16) float x[4][N], y[4][N];      // exchange between the four warps that share rows
    float4 par[PAR_SLOTS][UNIT];     // by unit and key: K's scale and middle (min + 8 scale) times log2(e) / sqrt(d_head), V's scale and middle
    alignas(4) uint8_t groups[GROUP_SLOTS][4];      // which of a quarter's two groups of 16 keys have a page, by unit
    alignas(16) int rowix[2][N];               // row of q and out, in d_head elements, of the query rows of an item and the next
    int64_t scratch[32];
    int64_t sums[1];                 // [n_seqs + 1]
};
template <int D> constexpr uint32_t smem_bytes(int n_seqs) { return Shape<D>::CTRL_AT + (uint32_t)sizeof(Ctrl) + 8 * (uint32_t)n_seqs + 1024; }
static_assert(offsetof(Ctrl, qs) % 16 == 0 && offsetof(Ctrl, fac) % 16 == 0 && offsetof(Ctrl, par) % 16 == 0, "rows are read in pairs");
static_assert(smem_bytes<128>(GHD_MAX_SEQS) <= 227 * 1024, "shared memory");

__device__ __forceinline__ void ld_frag(uint32_t taddr, uint32_t (&r)[4]) {      // 16 lanes x 8 columns, as an mma accumulator
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ld_cols8(uint32_t taddr, uint32_t (&r)[8]) {     // 32 lanes x 8 columns, a lane a thread
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ld_frag2(uint32_t taddr, uint32_t (&a)[4], uint32_t (&b)[4]) {      // ... x 16 columns
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]), "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                   "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void st_frag(uint32_t taddr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x1.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void stmatrix4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, const uint32_t* r) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// mbar_wait in few instructions: what this kernel executes over and over has to fit the instruction cache.  A wait takes at
// most *left looks (2^22, about a second); one that runs out sets it to 1, so that all later ones are short.  NAP:
// nanoseconds between two looks, for warps that are ahead of what they wait for.
constexpr uint32_t LOOKS = 1u << 22;
template <int NAP = 0>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile uint32_t* left, int* status, int code) {
    uint32_t ok, n = *left;
    if (NAP > 0)
        asm volatile("{\n\t.reg .pred p, q;\n\tWAIT_%=:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%2], %3;\n\t@p bra DONE_%=;\n\tnanosleep.u32 %4;\n\t"
                     "sub.u32 %1, %1, 1;\n\tsetp.ne.u32 q, %1, 0;\n\t@q bra WAIT_%=;\n\tDONE_%=:\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok), "+r"(n) : "r"(bar), "r"(parity), "n"(NAP) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\tWAIT_%=:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%2], %3;\n\t@p bra DONE_%=;\n\t"
                     "sub.u32 %1, %1, 1;\n\tsetp.ne.u32 q, %1, 0;\n\t@q bra WAIT_%=;\n\tDONE_%=:\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok), "+r"(n) : "r"(bar), "r"(parity) : "memory");
    if (__builtin_expect(!ok, 0)) {
        *left = 1;
        atomicCAS(status, DEV_OK, code);
    }
    return ok != 0;
}
__device__ __forceinline__ void wait_drain(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t spin = 0; spin < LOOKS && !mbar_try(bar, parity); ++spin) __nanosleep(64);
}
// One arrival for the whole warp: arrivals on one barrier are taken one by one, five cycles each.
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
template <int ID, int NT> __device__ __forceinline__ void named_sync() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(NT) : "memory"); }
__device__ __forceinline__ void part_sync(int part) { asm volatile("bar.sync %0, 128;" ::"r"(2 + part) : "memory"); }
__device__ __forceinline__ bool part_any(int part, bool v) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(v ? 1u : 0u), "r"(2 + part) : "memory");
    return r != 0;
}
// untiled copy to shared memory, counted on an mbarrier
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// two 32-bit products and sums in one instruction
__device__ __forceinline__ uint64_t bits2(float2 a) { return (uint64_t)__float_as_uint(a.x) | (uint64_t)__float_as_uint(a.y) << 32; }
__device__ __forceinline__ float2 pair2(uint64_t a) { return make_float2(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32))); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
    return pair2(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
    return pair2(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
    return pair2(r);
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// eight codes -> four packed pairs, nibbles in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t* r, const HalfMagic& m) {
    const uint32_t x = w >> 8;
    r[0] = centred_half<0>(w, m);
    r[1] = centred_half<4>(w, m);
    r[2] = centred_half<0>(x, m);
    r[3] = centred_half<4>(x, m);
}
template <int D>
__global__ void __launch_bounds__(THREADS, 1) k_attn_kv4_tc(const __grid_constant__ Kv4AttnParams p) {
    using SH = Shape<D>;
    constexpr int NB = N / 8 / PARTS;                // blocks of eight query rows of a softmax thread
    constexpr int PIECES = D / 32;                   // 16-byte pieces of a packed row
    constexpr uint32_t ROW = D / 2;                  // bytes of a packed row
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw), pad = (1024u - (raw_addr & 1023u)) & 1023u;
    uint8_t* base = smem_raw + pad;
    const uint32_t base_a = smem_u32(base);
    Ctrl* sm = reinterpret_cast<Ctrl*>(base + SH::CTRL_AT);
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // (the compiler sees that a warp has one number)

    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&sm->q_full), SOFT / 32);
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sm->k_full[b]), CONV / 64); mbar_init(smem_u32(&sm->k_empty[b]), 1);
            mbar_init(smem_u32(&sm->v_full[b]), CONV / 64); mbar_init(smem_u32(&sm->v_empty[b]), 1);
            mbar_init(smem_u32(&sm->s_full[b]), 1); mbar_init(smem_u32(&sm->s_empty[b]), SOFT / 32);
            mbar_init(smem_u32(&sm->p_full[b]), SOFT / 32); mbar_init(smem_u32(&sm->p_empty[b]), 1);
        }
        mbar_init(smem_u32(&sm->drain), 1);
        mbar_init(smem_u32(&sm->drain_pv), 1);
        for (int b = 0; b < 4 * (CONV / 32); ++b) mbar_init(smem_u32(&sm->c_full[b >> 2][b & 3]), 1);
        for (int b = 0; b < ITEMS; ++b) { mbar_init(smem_u32(&sm->item_full[b]), 1); mbar_init(smem_u32(&sm->item_empty[b]), CONV / 32 + 3); }      // unpacking warps, softmax, both issuers
        sm->looks = LOOKS;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == CW) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm->tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const Kv4View& w = p.w;
    const Kv4Tiling til{w.heads, p.group, N, UNIT, LEAD};
    tc_fence_before();
    const int64_t units = unit_sums(w, til, sm->sums, sm->scratch);      // two block barriers inside
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;
    volatile uint32_t* looks = &sm->looks;
    const int64_t per = kv4_units_per_cta(units, p.ctas);
    const int64_t u_beg = per * blockIdx.x, u_end = u_beg + per < units ? u_beg + per : units;
    // The k-th item of this CTA (take = 0: there are no more, or a wait has run out).  One thread looks; who takes it together
    // with others gets it from that thread, so that all of them go on or stop alike.
    auto item_get = [&](int k) -> Kv4Item {
        if (!wait<20>(smem_u32(&sm->item_full[k % ITEMS]), (k / ITEMS) & 1, looks, w.status, DEV_TIMEOUT_EPI)) { Kv4Item none{}; return none; }
        const Kv4Item it = sm->item[k % ITEMS];
        mbar_arrive(smem_u32(&sm->item_empty[k % ITEMS]));
        return it;
    };
    auto rows_of = [&](const Kv4Item& it) { const int r = it.q.n * p.group - it.tile * N; return r < N ? r : N; };
    auto cols_of = [&](int rows) { return (rows + 15) & ~15; };           // MMA N: a multiple of 16

    if (warp >= SW && warp < CW) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_CONV));
        const int quad = warp & 3;                                        // this warp's 32 keys of a unit
        const float sl2 = p.scale * KV4_LOG2E;
        const HalfMagic magic;
        // Every warp asks for its own rows by bulk copies into a ring of its own, STAGES - 1 units ahead and over the borders of
        // items: K's or V's codes (which), and the K warps the scales and minima of both.
        const int which = warp < SW + 4 ? 0 : 1, own = warp - SW, R = 1 << w.shift;
        const uint32_t ring = base_a + SH::ST_AT + which * UNIT * ROW + quad * 32 * ROW, pring = base_a + SH::ST_AT + 2 * UNIT * ROW + quad * 32 * 4;
        int items = 0, lseq = 0, lhead = 0, lch = 0, lend = 0, lkeys = 0, n = 0;      // load cursor; units asked for so far
        bool more = true;
        // page ids of the next sixteen units' two groups of 16 keys: lane 2 u + h has unit pbase + u
        int pages = -1, pbase = 0;
        auto look = [&]() {
            const int key = (lch + (lane >> 1)) * UNIT + quad * 32 + 16 * (lane & 1);
            pbase = lch;
            pages = lch + (lane >> 1) < lend && key < lkeys ? __ldg(w.table + (size_t)lseq * w.max_pages + (key >> w.shift)) : -1;
        };
        auto ask = [&]() {
            if (lch >= lend && more) {
                if (lane == 0) {
                    const Kv4Item it = item_get(items);
                    lseq = it.seq; lhead = it.head; lch = it.chunk0; lend = it.chunk0 + it.take; lkeys = it.keys;
                }
                ++items;
                lseq = __shfl_sync(0xffffffffu, lseq, 0);
                lhead = __shfl_sync(0xffffffffu, lhead, 0);
                lch = __shfl_sync(0xffffffffu, lch, 0);
                lend = __shfl_sync(0xffffffffu, lend, 0);
                lkeys = __shfl_sync(0xffffffffu, lkeys, 0);
                more = lend > lch;
                look();
            }
            if (lch >= lend) return;
            if (lch >= pbase + 16) look();
            const int page[2] = {__shfl_sync(0xffffffffu, pages, 2 * (lch - pbase)), __shfl_sync(0xffffffffu, pages, 2 * (lch - pbase) + 1)};
            if (lane == 0) {
                const int key0 = lch * UNIT + quad * 32, s_ = n % SH::STAGES;
                const uint32_t full = smem_u32(&sm->c_full[own][s_]);
                uint32_t there = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if ((unsigned)page[h] < (unsigned)w.n_pages) there |= 1u << h;
                    else if (key0 + 16 * h < lkeys) atomicCAS(w.input_status, DEV_OK, DEV_KV4_PAGE);
                }
                if (which == 0) sm->groups[n & (GROUP_SLOTS - 1)][quad] = (uint8_t)there;
                if (there) mbar_expect_tx(full, (there == 3u ? 2u : 1u) * 16 * (ROW + (which ? 0 : 8)));
                else mbar_arrive(full);
                const bool one = there == 3u && R >= 32;                  // 32 rows of one page: one copy of each kind
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    if (!((there >> h) & 1u) || (one && h)) continue;
                    const int r = (key0 + 16 * h) & (R - 1), rows = one ? 32 : 16;
                    const uint8_t* blk = p.pool + kv4_block_at(w, page[h], lhead);
                    bulk_load(ring + s_ * SH::ST_BYTES + 16 * h * ROW, blk + kv4_code_at(R, D, which, r), rows * ROW, full);
                    if (which == 0) {
                        bulk_load(pring + s_ * SH::ST_BYTES + 64 * h, blk + kv4_param_at(R, D, 2, 0, r), rows * 4, full);
                        bulk_load(pring + s_ * SH::ST_BYTES + 4 * UNIT + 64 * h, blk + kv4_param_at(R, D, 2, 1, r), rows * 4, full);
                    }
                }
            }
            ++lch;
            ++n;
        };
#pragma unroll 1
        for (int i = 0; i < SH::STAGES - 1; ++i) ask();
        // K: thread = key = tensor-memory lane.  V: a lane takes one 16-byte piece of a row at a time; eight lanes read 128 bytes in
        // a row, and their four stores go to eight different bank groups.
        const int row0 = quad * 32 + lane / PIECES, c = lane % PIECES, turn = D == 128 ? (c >> 1) << 1 : 0;
        constexpr int PER = 32 / PIECES;                                  // rows a step: a multiple of 8, so the swizzle of a lane's rows is one
        const uint32_t from = which == 0 ? ring + lane * ROW : ring + (lane / PIECES) * ROW + 16 * c, step = which == 0 ? 16 : PER * ROW;
        const uint32_t vt0 = base_a + SH::V_AT + (c >> 1) * V_SLAB + row0 * 128;
        uint32_t off[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) off[k] = (((c & 1) * 4 + (k ^ turn)) ^ (row0 & 7)) << 4;
        // what the unpacked rows go to (a tensor-memory block, a V tile), when it is free and when it is full
        const uint32_t empty = which == 0 ? smem_u32(&sm->k_empty[0]) : smem_u32(&sm->v_empty[0]), full = which == 0 ? smem_u32(&sm->k_full[0]) : smem_u32(&sm->v_full[0]);
#pragma unroll 1
        for (int i = 0; i < n; ++i) {                                     // (n runs ahead until the last unit has been asked for)
            const int b = i & 1, s_ = i % SH::STAGES;
            __syncwarp();                                                 // everybody has read the stage that is filled next
            ask();
            wait<40>(smem_u32(&sm->c_full[own][s_]), (i / SH::STAGES) & 1, looks, w.status, DEV_TIMEOUT_TMA);
            if (i >= 2) wait<100>(empty + 8 * b, ((i >> 1) - 1) & 1, looks, w.status, DEV_TIMEOUT_TMEM);
            uint32_t st = from + s_ * SH::ST_BYTES;
            uint4 x = lds128(st);
            if (which == 0) {
                const uint32_t at = pring + s_ * SH::ST_BYTES + 4 * lane;
                uint32_t kr, vr;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(kr) : "r"(at) : "memory");
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(vr) : "r"(at + 4 * UNIT) : "memory");
                const float2 kf = __half22float2(*reinterpret_cast<const __half2*>(&kr)), vf = __half22float2(*reinterpret_cast<const __half2*>(&vr));
                const float km = fmaf(8.f, kf.x, kf.y) * sl2;             // (km - km: NaN for a key of -inf, as in attn_kv4.cu)
                sm->par[i & (PAR_SLOTS - 1)][quad * 32 + lane] = make_float4(fmaf(kf.x, sl2, km - km), km, vf.x, fmaf(8.f, vf.x, vf.y));
            }
            tc_fence_after();
            uint32_t to = which == 0 ? tmem + SH::T_K + b * ROW + ((uint32_t)(quad * 32) << 16) : vt0 + b * SH::V_BYTES;
#pragma unroll 1
            for (int j = 0; j < PIECES; ++j) {
                uint32_t r[16];
                const bool swap = which != 0 && turn != 0;
                unpack8(swap ? x.z : x.x, r, magic); unpack8(swap ? x.w : x.y, r + 4, magic); unpack8(swap ? x.x : x.z, r + 8, magic); unpack8(swap ? x.y : x.w, r + 12, magic);
                st += step;
                if (j + 1 < PIECES) x = lds128(st);
                if (which == 0) {
                    st16(to, r);
                    to += 16;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) sts128(to + off[k], r + 4 * k);
                    to += PER * 128;
                }
            }
            if (which == 0) {
                st_wait();
                tc_fence_before();
            } else {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            warp_arrive(full + 8 * b);
        }
        // no copy is in flight when the block ends, whatever the others have given up
        if (lane == 0)
#pragma unroll 1
            for (int k = n > SH::STAGES ? n - SH::STAGES : 0; k < n; ++k) wait_drain(smem_u32(&sm->c_full[own][k % SH::STAGES]), (k / SH::STAGES) & 1);
    } else if (warp >= CW) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_ISSUE));
        if (warp == CW) {
        // ------------------------------------------------ issuer of S^T = K Q^T
        if (lane == 0) {
            const uint64_t q_desc = smem_desc_sw128(base_a);
            bool ok = true;
            int i = 0, items = 0;
#pragma unroll 1
            while (ok) {
                const Kv4Item it = item_get(items);
                if (it.take == 0) break;
                const uint32_t idesc = instr_desc_f16(cols_of(rows_of(it)), false);
                ok = wait(smem_u32(&sm->q_full), items & 1, looks, w.status, DEV_TIMEOUT_MMA);
                ++items;
#pragma unroll 1
                for (int k = 0; ok && k < it.take; ++k, ++i) {
                    const int b = i & 1;
                    ok = wait<30>(smem_u32(&sm->k_full[b]), (i >> 1) & 1, looks, w.status, DEV_TIMEOUT_MMA);
                    if (ok && i >= 2) ok = wait<30>(smem_u32(&sm->s_empty[b]), ((i >> 1) - 1) & 1, looks, w.status, DEV_TIMEOUT_TMEM);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int ks = 0; ks < D / 16; ++ks)                  // 16 channels: 8 columns of K, 32 bytes along Q's rows
                        mma_ts(tmem + SH::T_S + b * N, tmem + SH::T_K + b * (D / 2) + ks * 8,
                               q_desc + (uint64_t)((((ks >> 2) * N * 128) >> 4) + (ks & 3) * 2), idesc, ks > 0 ? 1u : 0u);
                    tc_commit(smem_u32(&sm->s_full[b]));
                    tc_commit(smem_u32(&sm->k_empty[b]));
                }
            }
            if (!ok) {
                tc_commit(smem_u32(&sm->drain));
                wait_drain(smem_u32(&sm->drain), 0);
            }
        }
        } else if (warp == CW + 1) {
        // ------------------------------------------------ issuer of O^T += V^T P^T
        if (lane == 0) {
            // both operands have the MMA's K dimension (keys) as rows of 128 bytes: 64 channels of V, 64 query rows of P
            const uint64_t v_desc = smem_desc_sw128(base_a + SH::V_AT, D == 128 ? V_SLAB : 0);   // d_head 64: channels 64 .. 127 repeat 0 .. 63
            const uint64_t p_desc = smem_desc_sw128(base_a + SH::P_AT, UNIT * 128);
            bool ok = true;
            int i = 0, items = 0;
#pragma unroll 1
            while (ok) {
                const Kv4Item it = item_get(items++);
                if (it.take == 0) break;
                const uint32_t idesc = instr_desc_f16(cols_of(rows_of(it)), true) | (1u << 15);
#pragma unroll 1
                for (int k = 0; ok && k < it.take; ++k, ++i) {
                    const int b = i & 1;
                    ok = wait<30>(smem_u32(&sm->v_full[b]), (i >> 1) & 1, looks, w.status, DEV_TIMEOUT_MMA);
                    if (ok) ok = wait<30>(smem_u32(&sm->p_full[b]), (i >> 1) & 1, looks, w.status, DEV_TIMEOUT_MMA);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int ks = 0; ks < UNIT / 16; ++ks)               // 16 keys: 16 rows of both tiles
                        tc_mma_f16(tmem + SH::T_O, v_desc + (uint64_t)((b * SH::V_BYTES + ks * 2048) >> 4), p_desc + (uint64_t)((b * SH::P_BYTES + ks * 2048) >> 4),
                                   idesc, (k > 0 || ks > 0) ? 1u : 0u);
                    tc_commit(smem_u32(&sm->v_empty[b]));
                    tc_commit(smem_u32(&sm->p_empty[b]));
                }
            }
            if (!ok) {
                tc_commit(smem_u32(&sm->drain_pv));
                wait_drain(smem_u32(&sm->drain_pv), 0);
            }
        }
        } else if (warp == CW + 2) {
        // ------------------------------------------------ scheduler
        if (lane == 0) {
            int k = 0;
            bool ok = true;
#pragma unroll 1
            for (Kv4Item it{}; ok;) {
                const auto seq_of = [&](int s_) { return kv4_load_seq(w, s_); };
                if (k == 0 && u_beg < u_end) it = kv4_find_item(til, sm->sums, w.n_seqs, seq_of, u_beg, u_end);
                else if (k > 0 && it.next < u_end) kv4_next_item(til, seq_of, it, u_end);
                else it.take = 0;
                if (it.take > 0) it.keys = kv4_tile_keys(til, it.q, it.tile);
                if (k >= ITEMS) ok = wait<500>(smem_u32(&sm->item_empty[k % ITEMS]), ((k / ITEMS) - 1) & 1, looks, w.status, DEV_TIMEOUT_EPI);
                sm->item[k % ITEMS] = it;
                mbar_arrive(smem_u32(&sm->item_full[k % ITEMS]));
                ++k;
                if (it.take == 0) break;
            }
        }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFT));
        // ------------------------------------------------ softmax warps
        // part: which pairs of blocks of eight query rows (part, part + PARTS, ...); quad: which 32 keys (tensor-memory lanes)
        const int part = warp >> 2, quad = warp & 3, g = lane >> 2, t = lane & 3, tid = threadIdx.x;
        auto col8 = [&](int j) { return 16 * (PARTS * (j >> 1) + part) + 8 * (j & 1); };      // first query row of this thread's block j
        int i = 0;                                                        // unit of this CTA
        // running sums and references of this thread's rows: rows 2 t + e of its blocks
        // `neg`: less what a row's scores are taken against, its reference, or 0 while it has none (its bit 2 j + e of `none`)
        float2 l[NB], ms[NB], neg[NB];
        uint32_t none = 0u;
        // Pass n finishes item n - 1 and begins item n: its queries are in place, and its first scores on the way, before the sums of
        // the one before go out.  (Shared words are double: a warp that is still writing sums out meets others in the next item.)
#pragma unroll 1
        for (int n = 0;; ++n) {
            if (n > 0) {
                // ---- sums of the rows over the four warps that share them
                // (eight lanes have parts of 16 sums: every exchange halves the sums that a lane still has, until lane g has those of
                // block g % 4, of weights or of middles)
                float2 a[2 * NB];
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    a[j] = l[j];
                    a[NB + j] = ms[j];
                }
#pragma unroll
                for (int h = NB, bit = 4; h >= 1; h >>= 1, bit >>= 1)
#pragma unroll
                    for (int k = 0; k < h; ++k) {
                        const float2 keep = g & bit ? a[k + h] : a[k], send = g & bit ? a[k] : a[k + h];
                        a[k] = add2(keep, make_float2(__shfl_xor_sync(0xffffffffu, send.x, 4 * bit), __shfl_xor_sync(0xffffffffu, send.y, 4 * bit)));
                    }
                *reinterpret_cast<float2*>(&(g & 4 ? sm->y : sm->x)[quad][col8(g & 3) + 2 * t]) = a[0];
                if (quad == 0 && g == 0) {
#pragma unroll
                    for (int j = 0; j < NB; ++j)
                        *reinterpret_cast<float2*>(&sm->fac[col8(j) + 2 * t]) = make_float2((none >> (2 * j)) & 1u ? -INFINITY : -neg[j].x, (none >> (2 * j + 1)) & 1u ? -INFINITY : -neg[j].y);
                }
            }
            if (tid == 0) sm->cur[n % 3] = item_get(n);
            named_sync<1, SOFT>();
            const Kv4Item& it = sm->cur[n % 3];                           // stays until the pass after the next
            const bool go = it.take > 0;
            const int rows = rows_of(it), cols = cols_of(rows);
            // ---- queries to shared memory, channels of a word in the order the nibbles come in; their sums
            constexpr int C8 = D / 8, MOST = (N * C8 + SOFT - 1) / SOFT;  // 16-byte pieces of a row, and at most of a thread
            uint4 v[MOST];
            if (go) {
#pragma unroll
                for (int z = 0; z < MOST; ++z) {                          // all loads first
                    const int x = tid + z * SOFT, rl = x / C8, c = x % C8, rr = it.tile * N + rl;
                    v[z] = make_uint4(0, 0, 0, 0);
                    if (rl < rows) {
                        const int ix = (it.q.row0 + rr / p.group) * p.q_heads + it.head * p.group + rr % p.group;
                        v[z] = __ldg(reinterpret_cast<const uint4*>((const __half*)p.q + (size_t)ix * D + 8 * c));
                        if (c == 0) sm->rowix[n & 1][rl] = ix;
                    }
                }
            }
            if (n > 0 && tid < N) {
                const float lsum = (sm->x[0][tid] + sm->x[1][tid]) + (sm->x[2][tid] + sm->x[3][tid]), mm = (sm->y[0][tid] + sm->y[1][tid]) + (sm->y[2][tid] + sm->y[3][tid]);
                sm->tot[tid] = make_float4(lsum, lsum == 0.f ? 0.f : 1.f / lsum, mm, sm->fac[tid]);
            }
            if (go) {
#pragma unroll
                for (int z = 0; z < MOST; ++z) {
                    const int x = tid + z * SOFT, rl = x / C8, c = x % C8;
                    const uint32_t r[4] = {__byte_perm(v[z].x, v[z].z, 0x5410), __byte_perm(v[z].x, v[z].z, 0x7632), __byte_perm(v[z].y, v[z].w, 0x5410), __byte_perm(v[z].y, v[z].w, 0x7632)};
                    if (rl < cols) sts128(base_a + (c >> 3) * N * 128 + rl * 128 + (((c & 7) ^ (rl & 7)) << 4), r);
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r[e])); s += f.x + f.y; }
#pragma unroll
                    for (int o = 1; o < C8; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                    if (c == 0) sm->qs[rl] = s;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                warp_arrive(smem_u32(&sm->q_full));
            }
            named_sync<1, SOFT>();                                        // totals and the queries' sums are read by everybody
            if (n > 0) {
            wait(smem_u32(&sm->p_empty[(i - 1) & 1]), ((i - 1) >> 1) & 1, looks, w.status, DEV_TIMEOUT_EPI);
            tc_fence_after();
            const Kv4Item& last = sm->cur[(n - 1) % 3];
            const int lrows = rows_of(last);
            const int64_t c0 = kv4_cta_of(last.first, per), c1 = kv4_cta_of(last.first + last.chunks - 1, per);
            const bool whole = c0 == c1;
            float* slot = p.part + ((size_t)blockIdx.x * 2 + ((int64_t)blockIdx.x == c0 ? 1 : 0)) * ((size_t)N * (D + 2));
            // lane m of the accumulator is channel (m & ~7) | {0 4 1 5 2 6 3 7}[m & 7]; a row's channels of this quarter are one store of the warp
            const int chn = quad * 32 + ((lane & ~7) | ((lane & 1) * 4) | ((lane & 7) >> 1));
            if (quad * 32 < D) {
#pragma unroll 1
                for (int j = 0; j < NB && col8(j) < lrows; ++j) {
                    uint32_t o[8];
                    const int r0 = col8(j), left = lrows - r0;
                    ld_cols8(tmem + SH::T_O + r0 + ((uint32_t)(quad * 32) << 16), o);
                    float4 tm[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) tm[x] = sm->tot[r0 + x];
                    const int4 ia = *reinterpret_cast<const int4*>(&sm->rowix[(n - 1) & 1][r0]), ib = *reinterpret_cast<const int4*>(&sm->rowix[(n - 1) & 1][r0 + 4]);
                    const int ix[8] = {ia.x, ia.y, ia.z, ia.w, ib.x, ib.y, ib.z, ib.w};
                    ld_wait();
                    if (whole) {
                        __half* out = (__half*)p.out + chn;
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            if (x < left) out[(size_t)ix[x] * D] = __float2half_rn((__uint_as_float(o[x]) + tm[x].z) * tm[x].y);
                    } else {
                        float* out = slot + r0 * D + chn;
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            if (x < left) __stcg(out + x * D, __uint_as_float(o[x]) + tm[x].z);
                    }
                }
            }
            if (!whole && tid < lrows) __stcg(reinterpret_cast<float2*>(slot + N * D + 2 * tid), make_float2(sm->tot[tid].w, sm->tot[tid].x));
            tc_fence_before();                                            // O^T has been read: the next item's first product may write it
            if (!whole) {
                named_sync<1, SOFT>();
                if (tid == 0) {
                    const int want = (int)(c1 - c0), old = arrive_at(p.counters + c0);
                    if (old == want) p.counters[c0] = 0;
                    sm->arrived = old == want;
                }
                named_sync<1, SOFT>();
                if (sm->arrived) merge_item<__half, D, 4>(p, last, N, lrows, c0, c1, warp, SW, nullptr, [] {});
            }
            }
            if (!go) break;
            none = 0u;                                                    // (no bits for blocks without rows)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                l[j] = ms[j] = neg[j] = make_float2(0.f, 0.f);
                if (col8(j) < cols) none |= 3u << 2 * j;
            }
            // The scores of a unit are fetched while the one before is worked on: s[j][h] has the 16 keys 16 h of block j.
            uint32_t s[NB][2][4];
            auto fetch = [&](int u) {
                const int b = u & 1;
                wait(smem_u32(&sm->s_full[b]), (u >> 1) & 1, looks, w.status, DEV_TIMEOUT_EPI);
                tc_fence_after();
                const uint32_t ts = tmem + SH::T_S + b * N + ((uint32_t)(quad * 32) << 16);
#pragma unroll
                for (int j = 0; j < NB; j += 2)
#pragma unroll
                    for (int h = 0; h < 2; ++h) ld_frag2(ts + col8(j) + ((uint32_t)(16 * h) << 16), s[j][h], s[j + 1][h]);
            };
            auto fetched = [&](int u) {
                ld_wait();
                tc_fence_before();
                warp_arrive(smem_u32(&sm->s_empty[u & 1]));
            };
            fetch(i);
            fetched(i);
#pragma unroll 1
            for (int k = 0; k < it.take; ++k, ++i) {
                const int b = i & 1, key0 = (it.chunk0 + k) * UNIT + quad * 32 + g;
                float ks[4], km[4], vs[4], vm[4], lv[4];                  // (lv: what V's scale adds to a product)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float4 f = sm->par[i & (PAR_SLOTS - 1)][quad * 32 + g + 8 * x];
                    ks[x] = f.x; km[x] = f.y; vs[x] = f.z; vm[x] = f.w;
                    lv[x] = scale_bits(f.z);
                }
                const uint32_t groups = *reinterpret_cast<const uint32_t*>(sm->groups[i & (GROUP_SLOTS - 1)]);
                const bool all = (it.chunk0 + k + 1) * UNIT <= it.q.len && groups == 0x03030303u;      // every key of the unit is visible to every row
                // Scores of key x and row e of block j (registers 2 (x & 1) + e of fragment x >> 1), in powers of two, less the base.
                float sc[NB][4][2], top = -INFINITY;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const float2 qq = *reinterpret_cast<const float2*>(&sm->qs[col8(j) + 2 * t]);
                    float tj = -INFINITY;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const float2 dot = make_float2(__uint_as_float(s[j][x >> 1][2 * (x & 1)]), __uint_as_float(s[j][x >> 1][2 * (x & 1) + 1]));
                        const float2 v = fma2(both(ks[x]), dot, fma2(both(km[x]), qq, neg[j]));
                        sc[j][x][0] = v.x;
                        sc[j][x][1] = v.y;
                        const float2 pr = add2(v, both(lv[x]));
                        tj = fmaxf(tj, fmaxf(pr.x, pr.y));
                    }
                    if (col8(j) < cols) top = fmaxf(top, tj);             // (blocks behind the tile's rows hold anything)
                }
                bool over = top > RAISE || none != 0u;                    // (a row's first keys may have had no page)
                uint32_t vis = 0xffffffffu;                               // bit 8 j + 4 e + x: row e of block j sees key x
                if (__builtin_expect(!all, 0)) {
                    // a lane looks up the warp's 32 keys for one of the part's 32 rows; the others get the word by shuffle
                    uint32_t word = sees(p, it.q, (it.tile * N + col8(lane >> 3) + (lane & 7)) / p.group, key0 - g - it.q.len);
                    word &= ((groups >> (8 * quad)) & 1u ? 0x0000ffffu : 0u) | ((groups >> (8 * quad)) & 2u ? 0xffff0000u : 0u);
                    vis = 0u;
                    over = k == 0;
#pragma unroll
                    for (int j = 0; j < NB; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t w32 = __shfl_sync(0xffffffffu, word, 8 * j + 2 * t + e) >> g;
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                const bool ok = (w32 >> (8 * x)) & 1u;
                                if (ok) vis |= 1u << (8 * j + 4 * e + x);
                                else sc[j][x][e] = -INFINITY;
                                over = over || (col8(j) < cols && sc[j][x][e] + lv[x] > ((none >> (2 * j + e)) & 1u ? -INFINITY : RAISE));
                            }
                        }
                }
                // Where one of the 128 threads of these rows finds a product too far above (and in an item's first unit), they agree
                // on new references.
                if (__builtin_expect(part_any(part, over), 0)) {
#pragma unroll
                    for (int j = 0; j < NB; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float m = fmaxf(fmaxf(sc[j][0][e] + lv[0], sc[j][1][e] + lv[1]), fmaxf(sc[j][2][e] + lv[2], sc[j][3][e] + lv[3]));
#pragma unroll
                            for (int sh = 4; sh < 32; sh <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, sh));
                            if (g == 0) sm->x[quad][col8(j) + 2 * t + e] = m;
                        }
                    part_sync(part);
#pragma unroll
                    for (int j = 0; j < NB; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int rl = col8(j) + 2 * t + e;
                            const bool had = !((none >> (2 * j + e)) & 1u);
                            const float up = fmaxf(fmaxf(sm->x[0][rl], sm->x[1][rl]), fmaxf(sm->x[2][rl], sm->x[3][rl])) - TOP;
                            float f = 1.f;
                            if (up > (had ? 0.f : -INFINITY)) {           // the new reference is `up` above the base
                                f = had ? ex2(-up) : 0.f;
                                none &= ~(1u << (2 * j + e));
                                (e ? neg[j].y : neg[j].x) -= up;
                                (e ? l[j].y : l[j].x) *= f;
                                (e ? ms[j].y : ms[j].x) *= f;
#pragma unroll
                                for (int x = 0; x < 4; ++x) sc[j][x][e] -= up;
                            }
                            if (quad == 0 && g == 0) sm->fac[rl] = f;
                        }
                    part_sync(part);
                    if (k > 0) {
                        // O^T holds the products of the units before once the last of them has completed (each P buffer's release
                        // is waited for again two units later, so its phases are seen one by one)
                        wait(smem_u32(&sm->p_empty[(i - 1) & 1]), ((i - 1) >> 1) & 1, looks, w.status, DEV_TIMEOUT_EPI);
                        tc_fence_after();
#pragma unroll 1
                        for (int j = 0; j < NB && col8(j) < cols; ++j) {  // this part's blocks of eight columns, both groups of 16 lanes
                            const float2 f = *reinterpret_cast<const float2*>(&sm->fac[col8(j) + 2 * t]);
                            const uint32_t to = tmem + SH::T_O + col8(j) + ((uint32_t)(quad * 32) << 16);
                            uint32_t o[2][4];
                            ld_frag(to, o[0]);
                            ld_frag(to + (16u << 16), o[1]);
                            ld_wait();
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[h][e] = __float_as_uint(__uint_as_float(o[h][e]) * ((e & 1) ? f.y : f.x));
                                st_frag(to + ((uint32_t)(16 * h) << 16), o[h]);
                            }
                        }
                        st_wait();
                        tc_fence_before();
                    }
                    part_sync(part);                                      // the exchange buffers may be written again
                }
                const bool more = k + 1 < it.take;
                if (more) fetch(i + 1);
                if (i >= 2) wait(smem_u32(&sm->p_empty[b]), ((i >> 1) - 1) & 1, looks, w.status, DEV_TIMEOUT_EPI);
                // (one straight run of instructions for the units that matter, where nothing is masked and every block has rows)
                auto weights = [&](auto plain) {
                    constexpr bool PLAIN = decltype(plain)::value;
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const int blk = col8(j) >> 3;
                        if (!PLAIN && 8 * blk >= cols) break;
                        uint32_t h4[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float2 pe = make_float2(ex2(sc[j][x][0]), ex2(sc[j][x][1]));
                            l[j] = add2(l[j], pe);
                            float2 pv = mul2(pe, both(vs[x])), m2 = fma2(pe, both(vm[x]), ms[j]);
                            if (!PLAIN) {                                 // by selection: what a key holds stays out of rows that do not see it
                                const uint32_t at = vis >> (8 * j + x);
                                if (!(at & 1u)) { pv.x = 0.f; m2.x = ms[j].x; }
                                if (!(at & 16u)) { pv.y = 0.f; m2.y = ms[j].y; }
                            }
                            ms[j] = m2;
                            const __half2 h2 = __floats2half2_rn(pv.x, pv.y);
                            h4[x] = *reinterpret_cast<const uint32_t*>(&h2);
                        }
                        // lane's matrix row: key 32 quad + lane, query rows 8 blk .. 8 blk + 7
                        stmatrix4(base_a + SH::P_AT + b * SH::P_BYTES + (quad * 32 + lane) * 128 + ((blk ^ (lane & 7)) << 4), h4[0], h4[1], h4[2], h4[3]);
                    }
                };
                if (__builtin_expect(all && col8(NB - 1) < cols, 1)) weights(std::true_type{});
                else weights(std::false_type{});
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                warp_arrive(smem_u32(&sm->p_full[b]));
                if (more) fetched(i + 1);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == CW) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

template <int D>
ghd_status launch_tc(ghd_ctx* c, Kv4AttnParams& p) {
    constexpr int VARIANT = 8 + (D == 64 ? 0 : 1);
    if (!(c->attr_kv4 >> VARIANT & 1)) {                                 // once a context, for as many sequences as a call takes
        if (cudaFuncSetAttribute(k_attn_kv4_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>(GHD_MAX_SEQS)) != cudaSuccess) {
            cudaGetLastError();
            return fail(c, GHD_ECUDA, "kv4_attention: cannot raise dynamic shared memory");
        }
        c->attr_kv4 |= 1u << VARIANT;
    }
    p.ctas = c->sm_count;
    c->path_count[GHD_PATH_KV4_TC]++;
    launch_k(c, false, k_attn_kv4_tc<D>, dim3(p.ctas), dim3(THREADS), smem_bytes<D>(p.w.n_seqs), p);
    return GHD_OK;
}

}  // namespace

// partials: 2 slots of [64][d_head + 2] floats a CTA, within the tile scratch of 2 x 256 x 128 floats an SM
ghd_status launch_attn_kv4_tc(ghd_ctx* c, Kv4AttnParams& p) {
    return c->cfg.d_head == 64 ? launch_tc<64>(c, p) : launch_tc<128>(c, p);
}

}  // namespace ghd

