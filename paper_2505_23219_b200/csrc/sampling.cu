// Sampling from logits with given random numbers: candidates drawn without replacement, and the verification of drafted
// tokens against the target's probabilities.
//
// A row of logits is one distribution, w_s = exp(l_s / temperature) up to a factor, in 64 bits: a token is decided by where a random
// number falls between running sums of up to 2^20 weights, whose borders 32 bits would move.
//
// The tokens lie in segments of 256 (32 lanes with 8 neighbours each), the segments in equal shares over the CTAs of a cluster, in
// order.  One pass over a row leaves the weight of every segment.  Weights are powers of two, 2^(l log2(e) / temperature - ref) with a
// whole number ref that is at least the largest exponent of the segment, so that sums with unlike references are added exactly but for
// the addition, by shifting exponents, and no second pass or exponential is needed once the row's largest logit is known.  What the CTAs
// have to know of each other goes through distributed shared memory, one cluster barrier for each exchange.  Where a random number
// falls is looked up over the CTAs, over a CTA's segments, over the lanes of one segment and over a lane's tokens, so that only one
// segment's weights are worked out again.
//
// What bounds it: chains of latencies.  10 draws from 5 rows of 32000: 20 us, 1.75 for each draw (where it falls, the segment's logits from
// the L2, two running sums over 32 lanes, the segment's weight again); 4 draws from 320 rows 35 us, 19 of them the pass over the rows at 1.4 instructions a cycle.
// A tree: 15 us when nothing was drawn, about 1 a level and 2 to 3 a rejected draw (29 with three of these); 48 trees of 64 nodes, row by row, 34.
#include <cstdio>

#include "internal.h"
#include "tc_common.cuh"

namespace ghd {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int MAX_CLUSTER = 8;
constexpr int RUN = 8, SEG = 32 * RUN;          // tokens of a lane, of a segment
constexpr int MAX_VOCAB = 1 << 20;
constexpr int VALUES = 4;                       // doubles that one exchange carries

struct Shared {
    double box[2][MAX_CLUSTER][VALUES];         // exchanges, by turns: what the CTAs of the cluster have sent
    double part[2][WARPS][2];                   // reference and weight of every warp's segments, of two rows
    double mine[VALUES];                        // what this CTA sends
    double share[MAX_CLUSTER];                  // weights of the CTAs' shares of the row
    uint32_t child[GHD_MAX_NODES / 32];         // children of the node, a bit each
    int32_t parent[GHD_MAX_NODES];
    int32_t token[GHD_MAX_NODES], draft[GHD_MAX_NODES];      // of the nodes: drafted token, draft row
    float uniform[GHD_MAX_NODES];
    double of_p[GHD_MAX_NODES], of_q[GHD_MAX_NODES];          // of the children of the node: their tokens' probabilities
    int32_t gone[GHD_MAX_NODES];                // tokens that are not in the distribution any more
    double taken[GHD_MAX_NODES];                // what rejected draws have taken from P, as multiples of Q
    double roots[16];
};

__device__ __forceinline__ void send(double* p, uint32_t rank, double v) {
    const uint32_t at = tc::mapa_shared(tc::smem_u32(p), rank);
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(v) : "memory");
}

__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// inclusive running sums over the lanes
__device__ __forceinline__ double warp_scan(double v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// 2^n of a whole number n <= 0; 0 below -1000.  1 where n is NaN: the difference of two references that are both infinite.
__device__ __forceinline__ double pow2_whole(double n) {
    if (!(n < 0.0)) return 1.0;
    return n < -1000.0 ? 0.0 : __hiloint2double((1023 + (int)n) << 20, 0);
}
// 2^(j / 16), rounded
__constant__ double ROOTS[16] = {
    1.0, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916,
    1.189207115002721, 1.241857812073484, 1.2968395546510096, 1.3542555469368927,
    1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543,
    1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474,
};
// 2^y of y <= 0, 0 below -1000.  Table-driven, after Tang (ACM TOMS 15, 1989): y = n / 16 + f with the nearest whole n, 2^(n / 16) from
// the table (in shared memory, a pair of banks to each entry) and the exponent, and the series of e^(f ln 2), whose first term left out is below
// 2^-50 for |f| <= 1/32: the borders between tokens move by that.  (The library's function takes any argument and about twice the
// instructions; 64-bit ones are what bounds the calls with many rows.)
__device__ __forceinline__ double pow2(double y, const double* roots) {
    constexpr double L = 0.693147180559945309417, MAGIC = 6755399441055744.0 / 16;         // 1.5 * 2^52 / 16: adding it rounds to a whole 16th
    constexpr double C1 = L, C2 = L * L / 2, C3 = L * L * L / 6, C4 = L * L * L * L / 24, C5 = L * L * L * L * L / 120, C6 = L * L * L * L * L * L / 720;
    const double t = y + MAGIC, f = y - (t - MAGIC);
    const int n = __double2loint(t);
    const double root = roots[n & 15];
    double r = fma(C6, f, C5);
    r = fma(r, f, C4);
    r = fma(r, f, C3);
    r = fma(r, f, C2);
    r = fma(r, f, C1);
    r = fma(r * f, root, root);
    r = __hiloint2double(__double2hiint(r) + (n >> 4 << 20), __double2loint(r));
    return (uint32_t)__double2hiint(y) > 0xc08f4000u ? 0.0 : r;      // (below -1000, by its bits)
}
// A float as a double by its bits (the conversion has a quarter of the other instructions' rate): numbers below 2^-126, zeros among them, come out
// below 2^-126, infinities as 2^128 (as good for weights: a temperature is at most 2^64); NaN is found by the row's maximum.
// COLD: temperatures below some 2^-60 bring what is below 2^-126 up to where it counts, and are served by kernels that convert (looking at each
// logit costs all calls 5 %, at the temperature 2 to 3).
constexpr double COLD_SCALE = 0x1p60;
template <bool COLD>
__device__ __forceinline__ double widen(float l) {
    if (COLD) return (double)l;
    const uint32_t b = __float_as_uint(l);
    return __hiloint2double((int)((b & 0x80000000u) | ((b & 0x7fffffffu) >> 3) + 0x38000000u), (int)(b << 29));
}
// The product is rounded before the difference: equal logits are equally likely however large they are.
template <bool COLD>
__device__ __forceinline__ double weight(float l, double scale, double ref, const double* roots) { return pow2(__dsub_rn(__dmul_rn(widen<COLD>(l), scale), ref), roots); }

// One row's distribution: 2^(l * scale - ref) / sum, scale = log2(e) / temperature.
template <bool COLD>
struct Dist {
    const float* row;
    double scale, ref, inv_sum;
    bool ok;
    const double* roots;
    __device__ __forceinline__ double of(float l) const { return __dmul_rn(weight<COLD>(l, scale, ref, roots), inv_sum); }
};

// This CTA's share of a row, and what the cluster has agreed on so far.
struct Team {
    Shared* s;
    double* seg;                                // [own segments] weights
    int rank, size, turn, warp, lane;
    int vocab;
    bool wide;                                  // all rows on 16-byte boundaries
    int seg0, segs;                             // own segments

    __device__ Team(Shared* sm, double* weights, int vocab_, bool wide_, int cluster) : s(sm), seg(weights), size(cluster), turn(0), vocab(vocab_), wide(wide_) {
        rank = cluster > 1 ? (int)tc::cluster_ctarank() : 0;
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        const int n = (vocab + SEG - 1) / SEG;
        seg0 = n * rank / cluster;
        segs = n * (rank + 1) / cluster - seg0;
        if (threadIdx.x < 16) s->roots[threadIdx.x] = ROOTS[threadIdx.x];
        if (cluster > 1) tc::cluster_sync_all();                   // everybody's shared memory is there
        else __syncthreads();
    }
    __device__ __forceinline__ int first_of(int sg) const { return sg * SEG + lane * RUN; }       // this lane's first token of a segment
    // RUN tokens from t on, -inf past the row's end
    __device__ __forceinline__ void load(const float* __restrict__ row, int t, float (&x)[RUN]) const {
        if (wide && t + RUN <= vocab) {
#pragma unroll
            for (int i = 0; i < RUN; i += 4) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(row + t + i));
                x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < RUN; ++i) x[i] = t + i < vocab ? __ldg(row + t + i) : -INFINITY;
        }
    }
    // mine[0 .. n) of every CTA, to be read from the returned box by everyone: one barrier of the cluster.
    // The box of the exchange before is still being read; the one before that has been left by everybody.
    __device__ double (*exchange(int n))[VALUES] {
        double (*box)[VALUES] = s->box[turn];
        __syncthreads();
        if (threadIdx.x < (unsigned)(size * n)) {
            const int to = threadIdx.x / n, i = threadIdx.x % n;
            if (size > 1) send(&box[rank][i], (uint32_t)to, s->mine[i]);
            else box[0][i] = s->mine[i];
        }
        if (size > 1) tc::cluster_sync_all();
        else __syncthreads();
        turn ^= 1;
        return box;
    }
    // what every CTA has sent as its share's weight -> the total
    __device__ double add_shares(double (*box)[VALUES]) {
        double sum = lane % MAX_CLUSTER < size ? box[lane % MAX_CLUSTER][0] : 0.0;
        if (threadIdx.x < (unsigned)size) s->share[threadIdx.x] = sum;
#pragma unroll
        for (int o = 1; o < MAX_CLUSTER; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        __syncthreads();
        return sum;
    }
};

// The weights of a segment's tokens in this lane: 0 of -inf, whatever the reference
template <bool COLD>
__device__ __forceinline__ double sum_of(const float (&x)[RUN], double scale, double ref, const double* roots) {
    double w[RUN];
    ref = ref == -INFINITY ? 0.0 : ref;
#pragma unroll
    for (int e = 0; e < RUN; ++e) w[e] = weight<COLD>(x[e], scale, ref, roots);
    return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
}

// One warp: weight of a segment and its reference, from this lane's logits
template <bool COLD>
__device__ __forceinline__ double segment_sum(const float (&x)[RUN], double scale, const double* roots, double& ref) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < RUN; ++e) top = max_nan(top, x[e]);
    top = warp_max(top);
    // NaN and infinity are kept apart from all numbers: a reference that no number gives
    ref = top < INFINITY ? ceil(__dmul_rn((double)top, scale)) : INFINITY;
    return warp_sum(sum_of<COLD>(x, scale, ref, roots));
}

// seg[] from the segments' own weights and references: the weights with the row's reference (not divided by the sum).  A token ends at 2^-1000 of that
// reference (see pow2), a segment's weight does not: what is below FAR is weighed again token by token, so that a segment has weight exactly where
// a token of it has.  Above FAR the tokens that end are 2^-60 of their segment.
constexpr double FAR = -940.0;
template <bool COLD, typename W, typename R>
__device__ void row_weights(Team& m, const Dist<COLD>& p, W weight_of, R ref_of) {
    bool far = false;
    for (int g = threadIdx.x; g < m.segs; g += THREADS) {
        const double d = ref_of(g) - p.ref, w = weight_of(g) * pow2_whole(d);
        m.seg[g] = w;
        far |= w > 0.0 && d < FAR;
    }
    if (!__syncthreads_or(far)) return;
#pragma unroll 1
    for (int g = m.warp; g < m.segs; g += WARPS) {
        if (!(m.seg[g] > 0.0 && ref_of(g) - p.ref < FAR)) continue;
        float x[RUN];
        m.load(p.row, m.first_of(m.seg0 + g), x);
        const double sum = warp_sum(sum_of<COLD>(x, p.scale, p.ref, p.roots));
        if (m.lane == 0) m.seg[g] = sum;
    }
    __syncthreads();
}

// Reference and sum of a row p and, if q.row is given, of a second one.  seg[] is left with p's weights (not divided by the sum),
// share[] has every CTA's part of p's sum.  -> whether a part is below FAR: then the sum of seg[] is right, share[] is not.
template <bool COLD>
__device__ bool measure(Team& m, Dist<COLD>& p, Dist<COLD>& q) {
    bool far = false;
    const int n = q.row ? 2 : 1;
    double ref[2] = {-INFINITY, -INFINITY}, all[2] = {0.0, 0.0};
#pragma unroll 1
    for (int g = m.warp; g < m.segs; g += WARPS) {
        float x[2][RUN];
        m.load(p.row, m.first_of(m.seg0 + g), x[0]);
        if (n == 2) m.load(q.row, m.first_of(m.seg0 + g), x[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i == 1 && n == 1) break;
            double r;
            const double sum = segment_sum<COLD>(x[i], i ? q.scale : p.scale, p.roots, r);
            if (i == 0 && m.lane == 0) { m.seg[g] = sum; m.seg[m.segs + g] = r; }
            const double both = fmax(ref[i], r);
            all[i] = all[i] * pow2_whole(ref[i] - both) + sum * pow2_whole(r - both);
            ref[i] = both;
        }
    }
    if (m.lane < n) { m.s->part[m.lane][m.warp][0] = m.lane ? ref[1] : ref[0]; m.s->part[m.lane][m.warp][1] = m.lane ? all[1] : all[0]; }
    __syncthreads();
    if (m.warp < n) {                                            // the warps' results of row `warp`
        const double r = m.lane < WARPS ? m.s->part[m.warp][m.lane][0] : -INFINITY, x = m.lane < WARPS ? m.s->part[m.warp][m.lane][1] : 0.0;
        const double both = warp_max(r), sum = warp_sum(x * pow2_whole(r - both));
        if (m.lane == 0) { m.s->mine[2 * m.warp] = both; m.s->mine[2 * m.warp + 1] = sum; }
    }
    double (*box)[VALUES] = m.exchange(2 * n);
    // every warp adds up what the CTAs have sent, a CTA to each of eight lanes
    const int c = m.lane % MAX_CLUSTER;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (i == 1 && n == 1) break;
        const double r = c < m.size ? box[c][2 * i] : -INFINITY;
        double both = r, sum = c < m.size ? box[c][2 * i + 1] : 0.0;
#pragma unroll
        for (int o = 1; o < MAX_CLUSTER; o <<= 1) both = fmax(both, __shfl_xor_sync(0xffffffffu, both, o));
        sum *= pow2_whole(r - both);
        if (i == 0) far = __any_sync(0xffffffffu, sum > 0.0 && r - both < FAR);
        if (i == 0 && threadIdx.x < (unsigned)m.size) m.s->share[threadIdx.x] = sum;
#pragma unroll
        for (int o = 1; o < MAX_CLUSTER; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        Dist<COLD>& d = i ? q : p;
        d.ref = both;
        d.inv_sum = 1.0 / sum;
        d.ok = both > -INFINITY && both < INFINITY && sum < INFINITY;
    }
    row_weights(m, p, [&](int g) { return m.seg[g]; }, [&](int g) { return m.seg[m.segs + g]; });
    return far;
}

// What a rejected draw leaves of P at a token.  One rounding, and the same wherever it is worked out: sums and the tokens in them must agree on
// where there is nothing.
__device__ __forceinline__ double take(double p, double q, double a) { return fmax(__fma_rn(-a, q, p), 0.0); }

// P and Q of this lane's tokens of segment g
template <bool COLD>
__device__ __forceinline__ void both_of(const Team& m, const Dist<COLD>& p, const Dist<COLD>& q, int g, double (&a)[RUN], double (&b)[RUN]) {
    float x[RUN], y[RUN];
    const int t = m.first_of(m.seg0 + g);
    m.load(p.row, t, x);
    m.load(q.row, t, y);
#pragma unroll
    for (int e = 0; e < RUN; ++e) {
        a[e] = p.of(x[e]);
        b[e] = q.of(y[e]);
    }
}
// ... after rejected draws: P less taken[0 .. steps) times Q, one after the other, and Q, both without the tokens gone[0 .. n)
__device__ __forceinline__ void leave(const Team& m, int g, int steps, int n, double (&a)[RUN], double (&b)[RUN]) {
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        const double w = m.s->taken[i];
#pragma unroll
        for (int e = 0; e < RUN; ++e) a[e] = take(a[e], b[e], w);
    }
#pragma unroll 1
    for (int i = 0; i < n; i += 32) {
        const int d = i + m.lane < n ? m.s->gone[i + m.lane] : -1;
        for (uint32_t here = __ballot_sync(0xffffffffu, d >= 0 && d / SEG == m.seg0 + g); here; here &= here - 1) {
            const int at = __shfl_sync(0xffffffffu, d, __ffs(here) - 1) - m.first_of(m.seg0 + g);
#pragma unroll
            for (int e = 0; e < RUN; ++e) if (at == e) a[e] = b[e] = 0.0;
        }
    }
}

// What is left after rejected draws (see leave): of P the weights of every own segment into seg[], of the CTAs' shares into share[] -> the total;
// of Q the sum -> rest.  Both are sums over what is left: 1 - Q(rejected) has no right digit where a rejected token holds all but 1e-16 of Q.
// keep (or null): room for P and Q of the own segments, which `kept` says are there from the rejection before.
template <bool COLD>
__device__ double total_left(Team& m, const Dist<COLD>& p, const Dist<COLD>& q, int steps, int n, double2* keep, bool kept, double& rest) {
    double all = 0.0, all_q = 0.0;
#pragma unroll 1
    for (int g = m.warp; g < m.segs; g += WARPS) {
        double a[RUN], b[RUN], sum = 0.0;
        double2* at = keep + g * SEG + m.lane;
        if (keep && kept) {
#pragma unroll
            for (int e = 0; e < RUN; ++e) {
                const double2 v = at[e * 32];
                a[e] = v.x;
                b[e] = v.y;
            }
        } else {
            both_of(m, p, q, g, a, b);
#pragma unroll
            for (int e = 0; e < RUN; ++e)
                if (keep) at[e * 32] = make_double2(a[e], b[e]);
        }
        leave(m, g, steps, n, a, b);
#pragma unroll
        for (int e = 0; e < RUN; ++e) {
            sum += a[e];
            all_q += b[e];
        }
        sum = warp_sum(sum);
        if (m.lane == 0) m.seg[g] = sum;
        all += sum;
    }
    all_q = warp_sum(all_q);
    if (m.lane == 0) { m.s->part[0][m.warp][0] = all; m.s->part[0][m.warp][1] = all_q; }
    __syncthreads();
    if (m.warp < 2) {
        const double sum = warp_sum(m.lane < WARPS ? m.s->part[0][m.lane][m.warp] : 0.0);
        if (m.lane == 0) m.s->mine[m.warp] = sum;
    }
    double (*box)[VALUES] = m.exchange(2);
    rest = m.lane % MAX_CLUSTER < m.size ? box[m.lane % MAX_CLUSTER][1] : 0.0;
#pragma unroll
    for (int o = 1; o < MAX_CLUSTER; o <<= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
    return m.add_shares(box);
}

// The CTA in whose share u times the total falls (the last one with weight where rounding leaves none) -> whether it is this one, and the
// sum of what lies before it
__device__ bool own_share(Team& m, double target, double& before) {
    int owner = -1, last = -1;
    double run = 0.0, start = 0.0, last_start = 0.0;
    for (int r = 0; r < m.size && owner < 0; ++r) {
        const double x = m.s->share[r];
        if (x > 0.0) { last = r; last_start = run; }
        if (run + x > target) { owner = r; start = run; }
        run += x;
    }
    if (owner < 0) { owner = last; start = last_start; }
    before = start;
    return owner == m.rank;
}

// One warp: the lane in whose running sum the target falls, the last one with weight where rounding leaves none, -1 where there is no weight;
// start: what lies before that lane.
__device__ __forceinline__ int lane_at(double run, double sum, double target, double& start) {
    const uint32_t over = __ballot_sync(0xffffffffu, sum > 0.0 && run > target), some = __ballot_sync(0xffffffffu, sum > 0.0);
    if (!some) return -1;
    const int k = over ? __ffs(over) - 1 : 31 - __clz(some);
    start = __shfl_sync(0xffffffffu, run - sum, k);
    return k;
}
__device__ __forceinline__ int lane_of(double sum, double before, double target, int lane, double& start) { return lane_at(before + warp_scan(sum, lane), sum, target, start); }
// One warp: the segment of seg[0 .. n) in which the target falls.  A lane has `per` neighbouring segments; k: the lane that it falls in.
__device__ __forceinline__ int segment_at(const double* seg, int n, int per, int k, double target, double& start) {
    if (k < 0) return -1;
    int found = -1, last = -1;
    double run = start, last_start = start;
    for (int g = k * per; g < min(n, (k + 1) * per); ++g) {      // (all lanes walk the owner's)
        const double x = seg[g];
        if (x > 0.0) { last = g; last_start = run; }
        if (x > 0.0 && run + x > target) { found = g; break; }
        run += x;
    }
    start = found < 0 ? last_start : run;
    return found < 0 ? last : found;
}
__device__ __forceinline__ int segment_of(const double* seg, int n, int per, double sum, double before, double target, int lane, double& start) {
    const int k = lane_of(sum, before, target, lane, start);
    return segment_at(seg, n, per, k, target, start);
}
// One warp: the token, from the weights w of the segment's tokens in this lane.  All lanes get it.
__device__ int token_of(const double (&w)[RUN], int t0, double before, double target, int lane) {
    double sum = 0.0, start;
#pragma unroll
    for (int e = 0; e < RUN; ++e) sum += w[e];
    const int k = lane_of(sum, before, target, lane, start);
    if (k < 0) return -1;
    int token = -1, last = -1;
    double run = start;
#pragma unroll
    for (int e = 0; e < RUN; ++e) {
        run += w[e];
        if (w[e] > 0.0) last = t0 + e;
        if (token < 0 && w[e] > 0.0 && run > target) token = t0 + e;
    }
    return __shfl_sync(0xffffffffu, token < 0 ? last : token, k);
}
// what a lane's neighbouring segments weigh
__device__ __forceinline__ double lane_sum(const double* seg, int n, int per, int lane) {
    double sum = 0.0;
    for (int g = lane * per; g < min(n, (lane + 1) * per); ++g) sum += seg[g];
    return sum;
}
// tokens that are gone have no weight
__device__ __forceinline__ void without(double (&w)[RUN], int t0, const int32_t* gone, int n) {
    for (int g = 0; g < n; ++g) {
        const int d = gone[g] - t0;
#pragma unroll
        for (int e = 0; e < RUN; ++e) w[e] = d == e ? 0.0 : w[e];
    }
}

// seg[] after measure(), without the tokens gone[0 .. n)
template <bool COLD>
__device__ void weigh_again(Team& m, const Dist<COLD>& p, int n) {
    __syncthreads();
#pragma unroll 1
    for (int i = m.warp; i < n; i += WARPS) {
        const int g = m.s->gone[i] / SEG - m.seg0;
        bool first = g >= 0 && g < m.segs;                       // one warp to a segment, that of the first of its tokens
        for (int k = 0; k < i && first; ++k) first = m.s->gone[k] / SEG - m.seg0 != g;
        if (!first) continue;
        float x[RUN];
        double w[RUN], sum = 0.0;
        const int t0 = m.first_of(m.seg0 + g);
        m.load(p.row, t0, x);
#pragma unroll
        for (int e = 0; e < RUN; ++e) w[e] = p.of(x[e]);
        without(w, t0, m.s->gone, n);
#pragma unroll
        for (int e = 0; e < RUN; ++e) sum += w[e];
        sum = warp_sum(sum);
        if (m.lane == 0) m.seg[g] = sum;
    }
    __syncthreads();
}
// share[] from seg[] -> the total
__device__ double total_again(Team& m) {
    if (m.warp == 0) {
        double sum = 0.0;
        for (int g = m.lane; g < m.segs; g += 32) sum += m.seg[g];
        sum = warp_sum(sum);
        if (m.lane == 0) m.s->mine[0] = sum;
    }
    return m.add_shares(m.exchange(1));
}

// Reference and sum of one row (or two) whose segments k_row_segments has weighed: every CTA for itself.
template <bool COLD>
__device__ void collect(Team& m, int n_segs, const double2* sp, const double2* sq, Dist<COLD>& p, Dist<COLD>& q) {
    const int n = q.row ? 2 : 1;
    double ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0, 0.0};
    for (int g = threadIdx.x; g < n_segs; g += THREADS) {
        const double2 v[2] = {sp[g], n == 2 ? sq[g] : make_double2(0.0, -INFINITY)};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const double both = fmax(ref[i], v[i].y);
            sum[i] = sum[i] * pow2_whole(ref[i] - both) + v[i].x * pow2_whole(v[i].y - both);
            ref[i] = both;
        }
    }
    const int c = m.lane % WARPS;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (i == 1 && n == 1) break;
        const double both = warp_max(ref[i]), all = warp_sum(sum[i] * pow2_whole(ref[i] - both));
        if (m.lane == 0) { m.s->part[i][m.warp][0] = both; m.s->part[i][m.warp][1] = all; }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (i == 1 && n == 1) break;
        const double r = m.s->part[i][c][0];
        double both = r, all = m.s->part[i][c][1];
#pragma unroll
        for (int o = 1; o < WARPS; o <<= 1) both = fmax(both, __shfl_xor_sync(0xffffffffu, both, o));
        all *= pow2_whole(r - both);
#pragma unroll
        for (int o = 1; o < WARPS; o <<= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
        Dist<COLD>& d = i ? q : p;
        d.ref = both;
        d.inv_sum = 1.0 / all;
        d.ok = both > -INFINITY && both < INFINITY && all < INFINITY;
    }
}

// random numbers are held in [0, 1 - 2^-24]
__device__ __forceinline__ double unit(float u) { return (double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }

// ---------------------------------------------------------------- candidates
// When the row has been measured its first CTA gets all segments' weights and draws alone, with one warp: what it takes to find a token
// is one segment's logits.
// HELD: CTAs to a SM.  Four hide more of each other's latencies (1000 rows of 32000, 4 draws each: 73 us against 85), three leave registers for
// a shorter chain of a draw (5 rows 11.8 us against 13.0, 320 rows 33.7 against 34.8): four from where there are rows for four.
template <int HELD, bool COLD>
__global__ void __launch_bounds__(THREADS, HELD) k_draft_sample(const float* __restrict__ logits, int vocab, bool wide, int cluster, double scale, int draws,
                                                          const float* __restrict__ uniforms, int32_t* __restrict__ cand, int* status) {
    extern __shared__ __align__(16) double weights[];
    __shared__ Shared sm;
    Team m(&sm, weights, vocab, wide, cluster);
    const int row = blockIdx.x / cluster;
    Dist<COLD> p{logits + (size_t)row * vocab, scale, 0.0, 1.0, false, sm.roots}, none{};
    measure(m, p, none);
    if (cluster > 1) {
        tc::cluster_sync_all();                                // (the first CTA's room behind its own segments is free)
        if (m.rank > 0)
            for (int g = threadIdx.x; g < m.segs; g += THREADS) send(weights + m.seg0 + g, 0, weights[g]);
        tc::cluster_sync_all();
    }
    if (m.rank > 0 || m.warp > 0) return;
    if (!p.ok && m.lane == 0) atomicCAS(status, DEV_OK, DEV_SAMPLE_DIST);
    p.inv_sum = 1.0;                                           // the weights as they are
    const int n = (vocab + SEG - 1) / SEG, per = (n + 31) / 32;
    const float u = m.lane < draws ? __ldg(uniforms + (size_t)row * GHD_MAX_TOPK + m.lane) : 0.f;
    double mine = lane_sum(weights, n, per, m.lane);
    int out = -1;
#pragma unroll 1
    for (int j = 0; j < draws && p.ok; ++j) {
        const double run = warp_scan(mine, m.lane), target = unit(__shfl_sync(0xffffffffu, u, j)) * __shfl_sync(0xffffffffu, run, 31);
        double start;
        const int k = lane_at(run, mine, target, start), sg = segment_at(weights, n, per, k, target, start);
        if (sg < 0) break;                                     // nothing is left
        float x[RUN];
        double w[RUN], sum = 0.0;
        const int t0 = m.first_of(sg);
        m.load(p.row, t0, x);
#pragma unroll
        for (int e = 0; e < RUN; ++e) w[e] = p.of(x[e]);
        // (lane i has drawn token i)
        for (uint32_t here = __ballot_sync(0xffffffffu, out >= 0 && out / SEG == sg); here; here &= here - 1) {
            const int d = __shfl_sync(0xffffffffu, out, __ffs(here) - 1) - t0;
#pragma unroll
            for (int e = 0; e < RUN; ++e) w[e] = d == e ? 0.0 : w[e];
        }
        const int t = token_of(w, t0, start, target, m.lane);
        if (t < 0) break;
        if (m.lane == j) out = t;
        // the segment's weight without it
#pragma unroll
        for (int e = 0; e < RUN; ++e) sum += t - t0 == e ? 0.0 : w[e];
        sum = warp_sum(sum);
        if (m.lane == 0) weights[sg] = sum;
        __syncwarp();
        if (m.lane == sg / per) mine = lane_sum(weights, n, per, m.lane);
    }
    if (m.lane < GHD_MAX_TOPK) cand[(size_t)row * GHD_MAX_TOPK + m.lane] = out;
}

// ---------------------------------------------------------------- verification
// A walk from the root.  At a node with target distribution P and draft distribution Q its children are looked at in order, with
// P_1 = P, Q_1 = Q: child x is accepted if u Q_j(x) < P_j(x); otherwise P_{j+1} = max(P_j - Q_j, 0) / its sum and Q_{j+1} = Q_j
// without x / its sum.  Neither is divided by its sum here: with p_j = W_j P_j, W_j the sum of p_j, and 1 / c_j the sum of Q without the rejected
// tokens, Q_j is c_j Q and p_{j+1} = max(p_j - c_j W_j Q, 0).  So a rejection leaves one number a_j = c_j W_j, from which, with the ones before it,
// a token's p is worked out at any time, and costs one pass over the vocabulary for both sums.  (max(P - (a_1 + .. + a_j) Q, 0) is the same without
// rounding, but a difference of numbers that agree to ever more digits.)  A rejected token has u Q_j >= P_j, u < 1, so P_{j+1} gives it nothing;
// it is taken out, so that rounding gives it nothing either.  Where p_j - a_j Q is nothing but rounding, p_j stays, without x.
// Candidates that nobody drew have Q = 1 at themselves: P_{j+1} is P_j without x.
// The segments' weights and references of all rows, of the targets and behind them of the drafts, a warp to a segment.  With few trees
// the walk below knows its rows one after the other only, and most SMs would wait; weighing all rows first costs less than it saves.
template <bool COLD>
__global__ void __launch_bounds__(THREADS, 4) k_row_segments(const float* __restrict__ logits, const float* __restrict__ draft, int n_rows, int n_draft, int vocab, bool wide, double scale,
                                                             double draft_scale, double2* __restrict__ out) {
    __shared__ Shared sm;
    pdl_trigger();
    Team m(&sm, nullptr, vocab, wide, 1);
    const int n = m.segs, total = (n_rows + n_draft) * n;
    for (int t = blockIdx.x * WARPS + m.warp; t < total; t += gridDim.x * WARPS) {
        const int row = t / n, g = t - row * n;
        const bool target = row < n_rows;
        float x[RUN];
        m.load(target ? logits + (size_t)row * vocab : draft + (size_t)(row - n_rows) * vocab, m.first_of(g), x);
        double ref;
        const double sum = segment_sum<COLD>(x, target ? scale : draft_scale, sm.roots, ref);
        if (m.lane == 0) out[t] = make_double2(sum, ref);
    }
}

// READY: k_row_segments has run.
template <bool READY, bool COLD>
__global__ void __launch_bounds__(THREADS, 2) k_accept_sampled(ghd_sampled a, int vocab, bool wide, double scale, double draft_scale, int cluster, int keep_at, const double2* __restrict__ ready,
                                                               ghd_accept_result* __restrict__ results, int* status) {
    extern __shared__ __align__(16) double weights[];
    __shared__ Shared sm;
    Team m(&sm, weights, vocab, wide, cluster);
    double2* keep = keep_at ? reinterpret_cast<double2*>(weights + keep_at) : nullptr;
    const int seq = blockIdx.x / cluster;
    ghd_accept_result* out = results + seq;
    const bool writes = m.rank == 0 && threadIdx.x == 0;
    auto record = [&](int code) { if (writes) atomicCAS(status, DEV_OK, code); };
    const int first = a.row_start ? __ldg(a.row_start + seq) : 0, end = a.row_start ? __ldg(a.row_start + seq + 1) : a.n_rows;
    int n = 0;
    if (first < 0 || end < first || end > a.n_rows || end - first > GHD_MAX_NODES) record(DEV_SAMPLE_TREE);
    else n = end - first;
    if (m.rank == 0)
        for (int i = threadIdx.x; i < GHD_MAX_NODES; i += THREADS) {
            out->nodes[i] = i == 0 && n > 0 ? 0 : -1;
            out->tokens[i] = -1;
        }
    if (threadIdx.x < GHD_MAX_NODES) {
        const int i = threadIdx.x, p = i < n ? __ldg(a.parent + first + i) : -1;
        const bool bad = i < n && (i == 0 ? p != -1 : p < 0 || p >= i);
        if (bad && m.rank == 0) atomicCAS(status, DEV_OK, DEV_SAMPLE_TREE);
        sm.parent[i] = bad ? -1 : p;
        sm.token[i] = i < n ? __ldg(a.tokens + first + i) : -1;
        sm.uniform[i] = i < n ? __ldg(a.uniforms + first + i) : 0.f;
        sm.draft[i] = i < n && a.draft_row ? __ldg(a.draft_row + first + i) : -1;
    }
    __syncthreads();
    const int n_segs = (vocab + SEG - 1) / SEG;
    if (READY) pdl_wait();
    int node = 0, depth = 0;
    while (n > 0) {
        if (threadIdx.x < GHD_MAX_NODES) {
            const uint32_t b = __ballot_sync(0xffffffffu, (int)threadIdx.x > node && sm.parent[threadIdx.x] == node);
            if (m.lane == 0) sm.child[m.warp] = b;
        }
        __syncthreads();
        bool any = false;
        for (int i = 0; i < GHD_MAX_NODES / 32; ++i) any |= sm.child[i] != 0;
        int drawn = sm.draft[node];
        if (any && drawn >= a.n_draft) {
            record(DEV_SAMPLE_DRAFT);
            drawn = -1;
        }
        Dist<COLD> p{a.logits + (size_t)(first + node) * vocab, scale, 0.0, 1.0, false, sm.roots}, q{};
        if (any && drawn >= 0) { q.row = a.draft_logits + (size_t)drawn * vocab; q.scale = draft_scale; q.roots = sm.roots; }
        // the children's logits are on their way while the rows are measured
        const int mine = threadIdx.x < GHD_MAX_NODES && (sm.child[m.warp % (GHD_MAX_NODES / 32)] >> m.lane & 1) ? sm.token[threadIdx.x] : -1;
        const bool look = mine >= 0 && mine < vocab;
        const float lp = look ? __ldg(p.row + mine) : 0.f, lq = look && q.row ? __ldg(q.row + mine) : 0.f;
        bool far = false;
        if (READY) collect(m, n_segs, ready + (size_t)(first + node) * n_segs, ready + (size_t)(a.n_rows + max(drawn, 0)) * n_segs, p, q);
        else far = measure(m, p, q);
        if (!p.ok || (q.row && !q.ok)) record(DEV_SAMPLE_DIST);
        if (threadIdx.x < GHD_MAX_NODES) {
            sm.of_p[threadIdx.x] = look ? p.of(lp) : 0.0;
            sm.of_q[threadIdx.x] = look && q.row ? q.of(lq) : 0.0;
        }
        __syncthreads();
        double W = 1.0, rest = 1.0;                            // rest: of what the children come from (Q, or P if they were not drawn) without the rejected tokens
        int n_gone = 0, steps = 0, next = -1;
        bool fresh = false;                                    // seg[] and share[] are of the weights as they are, their total is W
        if (p.ok && (!q.row || q.ok))
            for (int word = 0; word < GHD_MAX_NODES / 32 && next < 0; ++word)
                for (uint32_t bits = sm.child[word]; bits; bits &= bits - 1) {
                    const int c = 32 * word + __ffs(bits) - 1, x = sm.token[c];
                    if (x < 0 || x >= vocab) continue;
                    const double u = unit(sm.uniform[c]), px = sm.of_p[c];
                    if (q.row) {
                        const double qx = sm.of_q[c];
                        bool before = false;                   // a token that was rejected already is not drawn again
                        for (int g = 0; g < n_gone; ++g) before |= sm.gone[g] == x;
                        if (!(qx > 0.0) || before) continue;
                        const double c_j = 1.0 / fmax(rest, qx);
                        if (u * (qx * c_j) * W < px) { next = c; break; }
                        const double a_j = c_j * W;
                        __syncthreads();
                        if (threadIdx.x == 0) {
                            sm.gone[n_gone] = x;
                            sm.taken[steps] = a_j;
                        }
                        ++n_gone;
                        ++steps;
                        __syncthreads();
                        W = total_left(m, p, q, steps, n_gone, keep, fresh, rest);
                        if (W > 0.0) {
                            if (threadIdx.x < GHD_MAX_NODES) sm.of_p[threadIdx.x] = take(sm.of_p[threadIdx.x], sm.of_q[threadIdx.x], a_j);
                            __syncthreads();
                        } else {
                            W = total_left(m, p, q, --steps, n_gone, keep, true, rest);
                        }
                        fresh = true;
                    } else {
                        bool before = false;
                        for (int g = 0; g < n_gone; ++g) before |= sm.gone[g] == x;
                        if (before) continue;
                        if (u * fmax(rest, px) < px) { next = c; break; }
                        rest -= px;
                        __syncthreads();
                        if (threadIdx.x == 0) sm.gone[n_gone] = x;
                        ++n_gone;
                        __syncthreads();
                        if (px > 0.0 && rest < 0x1p-10) {      // the difference loses its digits (random numbers close to one get here)
                            W = total_left(m, p, p, 0, n_gone, nullptr, false, rest);
                            fresh = true;
                        }
                    }
                }
        if (next < 0) {
            if (!p.ok) {
                if (writes) out->tokens[depth] = 0;
            } else {
                // What is left of P: after rejected draws the weights of the last sum; otherwise P's own segments (not divided by the sum),
                // those with a token that is gone weighed again.
                double total = W;
                if (!fresh) {
                    p.inv_sum = 1.0;
                    if (READY) {
                        if (m.rank != 0) break;
                        // the first CTA has all of the row
                        m.size = 1;
                        m.seg0 = 0;
                        m.segs = n_segs;
                        const double2* row = ready + (size_t)(first + node) * n_segs;
                        row_weights(m, p, [&](int g) { return row[g].x; }, [&](int g) { return row[g].y; });
                    }
                    if (n_gone > 0) weigh_again(m, p, n_gone);
                    if (READY || n_gone > 0 || far) {
                        total = total_again(m);
                    } else {
                        total = 0.0;
                        for (int r = 0; r < m.size; ++r) total += sm.share[r];
                    }
                }
                const double target = unit(sm.uniform[0]) * total;
                double before, start;
                if (own_share(m, target, before) && m.warp == 0) {
                    const int per = (m.segs + 31) / 32, sg = segment_of(m.seg, m.segs, per, lane_sum(m.seg, m.segs, per, m.lane), before, target, m.lane, start);
                    const int g = max(sg, 0);
                    double w[RUN], v[RUN];
                    both_of(m, p, q.row ? q : p, g, w, v);
                    leave(m, g, steps, n_gone, w, v);
                    const int t = token_of(w, m.first_of(m.seg0 + g), start, target, m.lane);
                    if (m.lane == 0) out->tokens[depth] = t;
                }
            }
            break;
        }
        if (writes) {
            out->tokens[depth] = sm.token[next];
            out->nodes[depth + 1] = next;
        }
        ++depth;
        node = next;
        __syncthreads();                                       // child[] and gone[] are written again
    }
    if (writes) {
        out->n_matched = depth;
        out->n_emitted = n > 0 ? depth + 1 : 0;
    }
    if (cluster > 1) tc::cluster_sync_all();                   // nobody leaves while others may write to its shared memory
}

// CTAs to a row: as many as leave each of them room beside the others (`held` to a SM) and four segments
int cluster_for(const ghd_ctx* c, int rows, int vocab, int held) {
    const int64_t k = (int64_t)held * c->sm_count / rows, most = vocab / (4 * SEG);
    return (int)(k < 1 || most < 1 ? 1 : k > most ? (most > MAX_CLUSTER ? MAX_CLUSTER : most) : k > MAX_CLUSTER ? MAX_CLUSTER : k);
}
// room for a CTA's segments twice over (weights and references), and in a row's first CTA for the weights of all
size_t room_for(int vocab, int cluster) {
    const size_t n = ((size_t)vocab + SEG - 1) / SEG, own = (n + cluster - 1) / cluster;
    return sizeof(double) * (2 * own > n ? 2 * own : n);
}
// room for P and Q of a CTA's segments
size_t keep_for(int vocab, int cluster) { return ((size_t)(vocab + SEG - 1) / SEG + cluster - 1) / cluster * SEG * sizeof(double2); }
constexpr size_t MAX_ROOM = 96 * 1024;
// rows of four logits at a time (a null pointer is as good as any)
bool wide_rows(const ghd_ctx* c, const float* rows) { return c->cfg.vocab % 4 == 0 && ((uintptr_t)rows & 15) == 0; }
// log2(e) / temperature
double scale_of(float temperature) { return 1.44269504088896340736 / (double)temperature; }

ghd_status raise_room(ghd_ctx* c) {              // (a CTA with all segments of the largest vocabulary takes 64 KB)
    if (c->attr_sampling) return GHD_OK;
    const void* drafts[] = {(const void*)k_draft_sample<3, false>, (const void*)k_draft_sample<4, false>, (const void*)k_draft_sample<4, true>};
    const void* walks[] = {(const void*)k_accept_sampled<true, false>, (const void*)k_accept_sampled<false, false>, (const void*)k_accept_sampled<true, true>, (const void*)k_accept_sampled<false, true>};
    for (const void* f : drafts)
        if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)room_for(MAX_VOCAB, 1)) != cudaSuccess) return check_cuda(c, "sampling: shared memory");
    for (const void* f : walks)
        if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MAX_ROOM) != cudaSuccess) return check_cuda(c, "sampling: shared memory");
    c->attr_sampling = true;
    return GHD_OK;
}

}  // namespace

}  // namespace ghd

using namespace ghd;

extern "C" {

ghd_status ghd_draft_sample(ghd_ctx* c, const float* logits, int32_t n_rows, float temperature, int32_t n_draws, const float* uniforms, int32_t* cand) {
    if (!c) return GHD_EINVAL;
    if (n_rows < 0 || n_draws < 1 || n_draws > GHD_MAX_TOPK) return fail(c, GHD_EINVAL, "draft_sample: negative n_rows, or n_draws outside [1, 16]");
    if (!(temperature > 0.f) || !(temperature <= 0x1p64f)) return fail(c, GHD_EINVAL, "draft_sample: temperature outside (0, 2^64]");
    if (c->cfg.vocab > MAX_VOCAB) return fail(c, GHD_ESHAPE, "draft_sample: a vocabulary above 2^20");
    if (n_rows == 0) return GHD_OK;
    if (n_rows > (1 << 24)) return fail(c, GHD_EINVAL, "draft_sample: more than 2^24 rows");
    if (!logits || !uniforms || !cand) return fail(c, GHD_EINVAL, "draft_sample: null pointer");
    if (!c->ws) return fail(c, GHD_ENOSPACE, "no workspace set");
    OnDevice dev(c);
    const bool many = n_rows > 3 * c->sm_count;
    const int k = cluster_for(c, n_rows, c->cfg.vocab, many ? 4 : 3);
    ghd_status s = raise_room(c);
    if (s != GHD_OK) return s;
    const double scale = scale_of(temperature);
    launch_kc(c, false, k, scale > COLD_SCALE ? k_draft_sample<4, true> : many ? k_draft_sample<4, false> : k_draft_sample<3, false>, n_rows * k, THREADS, room_for(c->cfg.vocab, k), logits, c->cfg.vocab,
              wide_rows(c, logits), k, scale, n_draws, uniforms, cand, c->input_status);
    return check_cuda(c, "draft_sample");
}

ghd_status ghd_accept_sampled(ghd_ctx* c, const ghd_sampled* a, ghd_accept_result* results_dev) {
    if (!c || !a) return GHD_EINVAL;
    if (a->n_seqs < 1 || a->n_seqs > GHD_MAX_SEQS || a->n_rows < 0) return fail(c, GHD_EINVAL, "accept_sampled: n_seqs outside [1, 1024] or negative n_rows");
    if (!a->row_start && a->n_seqs != 1) return fail(c, GHD_EINVAL, "accept_sampled: several sequences without row_start");
    if (!a->row_start && a->n_rows > GHD_MAX_NODES) return fail(c, GHD_ETREE, "accept_sampled: a tree of more than 256 nodes");
    if (!(a->temperature > 0.f) || !(a->temperature <= 0x1p64f)) return fail(c, GHD_EINVAL, "accept_sampled: temperature outside (0, 2^64]");
    if (c->cfg.vocab > MAX_VOCAB) return fail(c, GHD_ESHAPE, "accept_sampled: a vocabulary above 2^20");
    if (!results_dev || (a->n_rows > 0 && (!a->parent || !a->tokens || !a->logits || !a->uniforms))) return fail(c, GHD_EINVAL, "accept_sampled: null pointer");
    if ((a->draft_row == nullptr) != (a->draft_logits == nullptr)) return fail(c, GHD_EINVAL, "accept_sampled: give both draft_row and draft_logits or neither");
    if (a->draft_row && (a->n_draft < 1 || !(a->draft_temperature > 0.f) || !(a->draft_temperature <= 0x1p64f)))
        return fail(c, GHD_EINVAL, "accept_sampled: no draft rows, or a draft temperature outside (0, 2^64]");
    if (!c->ws) return fail(c, GHD_ENOSPACE, "no workspace set");
    OnDevice dev(c);
    const int k = cluster_for(c, a->n_seqs, c->cfg.vocab, 2);
    ghd_status s = raise_room(c);
    if (s != GHD_OK) return s;
    c->entry_fresh = 1;
    const double scale = scale_of(a->temperature), draft_scale = a->draft_row ? scale_of(a->draft_temperature) : 0.0;
    // P and Q of a node's rows are kept from one rejected draw to the next where two CTAs' worth fits into a SM (trees of 64 nodes over 32000
    // tokens, us without / with: one 31 / 29.5, 48 of them 88 / 81)
    const size_t room = (room_for(c->cfg.vocab, k) + 15) / 16 * 16, keeps = keep_for(c->cfg.vocab, k);
    const bool keep = a->draft_row && room + keeps <= MAX_ROOM;
    const int keep_at = keep ? (int)(room / sizeof(double)) : 0;
    const bool wide = wide_rows(c, a->logits) && wide_rows(c, a->draft_logits);
    const bool cold = scale > COLD_SCALE || draft_scale > COLD_SCALE;
    const int64_t segs = ((int64_t)a->n_rows + (a->draft_row ? a->n_draft : 0)) * ((c->cfg.vocab + SEG - 1) / SEG);
    if (segs > 0 && segs <= SAMPLE_SEGS) {
        const int64_t most = 4 * c->sm_count, ctas = (segs + WARPS - 1) / WARPS;
        launch_k(c, false, cold ? k_row_segments<true> : k_row_segments<false>, (int)(ctas < most ? ctas : most), THREADS, 0, a->logits, a->draft_logits, a->n_rows, a->draft_row ? a->n_draft : 0, c->cfg.vocab, wide, scale, draft_scale,
                 (double2*)c->sample_segs);
        launch_kc(c, true, k, cold ? k_accept_sampled<true, true> : k_accept_sampled<true, false>, a->n_seqs * k, THREADS, room + (keep ? keeps : 0), *a, c->cfg.vocab, wide, scale, draft_scale, k, keep_at, (const double2*)c->sample_segs, results_dev, c->input_status);
    } else {
        launch_kc(c, false, k, cold ? k_accept_sampled<false, true> : k_accept_sampled<false, false>, a->n_seqs * k, THREADS, room + (keep ? keeps : 0), *a, c->cfg.vocab, wide, scale, draft_scale, k, keep_at, (const double2*)nullptr, results_dev, c->input_status);
    }
    return check_cuda(c, "accept_sampled");
}

}  // extern "C"
