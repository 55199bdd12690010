// Sampling from logits with given random numbers: candidates drawn without replacement, and the verification of drafted
// tokens against the target's probabilities.
//
// A row of logits is one distribution, w_s = exp((l_s - max) / temperature), in 64 bits: a token is decided by where a random
// number falls between running sums of up to 2^17 weights, whose borders 32 bits would move.
//
// The tokens lie in segments of 256 (32 lanes with 8 neighbours each; more in vocabularies above 2^20), the segments in equal
// shares over the CTAs of a cluster, in order.  One pass over a row leaves the weight of every segment, relative to the segment's largest
// logit until the row's is known: what the CTAs have to know of each other (a maximum, a sum) goes through distributed shared memory,
// one cluster barrier for each exchange.  Where a random number falls is then looked up over the CTAs, over a CTA's segments, over the
// lanes of one segment and over a lane's tokens, so that only one segment's weights are worked out again.
#include <cfloat>
#include <cstdio>

#include "internal.h"
#include "tc_common.cuh"

namespace ghd {

namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_SEGS = 4096;                  // of a row
constexpr int RUN = 8;                          // tokens of a lane worked on together
constexpr int VALUES = 4;                       // doubles that one exchange carries

struct Shared {
    double box[2][MAX_CLUSTER][VALUES];         // exchanges, by turns: what the CTAs of the cluster have sent
    double part[2][WARPS][2];                   // largest logit and weight of every warp's segments, of two rows
    double mine[VALUES];                        // what this CTA sends
    double share[MAX_CLUSTER];                  // weights of the CTAs' shares of the row
    uint32_t child[GHD_MAX_NODES / 32];         // children of the node, a bit each
    int32_t parent[GHD_MAX_NODES];
    int32_t gone[GHD_MAX_NODES];                // tokens that are not in the distribution any more
    int32_t token;
};

__device__ __forceinline__ void send(double* p, uint32_t rank, double v) {
    const uint32_t at = tc::mapa_shared(tc::smem_u32(p), rank);
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(v) : "memory");
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
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

// exp(l * scale - z), the product rounded before the difference: equal logits are equally likely however large they are
__device__ __forceinline__ double weight(float l, double scale, double z) { return exp(__dsub_rn(__dmul_rn((double)l, scale), z)); }

// One row's distribution: exp(l * scale - max) / sum, scale = 1 / temperature.
struct Dist {
    const float* row;
    double scale, max, inv_sum;
    bool ok;
    __device__ __forceinline__ double of(float l) const { return weight(l, scale, max) * inv_sum; }
    __device__ __forceinline__ double at(int t) const { return of(__ldg(row + t)); }
};

// This CTA's share of a row, and what the cluster has agreed on so far.
struct Team {
    Shared* s;
    double* seg;                                // [own segments] weights
    int rank, size, turn, warp, lane;
    int vocab, run, wide;                       // tokens of a lane in a segment (a multiple of RUN); rows on 16-byte boundaries
    int seg0, segs;                             // own segments

    __device__ Team(Shared* sm, double* weights, int vocab_, int run_, int cluster) : s(sm), seg(weights), size(cluster), turn(0), vocab(vocab_), run(run_) {
        rank = cluster > 1 ? (int)tc::cluster_ctarank() : 0;
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        wide = vocab % 4 == 0;
        const int n = (vocab + 32 * run - 1) / (32 * run);
        seg0 = (int)((long long)n * rank / cluster);
        segs = (int)((long long)n * (rank + 1) / cluster) - seg0;
        if (cluster > 1) tc::cluster_sync_all();                   // everybody's shared memory is there
    }
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
    __device__ __forceinline__ int first_of(int sg) const { return (sg * 32 + lane) * run; }       // this lane's first token of a segment
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
        double sum = 0.0;
        for (int r = 0; r < size; ++r) sum += box[r][0];
        if (threadIdx.x < (unsigned)size) s->share[threadIdx.x] = box[threadIdx.x][0];
        __syncthreads();
        return sum;
    }
};

// Maximum and sum of a row p and, if q.row is given, of a second one.  seg[] is left with p's weights (not divided by the sum),
// share[] has every CTA's part of p's sum.
__device__ void measure(Team& m, Dist& p, Dist& q) {
    const int n = q.row ? 2 : 1;
#pragma unroll 1
    for (int i = n - 1; i >= 0; --i) {
        const float* row = i ? q.row : p.row;
        const double scale = i ? q.scale : p.scale;
        // of the warp's segments: the largest logit so far, and the weight relative to it
        float top = -INFINITY;
        double all = 0.0;
#pragma unroll 1
        for (int g = m.warp; g < m.segs; g += WARPS) {
            float high = -INFINITY;
            double sum = 0.0;
#pragma unroll 1
            for (int c = 0; c < m.run; c += RUN) {
                float x[RUN];
                m.load(row, m.first_of(m.seg0 + g) + c, x);
                float now = x[0];
#pragma unroll
                for (int e = 1; e < RUN; ++e) now = fmaxf(now, x[e]);
                now = fmaxf(high, warp_max(now));                              // (a NaN is left out of the maximum, and makes the sum one)
                const double z = (double)now * scale;
                double add = 0.0;
#pragma unroll
                for (int e = 0; e < RUN; ++e) add += x[e] == -INFINITY ? 0.0 : weight(x[e], scale, z);
                sum = (high == -INFINITY ? sum : sum * weight(high, scale, z)) + warp_sum(add);
                high = now;
            }
            if (i == 0 && m.lane == 0) m.seg[g] = sum;
            if (i == 0 && m.lane == 0) m.seg[m.segs + g] = (double)high * scale;
            const float now = fmaxf(top, high);
            const double z = (double)now * scale;
            all = (top == -INFINITY ? all : all * weight(top, scale, z)) + (high == -INFINITY ? sum : sum * weight(high, scale, z));
            top = now;
        }
        if (m.lane == 0) { m.s->part[i][m.warp][0] = (double)top * scale; m.s->part[i][m.warp][1] = all; }
    }
    __syncthreads();
    if (m.warp < n) {                                            // the warps' results of row `warp`
        double best = m.lane < WARPS ? m.s->part[m.warp][m.lane][0] : -INFINITY;
        const double a = best, b = m.lane < WARPS ? m.s->part[m.warp][m.lane][1] : 0.0;
#pragma unroll
        for (int o = 16; o; o >>= 1) best = fmax(best, __shfl_xor_sync(0xffffffffu, best, o));
        const double all = warp_sum(a == -INFINITY ? b : b * exp(a - best));       // (b is 0 or NaN where there is no maximum)
        if (m.lane == 0) { m.s->mine[2 * m.warp] = best; m.s->mine[2 * m.warp + 1] = all; }
    }
    double (*box)[VALUES] = m.exchange(2 * n);
    const int r = m.lane < m.size ? m.lane : 0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        const double a = box[r][2 * i], b = box[r][2 * i + 1];
        double best = a;
#pragma unroll
        for (int o = 16; o; o >>= 1) best = fmax(best, __shfl_xor_sync(0xffffffffu, best, o));
        double share = m.lane < m.size ? (a == -INFINITY ? b : b * exp(a - best)) : 0.0;
        double sum = 0.0;
        for (int k = 0; k < m.size; ++k) sum += __shfl_sync(0xffffffffu, share, k);
        Dist& d = i ? q : p;
        d.max = best;
        d.inv_sum = 1.0 / sum;
        d.ok = best > -INFINITY && best < INFINITY && sum < INFINITY;
        if (i == 0 && m.warp == 0 && m.lane < m.size) m.s->share[m.lane] = share;
    }
    for (int g = threadIdx.x; g < m.segs; g += THREADS) {
        const double z = m.seg[m.segs + g];
        m.seg[g] = z == -INFINITY ? 0.0 : m.seg[g] * exp(z - p.max);
    }
    __syncthreads();
}

// The weights w(logit of p, logit of q, token) of every own segment into seg[], of the CTAs' shares into share[] -> the total.
template <typename W>
__device__ double total_of(Team& m, const float* p, const float* q, W w) {
    double all = 0.0;
#pragma unroll 1
    for (int g = m.warp; g < m.segs; g += WARPS) {
        double sum = 0.0;
#pragma unroll 1
        for (int c = 0; c < m.run; c += RUN) {
            float x[RUN], y[RUN];
            const int t = m.first_of(m.seg0 + g) + c;
            m.load(p, t, x);
            if (q) m.load(q, t, y);
#pragma unroll
            for (int e = 0; e < RUN; ++e) sum += t + e < m.vocab ? w(x[e], q ? y[e] : 0.f, t + e) : 0.0;
        }
        sum = warp_sum(sum);
        if (m.lane == 0) m.seg[g] = sum;
        all += sum;
    }
    if (m.lane == 0) m.s->part[0][m.warp][0] = all;
    __syncthreads();
    if (m.warp == 0) {
        const double sum = warp_sum(m.lane < WARPS ? m.s->part[0][m.lane][0] : 0.0);
        if (m.lane == 0) m.s->mine[0] = sum;
    }
    return m.add_shares(m.exchange(1));
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

// One warp: the first token whose running sum, `before` and seg[] in front, exceeds the target; weights as in total_of.  All lanes get it.
template <typename W>
__device__ int look_up(Team& m, double before, double target, const float* p, const float* q, W w) {
    // the segment
    int found = -1, held = -1;
    double start = before, held_start = before;
#pragma unroll 1
    for (int g0 = 0; g0 < m.segs && found < 0; g0 += 32) {
        const double x = g0 + m.lane < m.segs ? m.seg[g0 + m.lane] : 0.0;
        const double run = before + warp_scan(x, m.lane);
        const uint32_t over = __ballot_sync(0xffffffffu, x > 0.0 && run > target), some = __ballot_sync(0xffffffffu, x > 0.0);
        if (some) {
            const int k = 31 - __clz(some);
            held = g0 + k;
            held_start = __shfl_sync(0xffffffffu, run - x, k);
        }
        if (over) {
            const int k = __ffs(over) - 1;
            found = g0 + k;
            start = __shfl_sync(0xffffffffu, run - x, k);
        }
        before = __shfl_sync(0xffffffffu, run, 31);
    }
    if (found < 0) { found = held; start = held_start; }
    if (found < 0) return -1;
    // the lane, and the token
    double sum = 0.0;
    const int t0 = m.first_of(m.seg0 + found);
    auto weigh = [&](auto f) {
#pragma unroll 1
        for (int c = 0; c < m.run; c += RUN) {
            float x[RUN], y[RUN];
            m.load(p, t0 + c, x);
            if (q) m.load(q, t0 + c, y);
#pragma unroll
            for (int e = 0; e < RUN; ++e) f(t0 + c + e, t0 + c + e < m.vocab ? w(x[e], q ? y[e] : 0.f, t0 + c + e) : 0.0);
        }
    };
    weigh([&](int, double x) { sum += x; });
    const double run = start + warp_scan(sum, m.lane);
    const uint32_t over = __ballot_sync(0xffffffffu, sum > 0.0 && run > target), some = __ballot_sync(0xffffffffu, sum > 0.0);
    if (!some) return -1;
    const int k = over ? __ffs(over) - 1 : 31 - __clz(some);
    double at = run - sum;
    int token = -1, last = -1;
    weigh([&](int t, double x) {
        at += x;
        if (x > 0.0) last = t;
        if (token < 0 && x > 0.0 && at > target) token = t;
    });
    return __shfl_sync(0xffffffffu, token < 0 ? last : token, k);
}

// seg[] and share[] after measure(), without the tokens gone[0 .. n) -> the total
__device__ double total_without(Team& m, const Dist& p, int n) {
    __syncthreads();
#pragma unroll 1
    for (int i = m.warp; i < n; i += WARPS) {
        const int g = m.s->gone[i] / (32 * m.run) - m.seg0;
        bool first = g >= 0 && g < m.segs;                       // one warp to a segment, that of the first of its tokens
        for (int k = 0; k < i && first; ++k) first = m.s->gone[k] / (32 * m.run) - m.seg0 != g;
        if (!first) continue;
        double sum = 0.0;
#pragma unroll 1
        for (int c = 0; c < m.run; c += RUN) {
            float x[RUN];
            const int t = m.first_of(m.seg0 + g) + c;
            m.load(p.row, t, x);
#pragma unroll
            for (int e = 0; e < RUN; ++e) {
                double y = t + e < m.vocab ? p.of(x[e]) : 0.0;
                for (int k = 0; k < n; ++k) y = m.s->gone[k] == t + e ? 0.0 : y;
                sum += y;
            }
        }
        sum = warp_sum(sum);
        if (m.lane == 0) m.seg[g] = sum;
    }
    __syncthreads();
    if (m.warp == 0) {
        double sum = 0.0;
        for (int g = m.lane; g < m.segs; g += 32) sum += m.seg[g];
        sum = warp_sum(sum);
        if (m.lane == 0) m.s->mine[0] = sum;
    }
    return m.add_shares(m.exchange(1));
}

// random numbers are held in [0, 1 - 2^-24]
__device__ __forceinline__ double unit(float u) { return (double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }

// ---------------------------------------------------------------- candidates
// The CTA in whose share a draw falls is not the same every time, but what it takes to find the token is one segment's logits: when the
// shares are known the first CTA gets all segments' weights and draws alone, with one warp.
__global__ void __launch_bounds__(THREADS) k_draft_sample(const float* __restrict__ logits, int vocab, int run, int cluster, double scale, int draws,
                                                          const float* __restrict__ uniforms, int32_t* __restrict__ cand, int* status) {
    extern __shared__ double weights[];
    __shared__ Shared sm;
    Team m(&sm, weights, vocab, run, cluster);
    const int row = blockIdx.x / cluster;
    Dist p{logits + (size_t)row * vocab, scale, 0.0, 1.0, false}, none{};
    measure(m, p, none);
    const int n = (vocab + 32 * run - 1) / (32 * run);
    if (cluster > 1) {
        // (in the first CTA the room behind its own segments is free by now: measure's last barrier)
        tc::cluster_sync_all();
        if (m.rank > 0)
            for (int g = threadIdx.x; g < m.segs; g += THREADS) send(weights + m.seg0 + g, 0, weights[g]);
        tc::cluster_sync_all();
    }
    if (m.rank > 0 || m.warp > 0) return;
    m.segs = n;
    if (!p.ok && m.lane == 0) atomicCAS(status, DEV_OK, DEV_SAMPLE_DIST);
    p.inv_sum = 1.0;                                           // the weights as they are
    int out = -1, n_gone = 0;
#pragma unroll 1
    for (int j = 0; j < draws && p.ok; ++j) {
        double total = 0.0;
        for (int g = m.lane; g < n; g += 32) total += weights[g];
        total = warp_sum(total);
        if (!(total > 0.0)) break;                             // nothing is left
        auto w = [&](float l, float, int t) {
            double x = p.of(l);
            for (int g = 0; g < n_gone; ++g) x = sm.gone[g] == t ? 0.0 : x;
            return x;
        };
        const int t = look_up(m, 0.0, unit(__ldg(uniforms + (size_t)row * GHD_MAX_TOPK + j)) * total, p.row, nullptr, w);
        if (t < 0) break;
        if (m.lane == j) out = t;
        if (m.lane == 0) sm.gone[n_gone] = t;
        ++n_gone;
        __syncwarp();
        // the segment's weight without it
        const int sg = t / (32 * run);
        double sum = 0.0;
#pragma unroll 1
        for (int c = 0; c < run; c += RUN) {
            float x[RUN];
            const int t0 = m.first_of(sg) + c;
            m.load(p.row, t0, x);
#pragma unroll
            for (int e = 0; e < RUN; ++e) sum += t0 + e < vocab ? w(x[e], 0.f, t0 + e) : 0.0;
        }
        sum = warp_sum(sum);
        if (m.lane == 0) weights[sg] = sum;
        __syncwarp();
    }
    if (m.lane < GHD_MAX_TOPK) cand[(size_t)row * GHD_MAX_TOPK + m.lane] = out;
}

// ---------------------------------------------------------------- verification
// A walk from the root.  At a node with target distribution P and draft distribution Q its children are looked at in order, with
// P_1 = P, Q_1 = Q: child x is accepted if u Q_j(x) < P_j(x); otherwise P_{j+1} = max(P_j - Q_j, 0) / its sum and Q_{j+1} = Q_j
// without x / its sum.  Written out, P_j = max(P - beta_j Q, 0) / W_j with W_j its sum: subtracting Q_j = c_j Q from that gives
// beta_{j+1} = beta_j + c_j W_j, and c_j = 1 / (1 - Q(rejected)).  A rejected token has u Q_j >= P_j, u < 1, so P_{j+1} gives it
// nothing, and so do all later ones: beta only grows.  So two numbers are kept instead of two distributions, and a rejection costs
// one sum over the vocabulary.  Candidates that nobody drew have Q = 1 at themselves: P_{j+1} is P_j without x.
__global__ void __launch_bounds__(THREADS) k_accept_sampled(ghd_sampled a, int vocab, int run, int cluster, ghd_accept_result* __restrict__ results, int* status) {
    extern __shared__ double weights[];
    __shared__ Shared sm;
    Team m(&sm, weights, vocab, run, cluster);
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
    }
    __syncthreads();
    int node = 0, depth = 0;
    while (n > 0) {
        if (threadIdx.x < GHD_MAX_NODES) {
            const uint32_t b = __ballot_sync(0xffffffffu, (int)threadIdx.x > node && sm.parent[threadIdx.x] == node);
            if (m.lane == 0) sm.child[m.warp] = b;
        }
        __syncthreads();
        bool any = false;
        for (int i = 0; i < GHD_MAX_NODES / 32; ++i) any |= sm.child[i] != 0;
        int drawn = a.draft_row ? __ldg(a.draft_row + first + node) : -1;
        if (drawn >= a.n_draft) {
            record(DEV_SAMPLE_DRAFT);
            drawn = -1;
        }
        Dist p{a.logits + (size_t)(first + node) * vocab, 1.0 / (double)a.temperature, 0.0, 1.0, false}, q{};
        if (any && drawn >= 0) { q.row = a.draft_logits + (size_t)drawn * vocab; q.scale = 1.0 / (double)a.draft_temperature; }
        measure(m, p, q);
        if (!p.ok || (q.row && !q.ok)) record(DEV_SAMPLE_DIST);
        double beta = 0.0, W = 1.0, rejected = 0.0;
        int n_gone = 0, next = -1;
        bool fresh = false;                                    // seg[] and share[] are of the weights as they are, their total is W
        auto left = [&](float lp, float lq, int t) {
            const double x = p.of(lp);
            if (q.row) return fmax(x - beta * q.of(lq), 0.0);
            return x;
        };
        if (p.ok && (!q.row || q.ok))
            for (int word = 0; word < GHD_MAX_NODES / 32 && next < 0; ++word)
                for (uint32_t bits = sm.child[word]; bits; bits &= bits - 1) {
                    const int c = 32 * word + __ffs(bits) - 1, x = __ldg(a.tokens + first + c);
                    if (x < 0 || x >= vocab) continue;
                    const double u = unit(__ldg(a.uniforms + first + c)), px = p.at(x);
                    if (q.row) {
                        const double qx = q.at(x);
                        bool before = false;                   // a token that was rejected already is not drawn again
                        for (int g = 0; g < n_gone; ++g) before |= sm.gone[g] == x;
                        if (!(qx > 0.0) || before) continue;
                        const double c_j = 1.0 / fmax(1.0 - rejected, qx);
                        if (!(W > 0.0)) break;
                        if (u * qx * c_j * W < fmax(px - beta * qx, 0.0)) { next = c; break; }
                        beta += c_j * W;
                        rejected += qx;
                        W = total_of(m, p.row, q.row, left);
                        fresh = true;
                    } else {
                        bool before = false;
                        for (int g = 0; g < n_gone; ++g) before |= sm.gone[g] == x;
                        if (before) continue;
                        if (u * fmax(1.0 - rejected, px) < px) { next = c; break; }
                        rejected += px;
                    }
                    __syncthreads();
                    if (threadIdx.x == 0) sm.gone[n_gone] = x;
                    ++n_gone;
                    __syncthreads();
                }
        if (next < 0) {
            if (!p.ok) {
                if (writes) out->tokens[depth] = 0;
            } else {
                // What is left of P: after rejected draws the weights of the last sum; otherwise P's own segments (not divided by the sum),
                // those with a token that is gone weighed again.
                if (fresh && !(W > 0.0)) {
                    beta = 0.0;
                    fresh = false;
                    W = total_of(m, p.row, q.row, left);
                    fresh = true;
                }
                double total = W;
                if (!fresh) {
                    p.inv_sum = 1.0;
                    if (n_gone == 0 || q.row) {
                        total = 0.0;
                        for (int r = 0; r < m.size; ++r) total += m.s->share[r];
                        n_gone = 0;
                    } else {
                        total = total_without(m, p, n_gone);
                    }
                }
                const double target = unit(__ldg(a.uniforms + first)) * total;
                double before;
                if (own_share(m, target, before) && m.warp == 0) {
                    auto w = [&](float lp, float lq, int t) {
                        if (q.row && fresh) return left(lp, lq, t);
                        double x = p.of(lp);
                        for (int g = 0; g < n_gone; ++g) x = sm.gone[g] == t ? 0.0 : x;
                        return x;
                    };
                    const int t = look_up(m, before, target, p.row, fresh ? q.row : nullptr, w);
                    if (m.lane == 0) out->tokens[depth] = t;
                }
            }
            break;
        }
        if (writes) {
            out->tokens[depth] = __ldg(a.tokens + first + next);
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
    if (cluster > 1) tc::cluster_sync_all();
}

// CTAs to a row: as many as leave each of them a SM of its own and four segments to every warp's one
int cluster_for(const ghd_ctx* c, int rows, int vocab) {
    int k = MAX_CLUSTER;
    while (k > 1 && ((int64_t)k * rows > c->sm_count || vocab < 1024 * k)) k >>= 1;
    return k;
}
int run_for(int vocab) { return RUN * (int)(((int64_t)vocab + MAX_SEGS * 32 * RUN - 1) / (MAX_SEGS * 32 * RUN)); }
// room for a CTA's segments twice over (measure), and in a row's first CTA for all of them
size_t room_for(int vocab, int run, int cluster) {
    const size_t n = ((size_t)vocab + 32 * run - 1) / (32 * run), own = (n + cluster - 1) / cluster;
    return sizeof(double) * (2 * own > n ? 2 * own : n);
}

ghd_status raise_room(ghd_ctx* c) {              // (a CTA with all of 4096 segments takes 64 KB)
    if (c->attr_sampling) return GHD_OK;
    if (cudaFuncSetAttribute(k_draft_sample, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * MAX_SEGS * (int)sizeof(double)) != cudaSuccess ||
        cudaFuncSetAttribute(k_accept_sampled, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * MAX_SEGS * (int)sizeof(double)) != cudaSuccess)
        return check_cuda(c, "sampling: shared memory");
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
    if (!(temperature > 0.f) || !(temperature <= FLT_MAX)) return fail(c, GHD_EINVAL, "draft_sample: temperature is not a positive number");
    if (n_rows == 0) return GHD_OK;
    if (n_rows > (1 << 24)) return fail(c, GHD_EINVAL, "draft_sample: more than 2^24 rows");
    if (!logits || !uniforms || !cand) return fail(c, GHD_EINVAL, "draft_sample: null pointer");
    if (!c->ws) return fail(c, GHD_ENOSPACE, "no workspace set");
    const int k = cluster_for(c, n_rows, c->cfg.vocab);
    const int run = run_for(c->cfg.vocab);
    ghd_status s = raise_room(c);
    if (s != GHD_OK) return s;
    launch_kc(c, false, k, k_draft_sample, n_rows * k, THREADS, room_for(c->cfg.vocab, run, k), logits, c->cfg.vocab, run, k, 1.0 / (double)temperature, n_draws, uniforms, cand, c->input_status);
    return check_cuda(c, "draft_sample");
}

ghd_status ghd_accept_sampled(ghd_ctx* c, const ghd_sampled* a, ghd_accept_result* results_dev) {
    if (!c || !a) return GHD_EINVAL;
    if (a->n_seqs < 1 || a->n_seqs > GHD_MAX_SEQS || a->n_rows < 0) return fail(c, GHD_EINVAL, "accept_sampled: n_seqs outside [1, 1024] or negative n_rows");
    if (!a->row_start && a->n_seqs != 1) return fail(c, GHD_EINVAL, "accept_sampled: several sequences without row_start");
    if (!a->row_start && a->n_rows > GHD_MAX_NODES) return fail(c, GHD_ETREE, "accept_sampled: a tree of more than 256 nodes");
    if (!(a->temperature > 0.f) || !(a->temperature <= FLT_MAX)) return fail(c, GHD_EINVAL, "accept_sampled: temperature is not a positive number");
    if (!results_dev || (a->n_rows > 0 && (!a->parent || !a->tokens || !a->logits || !a->uniforms))) return fail(c, GHD_EINVAL, "accept_sampled: null pointer");
    if ((a->draft_row == nullptr) != (a->draft_logits == nullptr)) return fail(c, GHD_EINVAL, "accept_sampled: give both draft_row and draft_logits or neither");
    if (a->draft_row && (a->n_draft < 1 || !(a->draft_temperature > 0.f) || !(a->draft_temperature <= FLT_MAX)))
        return fail(c, GHD_EINVAL, "accept_sampled: no draft rows, or a draft temperature that is not a positive number");
    if (!c->ws) return fail(c, GHD_ENOSPACE, "no workspace set");
    const int k = cluster_for(c, a->n_seqs, c->cfg.vocab);
    const int run = run_for(c->cfg.vocab);
    ghd_status s = raise_room(c);
    if (s != GHD_OK) return s;
    launch_kc(c, false, k, k_accept_sampled, a->n_seqs * k, THREADS, room_for(c->cfg.vocab, run, k), *a, c->cfg.vocab, run, k, results_dev, c->input_status);
    return check_cuda(c, "accept_sampled");
}

}  // extern "C"
