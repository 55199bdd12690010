// Sampling from logits with given random numbers: candidates drawn without replacement, and the verification of drafted
// tokens against the target's probabilities.
//
// A row of logits is one distribution, w_s = exp((l_s - max) / temperature), in 64 bits: a token is decided by where a random
// number falls between running sums of up to 2^17 weights, whose borders 32 bits would move.  A cluster of CTAs works on a row;
// every warp owns a run of consecutive tokens, so that running sums are in the order of the tokens: over CTAs, over warps,
// and inside one warp's run, 32 tokens at a time.  What the CTAs have to know of each other (a maximum, a few sums) goes
// through distributed shared memory, one cluster barrier for each.
#include <cfloat>
#include <cstdio>

#include "internal.h"
#include "tc_common.cuh"

namespace ghd {

namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_CLUSTER = 8;
constexpr int VALUES = 4;                       // doubles that one exchange carries

struct Shared {
    double box[2][MAX_CLUSTER][VALUES];         // exchanges, by turns: what the CTAs of the cluster have sent
    double part[WARPS][2];                      // a value of every warp
    double run[WARPS];                          // weights of the warps' runs
    uint32_t child[GHD_MAX_NODES / 32];         // children of the node, a bit each
    int32_t parent[GHD_MAX_NODES];
    int32_t gone[GHD_MAX_NODES];                // tokens that are not in the distribution any more
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
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
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

// The tokens of this thread's warp, and what the cluster has agreed on so far.
struct Team {
    Shared* s;
    int rank, size, turn, warp, lane;
    int beg, end;                               // the warp's run

    __device__ Team(Shared* sm, int vocab, int cluster) : s(sm), size(cluster), turn(0) {
        rank = cluster > 1 ? (int)tc::cluster_ctarank() : 0;
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        const int per = ((vocab + cluster * WARPS - 1) / (cluster * WARPS) + 31) & ~31;       // whole 128-byte lines
        beg = min(vocab, (rank * WARPS + warp) * per);
        end = min(vocab, beg + per);
        if (cluster > 1) tc::cluster_sync_all();                   // everybody's shared memory is there
    }
    // v[0 .. n) of every CTA (thread 0's), to be read from the returned box by everyone: one barrier of the cluster.
    // The box of the exchange before is still being read; the one before that has been left by everybody.
    __device__ double (*exchange(const double* v, int n))[VALUES] {
        double (*box)[VALUES] = s->box[turn];
        if (threadIdx.x < (unsigned)(size * n)) {
            const int to = threadIdx.x / n, i = threadIdx.x % n;
            if (size > 1) send(&box[rank][i], (uint32_t)to, v[i]);
            else box[0][i] = v[i];
        }
        if (size > 1) tc::cluster_sync_all();
        else __syncthreads();
        turn ^= 1;
        return box;
    }
};

// exp((l - max) / temperature) / sum over one row
struct Dist {
    const float* row;
    double temp, max, sum;      // max: divided by the temperature
    bool ok;
    __device__ __forceinline__ double at(int t) const { return exp((double)__ldg(row + t) / temp - max) / sum; }
};

// Maximum and sum of one row or of two (q.row null: one).
__device__ void measure(Team& m, Dist& p, Dist& q) {
    double top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0, 0.0};
    const float* rows[2] = {p.row, q.row};
    const double temps[2] = {p.temp, q.temp};
    const int n = q.row ? 2 : 1;
    for (int i = 0; i < n; ++i) {
        float x = -INFINITY;
        for (int t = m.beg + m.lane; t < m.end; t += 32) x = fmaxf(x, __ldg(rows[i] + t));
        top[i] = warp_max((double)x / temps[i]);
        // (a NaN is left out of the maximum, and makes the sum one)
        for (int t = m.beg + m.lane; t < m.end; t += 32) {
            const float l = __ldg(rows[i] + t);
            sum[i] += l == -INFINITY ? 0.0 : exp((double)l / temps[i] - top[i]);
        }
        sum[i] = warp_sum(sum[i]);
    }
    __shared__ double v[VALUES];
    for (int i = 0; i < n; ++i) {
        __syncthreads();
        if (m.lane == 0) { m.s->part[m.warp][0] = top[i]; m.s->part[m.warp][1] = sum[i]; }
        __syncthreads();
        if (m.warp == 0) {
            const double a = m.lane < WARPS ? m.s->part[m.lane][0] : -INFINITY, b = m.lane < WARPS ? m.s->part[m.lane][1] : 0.0;
            const double best = warp_max(a);
            const double all = warp_sum(a == -INFINITY ? b : b * exp(a - best));       // (b is 0 or NaN where there is no maximum)
            if (m.lane == 0) { v[2 * i] = best; v[2 * i + 1] = all; }
        }
    }
    __syncthreads();
    double (*box)[VALUES] = m.exchange(v, 2 * n);
    for (int i = 0; i < n; ++i) {
        double best = -INFINITY, all = 0.0;
        for (int r = 0; r < m.size; ++r) best = fmax(best, box[r][2 * i]);
        for (int r = 0; r < m.size; ++r) all += box[r][2 * i] == -INFINITY ? box[r][2 * i + 1] : box[r][2 * i + 1] * exp(box[r][2 * i] - best);
        Dist& d = i ? q : p;
        d.max = best;
        d.sum = all;
        d.ok = best > -INFINITY && best < INFINITY && all < INFINITY;
    }
}

// Sums the weights w(t) of every warp's run and of the cluster -> their total.  run[] keeps the warps' sums.
template <typename W>
__device__ double total_of(Team& m, W w) {
    double sum = 0.0;
    for (int t = m.beg + m.lane; t < m.end; t += 32) sum += w(t);
    sum = warp_sum(sum);
    __shared__ double v[VALUES];
    __syncthreads();
    if (m.lane == 0) m.s->run[m.warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int i = 0; i < WARPS; ++i) all += m.s->run[i];
        v[0] = all;
    }
    __syncthreads();
    double (*box)[VALUES] = m.exchange(v, 1);
    double all = 0.0;
    for (int r = 0; r < m.size; ++r) all += box[r][0];
    return all;
}

// The first token whose running sum exceeds u times the total, after total_of with the same weights: -1 in all CTAs but the one
// that has it (and in that one for all threads but lane 0 of one warp).  Where rounding leaves none, the last one with weight.
template <typename W>
__device__ int pick(Team& m, double total, double u, W w) {
    double (*box)[VALUES] = m.s->box[m.turn ^ 1];
    const double target = u * total;
    int owner = -1, last = -1;
    double before = 0.0, start = 0.0, last_start = 0.0;
    for (int r = 0; r < m.size && owner < 0; ++r) {
        const double x = box[r][0];
        if (x > 0.0) { last = r; last_start = before; }
        if (before + x > target) { owner = r; start = before; }
        before += x;
    }
    if (owner < 0) { owner = last; start = last_start; }
    if (owner != m.rank) return -1;
    int mine = -1;
    last = -1;
    before = start;
    for (int i = 0; i < WARPS && mine < 0; ++i) {
        const double x = m.s->run[i];
        if (x > 0.0) { last = i; last_start = before; }
        if (before + x > target) { mine = i; start = before; }
        before += x;
    }
    if (mine < 0) { mine = last; start = last_start; }
    if (mine != m.warp) return -1;
    int found = -1, held = -1;
    for (int t0 = m.beg; t0 < m.end && found < 0; t0 += 32) {
        const int t = t0 + m.lane;
        const double x = t < m.end ? w(t) : 0.0;
        const double run = start + warp_scan(x, m.lane);
        const uint32_t over = __ballot_sync(0xffffffffu, x > 0.0 && run > target), some = __ballot_sync(0xffffffffu, x > 0.0);
        if (some) held = t0 + 31 - __clz(some);
        if (over) found = t0 + __ffs(over) - 1;
        start = __shfl_sync(0xffffffffu, run, 31);
    }
    if (found < 0) found = held;
    return m.lane == 0 ? found : -1;
}

// random numbers are held in [0, 1 - 2^-24]
__device__ __forceinline__ double unit(float u) { return (double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }

// ---------------------------------------------------------------- candidates
__global__ void __launch_bounds__(THREADS) k_draft_sample(const float* __restrict__ logits, int vocab, int cluster, double temp, int draws,
                                                          const float* __restrict__ uniforms, int32_t* __restrict__ cand, int* status) {
    __shared__ Shared sm;
    __shared__ int32_t token;
    Team m(&sm, vocab, cluster);
    const int row = blockIdx.x / cluster;
    Dist p{logits + (size_t)row * vocab, temp, 0.0, 1.0, false}, none{};
    measure(m, p, none);
    if (!p.ok && m.rank == 0 && threadIdx.x == 0) atomicCAS(status, DEV_OK, DEV_SAMPLE_DIST);
    int n_gone = 0;
    for (int j = 0; j < GHD_MAX_TOPK; ++j) {
        double total = 0.0;
        auto w = [&](int t) {
            for (int g = 0; g < n_gone; ++g)
                if (sm.gone[g] == t) return 0.0;
            return p.at(t);
        };
        if (j < draws && p.ok) total = total_of(m, w);
        if (!(total > 0.0)) {                                  // nothing is left, or no more is asked for
            if (m.rank == 0 && threadIdx.x == 0) cand[(size_t)row * GHD_MAX_TOPK + j] = -1;
            continue;
        }
        if (threadIdx.x == 0) token = -1;
        __syncthreads();
        const int t = pick(m, total, unit(__ldg(uniforms + (size_t)row * GHD_MAX_TOPK + j)), w);
        if (t >= 0) {
            cand[(size_t)row * GHD_MAX_TOPK + j] = t;
            token = t;
        }
        __syncthreads();
        if (token >= 0) {                                      // only this CTA's sums have to know
            if (threadIdx.x == 0) sm.gone[n_gone] = token;
            ++n_gone;
        }
        __syncthreads();
    }
    if (cluster > 1) tc::cluster_sync_all();                   // nobody leaves while others may write to its shared memory
}

// ---------------------------------------------------------------- verification
// A walk from the root.  At a node with target distribution P and draft distribution Q its children are looked at in order, with
// P_1 = P, Q_1 = Q: child x is accepted if u Q_j(x) < P_j(x); otherwise P_{j+1} = max(P_j - Q_j, 0) / its sum and Q_{j+1} = Q_j
// without x / its sum.  Written out, P_j = max(P - beta_j Q, 0) / W_j with W_j its sum: subtracting Q_j = c_j Q from that gives
// beta_{j+1} = beta_j + c_j W_j, and c_j = 1 / (1 - Q(rejected)).  A rejected token has u Q_j >= P_j, u < 1, so P_{j+1} gives it
// nothing, and so do all later ones: beta only grows.  So two numbers are kept instead of two distributions, and a rejection costs
// one sum over the vocabulary.  Candidates that nobody drew have Q = 1 at themselves: P_{j+1} is P_j without x.
__global__ void __launch_bounds__(THREADS) k_accept_sampled(ghd_sampled a, int vocab, int cluster, ghd_accept_result* __restrict__ results, int* status) {
    __shared__ Shared sm;
    Team m(&sm, vocab, cluster);
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
        Dist p{a.logits + (size_t)(first + node) * vocab, (double)a.temperature, 0.0, 1.0, false}, q{};
        if (any && drawn >= 0) { q.row = a.draft_logits + (size_t)drawn * vocab; q.temp = (double)a.draft_temperature; }
        measure(m, p, q);
        if (!p.ok || (q.row && !q.ok)) record(DEV_SAMPLE_DIST);
        double beta = 0.0, W = 1.0, rejected = 0.0;
        int n_gone = 0, next = -1;
        bool fresh = false;                                    // run[] and the last exchange are of the weights as they are
        auto left = [&](int t) {
            const double x = p.at(t);
            if (q.row) return beta > 0.0 ? fmax(x - beta * q.at(t), 0.0) : x;
            for (int g = 0; g < n_gone; ++g)
                if (sm.gone[g] == t) return 0.0;
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
                        W = total_of(m, left);
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
                if (!(W > 0.0)) { beta = 0.0; fresh = false; }
                const double total = fresh ? W : total_of(m, left);
                const int t = pick(m, total, unit(__ldg(a.uniforms + first)), left);
                if (t >= 0) out->tokens[depth] = t;
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

// CTAs to a row: as many as leave each of them a SM of its own and 1024 tokens
int cluster_for(const ghd_ctx* c, int rows, int vocab) {
    int k = MAX_CLUSTER;
    while (k > 1 && ((int64_t)k * rows > c->sm_count || vocab < 1024 * k)) k >>= 1;
    return k;
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
    launch_kc(c, false, k, k_draft_sample, n_rows * k, THREADS, 0, logits, c->cfg.vocab, k, (double)temperature, n_draws, uniforms, cand, c->input_status);
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
    launch_kc(c, false, k, k_accept_sampled, a->n_seqs * k, THREADS, 0, *a, c->cfg.vocab, k, results_dev, c->input_status);
    return check_cuda(c, "accept_sampled");
}

}  // extern "C"
