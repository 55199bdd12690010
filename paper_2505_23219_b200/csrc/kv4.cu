// The paged cache in 4 bits: append (rotation and quantisation on the way), read back, commit, and the C entry points.
#include <cmath>
#include <cstdio>

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

// min and max that keep a NaN (fminf and fmaxf drop it)
__device__ __forceinline__ float min_nan(float a, float b) { return (a != a) ? a : ((b != b) ? b : fminf(a, b)); }
__device__ __forceinline__ float max_nan(float a, float b) { return (a != a) ? a : ((b != b) ? b : fmaxf(a, b)); }

// Scale and minimum of a row whose D values a warp holds, D / 32 a lane.
template <typename T, int N>
__device__ __forceinline__ void row_params(const float (&x)[N], T& scale, T& mn) {
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) { lo = min_nan(lo, x[i]); hi = max_nan(hi, x[i]); }
    for (int o = 16; o > 0; o >>= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    mn = from_f<T>(lo);
    scale = from_f<T>((float)(((double)hi - (double)lo) / 15.0));
}

// Code of x.  The quotient decides between two codes, so it is taken in 64 bits where 32 could fall on the other
// side of a half: 32-bit subtraction and multiplication by a reciprocal are off by less than 2^-20 of the quotient
// (three roundings of 2^-24 and the reciprocal's own), which is below 16; nearer than 2^-15 to a half is redone.
__device__ __forceinline__ uint32_t code_of(float x, float mn, float scale, float inv) {
    if (scale == 0.f) return 0u;
    const float t = (x - mn) * inv;
    float r = rintf(t);
    if (!(fabsf(fabsf(t - r) - 0.5f) > 0x1p-15f) || !(fabsf(t) < 32.f)) r = (float)rint(((double)x - (double)mn) / (double)scale);
    r = fminf(fmaxf(r, 0.f), 15.f);
    return (uint32_t)r;
}

// One row of the call per grid column; the warps of its blocks (blockIdx.y, then warp) share the row's heads: first the K
// heads, then V, then q.  Lane l of a K or q head holds the pairs t = l P .. l P + P - 1 with both halves (P = D / 64), so
// the rotation needs no exchange; of a V head the 2 P channels from 2 P l on.
// The angles of the row (64-bit sincos, D / 2 of them) are worked out once per block.
template <typename T, int D>
__global__ void k_kv4_append(Kv4View w, RopeFreq fr, uint8_t* __restrict__ pool, const int32_t* __restrict__ pos, const T* q, int64_t q_ld,
                             const T* __restrict__ k, const T* __restrict__ v, int64_t kv_ld, T* q_out, int q_heads) {
    constexpr int P = D / 64, R2 = D / 2;
    __shared__ double cs[R2], sn[R2];
    __shared__ int owner;
    const int row = blockIdx.x;
    Kv4Seq sq;
    const int s = kv4_owner(w, row, &owner, &sq);
    if (s < 0) return;
    const int i = row - sq.row0, slot = sq.len + i;
    if (sq.bad && threadIdx.x == 0) atomicCAS(w.status, DEV_OK, DEV_KV4_ROWS);
    if (i < 0 || i >= sq.n) return;
    const bool stored = i < sq.n_new;
    const int p0 = pos ? __ldg(pos + row) : slot;
    for (int t = threadIdx.x; t < R2; t += blockDim.x) {
        double a, b;
        sincos((double)p0 * fr.f[t], &b, &a);
        cs[t] = a;
        sn[t] = b;
    }
    int page = -1;
    if (stored) page = kv4_page(w, s, slot);
    __syncthreads();
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const int R = 1 << w.shift, r = slot & (R - 1);
    constexpr int es = (int)sizeof(T);
    const int jobs = 2 * w.heads + (q ? q_heads : 0);
    for (int job = blockIdx.y * warps + (threadIdx.x >> 5); job < jobs; job += gridDim.y * warps) {
        if (job >= 2 * w.heads) {                                   // q: rotated in 32 bits, rounded once
            const int h = job - 2 * w.heads;
            const T* x = q + (int64_t)row * q_ld + (int64_t)h * D;
            T* y = q_out + ((int64_t)row * q_heads + h) * D;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const int t = lane * P + e;
                const float c0 = (float)cs[t], s0 = (float)sn[t], a = to_f<T>(x[t]), b = to_f<T>(x[t + R2]);
                y[t] = from_f<T>(a * c0 - b * s0);
                y[t + R2] = from_f<T>(b * c0 + a * s0);
            }
            continue;
        }
        if (page < 0) continue;
        const int which = job >= w.heads, h = which ? job - w.heads : job;
        float x[2 * P];
        const T* src = (which ? v : k) + (int64_t)row * kv_ld + (int64_t)h * D;
        if (which) {
#pragma unroll
            for (int e = 0; e < 2 * P; ++e) x[e] = to_f<T>(src[2 * P * lane + e]);
        } else {
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const int t = lane * P + e;
                const double a = (double)to_f<T>(src[t]), b = (double)to_f<T>(src[t + R2]);
                x[e] = (float)(a * cs[t] - b * sn[t]);
                x[P + e] = (float)(b * cs[t] + a * sn[t]);
            }
        }
        T scale, mn;
        row_params<T>(x, scale, mn);
        const float sf = to_f<T>(scale), mf = to_f<T>(mn), inv = 1.f / sf;
        uint8_t* blk = pool + kv4_block_at(w, page, h);
        uint8_t* codes = blk + kv4_code_at(R, D, which, r);
        uint32_t c[2 * P];
#pragma unroll
        for (int e = 0; e < 2 * P; ++e) c[e] = code_of(x[e], mf, sf, inv);
        if (which) {                                                // P consecutive bytes a lane
#pragma unroll
            for (int e = 0; e < P; ++e) codes[P * lane + e] = (uint8_t)(c[2 * e] | (c[2 * e + 1] << 4));
        } else if constexpr (P == 2) {                              // channels 2l, 2l + 1 and 64 + 2l, 64 + 2l + 1
            codes[lane] = (uint8_t)(c[0] | (c[1] << 4));
            codes[32 + lane] = (uint8_t)(c[2] | (c[3] << 4));
        } else {                                                    // channel l and 32 + l: the odd lane's code is the high half
            const uint32_t o0 = __shfl_down_sync(0xffffffffu, c[0], 1), o1 = __shfl_down_sync(0xffffffffu, c[1], 1);
            if (!(lane & 1)) {
                codes[lane / 2] = (uint8_t)(c[0] | (o0 << 4));
                codes[16 + lane / 2] = (uint8_t)(c[1] | (o1 << 4));
            }
        }
        if (lane == 0) {
            T* par = reinterpret_cast<T*>(blk + kv4_param_at(R, D, es, which, r));
            par[0] = scale;
            par[1] = mn;
        }
    }
}

// One row of the call per grid column, a warp per (head, K or V): lane l decodes D / 32 consecutive channels.
template <typename T, int D>
__global__ void k_kv4_read(Kv4View w, const uint8_t* __restrict__ pool, const int32_t* __restrict__ first, T* __restrict__ k_out,
                           T* __restrict__ v_out) {
    constexpr int N = D / 32;
    __shared__ int owner;
    const int row = blockIdx.x;
    Kv4Seq sq;
    const int s = kv4_owner(w, row, &owner, &sq);
    if (s < 0 || row < sq.row0) return;
    const int64_t slot = (int64_t)(first ? __ldg(first + s) : sq.len) + (row - sq.row0);
    if (slot < 0 || slot >= kv4_capacity(w)) {
        if (threadIdx.x == 0) atomicCAS(w.status, DEV_OK, DEV_KV4_ROWS);
        return;
    }
    const int page = kv4_page(w, s, (int)slot);
    if (page < 0) return;
    const int R = 1 << w.shift, r = (int)slot & (R - 1), lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (int job = blockIdx.y * warps + (threadIdx.x >> 5); job < 2 * w.heads; job += gridDim.y * warps) {
        const int which = job >= w.heads, h = which ? job - w.heads : job;
        T* out = which ? v_out : k_out;
        if (!out) continue;
        const uint8_t* blk = pool + kv4_block_at(w, page, h);
        const T* par = reinterpret_cast<const T*>(blk + kv4_param_at(R, D, (int)sizeof(T), which, r));
        const float sc = to_f<T>(par[0]), mn = to_f<T>(par[1]);
        const uint8_t* codes = blk + kv4_code_at(R, D, which, r) + lane * (N / 2);
        T* y = out + ((int64_t)row * w.heads + h) * D + lane * N;
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
            const uint32_t b = codes[e];
            y[2 * e] = from_f<T>(fmaf(sc, (float)(b & 15u), mn));
            y[2 * e + 1] = from_f<T>(fmaf(sc, (float)(b >> 4), mn));
        }
    }
}

// Block = one (pool, sequence, head); a lane owns one piece of a row: 16 bytes of K or V codes, or the scale and minimum
// of K or V.  Accepted nodes rise and nodes[j] >= j, so a lane that moves its piece in ascending j never reads a piece it
// has overwritten, and lanes own disjoint pieces: no synchronisation.
constexpr int COMMIT_POOLS = 64;
struct CommitPools { uint8_t* p[COMMIT_POOLS]; };

__global__ void k_kv4_commit(Kv4View w, CommitPools pools, int es, const ghd_accept_result* __restrict__ results) {
    const int s = blockIdx.y, head = blockIdx.x % w.heads, layer = blockIdx.x / w.heads, lane = threadIdx.x;
    const Kv4Seq sq = kv4_load_seq(w, s);
    if (sq.n <= 0) return;
    const ghd_accept_result* res = results + s;
    int m = res->n_matched;
    if (m > GHD_MAX_NODES - 1) m = GHD_MAX_NODES - 1;
    const int R = 1 << w.shift, D = w.d_head, half = D / 32;         // 16-byte pieces of a row's codes
    if (lane >= 2 * half + 2) return;
    uint8_t* pool = pools.p[layer];
    const int which = lane < half ? 0 : (lane < 2 * half ? 1 : lane - 2 * half);
    for (int j = 1; j <= m; ++j) {
        const int src = res->nodes[j];
        if (src == j) continue;
        if (src < j || src >= sq.n_new) {
            atomicCAS(w.status, DEV_OK, DEV_KV4_ROWS);
            continue;
        }
        const int from = sq.len + src, to = sq.len + j;
        const int pf = kv4_page(w, s, from), pt = kv4_page(w, s, to);
        if (pf < 0 || pt < 0) continue;
        const uint8_t* a = pool + kv4_block_at(w, pf, head);
        uint8_t* b = pool + kv4_block_at(w, pt, head);
        const int rf = from & (R - 1), rt = to & (R - 1);
        if (lane < 2 * half) {
            const int at = 16 * (lane - which * half);
            *reinterpret_cast<uint4*>(b + kv4_code_at(R, D, which, rt) + at) = *reinterpret_cast<const uint4*>(a + kv4_code_at(R, D, which, rf) + at);
        } else if (es == 2) {
            *reinterpret_cast<uint32_t*>(b + kv4_param_at(R, D, es, which, rt)) = *reinterpret_cast<const uint32_t*>(a + kv4_param_at(R, D, es, which, rf));
        } else {
            *reinterpret_cast<uint2*>(b + kv4_param_at(R, D, es, which, rt)) = *reinterpret_cast<const uint2*>(a + kv4_param_at(R, D, es, which, rf));
        }
    }
}

// The lengths grow behind the moves: by the accepted path, or by all new rows.
__global__ void k_kv4_advance(Kv4View w, int32_t* kv_len, const ghd_accept_result* __restrict__ results) {
    const int s = blockIdx.x * blockDim.x + threadIdx.x;
    if (s >= w.n_seqs) return;
    const Kv4Seq sq = kv4_seq(w.row_start[s], w.row_start[s + 1], w.n_rows, kv_len[s], kv4_capacity(w));
    if (sq.bad) atomicCAS(w.status, DEV_OK, DEV_KV4_ROWS);
    if (sq.n <= 0) return;
    int add = sq.n_new;
    if (results) {
        int m = results[s].n_matched;
        if (m < 0) m = 0;
        if (m > GHD_MAX_NODES - 1) m = GHD_MAX_NODES - 1;
        if (m + 1 > sq.n_new) atomicCAS(w.status, DEV_OK, DEV_KV4_ROWS);
        else add = m + 1;
    }
    kv_len[s] = sq.len + add;
}

// Blocks per row so that a few rows still spread over the device: one warp's job is short, a block start is not.
int row_blocks(const ghd_ctx* c, int n_rows, int jobs, int warps) {
    int y = (4 * c->sm_count) / (n_rows > 0 ? n_rows : 1);
    const int most = (jobs + warps - 1) / warps;
    if (y > most) y = most;
    return y < 1 ? 1 : y;
}

// A call works on its context's device whatever the current one is.
struct OnDevice {
    int before;
    bool moved;
    explicit OnDevice(const ghd_ctx* c) : before(-1), moved(false) {
        if (cudaGetDevice(&before) == cudaSuccess && before != c->device) moved = cudaSetDevice(c->device) == cudaSuccess;
    }
    ~OnDevice() { if (moved) cudaSetDevice(before); }
};

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

ghd_status check_kv4(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows) {
    if (!kv || !rows) return fail(c, GHD_EINVAL, "kv4: null description");
    if (kv->n_seqs < 1 || kv->n_seqs > GHD_MAX_SEQS) return fail(c, GHD_EINVAL, "kv4: n_seqs outside [1, GHD_MAX_SEQS]");
    if (kv->page_rows != 16 && kv->page_rows != 32 && kv->page_rows != 64 && kv->page_rows != 128)
        return fail(c, GHD_EINVAL, "kv4: page_rows is not 16, 32, 64 or 128");
    if (kv->n_pages < 1 || kv->max_pages < 1 || (int64_t)kv->max_pages * kv->page_rows > 0x7fffffffll) return fail(c, GHD_EINVAL, "kv4: bad page counts");
    if (kv->n_kv_heads < 1 || c->cfg.n_heads % kv->n_kv_heads) return fail(c, GHD_ESHAPE, "kv4: n_kv_heads does not divide n_heads");
    if (!kv->page_table || !kv->kv_len || !rows->row_start) return fail(c, GHD_EINVAL, "kv4: null page table, lengths or row starts");
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
    w.status = c->status;
    return w;
}

}  // namespace ghd

using namespace ghd;

extern "C" {

size_t ghd_kv4_pool_bytes(const ghd_ctx* c, const ghd_kv4* kv) {
    if (!c || !kv || kv->n_pages < 1 || kv->n_kv_heads < 1 || c->cfg.n_heads % kv->n_kv_heads ||
        (kv->page_rows != 16 && kv->page_rows != 32 && kv->page_rows != 64 && kv->page_rows != 128)) return 0;
    return (size_t)kv->n_pages * kv->n_kv_heads * kv4_block_bytes(kv->page_rows, c->cfg.d_head, c->cfg.dtype == GHD_F32 ? 4 : 2);
}

ghd_status ghd_kv4_append(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows, void* pool, const void* q, int64_t q_ld, const void* k,
                          const void* v, int64_t kv_ld, void* q_out) {
    if (!c) return GHD_EINVAL;
    ghd_status st = check_kv4(c, kv, rows);
    if (st != GHD_OK) return st;
    const ghd_model_cfg& m = c->cfg;
    const int D = m.d_head;
    if (!pool || !k || !v || (!q != !q_out)) return fail(c, GHD_EINVAL, "kv4_append: null pool, k or v, or only one of q and q_out");
    if (q_ld == 0) q_ld = (int64_t)m.n_heads * D;
    if (kv_ld == 0) kv_ld = (int64_t)kv->n_kv_heads * D;
    if (q_ld < (int64_t)m.n_heads * D || kv_ld < (int64_t)kv->n_kv_heads * D || q_ld % 8 || kv_ld % 8)
        return fail(c, GHD_EINVAL, "kv4_append: a leading dimension below the row's width, or not a multiple of 8");
    if (!aligned16(pool) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out)) return fail(c, GHD_EINVAL, "kv4_append: pointers must be 16-byte aligned");
    if (q == q_out && q && q_ld != (int64_t)m.n_heads * D) return fail(c, GHD_EINVAL, "kv4_append: q_out may be q only when q is contiguous");
    if (rows->n_rows == 0) return GHD_OK;
    OnDevice dev(c);
    RopeFreq fr;
    for (int t = 0; t < D / 2; ++t) fr.f[t] = pow((double)m.rope_theta, -2.0 * t / D);
    const Kv4View w = kv4_view(c, kv, rows);
    constexpr int WARPS = 8;
    const dim3 grid(rows->n_rows, row_blocks(c, rows->n_rows, 2 * kv->n_kv_heads + (q ? m.n_heads : 0), WARPS));
#define GHD_APPEND(T, DH) k_kv4_append<T, DH><<<grid, WARPS * 32, 0, c->cur>>>(w, fr, (uint8_t*)pool, rows->pos, (const T*)q, q_ld, (const T*)k, (const T*)v, kv_ld, (T*)q_out, m.n_heads)
    if (m.dtype == GHD_F32) { if (D == 64) GHD_APPEND(float, 64); else GHD_APPEND(float, 128); }
    else { if (D == 64) GHD_APPEND(__half, 64); else GHD_APPEND(__half, 128); }
#undef GHD_APPEND
    c->launches++;
    return check_cuda(c, "kv4_append");
}

ghd_status ghd_kv4_attention(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows, const void* pool, const void* q, void* out) {
    if (!c) return GHD_EINVAL;
    ghd_status st = check_kv4(c, kv, rows);
    if (st != GHD_OK) return st;
    if (!pool || !q || !out) return fail(c, GHD_EINVAL, "kv4_attention: null pool, q or out");
    if (!aligned16(pool) || !aligned16(q) || !aligned16(out)) return fail(c, GHD_EINVAL, "kv4_attention: pointers must be 16-byte aligned");
    if (rows->n_rows == 0) return GHD_OK;
    OnDevice dev(c);
    c->entry_fresh = c->opt_chain_calls ? 0 : 1;
    st = launch_attn_kv4(c, kv4_view(c, kv, rows), rows, pool, q, out);
    return st != GHD_OK ? st : check_cuda(c, "kv4_attention");
}

ghd_status ghd_kv4_read(ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows, const void* pool, const int32_t* first, void* k_out, void* v_out) {
    if (!c) return GHD_EINVAL;
    ghd_status st = check_kv4(c, kv, rows);
    if (st != GHD_OK) return st;
    if (!pool || (!k_out && !v_out)) return fail(c, GHD_EINVAL, "kv4_read: null pool, or neither output");
    if (!aligned16(pool) || !aligned16(k_out) || !aligned16(v_out)) return fail(c, GHD_EINVAL, "kv4_read: pointers must be 16-byte aligned");
    if (rows->n_rows == 0) return GHD_OK;
    OnDevice dev(c);
    const Kv4View w = kv4_view(c, kv, rows);
    constexpr int WARPS = 8;
    const dim3 grid(rows->n_rows, row_blocks(c, rows->n_rows, 2 * kv->n_kv_heads, WARPS));
#define GHD_READ(T, DH) k_kv4_read<T, DH><<<grid, WARPS * 32, 0, c->cur>>>(w, (const uint8_t*)pool, first, (T*)k_out, (T*)v_out)
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
    if (n_layers < 0 || (results && (n_layers < 1 || !pools))) return fail(c, GHD_EINVAL, "kv4_commit: no pools");
    for (int l = 0; results && l < n_layers; ++l)
        if (!pools[l] || !aligned16(pools[l])) return fail(c, GHD_EINVAL, "kv4_commit: a pool is null or not 16-byte aligned");
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
