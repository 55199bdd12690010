// Index arithmetic of the paged 4-bit cache and of the split of its attention's work over CTAs: plain integer
// functions, compiled for the device by nvcc and for the host by any C++ compiler (the CPU tests walk them there).
#pragma once

#include <stddef.h>
#include <stdint.h>

#ifdef __CUDACC__
#define GHD_HD __host__ __device__ __forceinline__
#define GHD_ROLLED _Pragma("unroll 1")      // these loops run once an item: short code matters, not their speed
#else
#define GHD_HD inline
#define GHD_ROLLED
#endif

namespace ghd {

// ---------------------------------------------------------------- a block: the rows of one head in one page
// K codes [R][d/2] | V codes [R][d/2] | K {scale, min} [R][2] | V {scale, min} [R][2]; es = bytes of a scale.
GHD_HD uint32_t kv4_block_bytes(int page_rows, int d_head, int es) { return (uint32_t)(page_rows * d_head + 4 * page_rows * es); }
GHD_HD uint32_t kv4_code_at(int page_rows, int d_head, int which, int row) { return (uint32_t)((which * page_rows + row) * (d_head / 2)); }
GHD_HD uint32_t kv4_param_at(int page_rows, int d_head, int es, int which, int row) {
    return (uint32_t)(page_rows * d_head + (which * page_rows + row) * 2 * es);
}

// ---------------------------------------------------------------- rows of a sequence
// What a sequence really has, whatever the device words hold: first row and number of rows inside the call's
// buffers, cache length and number of new rows inside the page table.  bad: something was out of range.
struct Kv4Seq {
    int row0, n;        // rows of the call
    int len, n_new;     // cache rows, and those of the n rows that the page table has room for
    bool bad;
};
GHD_HD Kv4Seq kv4_seq(int start, int end, int n_rows, int kv_len, int64_t capacity) {
    Kv4Seq q;
    q.bad = start < 0 || end < start || end > n_rows || kv_len < 0 || (int64_t)kv_len > capacity;
    q.row0 = start < 0 ? 0 : (start > n_rows ? n_rows : start);
    const int e = end > n_rows ? n_rows : end;
    q.n = e > q.row0 ? e - q.row0 : 0;
    q.len = kv_len < 0 ? 0 : ((int64_t)kv_len > capacity ? (int)capacity : kv_len);
    const int64_t room = capacity - q.len;
    q.n_new = (int64_t)q.n > room ? (int)room : q.n;
    q.bad = q.bad || q.n_new != q.n;
    return q;
}

// ---------------------------------------------------------------- the attention's work
// An item is one (sequence, key/value head, tile of query rows); a query row of an item is (new row i, query head of
// the group), numbered i * group + head.  Its keys are walked in chunks of `chunk` rows; a tile sees the cache and
// the new rows up to its last one.  The work is numbered in units in the order (sequence, head, tile): an item has
// `lead` units for what it costs whatever its length (queries in, sums out), then one for each chunk.
struct Kv4Tiling {
    int heads, group, tile_rows, chunk, lead;
};
GHD_HD int kv4_div(int64_t a, int b) { return a <= 0x7fffffff ? (int)((uint32_t)a / (uint32_t)b) : (int)(a / b); }     // a >= 0, b > 0
GHD_HD int kv4_tiles(const Kv4Tiling& t, int n) { return kv4_div((int64_t)n * t.group + t.tile_rows - 1, t.tile_rows); }
// keys that the rows of a tile may see
GHD_HD int kv4_tile_keys(const Kv4Tiling& t, const Kv4Seq& q, int tile) {
    const int last = kv4_div((int64_t)(tile + 1) * t.tile_rows - 1, t.group);        // number of the tile's last new row
    return q.len + (last < q.n_new ? last + 1 : q.n_new);
}
GHD_HD int kv4_tile_chunks(const Kv4Tiling& t, const Kv4Seq& q, int tile) {
    const int c = kv4_div((int64_t)kv4_tile_keys(t, q, tile) + t.chunk - 1, t.chunk);
    return c > 0 ? c : 1;               // a row that sees nothing still gets its zeros
}
// units of one head of a sequence
GHD_HD int64_t kv4_head_units(const Kv4Tiling& t, const Kv4Seq& q) {
    int64_t u = 0;
    GHD_ROLLED
    for (int i = 0, n = kv4_tiles(t, q.n); i < n; ++i) u += t.lead + kv4_tile_chunks(t, q, i);
    return u;
}
// a / b for what is mostly below 2^32 (64-bit divisions are long on the device)
GHD_HD int64_t kv4_cta_of(int64_t unit, int64_t per) { return ((uint64_t)unit | (uint64_t)per) <= 0xffffffffull ? (uint32_t)unit / (uint32_t)per : unit / per; }
// Every CTA takes `per` consecutive units (the last ones fewer or none), so a unit's CTA is unit / per.
GHD_HD int64_t kv4_units_per_cta(int64_t units, int ctas) { return units > 0 ? kv4_cta_of(units + ctas - 1, ctas) : 1; }

// The item that unit u belongs to, and the chunks of it that the run [u, u_end) takes (none when the run ends before the
// item's first chunk).  sums: exclusive sums of the sequences' units, n_seqs + 1 of them; seq_of(s) -> Kv4Seq;
// u < sums[n_seqs].
struct Kv4Item {
    int seq, head, tile, chunk0, chunks, take;
    int keys;                       // keys the tile may see (filled in by who needs it)
    int64_t first, next;            // unit of the item's first chunk; unit where the run goes on behind this item
    Kv4Seq q;
};
template <typename SeqOf>
GHD_HD Kv4Item kv4_find_item(const Kv4Tiling& t, const int64_t* sums, int n_seqs, SeqOf seq_of, int64_t u, int64_t u_end) {
    Kv4Item it;
    int lo = 0, hi = n_seqs - 1;    // the last sequence that starts at or before u: it has units, u is one of them
    GHD_ROLLED
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (sums[mid] <= u) lo = mid; else hi = mid - 1;
    }
    it.seq = lo;
    it.q = seq_of(lo);
    int64_t rem = u - sums[lo];
    const int64_t seq_units = sums[lo + 1] - sums[lo];
    int64_t head_units;
    if (seq_units <= 0x7fffffff) {  // 64-bit divisions are long on the device
        head_units = (uint32_t)seq_units / (uint32_t)t.heads;
        it.head = (int)((uint32_t)rem / (uint32_t)head_units);
    } else {
        head_units = seq_units / t.heads;
        it.head = (int)(rem / head_units);
    }
    rem -= it.head * head_units;
    it.tile = 0;
    GHD_ROLLED
    for (;;) {
        it.chunks = kv4_tile_chunks(t, it.q, it.tile);
        if (rem < t.lead + it.chunks) break;
        rem -= t.lead + it.chunks;
        ++it.tile;
    }
    it.first = u - rem + t.lead;
    it.next = it.first + it.chunks < u_end ? it.first + it.chunks : u_end;
    it.chunk0 = rem > t.lead ? (int)(rem - t.lead) : 0;
    const int64_t take = it.next - (it.first + it.chunk0);
    it.take = take > 0 ? (int)take : 0;
    it.keys = 0;
    return it;
}

// The item behind `it` in the same run, where the run goes on (it.next < u_end): no search and no division by what only the
// launch knows.
template <typename SeqOf>
GHD_HD void kv4_next_item(const Kv4Tiling& t, SeqOf seq_of, Kv4Item& it, int64_t u_end) {
    if (++it.tile >= kv4_tiles(t, it.q.n)) {
        it.tile = 0;
        if (++it.head == t.heads) {
            it.head = 0;
            GHD_ROLLED
            do it.q = seq_of(++it.seq); while (it.q.n == 0);        // there are units left, so there is one with rows
        }
    }
    it.chunks = kv4_tile_chunks(t, it.q, it.tile);
    it.first = it.next + t.lead;
    it.next = it.first + it.chunks < u_end ? it.first + it.chunks : u_end;
    it.chunk0 = 0;
    it.take = it.next > it.first ? (int)(it.next - it.first) : 0;
    it.keys = 0;
}

}  // namespace ghd
