// A cache whose rows lie in pages of a common pool, and a batch of new rows over it: what the kernels of the paged
// operators share.
#pragma once
#include "common.h"

namespace unigist {

constexpr int kMaxPagedRows = 1 << 23;  // rows of a sequence

// k, v: [n_pages, Hkv, page, D]; row j of sequence b is slot j % page of page table[b * cols + j / page].  An entry outside
// 0 .. n_pages - 1 is a page that is not there.  Division by `page` is a multiplication: for x < 2^24,
// x / page = mulhi(2 x, magic) >> shift with shift = ceil(log2 page), magic = ceil(2^(31 + shift) / page).
struct PagedKv {
    char* k;
    char* v;
    const float* kscale;  // E4M3: [Hkv] each
    const float* vscale;
    float* weight;        // [n_pages, Hkv, page] or null
    const int* table;
    int n_pages, page, cols, Hkv, D;
    unsigned magic;
    int shift;
};
// pages in front of row x, x < 2^24
__host__ __device__ inline int page_of(const PagedKv& c, int x) {
#ifdef __HIP_DEVICE_COMPILE__
    return (int)(__umulhi((unsigned)x << 1, c.magic) >> c.shift);
#else
    return (int)(((uint64_t)((unsigned)x << 1) * c.magic >> 32) >> c.shift);
#endif
}
__device__ __forceinline__ bool page_there(const PagedKv& c, int b, int pg) {
    return pg < c.cols && (unsigned)c.table[(size_t)b * c.cols + pg] < (unsigned)c.n_pages;
}
// A row's place in the pool, in rows of one kv head's D elements (below 2^31, which the host checks), or -1: no such page.
__device__ __forceinline__ int pool_row(const PagedKv& c, int b, int hk, int row) {
    if ((unsigned)row >= (unsigned)kMaxPagedRows) return -1;
    const int pg = page_of(c, row);
    if (pg >= c.cols) return -1;
    const int id = c.table[(size_t)b * c.cols + pg];
    if ((unsigned)id >= (unsigned)c.n_pages) return -1;
    return (id * c.Hkv + hk) * c.page + (row - pg * c.page);
}

// The new rows of a batch: those of sequence b are cu[b] .. cu[b+1] - 1 of T (cu null: one each), and the last ones of
// its kv_len[b] rows.  Values that cannot be are taken as the nearest that can, so that nothing outside the tensors is touched.
struct PagedBatch {
    const int* cu;
    const int* kv_len;
    int B, T;
    int max_new, max_kv;
};
struct PagedSeq {
    int t0, n;   // its rows of the batch
    int len;     // rows in use, the new ones among them
    int p0;      // position of its first new row (negative where len < n)
};
// how many new rows sequence b has
__device__ __forceinline__ int paged_new(const PagedBatch& x, int b) {
    if (!x.cu) return 1;
    const int t0 = min(max(x.cu[b], 0), x.T);
    return min(max(x.cu[b + 1], t0), x.T) - t0;
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch& x, int b) {
    PagedSeq s;
    s.t0 = x.cu ? min(max(x.cu[b], 0), x.T) : b;
    const int t1 = x.cu ? min(max(x.cu[b + 1], s.t0), x.T) : b + 1;
    s.n = t1 - s.t0;
    s.len = min(max(x.kv_len[b], 0), x.max_kv);
    s.p0 = s.len - s.n;
    return s;
}
// the sequence that row t of the batch belongs to: the last b with cu[b] <= t
__device__ __forceinline__ int seq_of_row(const PagedBatch& x, int t) {
    if (!x.cu) return t;
    int lo = 0, hi = x.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (x.cu[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// The mask as the rules of common.h take it (only the fields that win_lo, is_always, count_always and pos_of_always read).
struct PagedMask {
    int rp1, W, S, umode;
};
__host__ __device__ inline AttnShape mask_shape(const PagedMask& m) {
    AttnShape s = {};
    s.rp1 = m.rp1;
    s.W = m.W;
    s.S = m.S;
    s.umode = m.umode;
    return s;
}

// What a set of query rows at positions pf (the first, >= 0) to end - 1 walks: the `nfar` always-visible rows left of every
// window, which all of them see, then the rows wstart .. end - 1, which each sees by the rule.  Numbered through as `E` entries.
struct PagedWalk {
    int wstart, nfar, E;
};
__host__ __device__ inline PagedWalk paged_walk(const AttnShape& m, int pf, int end) {
    PagedWalk w;
    w.wstart = win_lo(m, pf);
    w.nfar = count_always(m, w.wstart);
    w.E = w.nfar + (end - w.wstart);
    return w;
}
__host__ __device__ inline int entry_row(const AttnShape& m, const PagedWalk& w, int e) {
    return e < w.nfar ? pos_of_always(m, e) : e - w.nfar + w.wstart;
}
// A row of entry e as the kernels fetch it: byte offset / 16 from k or v (the host checks that it fits), or place 0 of the
// pool with there = false where its page is not there.
struct PagedPlace {
    unsigned off;
    bool there;
};
// first half: the table entry of a row (-1: the table has none), second half: the place.  Apart, so that the load can be in flight.
__device__ __forceinline__ int page_id(const PagedKv& c, int b, int row) {
    const int pg = page_of(c, row);
    return pg < c.cols ? c.table[(size_t)b * c.cols + pg] : -1;
}
__device__ __forceinline__ PagedPlace place_of(const PagedKv& c, int hk, int row, int id, int row16) {
    PagedPlace p;
    p.there = (unsigned)id < (unsigned)c.n_pages;
    const unsigned at = ((unsigned)id * c.Hkv + hk) * c.page + (row - page_of(c, row) * c.page);
    p.off = p.there ? at * (unsigned)row16 : 0u;
    return p;
}

// Entries of a walk are shared out in at most S slices of about `want` entries, all of one length (a multiple of `unit`).
struct PagedSlices {
    int n, per;
};
__host__ __device__ inline PagedSlices paged_slices(int E, int S, int want, int unit) {
    PagedSlices x;
    x.n = (E + want - 1) / want;
    x.n = x.n > S ? S : x.n < 1 ? 1 : x.n;
    x.per = ((E + x.n - 1) / x.n + unit - 1) / unit * unit;
    x.n = x.per > 0 ? (E + x.per - 1) / x.per : 1;  // rounding up may leave fewer
    if (x.n < 1) x.n = 1;
    return x;
}
// Partial results of slices: per (unit, slice, column) the running reference m (exponent of 2) and sum l, and the
// accumulator of built-for width.
struct PagedParts {
    float* ml;   // [units][S][cols][2]
    float* acc;  // [units][S][cols][D]
    int S, want, cols;
    int groups;  // chunk kernel: parts of a slice, which its workgroup merges itself
    int units;   // chunk kernel: tiles x slices of a kv head that there is room for; more tiles than that are not sliced
};

// Scores of few columns in exponents of 2, -inf where a column does not see the entry: [B * Hkv][cols][pitch], pitch >= entries.
// Kept are those of the new rows whose attention counts, of sequences of at most `most` columns.
struct PagedScores {
    float* x;
    int cols, most;
    int pitch;
};

struct PagedAttn {
    PagedKv kv;
    PagedBatch batch;
    PagedMask mask;
    const bf16_t* q;
    bf16_t* out;
    float* lse;  // [Hq, T], may be null
    long long q_hs;
    int q_rs;
    int Hq;
    float scale;
    int weigh;    // new rows of each sequence, from the last, whose attention is added to the weights
    float decay;  // what was there is multiplied by this
};

// workspace; 0: more workgroups than a launch takes
size_t paged_attn_bytes(const PagedAttn& a, bool e4m3);
hipError_t launch_paged_attn(const PagedAttn& a, bool e4m3, void* ws, hipStream_t st);
hipError_t launch_paged_append(const PagedKv& c, const PagedBatch& x, bool e4m3, const bf16_t* k_new, const bf16_t* v_new, long long hs,
                               int rs, hipStream_t st);
// elem: bytes of an element
hipError_t launch_paged_evict(const PagedKv& src, const PagedKv& dst, int elem, const int* kv_len, const int* keep, int B, int max_kv,
                              int max_keep, int sinks, int recent, int* kept, int* rows_out, hipStream_t st);

}  // namespace unigist
