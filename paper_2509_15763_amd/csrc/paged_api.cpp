// C ABI of the paged operators: argument validation and dispatch.  As in api.cpp, nothing is allocated and nothing
// synchronises; what stands in device memory (page tables, lengths) is checked by the kernels.
#include <math.h>

#include "paged.h"

using namespace unigist;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// A descriptor as the kernels take it; values: they read or write numbers (and need the scales of codes).
unigist_status check_cache(const unigist_paged_cache* c, PagedKv* out, bool values = true) {
    if (!c) return UNIGIST_EINVAL;
    if (c->n_pages < 1 || c->page < 1 || c->table_cols < 1 || c->Hkv < 1 || c->D < 1) return UNIGIST_EINVAL;
    if (c->dt != UNIGIST_BF16 && c->dt != UNIGIST_E4M3) return UNIGIST_EUNSUPPORTED;
    if (c->D < 8 || c->D > 128 || c->D % (c->dt == UNIGIST_E4M3 ? 16 : 8) != 0) return UNIGIST_EUNSUPPORTED;
    // rows of the pool are counted in 31 bits
    if ((long long)c->n_pages * c->Hkv > 0x7fffffffLL || (long long)c->n_pages * c->Hkv * c->page > 0x7fffffffLL || c->Hkv > 65535)
        return UNIGIST_EUNSUPPORTED;
    // ... and its bytes, in steps of 16, in 32
    if ((long long)c->n_pages * c->Hkv * c->page * c->D * (c->dt == UNIGIST_E4M3 ? 1 : 2) > 1LL << 36) return UNIGIST_EUNSUPPORTED;
    if (!c->k || !c->v || !c->table || !aligned16(c->k) || !aligned16(c->v)) return UNIGIST_EINVAL;
    if (values && c->dt == UNIGIST_E4M3 && (!c->k_scale || !c->v_scale)) return UNIGIST_EINVAL;
    PagedKv p;
    p.k = (char*)c->k;
    p.v = (char*)c->v;
    p.kscale = c->dt == UNIGIST_E4M3 ? c->k_scale : nullptr;
    p.vscale = c->dt == UNIGIST_E4M3 ? c->v_scale : nullptr;
    p.weight = c->weight;
    p.table = c->table;
    p.n_pages = c->n_pages;
    p.page = c->page;
    p.cols = c->table_cols;
    p.Hkv = c->Hkv;
    p.D = c->D;
    p.shift = 0;
    while ((1LL << p.shift) < c->page) ++p.shift;
    const uint64_t two = (uint64_t)1 << (31 + p.shift);  // shift <= 31
    p.magic = (unsigned)((two + c->page - 1) / c->page);
    *out = p;
    return UNIGIST_OK;
}

unigist_status check_batch(int B, int T, const int* cu, const int* kv_len) {
    if (B < 1 || T < 0 || !kv_len || (!cu && T != B)) return UNIGIST_EINVAL;
    if (B > 65535 || T > kMaxPagedRows) return UNIGIST_EUNSUPPORTED;
    return UNIGIST_OK;
}

unigist_status check_attn(const unigist_paged_cache* c, int B, int Hq, int T, const int* cu, const int* kv_len, int max_new, int max_kv,
                          int r, int W, int sinks, int window_mode, int weigh, PagedAttn* a) {
    unigist_status st = check_cache(c, &a->kv);
    if (st == UNIGIST_OK) st = check_batch(B, T, cu, kv_len);
    if (st != UNIGIST_OK) return st;
    if (Hq < 1 || Hq % c->Hkv != 0 || max_new < 1 || max_kv < 1 || r < 1 || W < 1 || sinks < 0 || weigh < 0) return UNIGIST_EINVAL;
    if (window_mode != UNIGIST_WINDOW_SLIDING && window_mode != UNIGIST_WINDOW_UNITS) return UNIGIST_EINVAL;
    if (max_kv > kMaxPagedRows || Hq > 65535 || (long long)B * c->Hkv > 0x7fffffffLL / 64) return UNIGIST_EUNSUPPORTED;
    if ((long long)Hq * (T > 0 ? T : 1) > 0x7fffffffLL) return UNIGIST_EUNSUPPORTED;
    if (weigh > 0 && !c->weight) return UNIGIST_EINVAL;
    const int far = kMaxPagedRows + 1;  // beyond every position
    a->batch = {cu, kv_len, B, T, max_new < T ? max_new : (T > 0 ? T : 1), max_kv};
    a->mask = {r >= far ? far : r + 1, W > far ? far : W, sinks > far ? far : sinks, window_mode == UNIGIST_WINDOW_UNITS};
    a->Hq = Hq;
    a->scale = 1.0f / sqrtf((float)c->D);
    a->weigh = weigh;
    return UNIGIST_OK;
}

}  // namespace

extern "C" unigist_status unigist_paged_append(const unigist_paged_cache* c, const void* k_new, const void* v_new, long long head_stride,
                                               long long row_stride, int B, int T, const int* cu, const int* kv_len, void* hip_stream) {
    PagedKv kv;
    unigist_status st = check_cache(c, &kv);
    if (st == UNIGIST_OK) st = check_batch(B, T, cu, kv_len);
    if (st != UNIGIST_OK) return st;
    if (T == 0) return UNIGIST_OK;
    if (!k_new || !v_new || !aligned16(k_new) || !aligned16(v_new)) return UNIGIST_EINVAL;
    if (head_stride % 8 != 0 || row_stride % 8 != 0 || row_stride < c->D || head_stride < 0) return UNIGIST_EINVAL;
    if (row_stride > 0x7fffffffLL || (long long)T * c->Hkv > 0x7fffffffLL - 16) return UNIGIST_EUNSUPPORTED;
    const PagedBatch x = {cu, kv_len, B, T, T, kMaxPagedRows};
    hipError_t e = launch_paged_append(kv, x, c->dt == UNIGIST_E4M3, (const bf16_t*)k_new, (const bf16_t*)v_new, head_stride, (int)row_stride,
                                       (hipStream_t)hip_stream);
    return e == hipSuccess ? UNIGIST_OK : UNIGIST_ELAUNCH;
}

extern "C" size_t unigist_paged_attn_workspace(const unigist_paged_cache* c, int B, int Hq, int T, int max_new, int max_kv, int r, int W,
                                               int sinks, int window_mode, int weigh) {
    PagedAttn a = {};
    const int any = 0;  // lengths are not read on the host
    if (check_attn(c, B, Hq, T, &any, &any, max_new, max_kv, r, W, sinks, window_mode, weigh, &a) != UNIGIST_OK) return 0;
    return paged_attn_bytes(a, c->dt == UNIGIST_E4M3);
}

extern "C" unigist_status unigist_paged_attn(const unigist_paged_cache* c, const void* q, void* out, float* lse, int B, int Hq, int T,
                                             const int* cu, const int* kv_len, int max_new, int max_kv, int r, int W, int sinks,
                                             int window_mode, long long q_head_stride, long long q_row_stride, int weigh, float decay,
                                             void* workspace, size_t workspace_bytes, void* hip_stream) {
    PagedAttn a = {};
    unigist_status st = check_attn(c, B, Hq, T, cu, kv_len, max_new, max_kv, r, W, sinks, window_mode, weigh, &a);
    if (st != UNIGIST_OK) return st;
    if (weigh > 0 && (!lse || !(decay >= 0.f) || isinf(decay))) return UNIGIST_EINVAL;
    if (T == 0) return UNIGIST_OK;
    if (!q || !out || !aligned16(q) || !aligned16(out)) return UNIGIST_EINVAL;
    if (Hq > 1 && q_head_stride < c->D) return UNIGIST_EINVAL;  // heads of out on each other
    if (weigh > 0 && q == out) return UNIGIST_EINVAL;  // the weights are made from q once out is there
    if (q_head_stride % 8 != 0 || q_row_stride % 8 != 0 || q_row_stride < c->D || q_head_stride < 0) return UNIGIST_EINVAL;
    if (q_row_stride > 0x7fffffffLL) return UNIGIST_EUNSUPPORTED;
    const bool e4m3 = c->dt == UNIGIST_E4M3;
    const size_t need = paged_attn_bytes(a, e4m3);
    if (need == 0) return UNIGIST_EUNSUPPORTED;
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need) return UNIGIST_EINVAL;
    a.q = (const bf16_t*)q;
    a.out = (bf16_t*)out;
    a.lse = lse;
    a.q_hs = q_head_stride;
    a.q_rs = (int)q_row_stride;
    a.decay = decay;
    hipError_t e = launch_paged_attn(a, e4m3, workspace, (hipStream_t)hip_stream);
    return e == hipSuccess ? UNIGIST_OK : UNIGIST_ELAUNCH;
}

extern "C" unigist_status unigist_paged_evict(const unigist_paged_cache* src, const unigist_paged_cache* dst, int B, const int* kv_len,
                                              const int* keep, int max_kv, int max_keep, int sinks, int recent, int* kept, int* rows_out,
                                              void* hip_stream) {
    PagedKv a, b;
    unigist_status st = check_cache(src, &a, false);
    if (st == UNIGIST_OK) st = check_cache(dst, &b, false);
    if (st != UNIGIST_OK) return st;
    if (src->Hkv != dst->Hkv || src->D != dst->D || src->dt != dst->dt || !src->weight) return UNIGIST_EINVAL;
    if (B < 1 || max_kv < 1 || max_keep < 1 || sinks < 0 || recent < 0) return UNIGIST_EINVAL;
    if (!kv_len || !keep || !kept || !rows_out) return UNIGIST_EINVAL;
    if (max_kv > kMaxPagedRows || max_keep > kMaxPagedRows || B > 65535) return UNIGIST_EUNSUPPORTED;
    hipError_t e = launch_paged_evict(a, b, src->dt == UNIGIST_E4M3 ? 1 : 2, kv_len, keep, B, max_kv, max_keep, sinks, recent, kept, rows_out,
                                      (hipStream_t)hip_stream);
    return e == hipSuccess ? UNIGIST_OK : UNIGIST_ELAUNCH;
}
