// Rows of a paged cache moved about: the new rows of a batch into their pages, and the rows of most weight into new pages.
#include <algorithm>

#include "paged.h"

namespace unigist {
namespace {

__device__ __forceinline__ float clamp448(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }

// ---------------------------------------------------------------------------------------------
// Append.  A lane moves 8 elements (16 bytes of bf16): D / 8 lanes a row, K and V of it.  Codes are RNE(clamp(x / scale,
// +-448)) with one correctly rounded division, as unigist_quantize_e4m3 makes them.
template <bool E4M3>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedKv c, PagedBatch x, const bf16_t* __restrict__ k_new,
                                                           const bf16_t* __restrict__ v_new, long long hs, int rs) {
    const int per_row = c.D / 8;
    const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row_id = idx / per_row;
    const int d = (int)(idx - row_id * per_row) * 8;
    const int t = (int)(row_id / c.Hkv), h = (int)(row_id - (long long)t * c.Hkv);
    if (t >= x.T) return;
    const int b = seq_of_row(x, t);
    const PagedSeq s = paged_seq(x, b);
    if (t < s.t0 || t >= s.t0 + s.n) return;  // behind the last sequence
    const int at = pool_row(c, b, h, s.p0 + (t - s.t0));
    if (at < 0) return;
    const size_t from = (size_t)h * hs + (size_t)t * rs + d, to = (size_t)at * c.D + d;
    const u32x4 kx = *(const u32x4*)(k_new + from), vx = *(const u32x4*)(v_new + from);
    if (E4M3) {
        auto code = [](u32x4 w, float s) {
            u32x2 y;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float a = __uint_as_float(w[2 * i] << 16), b2 = __uint_as_float(w[2 * i] & 0xffff0000u);
                const float e = __uint_as_float(w[2 * i + 1] << 16), f = __uint_as_float(w[2 * i + 1] & 0xffff0000u);
                int r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(__fdiv_rn(a, s)), clamp448(__fdiv_rn(b2, s)), 0, false);
                y[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(clamp448(__fdiv_rn(e, s)), clamp448(__fdiv_rn(f, s)), r, true);
            }
            return y;
        };
        *(u32x2*)(c.k + to) = code(kx, c.kscale[h]);
        *(u32x2*)(c.v + to) = code(vx, c.vscale[h]);
    } else {
        *(u32x4*)(c.k + 2 * to) = kx;
        *(u32x4*)(c.v + 2 * to) = vx;
    }
    if (d == 0 && c.weight) c.weight[at] = 0.f;
}

// ---------------------------------------------------------------------------------------------
// Eviction, first part: which rows stay.  A workgroup takes one kv head of one sequence.  Rows are ordered by a 32-bit key
// that grows with the weight (the float's bits, made monotone; protected rows the largest, NaN the least); the keep-th
// largest key is found digit by digit from histograms in LDS, then the rows above it and as many of those equal to it as are
// left to take, lowest first, are numbered in row order.  Bound by latency: the keys are fetched once, kPer at a time in
// flight (a page's number, then the weight), and stay in LDS, up to kCached of them (the rest are fetched again in each of
// the five passes); the numbering takes a contiguous stretch of rows per wave, counted first, so that it needs one barrier.
constexpr int kSel = 1024;  // threads
constexpr int kBins = 4096;
constexpr int kPer = 8;
constexpr int kCached = 32768;

__device__ __forceinline__ unsigned weight_key(float w) {
    if (w != w) return 0u;
    const unsigned u = __float_as_uint(w + 0.f);  // -0 as 0
    const unsigned m = (u >> 31) ? ~u : (u | 0x80000000u);
    return m < 0xfffffffeu ? m : 0xfffffffeu;
}

__global__ __launch_bounds__(kSel) void paged_select_kernel(PagedKv c, PagedKv to, const int* __restrict__ kv_len, const int* __restrict__ keep,
                                                            int max_kv, int max_keep, int sinks, int recent, int* __restrict__ kept,
                                                            int* __restrict__ rows_out) {
    constexpr int kWaves = kSel / 64;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    extern __shared__ unsigned cache[];  // min(max_kv, kCached) keys
    __shared__ int hist[kBins];
    __shared__ int part[kWaves], part2[kWaves];
    __shared__ int found, above, bad;
    int* list = kept + ((size_t)b * c.Hkv + h) * max_keep;
    const int len = kv_len[b], want = keep[b];
    const int stay = min(want, len);  // rows that stay
    if (tid == 0) bad = len < 0 || len > max_kv || want < 0 || want > max_keep;
    __syncthreads();
    if (!bad) {  // every page of the rows there are, and of those that stay, has to be there
        int missing = 0;
        for (int pg = tid, n = len ? page_of(c, len - 1) + 1 : 0; pg < n; pg += kSel) missing |= !page_there(c, b, pg);
        for (int pg = tid, n = stay ? page_of(to, stay - 1) + 1 : 0; pg < n; pg += kSel) missing |= !page_there(to, b, pg);
        if (missing) bad = 1;
    }
    __syncthreads();
    const bool refused = bad;
    if (h == 0 && tid == 0) rows_out[b] = refused ? -1 : stay;
    for (int i = (refused ? 0 : stay) + tid; i < max_keep; i += kSel) list[i] = -1;
    if (refused || stay == 0) return;

    auto is_safe = [&](int j) { return j < sinks || j >= len - recent; };
    auto fetch = [&](int j0, unsigned (&key)[kPer]) {  // of the rows j0 + kSel * i, those that there are
        int at[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) at[i] = pool_row(c, b, h, min(j0 + kSel * i, len - 1));
#pragma unroll
        for (int i = 0; i < kPer; ++i) key[i] = weight_key(c.weight[at[i]]);
#pragma unroll
        for (int i = 0; i < kPer; ++i) key[i] = is_safe(j0 + kSel * i) ? 0xffffffffu : key[i];
    };
    const int cached = min(len, kCached);
    for (int j0 = tid; j0 < cached; j0 += kSel * kPer) {
        unsigned key[kPer];
        fetch(j0, key);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (j0 + kSel * i < cached) cache[j0 + kSel * i] = key[i];
    }
    unsigned limit = 0u;  // the stay-th largest key
    int left = stay;      // rows still to take among those that share its leading digits
    const int shifts[3] = {20, 10, 0}, bits[3] = {12, 10, 10};
#pragma unroll 1
    for (int p = 0; p < 3; ++p) {
        const int bins = 1 << bits[p], up = shifts[p] + bits[p], down = shifts[p];
        for (int i = tid; i < bins; i += kSel) hist[i] = 0;
        __syncthreads();
        auto count = [&](unsigned key) {
            if (up == 32 || ((key ^ limit) >> up) == 0u) atomicAdd(&hist[(key >> down) & (bins - 1)], 1);
        };
        for (int j = tid; j < cached; j += kSel) count(cache[j]);
        for (int j0 = cached + tid; j0 < len; j0 += kSel * kPer) {
            unsigned key[kPer];
            fetch(j0, key);
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (j0 + kSel * i < len) count(key[i]);
        }
        __syncthreads();
        // bins per thread from the top: thread 0 has the largest digits
        const int per = bins / kSel;
        int own = 0;
        for (int i = 0; i < per; ++i) own += hist[bins - 1 - (tid * per + i)];
        int sum = own;  // of this thread and those above it
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(sum, off, 64);
            if (lane >= off) sum += o;
        }
        if (lane == 63) part[wave] = sum;
        __syncthreads();
        for (int w = 0; w < wave; ++w) sum += part[w];
        if (sum >= left && sum - own < left) {  // the digit is among this thread's
            int before = sum - own;
            for (int i = 0; i < per; ++i) {
                const int bin = bins - 1 - (tid * per + i);
                if (before + hist[bin] >= left) {
                    found = bin;
                    above = before;
                    break;
                }
                before += hist[bin];
            }
        }
        __syncthreads();
        limit |= (unsigned)found << down;
        left -= above;
        __syncthreads();
    }
    // ---- numbering: wave w takes the rows [w * seg, (w + 1) * seg)
    const int seg = ((len + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int j0 = wave * seg, j1 = min(len, j0 + seg);
    auto key_at = [&](int j) {
        if (j >= j1) return 0u;
        if (j < cached) return cache[j];
        return is_safe(j) ? 0xffffffffu : weight_key(c.weight[pool_row(c, b, h, j)]);
    };
    int over = 0, ties = 0;  // rows above the limit and at it in the rows of the waves so far
    for (int j = j0; j < j1; j += 64) {
        const unsigned key = key_at(j + lane);
        over += __popcll(__builtin_amdgcn_ballot_w64(key > limit));
        ties += __popcll(__builtin_amdgcn_ballot_w64(j + lane < j1 && key == limit));
    }
    if (lane == 0) {
        part[wave] = over;
        part2[wave] = ties;
    }
    __syncthreads();
    over = ties = 0;
    for (int w = 0; w < wave; ++w) {
        over += part[w];
        ties += part2[w];
    }
    const unsigned long long before = (1ull << lane) - 1ull;
    for (int j = j0; j < j1; j += 64) {
        const unsigned key = key_at(j + lane);
        const unsigned long long ob = __builtin_amdgcn_ballot_w64(key > limit);
        const unsigned long long tb = __builtin_amdgcn_ballot_w64(j + lane < j1 && key == limit);
        const int tie_at = ties + __popcll(tb & before), taken = min(tie_at, left);  // ties in front of this row that are taken
        if ((ob >> lane & 1) || ((tb >> lane & 1) && tie_at < left)) list[over + __popcll(ob & before) + taken] = j + lane;
        over += __popcll(ob);
        ties += __popcll(tb);
    }
}

// Second part: the rows that stay are copied in order, 16 bytes a lane, K and V and the weight of a row.
__global__ __launch_bounds__(256) void paged_gather_kernel(PagedKv c, PagedKv to, int row_bytes, int max_keep, const int* __restrict__ kept,
                                                           const int* __restrict__ rows_out) {
    const int h = blockIdx.y, b = blockIdx.z, per_row = row_bytes / 16;
    const int i = (int)(((long long)blockIdx.x * 256 + threadIdx.x) / per_row);
    const int o = (int)(((long long)blockIdx.x * 256 + threadIdx.x) - (long long)i * per_row) * 16;
    if (i >= rows_out[b]) return;  // -1 for a sequence left alone
    const int j = kept[((size_t)b * c.Hkv + h) * max_keep + i];
    const int from = pool_row(c, b, h, j), at = pool_row(to, b, h, i);
    if (from < 0 || at < 0) return;
    const size_t f = (size_t)from * row_bytes + o, t = (size_t)at * row_bytes + o;
    *(u32x4*)(to.k + t) = *(const u32x4*)(c.k + f);
    *(u32x4*)(to.v + t) = *(const u32x4*)(c.v + f);
    if (o == 0 && to.weight) to.weight[at] = c.weight[from];
}

}  // namespace

hipError_t launch_paged_append(const PagedKv& c, const PagedBatch& x, bool e4m3, const bf16_t* k_new, const bf16_t* v_new, long long hs,
                               int rs, hipStream_t st) {
    const long long lanes = (long long)x.T * c.Hkv * (c.D / 8), blocks = (lanes + 255) / 256;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    if (e4m3) paged_append_kernel<true><<<dim3((unsigned)blocks), 256, 0, st>>>(c, x, k_new, v_new, hs, rs);
    else paged_append_kernel<false><<<dim3((unsigned)blocks), 256, 0, st>>>(c, x, k_new, v_new, hs, rs);
    return hipGetLastError();
}

hipError_t launch_paged_evict(const PagedKv& src, const PagedKv& dst, int elem, const int* kv_len, const int* keep, int B, int max_kv,
                              int max_keep, int sinks, int recent, int* kept, int* rows_out, hipStream_t st) {
    const unsigned lds = (unsigned)std::min(max_kv, kCached) * 4u;
    paged_select_kernel<<<dim3(src.Hkv, B), kSel, lds, st>>>(src, dst, kv_len, keep, max_kv, max_keep, sinks, recent, kept, rows_out);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int row_bytes = src.D * elem;
    const long long lanes = (long long)max_keep * (row_bytes / 16);
    paged_gather_kernel<<<dim3((unsigned)((lanes + 255) / 256), src.Hkv, B), 256, 0, st>>>(src, dst, row_bytes, max_keep, kept, rows_out);
    return hipGetLastError();
}

}  // namespace unigist
