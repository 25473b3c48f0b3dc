// Rows of a paged cache moved about: the new rows of a batch into their pages, and the rows of most weight into new pages.
#include "paged.h"

namespace unigist {
namespace {

__device__ __forceinline__ float clamp448(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }

// ---------------------------------------------------------------------------------------------
// Append.  A lane moves 8 elements (16 bytes of bf16), 16 lanes a row (those that a smaller head dimension has), K and V of
// it.  Bound by the rows' bytes; for a token a sequence by latency.  Codes are RNE(clamp(x / scale, +-448)) with one correctly
// rounded division, as unigist_quantize_e4m3 makes them.
constexpr unsigned kAppendBlocks = 1u << 20;  // a row of the grid: a launch takes fewer than 2^32 threads an axis
template <bool E4M3>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedKv c, PagedBatch x, const bf16_t* __restrict__ k_new,
                                                           const bf16_t* __restrict__ v_new, long long hs, int rs) {
    const int row_id = (blockIdx.y * kAppendBlocks + blockIdx.x) * 16 + threadIdx.x / 16, d = (threadIdx.x & 15) * 8;
    const int t = row_id / c.Hkv, h = row_id - t * c.Hkv;
    if (t >= x.T || d >= c.D) return;
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
// left to take, lowest first, are numbered in row order.  Bound by latency: a thread holds the keys of PER rows, kSel apart, in
// registers (two of 32 in scratch; all pages' numbers and then all weights in flight); sequences of more than PER * kSel rows are fetched again,
// block by block, in each of the passes.  Rows are numbered from the counts of every 64 rows, scanned once.
// 8 heads of 32768 rows 30 us (44.8 with the keys in LDS, eight in flight and a wave numbering a stretch of rows), 64 x 8 of 2304 16 (20.2).
constexpr int kSel = 1024;  // threads
constexpr int kBins = 4096;

__device__ __forceinline__ unsigned weight_key(float w) {
    if (w != w) return 1u;  // 0: rows past the end, which no pass has to tell apart then
    const unsigned u = __float_as_uint(w + 0.f);  // -0 as 0
    const unsigned m = (u >> 31) ? ~u : (u | 0x80000000u);
    return m < 0xfffffffeu ? m : 0xfffffffeu;
}

template <int PER>
__global__ __launch_bounds__(kSel) void paged_select_kernel(PagedKv c, PagedKv to, const int* __restrict__ kv_len, const int* __restrict__ keep,
                                                            int max_kv, int max_keep, int sinks, int recent, int* __restrict__ kept,
                                                            int* __restrict__ rows_out) {
    constexpr int kWaves = kSel / 64, kGroups = PER * kWaves;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __shared__ int hist[kBins];
    __shared__ int part[kWaves];
    __shared__ int overs[kGroups], ties[kGroups];  // per 64 rows of a block: those above the limit and at it, then in front of them
    __shared__ int found, above, bad, sums[2];
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

    // ---- keys of the rows block * PER * kSel + i * kSel + tid
    const int nblocks = (len + PER * kSel - 1) / (PER * kSel);
    unsigned key[PER];
    constexpr int BATCH = PER < 8 ? PER : 8;
    auto fetch = [&](int base) {  // every page is there; rows past the end repeat the last
        int at[PER];
#pragma unroll
        for (int g = 0; g < PER; g += BATCH) {
            if (base + g * kSel >= len) break;
#pragma unroll
            for (int i = g; i < g + BATCH; ++i) at[i] = c.table[(size_t)b * c.cols + page_of(c, min(base + i * kSel + tid, len - 1))];
        }
#pragma unroll
        for (int g = 0; g < PER; g += BATCH) {
            if (base + g * kSel >= len) break;
#pragma unroll
            for (int i = g; i < g + BATCH; ++i) {
                const int j = min(base + i * kSel + tid, len - 1);
                key[i] = __float_as_uint(c.weight[(at[i] * c.Hkv + h) * c.page + (j - page_of(c, j) * c.page)]);
            }
        }
#pragma unroll
        for (int g = 0; g < PER; g += BATCH) {
            if (base + g * kSel >= len) break;
#pragma unroll
            for (int i = g; i < g + BATCH; ++i) {
                const int j = base + i * kSel + tid;
                key[i] = j >= len ? 0u : j < sinks || j >= len - recent ? 0xffffffffu : weight_key(__uint_as_float(key[i]));
            }
        }
    };
    if (nblocks == 1) fetch(0);
    unsigned limit = 0u;  // the stay-th largest key
    int left = stay;      // rows still to take among those that share its leading digits
#pragma unroll 1
    for (int p = 0; p < 3; ++p) {
        const int down = p == 0 ? 20 : p == 1 ? 10 : 0, up = p == 0 ? 32 : p == 1 ? 20 : 10, bins = 1 << (up - down);
        for (int i = tid; i < bins; i += kSel) hist[i] = 0;
        __syncthreads();
#pragma unroll 1
        for (int k = 0; k < nblocks; ++k) {
            const int base = k * PER * kSel;
            if (nblocks > 1) fetch(base);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (base + i * kSel >= len) break;
                if (p == 0 || ((key[i] ^ limit) >> up) == 0u) atomicAdd(&hist[(key[i] >> down) & (bins - 1)], 1);
            }
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
    // ---- numbering
    int over0 = 0, ties0 = 0;  // of the blocks so far
#pragma unroll 1
    for (int k = 0; k < nblocks; ++k) {
        const int base = k * PER * kSel;
        if (nblocks > 1) fetch(base);
        int no = 0, nt = 0;  // lane i: of the wave's i-th 64 rows
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (base + i * kSel >= len) break;
            const int o = __popcll(__builtin_amdgcn_ballot_w64(key[i] > limit)), t = __popcll(__builtin_amdgcn_ballot_w64(key[i] == limit));
            no = lane == i ? o : no;
            nt = lane == i ? t : nt;
        }
        if (lane < PER) {
            overs[lane * kWaves + wave] = no;
            ties[lane * kWaves + wave] = nt;
        }
        __syncthreads();
        if (wave < 2) {  // one wave scans each
            int* x = wave ? ties : overs;
            int own[kGroups / 64], sum = 0;
#pragma unroll
            for (int i = 0; i < kGroups / 64; ++i) {
                own[i] = sum;
                sum += x[lane * (kGroups / 64) + i];
            }
            int all = sum;
            for (int off = 1; off < 64; off <<= 1) {
                const int o = __shfl_up(all, off, 64);
                if (lane >= off) all += o;
            }
#pragma unroll
            for (int i = 0; i < kGroups / 64; ++i) x[lane * (kGroups / 64) + i] = all - sum + own[i];
            if (lane == 63) sums[wave] = all;
        }
        __syncthreads();
        const int at_o = over0 + overs[min(lane, PER - 1) * kWaves + wave], at_t = ties0 + ties[min(lane, PER - 1) * kWaves + wave];
        auto in_front = [&](bool x, int from) __attribute__((always_inline)) {
            const unsigned long long m = __builtin_amdgcn_ballot_w64(x);
            return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, (unsigned)from));
        };
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (base + i * kSel >= len) break;
            const int j = base + i * kSel + tid;
            const bool is_over = key[i] > limit, is_tie = key[i] == limit;  // limit > 0
            const int o = in_front(is_over, __builtin_amdgcn_readlane(at_o, i)), t = in_front(is_tie, __builtin_amdgcn_readlane(at_t, i));
            if (is_over || (is_tie && t < left)) list[o + min(t, left)] = j;  // in front of it: o rows above the limit, t at it
        }
        over0 += sums[0];
        ties0 += sums[1];
        __syncthreads();
    }
}

// Second part: the rows that stay are copied in order, 16 bytes a lane, K and V and the weight of a row.
__global__ __launch_bounds__(256) void paged_gather_kernel(PagedKv c, PagedKv to, int row_bytes, int max_keep, const int* __restrict__ kept,
                                                           const int* __restrict__ rows_out) {
    const int h = blockIdx.y, b = blockIdx.z, per_row = row_bytes / 16;
    const int at_lane = blockIdx.x * 256 + threadIdx.x, i = at_lane / per_row, o = (at_lane - i * per_row) * 16;  // 2^23 rows of 16 at most
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
    const unsigned blocks = (unsigned)(((long long)x.T * c.Hkv + 15) / 16);
    const dim3 grid(blocks < kAppendBlocks ? blocks : kAppendBlocks, (blocks + kAppendBlocks - 1) / kAppendBlocks);
    if (e4m3) paged_append_kernel<true><<<grid, 256, 0, st>>>(c, x, k_new, v_new, hs, rs);
    else paged_append_kernel<false><<<grid, 256, 0, st>>>(c, x, k_new, v_new, hs, rs);
    return hipGetLastError();
}

hipError_t launch_paged_evict(const PagedKv& src, const PagedKv& dst, int elem, const int* kv_len, const int* keep, int B, int max_kv,
                              int max_keep, int sinks, int recent, int* kept, int* rows_out, hipStream_t st) {
    auto go = [&](auto kern) {
        kern<<<dim3(src.Hkv, B), kSel, 0, st>>>(src, dst, kv_len, keep, max_kv, max_keep, sinks, recent, kept, rows_out);
    };
    max_kv <= 4 * kSel ? go(paged_select_kernel<4>) : go(paged_select_kernel<32>);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int row_bytes = src.D * elem;
    const long long lanes = (long long)max_keep * (row_bytes / 16);
    paged_gather_kernel<<<dim3((unsigned)((lanes + 255) / 256), src.Hkv, B), 256, 0, st>>>(src, dst, row_bytes, max_keep, kept, rows_out);
    return hipGetLastError();
}

}  // namespace unigist
