// Attention over a paged cache: the choice of kernels, the merge of slices, and the weight that the cached rows receive.
#include <algorithm>

#include "paged_common.h"

namespace unigist {

hipError_t launch_paged_decode(const PagedAttn& a, bool e4m3, const PagedParts& parts, const PagedScores& scores, int cols, hipStream_t st);
hipError_t launch_paged_chunk(const PagedAttn& a, bool e4m3, const PagedParts& parts, long long blocks, int min_cols, hipStream_t st);

namespace {

// ---------------------------------------------------------------------------------------------
// Merge of the slices of a column, nothing but latency and the partial results' bytes.  A slice in which the column sees nothing has l = 0
// and is left out; one with scores that are no numbers has l = NaN and any m.
__device__ __forceinline__ float slice_weight(f32x2 ml, float mm) {
    return ml[1] == 0.f ? 0.f : ml[0] == mm ? 1.f : __builtin_amdgcn_exp2f(ml[0] - mm);
}

// (Sequence, kv head) pairs of the decode kernel: W waves a column, each taking every W-th slice; all loads of up to kBatch
// slices of a wave are in flight.
constexpr int kBatch = 8;
template <int D, int W>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedAttn a, PagedParts parts) {
    constexpr int C = (D + 63) / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave % W, col = blockIdx.x * (4 / W) + wave / W, hk = blockIdx.y, b = blockIdx.z;
    const int Hkv = a.kv.Hkv, G = a.Hq / Hkv;
    __shared__ float sums[4][64 * C];
    const PagedSeq s = paged_seq(a.batch, b);
    const int ncol = s.n * G;
    bool mine = ncol <= parts.cols && col < ncol && s.len > 0;
    const int E = mine ? paged_walk(mask_shape(a.mask), max(s.p0, 0), s.len).E : 0;
    const int n = paged_slices(E, parts.S, parts.want, 128).n;
    mine = mine && n > 1;
    float acc[C], mm = -INFINITY, ll = 0.f;
#pragma unroll
    for (int k = 0; k < C; ++k) acc[k] = 0.f;
    if (mine) {
        const size_t stride = parts.cols, at0 = ((size_t)b * Hkv + hk) * parts.S * stride + col;  // columns between slices
        float x[kBatch][C];
        auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
#pragma unroll
                for (int k = 0; k < C; ++k) x[i][k] = parts.acc[(at0 + min(s0 + W * i, n - 1) * stride) * D + min(64 * k + lane, D - 1)];
        };
        load(part);
        const f32x2 ml = lane < n ? *(const f32x2*)(parts.ml + 2 * (at0 + lane * stride)) : f32x2{-INFINITY, 0.f};  // n <= 64
        mm = ml[0];
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) mm = fmaxf(mm, __shfl_xor(mm, off, 64));
        const float wgt = slice_weight(ml, mm);
        const unsigned long long has = __builtin_amdgcn_ballot_w64(!(ml[1] == 0.f));
        ll = wgt * ml[1];
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) ll += __shfl_xor(ll, off, 64);
        for (int s0 = part; s0 < n; s0 += W * kBatch) {
            if (s0 != part) load(s0);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int t = s0 + W * i;
                const float f = __shfl(wgt, t < n ? t : 0, 64);
                if (t < n && (has >> t & 1))
#pragma unroll
                    for (int k = 0; k < C; ++k) acc[k] += f * x[i][k];
            }
        }
    }
    if (W > 1) {
#pragma unroll
        for (int k = 0; k < C; ++k) sums[wave][64 * k + lane] = acc[k];
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int k = 0; k < C; ++k) acc[k] = (sums[wave][64 * k + lane] + sums[wave + 1][64 * k + lane]) + (sums[wave + 2][64 * k + lane] + sums[wave + 3][64 * k + lane]);
    }
    if (!mine) return;
    const int i = col / G, hq = hk * G + (col - i * G), t = s.t0 + i;
#pragma unroll
    for (int k = 0; k < C; ++k)
        if (64 * k + lane < a.kv.D)
            Elem<bf16_t>::store(a.out + (size_t)hq * a.q_hs + (size_t)t * a.q_rs + 64 * k + lane, ll == 0.f ? 0.f : acc[k] / ll);
    if (lane == 0 && a.lse) a.lse[(size_t)hq * a.batch.T + t] = ll == 0.f ? -INFINITY : mm * kLn2 + __builtin_amdgcn_logf(ll) * kLn2;
}

// Tiles of the chunk kernel: 16 columns a workgroup, 16 lanes a column (a lane has the columns 4 (lane % 16) + 64 k .. + 3 of
// D), eight slices in flight.
template <int D>
__global__ __launch_bounds__(256) void paged_combine_chunk_kernel(PagedAttn a, PagedParts parts, int min_cols) {
    constexpr int C = (D + 63) / 64, NB = 8;
    const int sub = threadIdx.x & 15, hk = blockIdx.y, tile = blockIdx.x;
    const int Hkv = a.kv.Hkv, G = a.Hq / Hkv;
    const PagedTiles tiles = count_tiles(a.batch, G, min_cols);
    const int S = slices_of(parts, tiles.total);
    if (S <= 1 || tile >= tiles.total) return;
    int nth;
    const int b = seq_of_tile(a.batch, G, min_cols, tiles, tile, nth);
    const PagedSeq s = paged_seq(a.batch, b);
    const int ncol = s.n * G, c0 = nth * kChunkCols, col = c0 + blockIdx.z * 16 + (threadIdx.x >> 4);
    if ((unsigned)nth * kChunkCols >= (unsigned)ncol || col >= ncol) return;
    const int pe = s.p0 + (min(c0 + kChunkCols, ncol) - 1) / G;
    const int E = pe >= 0 ? paged_walk(mask_shape(a.mask), max(s.p0 + c0 / G, 0), pe + 1).E : 0;
    const int n = paged_slices(E, S, parts.want, 32).n;
    if (n <= 1) return;
    const size_t at0 = (((size_t)tile * Hkv + hk) * S) * kChunkCols + (col - c0);
    const f32x2* ml = (const f32x2*)parts.ml + at0;
    f32x4 acc[C], x[NB][C];
    f32x2 y[NB];
    auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const size_t at = (size_t)min(s0 + i, n - 1) * kChunkCols;
            y[i] = ml[at];
#pragma unroll
            for (int k = 0; k < C; ++k) x[i][k] = *(const f32x4*)(parts.acc + (at0 + at) * D + min(64 * k + 4 * sub, D - 4));
        }
    };
    float mm = -INFINITY, ll = 0.f;
#pragma unroll
    for (int k = 0; k < C; ++k) acc[k] = zero4();
    for (int s0 = 0; s0 < n; s0 += NB) {
        load(s0);
        float top = mm;
#pragma unroll
        for (int i = 0; i < NB; ++i) top = fmaxf(top, y[i][0]);
        const float old = slice_weight(f32x2{mm, ll}, top);
        ll *= old;
#pragma unroll
        for (int k = 0; k < C; ++k) acc[k] *= old;
        mm = top;
#pragma unroll
        for (int i = 0; i < NB; ++i)
            if (s0 + i < n && !(y[i][1] == 0.f)) {
                const float f = slice_weight(y[i], mm);
                ll += f * y[i][1];
#pragma unroll
                for (int k = 0; k < C; ++k) acc[k] += f * x[i][k];
            }
    }
    const int i = col / G, hq = hk * G + (col - i * G), t = s.t0 + i;
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll
    for (int k = 0; k < C; ++k)
        if (64 * k + 4 * sub < a.kv.D) {
            u32x2 w2;
            w2[0] = pack_bf16x2(acc[k][0] * inv, acc[k][1] * inv);
            w2[1] = pack_bf16x2(acc[k][2] * inv, acc[k][3] * inv);
            *(u32x2*)(a.out + (size_t)hq * a.q_hs + (size_t)t * a.q_rs + 64 * k + 4 * sub) = w2;
        }
    if (sub == 0 && a.lse) a.lse[(size_t)hq * a.batch.T + t] = ll == 0.f ? -INFINITY : mm * kLn2 + __builtin_amdgcn_logf(ll) * kLn2;
}

// ---------------------------------------------------------------------------------------------
// Weights of a sequence of many columns: the scores of the last new rows once more, summed over columns instead of keys.  A
// wave holds 128 keys of one kv head (A operand K, in registers); the columns come in chunks of 64 through two LDS stages
// (B operand Q^T, direct loads, chunks swizzled as in the attention kernels) with their position, the start of their window
// and their lse, and exp(score - lse) of the visible pairs adds up per lane, over a lane's 16 columns at the end.
// Bound by the matrix pipe and the exponentials, K is read once.
constexpr int kWeighKeys = 512, kWeighCols = 64;
template <int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void paged_weigh_kernel(PagedAttn a, int min_cols) {
    constexpr int KS = D / 32, CH = D <= 64 ? 8 : 16, RPI = 64 / CH, IPW = 16 / RPI;
    __shared__ __attribute__((aligned(1024))) char qs[2][kWeighCols * CH * 16];
    __shared__ float ls[2][kWeighCols];
    __shared__ int ps[2][kWeighCols], los[2][kWeighCols];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g4 = lane >> 4;
    const int hk = blockIdx.y, b = blockIdx.z, wg0 = blockIdx.x * kWeighKeys, j0 = wg0 + 128 * w;
    const int G = a.Hq / a.kv.Hkv, Dt = a.kv.D;
    const PagedSeq s = paged_seq(a.batch, b);
    const int ncol = s.n * G;
    if (wg0 >= s.len || ncol <= min_cols) return;
    const AttnShape m = mask_shape(a.mask);
    const float c = a.scale * (E4M3 ? a.kv.kscale[hk] : 1.f) * kLog2e;

    // ---- this wave's keys
    bf16x8 kf[2][4][KS];  // keys j0 + 64 half + 16 kb + r16
    const int row_bytes = Dt * (E4M3 ? 1 : 2), row16 = row_bytes / 16;
    unsigned long long gone[2];
    PagedPlace mine[2];
    int id[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) id[half] = page_id(a.kv, b, min(j0 + 64 * half + lane, s.len - 1));
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        mine[half] = place_of(a.kv, hk, min(j0 + 64 * half + lane, s.len - 1), id[half], row16);
        gone[half] = __builtin_amdgcn_ballot_w64(!mine[half].there || j0 + 64 * half + lane >= s.len);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            const char* p = a.kv.k + ((size_t)(unsigned)__shfl((int)mine[half].off, 16 * kb + r16, 64) << 4);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int e = 32 * ks + 8 * g4;
                u32x4 x = {0u, 0u, 0u, 0u};
                if (e < Dt) {
                    if constexpr (E4M3) {
                        const u32x2 y = *(const u32x2*)(p + e);
                        const u32x2 p0 = widen4(y[0]), p1 = widen4(y[1]);
                        x = u32x4{p0[0], p0[1], p1[0], p1[1]};
                    } else {
                        x = *(const u32x4*)(p + 2 * e);
                    }
                }
                kf[half][kb][ks] = __builtin_bit_cast(bf16x8, x);
            }
        }
    float sum[2][4][4] = {};

    // ---- columns, from the first new row that counts and sees any of these keys
    const int i0 = max(max(0, s.n - a.weigh), wg0 - s.p0);
    const int c0 = i0 * G, nchunks = (ncol - c0 + kWeighCols - 1) / kWeighCols;
    auto issue = [&](int ch, int buf) {
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int row = (w * IPW + i) * RPI + lane / CH, col = min(c0 + ch * kWeighCols + row, ncol - 1);
            const int n = col / G, h = col - n * G, sc = (lane % CH) ^ swz16<CH>(row);
            const bf16_t* q = a.q + (size_t)(hk * G + h) * a.q_hs + (size_t)(s.t0 + n) * a.q_rs + (8 * sc < Dt ? 8 * sc : 0);
            g2l16(q, &qs[buf][(w * IPW + i) * 1024]);
        }
        if (tid < kWeighCols) {
            const int col = min(c0 + ch * kWeighCols + tid, ncol - 1), n = col / G, h = col - n * G, p = s.p0 + n;
            const float x = a.lse[(size_t)(hk * G + h) * a.batch.T + s.t0 + n];
            // a column past the end, or one that sees nothing, sees no key here
            const bool none = c0 + ch * kWeighCols + tid >= ncol || x == -INFINITY;
            ls[buf][tid] = none ? 0.f : x * kLog2e;
            ps[buf][tid] = none ? -1 : p;
            los[buf][tid] = none || p < 0 ? 0x7fffffff : win_lo(m, p);
        }
    };
    if (nchunks > 0) issue(0, 0);
    for (int ch = 0; ch < nchunks; ++ch) {
        const int buf = ch & 1;
        wait_vmem();
        __syncthreads();
        if (ch + 1 < nchunks) issue(ch + 1, buf ^ 1);
        if (j0 >= s.len) continue;  // a wave without keys only stages
#pragma unroll
        for (int cb = 0; cb < kWeighCols / 16; ++cb) {
            const int p = ps[buf][16 * cb + r16], lo = los[buf][16 * cb + r16];
            const float l2 = ls[buf][16 * cb + r16];
            if (__builtin_amdgcn_ballot_w64(p >= j0) == 0ull) continue;
            bf16x8 qf[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                u32x4 x = *(const u32x4*)(qs[buf] + 16 * cb * CH * 16 + row16_lane_off<CH>(ks));
                if (D > Dt && 32 * ks + 8 * g4 >= Dt) x = u32x4{0u, 0u, 0u, 0u};
                qf[ks] = __builtin_bit_cast(bf16x8, x);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int jh = j0 + 64 * half;
                f32x4 sa[4];
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) {
                    sa[kb] = zero4();
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) sa[kb] = mfma16(kf[half][kb][ks], qf[ks], sa[kb]);
                }
                if (gone[half] != 0ull || __builtin_amdgcn_ballot_w64(p < jh + 63 || lo > jh) != 0ull) {
                    unsigned gists[2] = {0u, 0u};
                    if (__builtin_amdgcn_ballot_w64(p >= 0 && lo > jh) != 0ull) {
                        const unsigned long long g = __builtin_amdgcn_ballot_w64(is_always(m, jh + lane));
                        gists[0] = (unsigned)g;
                        gists[1] = (unsigned)(g >> 32);
                    }
#pragma unroll
                    for (int kb = 0; kb < 4; ++kb) {
                        const int j = jh + 32 * (kb / 2);
                        const unsigned vis =
                            p < 0 ? 0u : (bits_below(p - j + 1) & (~bits_below(lo - j) | gists[kb / 2]) & ~(unsigned)(gone[half] >> (32 * (kb / 2))));
#pragma unroll
                        for (int i = 0; i < 4; ++i) {  // an lse that is no number concerns the keys its row sees and no others
                            const float x = __builtin_amdgcn_exp2f(fmaf(sa[kb][i], c, -l2));
                            sum[half][kb][i] += (vis >> (16 * (kb % 2) + 4 * g4 + i)) & 1u ? x : 0.f;
                        }
                    }
                } else {
#pragma unroll
                    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sum[half][kb][i] += __builtin_amdgcn_exp2f(fmaf(sa[kb][i], c, -l2));
                }
            }
        }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float own = 0.f;  // lane r16 ends with the key 16 (r16 / 4) + 4 g4 + r16 % 4
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = row16_sum(sum[half][kb][i]);
                if (r16 == 4 * kb + i) own = x;
            }
        const int j = j0 + 64 * half + 16 * (r16 >> 2) + 4 * g4 + (r16 & 3);
        const int at = j < s.len ? pool_row(a.kv, b, hk, j) : -1;
        if (at >= 0) a.kv.weight[at] = a.decay == 0.f ? own : fmaf(a.decay, a.kv.weight[at], own);
    }
}

// Weights of a sequence of few columns, from the scores that the decode kernel has left: one lane per row.
__global__ __launch_bounds__(256) void paged_weigh_few_kernel(PagedAttn a, PagedScores scores) {
    const int hk = blockIdx.y, b = blockIdx.z, j = blockIdx.x * 256 + threadIdx.x;
    const int G = a.Hq / a.kv.Hkv;
    const PagedSeq s = paged_seq(a.batch, b);
    const int ncol = s.n * G;
    if (ncol == 0 || ncol > scores.most || j >= s.len) return;
    const int at = pool_row(a.kv, b, hk, j);
    if (at < 0) return;
    const AttnShape m = mask_shape(a.mask);
    const PagedWalk walk = paged_walk(m, max(s.p0, 0), s.len);
    const int e = j >= walk.wstart ? walk.nfar + j - walk.wstart : is_always(m, j) ? count_always(m, j) : -1;
    float sum = 0.f;
    if (e >= 0) {
        const float* x = scores.x + ((size_t)b * a.kv.Hkv + hk) * scores.cols * scores.pitch + e;
        const int i0 = max(0, s.n - a.weigh);
        for (int i = i0; i < s.n; ++i)
            for (int g = 0; g < G; ++g) {
                const float lse = a.lse[(size_t)(hk * G + g) * a.batch.T + s.t0 + i];
                const float y = x[(size_t)((i - i0) * G + g) * scores.pitch];
                if (lse != -INFINITY && y != -INFINITY) sum += __builtin_amdgcn_exp2f(fmaf(-lse, kLog2e, y));
            }
    }
    a.kv.weight[at] = a.decay == 0.f ? sum : fmaf(a.decay, a.kv.weight[at], sum);
}

// ---------------------------------------------------------------------------------------------
// The launch: sequences of few columns (new rows x heads of a group) go to the decode kernel, the others to the chunk
// kernel; a batch that may hold both launches both, and each leaves the other's sequences.  The chunk kernel's workgroups are numbered
// over the tiles that there are.
// Scores of few columns are kept for the weights, 4 bytes a key and column that counts for the 128 to 256 that reading K again takes, up
// to this much memory.
constexpr int kOneSlice = 384, kLongSlice = 2048;
constexpr size_t kMostScores = (size_t)1 << 30;
// Partial results of the decode kernel's slices: at most this much.  S slices of the longest sequence are kept for every one (4.3 GB
// for 1024 sequences of up to 128K rows, 8 kv heads); so many sequences fill the CUs with longer slices too.
constexpr size_t kMostParts = (size_t)1 << 30;
// Partial results of the chunk kernel: for twice the tiles that the batch has if every sequence has new rows and one of them the chunk,
// and for as many as this holds.  A batch of more tiles is cut in fewer slices each, which fill the CUs as well.
constexpr size_t kChunkParts = (size_t)64 << 20;
struct Plan {
    int few;      // columns that the decode kernel takes at most (0: not launched)
    bool chunk;   // is the chunk kernel launched?
    int ntiles;   // of a kv head at most
    long long blocks;  // workgroups of the chunk kernel
    PagedParts dec, chk;
    PagedScores scores;  // x null: not kept
    bool keep_scores;
    size_t bytes;
};

// How the walks of a launch's `busy` tiles are cut, the longest of E entries, avg in the mean: the split whose end comes first,
// in steps of 32 entries (about 1 us at D = 128).  A CU has room for two workgroups of four waves or one of eight that takes a
// slice in two halves; a step takes two workgroups 1.08, two halves 1.2 and a lone workgroup 1.0, starting and ending a workgroup about
// 5, the merge of slices 8 and the time of the partial results' bytes.  us, by this / by as many slices as fill the CUs, in halves
// up to 256 tiles (32/8 heads): 2048 tokens from the first 60 / 72, 512 at 32K 312 / 331, 64 at 1000 22.2 / 25.0, 64 at 32K 58.1 / 58.9;
// 8/1 heads, 700 at 32K 127 / 138.
struct ChunkSplit {
    int groups, S;
};
ChunkSplit split_chunks(long busy, int E, double avg) {
    ChunkSplit best = {1, 1};
    double least = 1e30;
    for (int g = 1; g <= 2; ++g)
        for (int S = 1; S <= 32 && (S == 1 || E / S >= 256); ++S) {
            const long wgs = busy * S, slots = g == 1 ? 512 : 256, rounds = (wgs + slots - 1) / slots;
            const double steps = std::max((double)E, rounds * avg) / 32.0 / (S * g);
            const double t = steps * (g == 2 ? 1.2 : wgs > 256 ? 1.08 : 1.0) + 5.0 * rounds + (S > 1 ? 8.0 + 0.026 * wgs : 0.0);
            if (t < least) {
                least = t;
                best = {g, S};
            }
        }
    return best;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int built_for(int D) { return D <= 64 ? 64 : D <= 96 ? 96 : 128; }

Plan make_plan(const PagedAttn& a, char* ws) {
    Plan p = {};
    const int G = a.Hq / a.kv.Hkv, Hkv = a.kv.Hkv, B = a.batch.B, T = a.batch.T, D = built_for(a.kv.D);
    const AttnShape m = mask_shape(a.mask);
    const long most = (long)a.batch.max_new * G;  // columns of a sequence at most
    // Where a batch has long chunks, the others are mostly single tokens: 16 columns, two workgroups a CU (32: one), if a token has no more.
    p.few = most <= 16 || (most > 32 && G <= 16) ? 16 : 32;
    p.chunk = most > p.few;
    if (B == 1 && p.chunk) p.few = 0;
    size_t off = 0;
    auto place = [&](PagedParts& x, size_t slices, int cols) {  // slices: of all units
        x.cols = cols;
        if (x.S <= 1) return;
        const size_t n = slices * cols;
        x.ml = (float*)(ws + off);
        off += align256(n * 2 * sizeof(float));
        x.acc = (float*)(ws + off);
        off += align256(n * D * sizeof(float));
    };
    if (p.few) {
        const int E = paged_walk(m, a.batch.max_kv - 1, a.batch.max_kv).E;
        const long units = (long)B * Hkv;
        int want = (int)std::min<long>(((long)E * units + 255) / 256, kLongSlice);
        want = std::max(want, E <= kOneSlice ? E : 128);
        const size_t one = (size_t)units * std::min<long>(p.few, most) * (D + 2) * sizeof(float);  // a slice of each
        const int most_slices = (int)std::max<size_t>(1, std::min<size_t>(64, kMostParts / one));  // the merge takes 64
        want = std::max(want, (E + most_slices - 1) / most_slices);
        p.dec.want = (want + 127) / 128 * 128;
        p.dec.S = std::min(64, std::max(1, (E + p.dec.want - 1) / p.dec.want));
        place(p.dec, (size_t)units * p.dec.S, (int)std::min<long>(p.few, most));
    }
    if (p.chunk) {
        const long cols = (long)T * G, busy = (cols + kChunkCols - 1) / kChunkCols * Hkv;  // tiles of all heads
        p.ntiles = (int)(cols / kChunkCols + std::min<long>(B, cols / (p.few + 1)));          // a sequence that has any is of more than `few` columns
        const int rows = std::min(a.batch.max_new, kChunkCols / G + 1);
        const int E = paged_walk(m, std::max(0, a.batch.max_kv - rows), a.batch.max_kv).E;  // the last tile of the longest walk
        const int first = std::max(0, a.batch.max_kv - a.batch.max_new);
        const int E0 = paged_walk(m, first, std::min(first + rows, a.batch.max_kv)).E;        // and its sequence's first
        const ChunkSplit x = split_chunks(busy, E, 0.5 * ((double)E + E0));
        p.chk.groups = x.groups;
        p.chk.S = x.S;
        p.chk.want = x.S == 1 ? 1 << 24 : (E + x.S - 1) / x.S;
        const long chunk = std::max<long>(T - B + 1, std::min(a.batch.max_new, T)) * G;  // columns of the chunk if the others are tokens
        const long room = std::max<long>(2 * (chunk / kChunkCols + 1) * x.S, kChunkParts / ((size_t)Hkv * kChunkCols * (D + 2) * sizeof(float)));
        p.chk.units = x.S == 1 ? p.ntiles : (int)std::min<long>(room, (long)p.ntiles * x.S);
        p.blocks = (long long)std::max(p.chk.units, p.ntiles) * Hkv;
        place(p.chk, (size_t)p.chk.units * Hkv, kChunkCols);
    }
    if (p.few && a.weigh) {
        p.scores.most = p.dec.cols;
        p.scores.cols = (int)std::min<long>(p.dec.cols, (long)a.weigh * G);
        p.scores.pitch = (a.batch.max_kv + 127) / 128 * 128;
        const size_t n = (size_t)B * Hkv * p.scores.cols * p.scores.pitch * sizeof(float);
        p.keep_scores = n <= kMostScores;
        if (p.keep_scores) {
            p.scores.x = (float*)(ws + off);
            off += align256(n);
        }
    }
    // an axis of a launch takes fewer than 2^32 threads
    p.bytes = p.blocks * 256 * std::max(p.chk.groups, 1) > 0xffffffffLL ? 0 : std::max<size_t>(off, 256);
    return p;
}

template <int D>
hipError_t launch_combine(const PagedAttn& a, const Plan& p, hipStream_t st) {
    if (p.few && p.dec.S > 1) {
        const int cols = p.dec.cols;
        if (p.dec.S > kBatch) paged_combine_kernel<D, 4><<<dim3(cols, a.kv.Hkv, a.batch.B), 256, 0, st>>>(a, p.dec);
        else paged_combine_kernel<D, 1><<<dim3((cols + 3) / 4, a.kv.Hkv, a.batch.B), 256, 0, st>>>(a, p.dec);
    }
    if (p.chunk && p.chk.S > 1)
        paged_combine_chunk_kernel<D><<<dim3(std::min(p.ntiles, p.chk.units / 2), a.kv.Hkv, kChunkCols / 16), 256, 0, st>>>(a, p.chk, p.few);
    return hipGetLastError();
}

}  // namespace

size_t paged_attn_bytes(const PagedAttn& a, bool) { return make_plan(a, nullptr).bytes; }

hipError_t launch_paged_attn(const PagedAttn& a, bool e4m3, void* ws, hipStream_t st) {
    const Plan p = make_plan(a, (char*)ws);
    hipError_t e = hipSuccess;
    if (p.chunk) e = launch_paged_chunk(a, e4m3, p.chk, p.blocks, p.few, st);
    if (e == hipSuccess && p.few) e = launch_paged_decode(a, e4m3, p.dec, p.keep_scores ? p.scores : PagedScores{}, p.few, st);
    const int D = built_for(a.kv.D);
    if (e == hipSuccess) e = D == 64 ? launch_combine<64>(a, p, st) : D == 96 ? launch_combine<96>(a, p, st) : launch_combine<128>(a, p, st);
    if (e != hipSuccess || !a.weigh) return e;
    if (p.keep_scores) {
        paged_weigh_few_kernel<<<dim3((a.batch.max_kv + 255) / 256, a.kv.Hkv, a.batch.B), 256, 0, st>>>(a, p.scores);
        e = hipGetLastError();
        if (e != hipSuccess || !p.chunk) return e;
    }
    const int min_cols = p.keep_scores ? p.scores.most : 0;
    auto go = [&](auto kern) { kern<<<dim3((a.batch.max_kv + kWeighKeys - 1) / kWeighKeys, a.kv.Hkv, a.batch.B), 256, 0, st>>>(a, min_cols); };
    if (D == 64) e4m3 ? go(paged_weigh_kernel<64, true>) : go(paged_weigh_kernel<64, false>);
    else if (D == 96) e4m3 ? go(paged_weigh_kernel<96, true>) : go(paged_weigh_kernel<96, false>);
    else e4m3 ? go(paged_weigh_kernel<128, true>) : go(paged_weigh_kernel<128, false>);
    return hipGetLastError();
}

}  // namespace unigist
