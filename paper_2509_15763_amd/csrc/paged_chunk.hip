// Attention of many new rows per sequence over a paged cache: prompt chunks.
//
// The (new row, query head of the group) pairs of one kv head of one sequence are columns, heads first; a workgroup takes
// 128 of them, a wave 32 (two 16-column blocks), and walks the entries that they see 32 at a time: S^T = K Q^T and
// O^T += V^T P^T on v_mfma_f32_16x16x32_bf16 as in the forward kernel, K and V tiles through two LDS stages, one barrier a
// step.  With heads first, the heads of a group share every tile, and 128 columns span only 128 / G positions: fewer
// masked steps at the diagonal and the window's edge.  P is rounded to bf16 for the second product, sums and accumulators are fp32 (out
// differs from 64 bits by 2.3e-3 of its norm, where the store alone makes 1.7e-3).
//   bf16: direct global -> LDS loads; codes: through registers, widened once per workgroup on the way.
// Places: 256 entries (eight steps) at a time, one per thread, into one of two tables in LDS; the table entries of the next
// 256 are loaded a block ahead and the places of a step are read from LDS one step ahead.
// Few workgroups: a lone wave per SIMD took about 2000 cycles a step where two together took 2200 (now 1900), so the entries of a
// tile are shared out in slices, two to a workgroup of eight waves (GROUPS, merged through LDS), and from there on to workgroups (merged by
// paged_combine_chunk_kernel).
#include "paged_common.h"

namespace unigist {
namespace {

constexpr int BN = 32;   // entries per step
constexpr int NT = 256;
constexpr int kBlock = 256;  // entries per block of places
constexpr float kLazy = 8.f;         // slack of the softmax reference, in exp2 units
constexpr float kBigSum = 16384.f;   // a partial sum above this sends the step through the maximum search

template <int D>
struct ChunkSmem {
    static constexpr int CH = D <= 64 ? 8 : 16;
    char k[2][BN * CH * 16];
    char v[2][BN * CH * 16];
    unsigned places[2][kBlock];
    unsigned gone[2][kBlock / 32];  // a bit per entry that is not there
};

template <int D, bool E4M3, int GROUPS>
__global__ __launch_bounds__(NT * GROUPS, 2) void paged_chunk_kernel(PagedAttn a, PagedParts parts, int min_cols) {
    constexpr int KS = D / 32, DB = D / 16, CH = D <= 64 ? 8 : 16;
    constexpr int RPI = 64 / CH;       // tile rows of one direct load
    constexpr int IPW = BN / RPI / 4;  // direct loads per wave, matrix and tile
    constexpr int PPR = CH / 2;        // 16-code pieces of a row
    constexpr int PCS = BN * PPR;      // pieces of a tile: 256 or 128
    constexpr int kMerge = GROUPS > 1 ? 4 * 64 * (DB * 2 * 16 + 2 * 8) : 0, kStages = GROUPS * (int)sizeof(ChunkSmem<D>);
    __shared__ __attribute__((aligned(1024))) char smem[kStages > kMerge ? kStages : kMerge];
    const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    ChunkSmem<D>& sm = ((ChunkSmem<D>*)smem)[group];

    const int tid = threadIdx.x % NT, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);  // inside the group
    const int r16 = lane & 15, g4 = lane >> 4;
    const int Hkv = a.kv.Hkv, G = a.Hq / Hkv, Dt = a.kv.D;

    // ---- which kv head, slice and tile: late tiles, which walk further, first
    const int hk = blockIdx.x % Hkv, rest = blockIdx.x / Hkv;
    const PagedTiles tiles = count_tiles(a.batch, G, min_cols);
    const int S = slices_of(parts, tiles.total), slice = rest % S, tile = tiles.total - 1 - rest / S;
    if (tile < 0) return;
    int nth;
    const int b = seq_of_tile(a.batch, G, min_cols, tiles, tile, nth);
    const PagedSeq s = paged_seq(a.batch, b);
    const int ncol = s.n * G, c0 = nth * kChunkCols;
    if ((unsigned)nth * kChunkCols >= (unsigned)ncol) return;  // boundaries that decrease
    const AttnShape m = mask_shape(a.mask);
    const int c1 = min(c0 + kChunkCols, ncol) - 1;  // last column
    const int pf = s.p0 + c0 / G, pe = s.p0 + c1 / G;
    PagedWalk walk = {0, 0, 0};
    if (pe >= 0) walk = paged_walk(m, max(pf, 0), pe + 1);
    const PagedSlices sl = paged_slices(walk.E, S, parts.want, BN);
    if (slice >= sl.n) return;
    const int a0 = slice * sl.per, a1 = min(walk.E, a0 + sl.per);                   // the workgroup's entries
    const int per = ((a1 - a0 + GROUPS - 1) / GROUPS + BN - 1) / BN * BN;          // of them a group's
    const int e0 = min(a1, a0 + group * per), e1 = min(a1, e0 + per);
    const int nsteps = (e1 - e0 + BN - 1) / BN;
    const int nmeet = GROUPS > 1 ? (min(per, a1 - a0) + BN - 1) / BN : nsteps;     // both groups meet at every step of the first, which has no fewer

    // ---- the wave's columns
    const int cw = c0 + 32 * wv;  // first
    const bool live_wave = cw <= c1;
    int pos[2], lo[2];
    bf16x8 qf[2][KS];
    f32x4 o[DB][2];
    float mr[2], l[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int col = min(cw + 16 * qb + r16, c1), i = col / G, h = col - i * G;  // columns past the end shadow the last
        pos[qb] = s.p0 + i;
        lo[qb] = pos[qb] >= 0 ? win_lo(m, pos[qb]) : 0;
        const bf16_t* q = a.q + (size_t)(hk * G + h) * a.q_hs + (size_t)(s.t0 + i) * a.q_rs;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x4 z = {0u, 0u, 0u, 0u};  // columns past the tensors' head dimension are zero
            if (32 * ks + 8 * g4 < Dt) z = *(const u32x4*)(q + 32 * ks + 8 * g4);
            qf[qb][ks] = __builtin_bit_cast(bf16x8, z);
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db][qb] = zero4();
        mr[qb] = -INFINITY;
        l[qb] = 0.f;
    }
    const int p_first = s.p0 + min(cw, c1) / G, p_last = s.p0 + min(cw + 31, c1) / G;
    const int lo_last = p_last >= 0 ? win_lo(m, p_last) : 0;
    bool need_max = true;
    const float c = a.scale * (E4M3 ? a.kv.kscale[hk] : 1.f) * kLog2e;

    // ---- staging
    const int row_bytes = Dt * (E4M3 ? 1 : 2), row16 = row_bytes / 16;
    const int lrow = lane / CH;
    const char *kl[IPW], *vl[IPW];  // bf16: with the byte offset of the lane's (swizzled) chunk inside its row, per load
    int rr[IPW];                    // row of the tile
    // codes: piece tid of K (and of V, D > 64), or for D = 64 threads 0 .. 127 a piece of K, the others one of V
    const int piece = tid % PCS, prow = piece / PPR, pcol = piece % PPR;
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
        rr[i] = E4M3 ? prow : (wv * IPW + i) * RPI + lrow;
        const int sc = (lane % CH) ^ swz16<CH>(rr[i]);
        const int off = E4M3 ? (16 * pcol < row_bytes ? 16 * pcol : 0) : (16 * sc < row_bytes ? 16 * sc : 0);  // a chunk the rows do not have: any
        kl[i] = a.kv.k + off;
        vl[i] = a.kv.v + off;
    }
    auto row_of = [&](int j) { return entry_row(m, walk, max(min(e0 + kBlock * j + tid, e1 - 1), 0)); };
    auto put = [&](int j, int id) {
        const PagedPlace p = place_of(a.kv, hk, row_of(j), id, row16);
        sm.places[j & 1][tid] = p.off;
        const unsigned long long gone = __builtin_amdgcn_ballot_w64(!p.there || e0 + kBlock * j + tid >= e1);
        if (lane == 0) {
            sm.gone[j & 1][2 * wv] = (unsigned)gone;
            sm.gone[j & 1][2 * wv + 1] = (unsigned)(gone >> 32);
        }
    };
    // Places (and missing entries) of tile `it`, in the registers of its parity: read a step before they are needed, behind the
    // tile's own reads of LDS (in front of them 2.5 % slower on a long chunk), and without a condition, since values that meet in
    // one register behind a branch are waited for there.  The tables hold something for two steps past the end too.
    unsigned at[2][IPW], gone_at[2];
    auto places_of = [&](int it, int odd) __attribute__((always_inline)) {
        const int j = (it >> 3) & 1;
#pragma unroll
        for (int i = 0; i < (E4M3 ? 1 : IPW); ++i) at[odd][i] = sm.places[j][(it & 7) * BN + rr[i]];
        gone_at[odd] = sm.gone[j][it & 7];
    };
    u32x4 ck, cv;  // codes on their way
    auto issue = [&](int buf) {  // tile `it` goes to stage it % 2, from the places of that parity
        if constexpr (E4M3) {
            const size_t off = (size_t)at[buf][0] << 4;
            if (PCS == NT || tid < PCS) ck = *(const u32x4*)(kl[0] + off);
            if (PCS == NT || tid >= PCS) cv = *(const u32x4*)(vl[0] + off);
        } else {
#pragma unroll
            for (int i = 0; i < IPW; ++i) {
                const size_t off = (size_t)at[buf][i] << 4;
                g2l16(kl[i] + off, &sm.k[buf][(wv * IPW + i) * 1024]);
                g2l16(vl[i] + off, &sm.v[buf][(wv * IPW + i) * 1024]);
            }
        }
    };
    auto land = [&](int buf) {  // codes widened into the stage
        auto store = [&](char* tile, const u32x4& x) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const u32x2 p0 = widen4(x[2 * t]), p1 = widen4(x[2 * t + 1]);
                *(u32x4*)(tile + prow * (CH * 16) + (((2 * pcol + t) ^ swz16<CH>(prow)) << 4)) = u32x4{p0[0], p0[1], p1[0], p1[1]};
            }
        };
        if (PCS == NT || tid < PCS) store(sm.k[buf], ck);
        if (PCS == NT || tid >= PCS) store(sm.v[buf], cv);
    };

    int koff[KS], voff[DB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = row16_lane_off<CH>(ks);
#pragma unroll
    for (int db = 0; db < DB; ++db) voff[db] = tr16_lane_off16<CH>(db);

    // Masked tiles whose V holds numbers that are not finite, or which miss a row's page, are left for a second walk over the steps
    // from the first of them to the last: their product is many times as long, and where the two meet in one step, every step
    // copies its accumulators (4096 tokens at 28K: 2103 us with both in one step, 1955 us so).
    int c_first = 0x7fffffff, c_last = -1;
    auto tile_step = [&](auto bufc, auto carefulc, int it, unsigned gone) __attribute__((always_inline)) {
        constexpr int BUF = decltype(bufc)::value;
        constexpr bool CAREFUL = decltype(carefulc)::value;
        const char* kt = sm.k[BUF];
        const char* vt = sm.v[BUF];
        const int base = e0 + it * BN;
        const int top = base + BN - 1 - walk.nfar + walk.wstart, bot = max(base, walk.nfar) - walk.nfar + walk.wstart;  // rows of the window part
        if (!live_wave || p_last < 0 || (base >= walk.nfar && bot > p_last)) return;
        const bool masked = gone != 0u || p_first < 0 || (base + BN > walk.nfar && (top > p_first || bot < lo_last));
        if (CAREFUL && !masked) return;

        // ---- S^T = K Q^T, the K fragments read two ahead of their MFMAs
        f32x4 sa[2][2];
        {
            constexpr int N = 2 * KS, PFK = 2;
            bf16x8 fk[N];
            auto fetch = [&](int n) __attribute__((always_inline)) { fk[n] = *(const bf16x8*)(kt + (n / KS) * 16 * CH * 16 + koff[n % KS]); };
#pragma unroll
            for (int n = 0; n < PFK; ++n) fetch(n);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n + PFK < N) fetch(n + PFK);
                const int kb = n / KS, ks = n % KS;
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) sa[kb][qb] = mfma16(fk[n], qf[qb][ks], ks == 0 ? zero4() : sa[kb][qb]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (masked) {
            const unsigned gists = bot < lo_last ? (unsigned)__builtin_amdgcn_ballot_w64(lane < BN && base + lane >= walk.nfar &&
                                                                                         is_always(m, base + lane - walk.nfar + walk.wstart))
                                                 : 0u;
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                const unsigned vis = entry_bits(walk, base, pos[qb], lo[qb], gists, gone) >> (4 * g4);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((vis >> (16 * kb + i)) & 1u)) sa[kb][qb][i] = -INFINITY;
            }
            unsigned odd = 0u;
#pragma unroll
            for (int t = 0; t < BN * CH / 64; ++t) {
                const u32x4 x = *(const u32x4*)(vt + (t * 64 + lane) * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= not_finite2(x[e]);
            }
            // A row whose page is not there stands for one of another sequence, which may change between the walks.
            const bool missing = (gone & bits_below(e1 - base)) != 0u;
            const bool careful = missing || __builtin_amdgcn_ballot_w64((odd & 0x80008000u) != 0u) != 0ull;
            if (careful != CAREFUL) {
                if (!CAREFUL) {
                    c_first = min(c_first, it);
                    c_last = it;
                }
                return;
            }
        }

        // ---- online softmax: a column is spread over the 4 lanes r16 + 16 g4; its reference is kept identical on them
        u32x4 pk[2];
        float ls[2];
        auto exps = [&](int qb, float mc) __attribute__((always_inline)) {
            float p[8];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) p[4 * kb + i] = __builtin_amdgcn_exp2f(fmaf(sa[kb][qb][i], c, -mc));
            ls[qb] = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
            for (int t = 0; t < 4; ++t) pk[qb][t] = pack_bf16x2(p[2 * t], p[2 * t + 1]);
        };
        bool with_max = need_max;
        if (!with_max) {
            exps(0, mr[0] * c);
            exps(1, mr[1] * c);
            with_max = __builtin_amdgcn_ballot_w64(!(ls[0] <= kBigSum) || !(ls[1] <= kBigSum)) != 0ull;
        }
        if (with_max) {
            bool any_inf = false;
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                float mx = sa[0][qb][0];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sa[kb][qb][i]);
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const bool grow = (mx - mr[qb]) * c > kLazy;
                if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
                    const float m_new = grow ? mx : mr[qb];
                    const float alpha = grow ? __builtin_amdgcn_exp2f((mr[qb] - m_new) * c) : 1.f;  // m = -inf gives 0
                    l[qb] *= alpha;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[db][qb][i] *= alpha;
                    mr[qb] = m_new;
                }
                exps(qb, (mr[qb] == -INFINITY ? 0.f : mr[qb]) * c);
                any_inf = any_inf || mr[qb] == -INFINITY;
            }
            need_max = __builtin_amdgcn_ballot_w64(any_inf) != 0ull;
        }
        l[0] += ls[0];
        l[1] += ls[1];

        // ---- O^T += V^T P^T
        if constexpr (CAREFUL) {
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                bf16x8 vf = tr16_frag16<CH>(vt + voff[db], 0);
                careful_v(vf, pk, o[db]);
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) o[db][qb] = mfma16(vf, __builtin_bit_cast(bf16x8, pk[qb]), o[db][qb]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            constexpr int PFV = 2;
            s16x4 x0[DB], x1[DB];
            auto fetch = [&](int db) __attribute__((always_inline)) {
                const char* p = vt + voff[db];
                x0[db] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
                x1[db] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * CH * 16));
            };
#pragma unroll
            for (int db = 0; db < PFV; ++db) fetch(db);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                if (db + PFV < DB) fetch(db + PFV);
                const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x0[db], x1[db], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) o[db][qb] = mfma16(vf, __builtin_bit_cast(bf16x8, pk[qb]), o[db][qb]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    auto walk_steps = [&](auto carefulc, int from, int to) __attribute__((always_inline)) {  // from: a multiple of 8
        const int end = min(nsteps, to);
        put(from >> 3, page_id(a.kv, b, row_of(from >> 3)));
        int ahead = page_id(a.kv, b, row_of((from >> 3) + 1));
        __syncthreads();
        places_of(from, 0);
        if (GROUPS == 1 || from < end) issue(0);
        if (E4M3 && (GROUPS == 1 || from < end)) land(0);
        places_of(from + 1, 1);
        // One step: the other stage is filled for the next one meanwhile.  Places of block j + 1 are written in the middle of block
        // j, over those of block j - 1, which were read for the last time two steps before its end.
        auto one = [&](auto bufc, int it) __attribute__((always_inline)) {
            constexpr int BUF = decltype(bufc)::value;
            if (!E4M3) wait_vmem();  // this wave's part of tile `it` has landed
            __syncthreads();         // ... and everyone's; everyone is also done reading the other stage
            const unsigned gone = __builtin_amdgcn_readfirstlane(gone_at[BUF]);
            if ((it & 7) == 4) {
                put((it >> 3) + 1, ahead);
                ahead = page_id(a.kv, b, row_of((it >> 3) + 2));
            }
            const bool more = it + 1 < end;
            if (more) issue(BUF ^ 1);
            if (GROUPS == 1 || it < end) tile_step(bufc, carefulc, it, gone);
            places_of(it + 2, BUF);
            if (E4M3 && more) land(BUF ^ 1);
        };
        for (int it = from; it < to; it += 2) {
            one(std::integral_constant<int, 0>{}, it);
            if (it + 1 < to) one(std::integral_constant<int, 1>{}, it + 1);
        }
    };
    if (nmeet > 0) {
        walk_steps(std::false_type{}, 0, nmeet);
        int* left = (int*)((ChunkSmem<D>*)smem)[0].places;  // [waves of the workgroup][first, last]
        __syncthreads();                                    // the tables are dead
        if (lane == 0) {
            left[2 * (group * 4 + wv)] = c_first;
            left[2 * (group * 4 + wv) + 1] = c_last;
        }
        __syncthreads();
        int first = 0x7fffffff, last = -1;
#pragma unroll
        for (int w = 0; w < 4 * GROUPS; ++w) {
            first = min(first, left[2 * w]);
            last = max(last, left[2 * w + 1]);
        }
        if (last >= 0) {  // alike in all waves
            __syncthreads();
            walk_steps(std::true_type{}, first & ~7, last + 1);
        }
    }

    if constexpr (GROUPS > 1) {  // the second group's waves leave their part to those of the first: same columns, same lanes
        f32x4* mo = (f32x4*)smem;                                            // [4 waves][DB][2][64 lanes]
        f32x2* ml = (f32x2*)(smem + 4 * DB * 2 * 64 * 16);                   // [4 waves][2][64 lanes]
        __syncthreads();  // the stages are dead
        if (group == 1) {
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                ml[(wv * 2 + qb) * 64 + lane] = f32x2{mr[qb], l[qb]};
#pragma unroll
                for (int db = 0; db < DB; ++db) mo[((wv * DB + db) * 2 + qb) * 64 + lane] = o[db][qb];
            }
        }
        __syncthreads();
        if (group == 1) return;
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const f32x2 x = ml[(wv * 2 + qb) * 64 + lane];
            const float mm = fmaxf(mr[qb], x[0]);
            const float f = mr[qb] == mm ? 1.f : __builtin_amdgcn_exp2f((mr[qb] - mm) * c), g = x[0] == mm ? 1.f : __builtin_amdgcn_exp2f((x[0] - mm) * c);
            l[qb] = l[qb] * f + x[1] * g;
            mr[qb] = mm;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db][qb] = o[db][qb] * f + mo[((wv * DB + db) * 2 + qb) * 64 + lane] * g;
        }
    }

    // ---- epilogue
    if (!live_wave) return;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        float lt = l[qb];
        lt += __shfl_xor(lt, 16, 64);
        lt += __shfl_xor(lt, 32, 64);
        const int col = cw + 16 * qb + r16;
        if (col > c1) continue;
        const float vmul = E4M3 ? a.kv.vscale[hk] : 1.f;
        if (sl.n > 1) {
            const size_t at_col = (((size_t)tile * Hkv + hk) * S + slice) * kChunkCols + (col - c0);
            if (g4 == 0) *(f32x2*)(parts.ml + 2 * at_col) = f32x2{mr[qb] * c, lt};
#pragma unroll
            for (int db = 0; db < DB; ++db) *(f32x4*)(parts.acc + at_col * D + 16 * db + 4 * g4) = o[db][qb] * vmul;
            continue;
        }
        const float inv = lt == 0.f ? 0.f : vmul / lt;
        const int i = col / G, hq = hk * G + (col - i * G), t = s.t0 + i;
        bf16_t* op = a.out + (size_t)hq * a.q_hs + (size_t)t * a.q_rs + 4 * g4;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            if (16 * db + 4 * g4 >= Dt) continue;
            u32x2 w2;
            w2[0] = pack_bf16x2(o[db][qb][0] * inv, o[db][qb][1] * inv);
            w2[1] = pack_bf16x2(o[db][qb][2] * inv, o[db][qb][3] * inv);
            *(u32x2*)(op + 16 * db) = w2;
        }
        if (g4 == 0 && a.lse) a.lse[(size_t)hq * a.batch.T + t] = lt == 0.f ? -INFINITY : mr[qb] * c * kLn2 + __builtin_amdgcn_logf(lt) * kLn2;
    }
}

}  // namespace

hipError_t launch_paged_chunk(const PagedAttn& a, bool e4m3, const PagedParts& parts, long long blocks, int min_cols, hipStream_t st) {
    auto go = [&](auto kern) { kern<<<dim3((unsigned)blocks), NT * parts.groups, 0, st>>>(a, parts, min_cols); };
    auto pick = [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (parts.groups == 1) e4m3 ? go(paged_chunk_kernel<D, true, 1>) : go(paged_chunk_kernel<D, false, 1>);
        else e4m3 ? go(paged_chunk_kernel<D, true, 2>) : go(paged_chunk_kernel<D, false, 2>);
    };
    if (a.kv.D <= 64) pick(std::integral_constant<int, 64>{});
    else if (a.kv.D <= 96) pick(std::integral_constant<int, 96>{});
    else pick(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace unigist
