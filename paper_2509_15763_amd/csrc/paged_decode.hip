// Attention of few new rows per sequence over a paged cache: single tokens and drafts.
//
// The (new row, query head of the group) pairs of one kv head of one sequence are columns, up to 16 or 32 of them; a
// workgroup takes all of them and a slice of the entries that they walk, so that each key and value is read once: the op is
// bound by the cache bytes.  A wave takes 32 entries per iteration, the workgroup's four 128:
//   S^T = K Q^T     v_mfma_f32_16x16x32_bf16, A = K rows straight from memory (lane r16 + 16 g4: key r16, 16 bytes at 64 t + 16 g4),
//                   B = Q^T in registers;
//   softmax         a column is spread over four lanes, its reference is raised lazily, the sum is a per-lane partial; no
//                   maximum is searched in the common iteration;
//   O^T += V^T P^T  P in place as the B operand; V through a wave-private LDS tile (codes widened) and back transposed.
// P is rounded to bf16 before the second product, as the matrix cores take it and as the forward kernel does; its sum is of the
// unrounded values, sums and accumulators are fp32.  The rounding is as large as that of the stored result: out differs from 64 bits by
// 2.3e-3 of its norm where the store alone makes 1.7e-3.
// Rows lie wherever the table says.  A wave works out the places of 64 entries (two iterations) at a time, one per lane:
// the table entries of two pairs ahead are loaded early, and the places go through a wave-private table in LDS from which
// every lane reads those of the rows it fetches.  The loads of the next 32 entries are issued before the work on these.
#include "paged_common.h"

namespace unigist {
namespace {

constexpr int NT = 256;
constexpr float kSlack = 8.f;       // the reference is raised when a score exceeds it by 2^kSlack
constexpr float kBigSum = 16384.f;  // a partial sum above this sends the iteration through the maximum search

// D: built-for head dimension (64, 96, 128), FULL: known to be the tensors' too (at 128, where the addresses'
// registers decide between one and two workgroups per CU), NB: 16-column blocks
template <int D, bool FULL, bool E4M3, int NB>
__global__ __launch_bounds__(NT, NB == 1 && (FULL || D < 128 || E4M3) ? (D == 64 ? 3 : 2) : 1) void paged_decode_kernel(PagedAttn a, PagedParts parts, PagedScores scores) {
    constexpr int KS = D / 32, DB = D / 16, CH = D <= 64 ? 8 : 16;  // k-steps, blocks of O^T, 16-byte chunks of an LDS row
    constexpr int NK = E4M3 ? KS / 2 : KS;                          // 16-byte loads of a K row per lane
    constexpr int NH = E4M3 ? KS % 2 : 0;                           // 8-byte ones behind them
    constexpr int LPR = E4M3 ? CH / 2 : CH;                         // lanes of a V row
    constexpr int NLV = LPR / 2;                                    // V loads per lane: rows NLV (lane / LPR) + j of 32
    constexpr int COLS = 16 * NB;
    constexpr int PD = D + 4;  // floats between columns of the merge buffer
    constexpr int kTile = 32 * CH * 16, kMerge = 4 * COLS * (PD + 2) * 4;
    __shared__ __attribute__((aligned(1024))) char smem[4 * kTile > kMerge ? 4 * kTile : kMerge];
    __shared__ __attribute__((aligned(16))) unsigned places[4][2][64];

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g4 = lane >> 4;
    const int hk = blockIdx.x, b = blockIdx.y, slice = blockIdx.z;
    const int G = a.Hq / a.kv.Hkv;
    const PagedSeq s = paged_seq(a.batch, b);
    const int ncol = s.n * G;
    if (ncol == 0 || ncol > parts.cols) return;  // parts.cols <= COLS
    const AttnShape m = mask_shape(a.mask);
    const int p_last = s.len - 1, p_first = s.p0;
    PagedWalk walk = {0, 0, 0};
    if (s.len > 0) walk = paged_walk(m, max(p_first, 0), s.len);
    const PagedSlices sl = paged_slices(walk.E, parts.S, parts.want, 128);
    if (slice >= sl.n) return;
    const int e0 = slice * sl.per, e1 = min(walk.E, e0 + sl.per);
    const float c = a.scale * (E4M3 ? a.kv.kscale[hk] : 1.f) * kLog2e;  // exp(x * scale) = exp2(x * c)

    // ---- columns: B operand Q^T, positions
    bf16x8 qf[NB][KS];
    int pos[NB], lo[NB];
    const int Dt = FULL ? D : a.kv.D;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int col = min(16 * nb + r16, ncol - 1), i = col / G, h = col - i * G;  // columns past the end shadow the last
        pos[nb] = p_first + i;
        lo[nb] = pos[nb] >= 0 ? win_lo(m, pos[nb]) : 0;
        const bf16_t* q = a.q + (size_t)(hk * G + h) * a.q_hs + (size_t)(s.t0 + i) * a.q_rs;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int e = !E4M3 || ks >= 2 * NK ? 32 * ks + 8 * g4 : 64 * (ks / 2) + 16 * g4 + 8 * (ks % 2);
            u32x4 z = {0u, 0u, 0u, 0u};
            if (e < Dt) z = *(const u32x4*)(q + e);
            qf[nb][ks] = __builtin_bit_cast(bf16x8, z);
        }
    }
    const int lo_last = p_last >= 0 ? win_lo(m, p_last) : 0;
    f32x4 o[DB][NB];
    float mr[NB], l[NB];
    bool need_max = true;  // until every column of the wave has a reference
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db][nb] = zero4();
        mr[nb] = -INFINITY;
        l[nb] = 0.f;
    }

    const int row_bytes = Dt * (E4M3 ? 1 : 2), row16 = row_bytes / 16;
    char* vt = smem + w * kTile;
    int toff[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) toff[db] = tr16_lane_off16<CH>(db);
    // pieces that a row does not have: its first one again (their q is zero, their columns of O are not stored)
    auto piece = [&](int at) { return FULL || at < row_bytes ? at : 0; };
    const char* kl[FULL ? 1 : NK + NH];  // FULL: piece t lies at a constant distance
    const char* kh = a.kv.k + piece(64 * NK + 8 * g4);
    if constexpr (FULL) {
        kl[0] = a.kv.k + 16 * g4;
    } else {
#pragma unroll
        for (int t = 0; t < NK; ++t) kl[t] = a.kv.k + piece(64 * t + 16 * g4);
    }
    const char* vl = a.kv.v + piece(16 * (lane % LPR));

    // ---- places: of the entries `base` + lane (lanes 0 .. 31) and `base` + 96 + lane, i.e. of this iteration and the next
    unsigned* pl = &places[w][0][0];
    auto entry_of = [&](int base) { return base + (lane < 32 ? lane : 96 + lane); };
    auto row_of = [&](int base) { return entry_row(m, walk, min(entry_of(base), e1 - 1)); };
    auto put = [&](int base, int id, int half) -> unsigned long long {  // -> entries that are not there
        const PagedPlace p = place_of(a.kv, hk, row_of(base), id, row16);
        pl[half * 64 + lane] = p.off;
        return __builtin_amdgcn_ballot_w64(!p.there || entry_of(base) >= e1);
    };

    struct Tile {
        u32x4 kw[2][NK > 0 ? NK : 1], vw[NLV];
        u32x2 kx[2];
    };
    auto load = [&](Tile& x, const unsigned* at) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const size_t off = (size_t)at[16 * kb + r16] << 4;
#pragma unroll
            for (int t = 0; t < NK; ++t) x.kw[kb][t] = *(const u32x4*)((FULL ? kl[0] + 64 * t : kl[t]) + off);
            if (NH) x.kx[kb] = *(const u32x2*)(kh + off);
        }
        unsigned vo[NLV];
#pragma unroll
        for (int j = 0; j < NLV; ++j) vo[j] = at[NLV * (lane / LPR) + j];
#pragma unroll
        for (int j = 0; j < NLV; ++j) x.vw[j] = *(const u32x4*)(vl + ((size_t)vo[j] << 4));
    };
    auto step = [&](const Tile& x, int base, unsigned gone) __attribute__((always_inline)) {
        // ---- S^T = K Q^T
        f32x4 sa[NB][2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) sa[nb][kb] = zero4();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                u32x4 kf;
                if constexpr (E4M3) {
                    unsigned w0, w1;
                    if (ks < 2 * NK) {
                        w0 = x.kw[kb][ks / 2][2 * (ks % 2)];
                        w1 = x.kw[kb][ks / 2][2 * (ks % 2) + 1];
                    } else {
                        w0 = x.kx[kb][0];
                        w1 = x.kx[kb][1];
                    }
                    const u32x2 p0 = widen4(w0), p1 = widen4(w1);
                    kf = u32x4{p0[0], p0[1], p1[0], p1[1]};
                } else {
                    kf = x.kw[kb][ks];
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) sa[nb][kb] = mfma16(__builtin_bit_cast(bf16x8, kf), qf[nb][ks], sa[nb][kb]);
            }
        }
        // ---- V rows into the wave's tile
        unsigned odd = 0u;
#pragma unroll
        for (int j = 0; j < NLV; ++j) {
            const int row = NLV * (lane / LPR) + j;
            char* to = vt + row * (CH * 16);
            if constexpr (E4M3) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x2 p0 = widen4(x.vw[j][2 * t]), p1 = widen4(x.vw[j][2 * t + 1]);
                    *(u32x4*)(to + (((2 * (lane % LPR) + t) ^ swz16<CH>(row)) << 4)) = u32x4{p0[0], p0[1], p1[0], p1[1]};
                }
            } else {
                *(u32x4*)(to + (((lane % LPR) ^ swz16<CH>(row)) << 4)) = x.vw[j];
            }
        }
        // ---- mask, where an entry may be invisible to a column
        const int top = base + 31 - walk.nfar + walk.wstart, bot = max(base, walk.nfar) - walk.nfar + walk.wstart;  // rows of the window part
        const bool masked = gone != 0u || p_first < 0 || (base + 31 >= walk.nfar && (top > p_first || bot < lo_last));
        if (masked) {
            const unsigned gists = bot < lo_last ? (unsigned)__builtin_amdgcn_ballot_w64(lane < 32 && base + lane >= walk.nfar &&
                                                                                         is_always(m, base + lane - walk.nfar + walk.wstart))
                                                 : 0u;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const unsigned vis = entry_bits(walk, base, pos[nb], lo[nb], gists, gone) >> (4 * g4);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((vis >> (16 * kb + i)) & 1u)) sa[nb][kb][i] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < NLV; ++j)
#pragma unroll
                for (int t = 0; t < 4; ++t) odd |= E4M3 ? not_finite4(x.vw[j][t]) & 0x80808080u : not_finite2(x.vw[j][t]) & 0x80008000u;
        }
        if (scores.x) {  // base + 31 < pitch: base is a multiple of 32 below the entries, pitch one of 128 no smaller
            const int skip = max(0, s.n - a.weigh) * G;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                if (16 * nb + r16 < ncol && 16 * nb + r16 >= skip) {
                    float* x = scores.x + (((size_t)b * a.kv.Hkv + hk) * scores.cols + (16 * nb + r16 - skip)) * scores.pitch + base + 4 * g4;
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) *(f32x4*)(x + 16 * kb) = sa[nb][kb] * c;
                }
        }
        // ---- softmax against the running references; only where a partial sum has grown too large, or a column has none yet, the
        // maximum is searched and the references raised
        u32x4 pk[NB];
        float ls[NB];
        auto exps = [&](int nb) __attribute__((always_inline)) {
            const float mc = (mr[nb] == -INFINITY ? 0.f : mr[nb]) * c;
            float p[8];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) p[4 * kb + i] = __builtin_amdgcn_exp2f(fmaf(sa[nb][kb][i], c, -mc));
            ls[nb] = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
            for (int t = 0; t < 4; ++t) pk[nb][t] = pack_bf16x2(p[2 * t], p[2 * t + 1]);
        };
        bool search = need_max;
        if (!search) {
            bool big = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                exps(nb);
                big = big || !(ls[nb] <= kBigSum);
            }
            search = __builtin_amdgcn_ballot_w64(big) != 0ull;
        }
        if (search) {
            bool none = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const f32x4 &s0 = sa[nb][0], &s1 = sa[nb][1];
                float mx = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                if ((mx - mr[nb]) * c > kSlack) {  // same decision on the four lanes of a column
                    const float alpha = __builtin_amdgcn_exp2f((mr[nb] - mx) * c);  // m = -inf gives 0
                    l[nb] *= alpha;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[db][nb][i] *= alpha;
                    mr[nb] = mx;
                }
                exps(nb);
                none = none || mr[nb] == -INFINITY;
            }
            need_max = __builtin_amdgcn_ballot_w64(none) != 0ull;
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) l[nb] += ls[nb];
        // ---- O^T += V^T P^T (the tile writes above are this wave's own: LDS operations of a wave complete in order)
        const bool careful = __builtin_amdgcn_ballot_w64(odd != 0u) != 0ull;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            bf16x8 vf = tr16_frag16<CH>(vt + toff[db], 0);
            if (careful) careful_v(vf, pk, o[db]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o[db][nb] = mfma16(vf, __builtin_bit_cast(bf16x8, pk[nb]), o[db][nb]);
        }
    };

    int base = e0 + 32 * w;
    if (base < e1) {
        Tile ta, tb;
        int ahead = page_id(a.kv, b, row_of(base));
        unsigned long long gone = put(base, ahead, 0);
        ahead = page_id(a.kv, b, row_of(base + 256));
        load(ta, pl);
        for (int half = 0;; half ^= 1) {  // loads behind the last entries repeat the last row
            const unsigned long long next = put(base + 256, ahead, half ^ 1);
            ahead = page_id(a.kv, b, row_of(base + 512));
            load(tb, pl + half * 64 + 32);
            step(ta, base, (unsigned)gone);
            if (base + 128 >= e1) break;
            load(ta, pl + (half ^ 1) * 64);
            step(tb, base + 128, (unsigned)(gone >> 32));
            if ((base += 256) >= e1) break;
            gone = next;
        }
    }

    // ---- merge the four waves (the tiles are dead: their memory takes the partials)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l[nb] += __shfl_xor(l[nb], 16, 64);
        l[nb] += __shfl_xor(l[nb], 32, 64);
    }
    __syncthreads();
    float* pm = (float*)smem;       // [4 waves][COLS]
    float* psum = pm + 4 * COLS;    // [4 waves][COLS]
    float* po = psum + 4 * COLS;    // [4 waves][COLS][PD]
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        if (16 * nb + r16 >= ncol) continue;
        if (g4 == 0) {
            pm[w * COLS + 16 * nb + r16] = mr[nb];
            psum[w * COLS + 16 * nb + r16] = l[nb];
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) *(f32x4*)(po + (w * COLS + 16 * nb + r16) * PD + 16 * db + 4 * g4) = o[db][nb];
    }
    __syncthreads();
    const float vmul = E4M3 ? a.kv.vscale[hk] : 1.f;
    const size_t unit = ((size_t)b * a.kv.Hkv + hk) * parts.S + slice;
    for (int idx = tid; idx < ncol * D; idx += NT) {
        const int col = idx / D, d = idx % D;
        float mm = -INFINITY, ll = 0.f, x = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) mm = fmaxf(mm, pm[t * COLS + col]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float lt = psum[t * COLS + col], mt = pm[t * COLS + col];
            if (lt != 0.f) {  // a wave that saw nothing has left zeros; a score that is no number leaves m and a sum that is none
                const float wgt = mt == mm ? 1.f : __builtin_amdgcn_exp2f((mt - mm) * c);
                ll += wgt * lt;
                x += wgt * po[(t * COLS + col) * PD + d];
            }
        }
        if (sl.n > 1) {
            if (d == 0) *(f32x2*)(parts.ml + 2 * (unit * parts.cols + col)) = f32x2{mm * c, ll};
            parts.acc[(unit * parts.cols + col) * D + d] = x * vmul;
            continue;
        }
        const int i = col / G, hq = hk * G + (col - i * G), t = s.t0 + i;
        if (d < Dt) Elem<bf16_t>::store(a.out + (size_t)hq * a.q_hs + (size_t)t * a.q_rs + d, ll == 0.f ? 0.f : x * vmul / ll);
        if (d == 0 && a.lse) a.lse[(size_t)hq * a.batch.T + t] = ll == 0.f ? -INFINITY : mm * c * kLn2 + __builtin_amdgcn_logf(ll) * kLn2;
    }
}

}  // namespace

hipError_t launch_paged_decode(const PagedAttn& a, bool e4m3, const PagedParts& parts, const PagedScores& scores, int cols, hipStream_t st) {
    // Slices last: workgroup ids go round the XCDs, and with 2, 4 or 8 slices next to each other an XCD would get the same ones of
    // every sequence, the last ones empty where lengths differ (slices of 2048, lengths spread from 1/16 up: 64 x 8000 E4M3 rows 139 -> 116
    // us, 64 x 8000 at D = 96 180 -> 159, 64 x 3000 100 -> 91; equal lengths 0 to 1 % slower).
    const dim3 grid(a.kv.Hkv, a.batch.B, parts.S);
    auto go = [&](auto kern) { kern<<<grid, NT, 0, st>>>(a, parts, scores); };
    auto pick = [&](auto d, auto full) {
        constexpr int D = decltype(d)::value;
        constexpr bool FULL = decltype(full)::value;
        if (cols <= 16) e4m3 ? go(paged_decode_kernel<D, FULL, true, 1>) : go(paged_decode_kernel<D, FULL, false, 1>);
        else e4m3 ? go(paged_decode_kernel<D, FULL, true, 2>) : go(paged_decode_kernel<D, FULL, false, 2>);
    };
    if (a.kv.D <= 64) pick(std::integral_constant<int, 64>{}, std::false_type{});
    else if (a.kv.D <= 96) pick(std::integral_constant<int, 96>{}, std::false_type{});
    else if (a.kv.D < 128) pick(std::integral_constant<int, 128>{}, std::false_type{});
    else pick(std::integral_constant<int, 128>{}, std::true_type{});
    return hipGetLastError();
}

}  // namespace unigist
