// Device code that the paged attention kernels share.
#pragma once
#include "mfma_common.h"
#include "paged.h"

namespace unigist {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kChunkCols = 128;  // (row, head) columns of a workgroup of the chunk kernel

// The chunk kernel's tiles, of kChunkCols columns each: those of sequence 0, then of sequence 1, .. for sequences of more than
// min_cols columns; the others have none.  Every wave counts them for itself, a lane the sequences lane * per .. of them, so that
// launch and workspace go by the work of a batch and not by its number of sequences.
struct PagedTiles {
    int total;
    int per, upto, own;  // per lane: sequences of a lane, tiles up to and with them, tiles of them
};
__device__ __forceinline__ int tiles_of(const PagedBatch& x, int G, int min_cols, int b) {
    const int ncol = b < x.B ? paged_new(x, b) * G : 0;
    return ncol > min_cols ? (ncol + kChunkCols - 1) / kChunkCols : 0;
}
__device__ __forceinline__ int scan64(int own) {  // sum of the lanes up to and with this one
    int sum = own;
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8: rows of 16 lanes
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xf, 0xf, false);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xf, 0xf, false);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xf, 0xf, false);
    const int row = (threadIdx.x & 63) >> 4;
    const int r0 = __builtin_amdgcn_readlane(sum, 15), r1 = r0 + __builtin_amdgcn_readlane(sum, 31), r2 = r1 + __builtin_amdgcn_readlane(sum, 47);
    return sum + (row == 0 ? 0 : row == 1 ? r0 : row == 2 ? r1 : r2);
}
__device__ __forceinline__ PagedTiles count_tiles(const PagedBatch& x, int G, int min_cols) {
    PagedTiles t;
    t.per = (x.B + 63) / 64;
    t.own = 0;
    if (x.B == 1) {
        t.total = t.upto = t.own = __builtin_amdgcn_readfirstlane(tiles_of(x, G, min_cols, 0));
        return t;
    }
    const int b0 = (int)(threadIdx.x & 63) * t.per;
    for (int i = 0; i < t.per; ++i) t.own += tiles_of(x, G, min_cols, b0 + i);
    t.upto = scan64(t.own);
    t.total = __builtin_amdgcn_readlane(t.upto, 63);
    return t;
}
// The sequence of tile 0 <= tile < total, and which of its tiles it is.
__device__ __forceinline__ int seq_of_tile(const PagedBatch& x, int G, int min_cols, const PagedTiles& t, int tile, int& j) {
    j = tile;
    if (x.B == 1) return 0;
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(t.upto > tile));
    j -= __builtin_amdgcn_readlane(t.upto - t.own, at);
    if (t.per == 1) return at;
    for (int b0 = at * t.per; b0 < x.B; b0 += 64) {  // among the lane's sequences, 64 at a time; tile lies in one of them
        const int b = b0 + (int)(threadIdx.x & 63), own = b < (at + 1) * t.per ? tiles_of(x, G, min_cols, b) : 0, upto = scan64(own);
        const unsigned long long behind = __builtin_amdgcn_ballot_w64(upto > j);
        if (behind != 0ull) {
            const int l = __builtin_ctzll(behind);
            j -= __builtin_amdgcn_readlane(upto - own, l);
            return b0 + l;
        }
        j -= __builtin_amdgcn_readlane(upto, 63);
    }
    return 0;  // boundaries that decrease
}
// Slices of a tile: as many as there is room for, at most S.
__device__ __forceinline__ int slices_of(const PagedParts& parts, int total) {
    return parts.S == 1 || (long long)total * parts.S <= parts.units ? parts.S : max(1, parts.units / total);
}

__device__ __forceinline__ unsigned bits_below(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// Which of the 32 entries from e on does a query at position p see?  gists: bits of the always-visible ones among them
// (window part); gone: bits of entries that are not there.
__device__ __forceinline__ unsigned entry_bits(const PagedWalk& w, int e, int p, int lo, unsigned gists, unsigned gone) {
    if (p < 0) return 0u;
    const int j0 = e - w.nfar + w.wstart;  // the row of entry e, were it in the window part
    return (bits_below(w.nfar - e) | (bits_below(p - j0 + 1) & (~bits_below(lo - j0) | gists))) & ~gone;
}

// 32 bits of two bf16: is one of them infinite or not a number?  Accumulated over words; bits 15 and 31 tell.
__device__ __forceinline__ unsigned not_finite2(unsigned w) { return (w & 0x7f807f80u) + 0x00800080u; }
// four E4M3 codes: bits 7, 15, 23, 31
__device__ __forceinline__ unsigned not_finite4(unsigned w) { return (w & 0x7f7f7f7fu) + 0x01010101u; }

// four E4M3 codes -> four bf16 (exact)
__device__ __forceinline__ u32x2 widen4(unsigned w) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    u32x2 r;
    r[0] = pack_bf16x2(lo[0], lo[1]);
    r[1] = pack_bf16x2(hi[0], hi[1]);
    return r;
}

// Before o[..] += V^T P^T (blocks of 16 x 16) where V may hold values that are not finite and some columns do not see all of its
// rows: a product with P = 0 would carry them over.  What is not finite is counted by products of ones, apart for +inf and
// -inf (not a number is both), and enters the columns that give it any weight; vf is left with the finite part.
template <int N>
__device__ __forceinline__ void careful_v(bf16x8& vf, const u32x4 (&p)[N], f32x4 (&o)[N]) {
    u32x4 v = __builtin_bit_cast(u32x4, vf), up, down;
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // two bf16 a word: a truth value is bit 15 or 31
        const unsigned odd = ((v[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        const unsigned nan = ((v[i] & 0x007f007fu) + 0x007f007fu) << 8;
        up[i] = ((odd & (~v[i] | nan)) >> 15) * 0x3f80u;  // 1 in bf16
        down[i] = ((odd & (v[i] | nan)) >> 15) * 0x3f80u;
        v[i] &= ~((odd >> 15) * 0xffffu);
    }
    vf = __builtin_bit_cast(bf16x8, v);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        u32x4 has;
#pragma unroll
        for (int i = 0; i < 4; ++i) has[i] = ((((p[n][i] & 0x7fff7fffu) + 0x7fff7fffu) & 0x80008000u) >> 15) * 0x3f80u;
        const f32x4 u = mfma16(__builtin_bit_cast(bf16x8, up), __builtin_bit_cast(bf16x8, has), zero4());
        const f32x4 d = mfma16(__builtin_bit_cast(bf16x8, down), __builtin_bit_cast(bf16x8, has), zero4());
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (u[i] > 0.f) o[n][i] += INFINITY;
            if (d[i] > 0.f) o[n][i] -= INFINITY;
        }
    }
}

}  // namespace unigist
