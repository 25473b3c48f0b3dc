// Device code that the paged attention kernels share.
#pragma once
#include "mfma_common.h"
#include "paged.h"

namespace unigist {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kChunkCols = 128;  // (row, head) columns of a workgroup of the chunk kernel

// Tiles of kChunkCols columns are numbered from floor(t0 * G / kChunkCols) + b on for sequence b, whose first new row is t0: that
// leaves room for the ceil(n * G / kChunkCols) that it has.
__device__ __forceinline__ int first_tile(int t0, int G, int b) { return (int)((unsigned)(t0 * G) / kChunkCols) + b; }
// the sequence that a tile belongs to: the last one whose numbers begin at or below it; 64 sequences a step
__device__ __forceinline__ int seq_of_tile(const PagedBatch& x, int G, int tile) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int b0 = 0; b0 < x.B; b0 += 64) {
        const int b = b0 + lane;
        const bool below = b < x.B && first_tile(x.cu ? min(max(x.cu[b], 0), x.T) : b, G, b) <= tile;
        const unsigned long long bits = __builtin_amdgcn_ballot_w64(below);
        n += __popcll(bits);
        if (~bits != 0ull) break;
    }
    return max(n - 1, 0);
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
