// Device code that the paged attention kernels share.
#pragma once
#include "mfma_common.h"
#include "paged.h"

namespace unigist {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kChunkCols = 128;  // (row, head) columns of a workgroup of the chunk kernel

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

// O^T += V^T P^T key by key, for a tile of 32 rows of which some hold values that are not finite and some columns do not
// see all: a product with P = 0 would carry them over.  vt: the tile in LDS (bf16, swizzled); pk: P of a 16-column block
// as the B operand, zero where a column does not see a key.  Rare, so as small as it can be.
template <int DB, int CH>
__device__ __forceinline__ void careful_pv(const char* vt, const u32x4 pk, f32x4 (&o)[DB]) {
    const int lane = threadIdx.x & 63, r16 = lane & 15, g4 = lane >> 4;
#pragma unroll 1
    for (int key = 0; key < 32; ++key) {
        const int word = 2 * (key >> 4) + ((key & 3) >> 1);
        const unsigned mine = word == 0 ? pk[0] : word == 1 ? pk[1] : word == 2 ? pk[2] : pk[3];
        const unsigned two = (unsigned)__shfl((int)mine, ((key & 15) >> 2) * 16 + r16, 64);
        const float p = __uint_as_float(key & 1 ? two & 0xffff0000u : two << 16);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const u32x2 v = *(const u32x2*)(vt + key * (CH * 16) + (((2 * db + (g4 >> 1)) ^ swz16<CH>(key)) << 4) + (g4 & 1) * 8);
            if (p != 0.f) {
                o[db][0] += p * __uint_as_float(v[0] << 16);
                o[db][1] += p * __uint_as_float(v[0] & 0xffff0000u);
                o[db][2] += p * __uint_as_float(v[1] << 16);
                o[db][3] += p * __uint_as_float(v[1] & 0xffff0000u);
            }
        }
    }
}

}  // namespace unigist
