// Attention of the new rows of a batch over a paged cache, and the attention weight that the cached rows receive.
#include "paged.h"

namespace unigist {
namespace {

__device__ __forceinline__ void load8(const PagedKv& c, const char* pool, bool e4m3, int at, int d, float (&x)[8]) {
    if (e4m3) {
        const u32x2 w = *(const u32x2*)(pool + (size_t)at * c.D + d);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
            x[4 * i] = lo[0], x[4 * i + 1] = lo[1], x[4 * i + 2] = hi[0], x[4 * i + 3] = hi[1];
        }
    } else {
        const u32x4 w = *(const u32x4*)(pool + ((size_t)at * c.D + d) * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// One wave per query row and head: 16 lanes a key, four keys at a time, running maximum and sum.
__global__ __launch_bounds__(64) void paged_attn_simple_kernel(PagedAttn a, bool e4m3) {
    const int t = blockIdx.x, hq = blockIdx.y, lane = threadIdx.x, sub = lane & 15, grp = lane >> 4;
    const int b = seq_of_row(a.batch, t), hk = hq / (a.Hq / a.kv.Hkv);
    const PagedSeq s = paged_seq(a.batch, b);
    if (t < s.t0 || t >= s.t0 + s.n) return;
    const AttnShape m = mask_shape(a.mask);
    const int p = s.p0 + (t - s.t0), d = 8 * sub;
    const bool have = d < a.kv.D;
    const float sc = a.scale * (a.kv.kscale ? a.kv.kscale[hk] : 1.f);
    float q[8] = {}, acc[8] = {}, mx = -INFINITY, l = 0.f;
    const size_t at_q = (size_t)hq * a.q_hs + (size_t)t * a.q_rs + d;
    if (have)
        for (int i = 0; i < 8; ++i) q[i] = bf16_to_f32(a.q[at_q + i]) * sc;
    for (int j = grp; j <= p; j += 4) {
        if (!is_always(m, j) && j < win_lo(m, p)) continue;
        const int at = pool_row(a.kv, b, hk, j);
        if (at < 0) continue;
        float k[8] = {}, v[8] = {}, x = 0.f;
        if (have) {
            load8(a.kv, a.kv.k, e4m3, at, d, k);
            load8(a.kv, a.kv.v, e4m3, at, d, v);
        }
        for (int i = 0; i < 8; ++i) x = fmaf(q[i], k[i], x);
        for (int off = 1; off < 16; off <<= 1) x += __shfl_xor(x, off, 16);
        const float mn = fmaxf(mx, x), old = mx == -INFINITY ? 0.f : __expf(mx - mn), w = mn == -INFINITY ? 0.f : __expf(x - mn);
        l = l * old + w;
        for (int i = 0; i < 8; ++i) acc[i] = acc[i] * old + w * v[i];
        mx = mn;
    }
    for (int off = 16; off < 64; off <<= 1) {
        const float om = __shfl_xor(mx, off, 64), mn = fmaxf(mx, om);
        const float f = mx == -INFINITY ? 0.f : __expf(mx - mn), g = om == -INFINITY ? 0.f : __expf(om - mn);
        l = l * f + __shfl_xor(l, off, 64) * g;
        for (int i = 0; i < 8; ++i) acc[i] = acc[i] * f + __shfl_xor(acc[i], off, 64) * g;
        mx = mn;
    }
    const float inv = (a.kv.vscale ? a.kv.vscale[hk] : 1.f) / l;
    if (grp == 0 && have)
        for (int i = 0; i < 8; ++i) a.out[at_q + i] = f32_to_bf16(mx == -INFINITY ? 0.f : acc[i] * inv);
    if (a.lse && lane == 0) a.lse[(size_t)hq * a.batch.T + t] = mx == -INFINITY ? -INFINITY : mx + __logf(l);
}

// One lane per cached row: the sum over the last new rows and the heads of the group of exp(score - lse).
__global__ __launch_bounds__(64) void paged_weigh_simple_kernel(PagedAttn a, bool e4m3) {
    const int b = blockIdx.z, hk = blockIdx.y, j = blockIdx.x * 64 + threadIdx.x, G = a.Hq / a.kv.Hkv;
    const PagedSeq s = paged_seq(a.batch, b);
    if (j >= s.len || s.n == 0) return;
    const int at = pool_row(a.kv, b, hk, j);
    if (at < 0) return;
    const AttnShape m = mask_shape(a.mask);
    const float sc = a.scale * (a.kv.kscale ? a.kv.kscale[hk] : 1.f);
    float sum = 0.f;
    for (int i = max(0, s.n - a.weigh); i < s.n; ++i) {
        const int p = s.p0 + i;
        if (j > p || (!is_always(m, j) && j < win_lo(m, p))) continue;
        for (int g = 0; g < G; ++g) {
            const int hq = hk * G + g, t = s.t0 + i;
            const bf16_t* q = a.q + (size_t)hq * a.q_hs + (size_t)t * a.q_rs;
            float x = 0.f;
            for (int d = 0; d < a.kv.D; d += 8) {
                float k[8];
                load8(a.kv, a.kv.k, e4m3, at, d, k);
                for (int e = 0; e < 8; ++e) x = fmaf(bf16_to_f32(q[d + e]), k[e], x);
            }
            const float lse = a.lse[(size_t)hq * a.batch.T + t];
            if (lse != -INFINITY) sum += __expf(x * sc - lse);
        }
    }
    a.kv.weight[at] = a.decay == 0.f ? sum : a.decay * a.kv.weight[at] + sum;
}

}  // namespace

size_t paged_attn_bytes(const PagedAttn& a, bool e4m3) { return 256; }

hipError_t launch_paged_attn(const PagedAttn& a, bool e4m3, void* ws, hipStream_t st) {
    paged_attn_simple_kernel<<<dim3(a.batch.T, a.Hq), 64, 0, st>>>(a, e4m3);
    if (a.weigh)
        paged_weigh_simple_kernel<<<dim3((a.batch.max_kv + 63) / 64, a.kv.Hkv, a.batch.B), 64, 0, st>>>(a, e4m3);
    return hipGetLastError();
}

}  // namespace unigist
