// Attention of a step's tokens over the paged 8-bit cache: the prefix, and inside the step each token's ancestors (a tree's bitmask)
// or predecessors (a chain).
#pragma once

#include "kv_common.cuh"

namespace ot {

struct KvAttend {
    KvShape shape;
    KvStep step;
    KvRows q, out;
    const uint8_t *kc, *vc;
    const float *ks, *vs;
    const int32_t* table;
    float* lse;
    float scale;
    int wide_q, wide_out;
    int* status;
};

// Whether token i of a step sees token j of it.
__device__ __forceinline__ bool kv_sees(const KvStep& st, int b, int i, int j) {
    if (j == i || j == 0) return true;
    if (!st.mask) return j < i;
    if (i == 0) return false;
    const int W = (st.T - 1 + 63) >> 6;
    return (st.mask[((long long)b * (st.T - 1) + i - 1) * W + ((j - 1) >> 6)] >> ((j - 1) & 63)) & 1ull;
}

// One warp per (sequence, token, query head): 32 keys at a time, a lane per key for the scores, a lane per D/32 elements for the values.
template <int D, class T>
__global__ void __launch_bounds__(128) kv_attend_plain_kernel(const __grid_constant__ KvAttend a) {
    grid_dependency_wait();
    __shared__ float qs[4][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long row = (long long)blockIdx.x * 4 + warp;
    if (row >= (long long)a.step.B * a.step.T * a.shape.q_heads) return;
    const int hq = (int)(row % a.shape.q_heads), j = (int)(row / a.shape.q_heads % a.step.T), b = (int)(row / a.shape.q_heads / a.step.T);
    int len, tokens;
    if (!kv_sequence(a.shape, a.step, b, len, tokens, a.status) || j >= tokens) return;
    const int h = hq / (a.shape.q_heads / a.shape.kv_heads);
    const uint16_t* q = a.q.data + b * a.q.batch + j * a.q.token + hq * a.q.head;
    for (int d = lane; d < D; d += 32) qs[warp][d] = to_float2<T>(q[d]).x;
    __syncwarp();
    float m = -INFINITY, l = 0.f, o[D / 32];
    for (int d = 0; d < D / 32; ++d) o[d] = 0.f;
    for (int s0 = 0; s0 < len + tokens; s0 += 32) {
        const int s = s0 + lane;
        const bool see = s < len || (s < len + tokens && kv_sees(a.step, b, j, s - len));
        const int id = s < len + tokens ? max(0, kv_page(a.shape, a.table, b, s >> a.shape.page_shift, a.status)) : 0;
        const long long head = (long long)id * a.shape.kv_heads + h;
        float x = -INFINITY;
        if (see) {
            const uint16_t* k = reinterpret_cast<const uint16_t*>(a.kc + (head * a.shape.page + (s & (a.shape.page - 1))) * D);
            x = 0.f;
            for (int d = 0; d < D / 2; ++d) {
                const float2 kk = to_float2<__half>(from_e4m3x2(k[d]));
                x += qs[warp][2 * d] * kk.x + qs[warp][2 * d + 1] * kk.y;
            }
            x *= a.ks[head] * a.scale;
        }
        const float top = warp_max_f32(x), was = m;
        m = fmaxf(m, top);
        if (m == -INFINITY && !__any_sync(0xFFFFFFFFu, x != x)) continue;
        const float p = see ? expf(x - m) : 0.f, fade = was == -INFINITY ? 0.f : expf(was - m);
        float sum = p;
        for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, w);
        l = l * fade + sum;
        for (int d = 0; d < D / 32; ++d) o[d] *= fade;
        const unsigned on = __ballot_sync(0xFFFFFFFFu, see);
        for (int t = 0; t < 32; ++t) {
            const float pt = __shfl_sync(0xFFFFFFFFu, p, t);
            const long long ht = __shfl_sync(0xFFFFFFFFu, head, t);
            if (!(on >> t & 1)) continue;
            const uint8_t* v = a.vc + (ht * a.shape.page + ((s0 + t) & (a.shape.page - 1))) * D + lane * (D / 32);
            const float w = pt * a.vs[ht];
            for (int d = 0; d < D / 32; ++d) o[d] += w * to_float2<__half>(from_e4m3x2(v[d])).x;
        }
    }
    uint16_t* out = const_cast<uint16_t*>(a.out.data) + b * a.out.batch + j * a.out.token + hq * a.out.head;
    for (int d = 0; d < D / 32; ++d) out[lane * (D / 32) + d] = (uint16_t)from_float2<T>(o[d] / l, 0.f);
    if (a.lse && lane == 0) a.lse[((long long)b * a.step.T + j) * a.shape.q_heads + hq] = m + logf(l);
}

}  // namespace ot
