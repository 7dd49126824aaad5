// Keys and values of a step into the paged 8-bit cache; queries and keys normed per head and rotated on the way.
//
//   x' = x * rsqrt(mean(x^2) + eps) * w        (where a weight is given)
//   (a, b) -> (a cos - b sin, b cos + a sin)   for the pairs of the rotated part
//   page scale s = max(s of the page's older entries, 2^ceil(log2(max |x'| / 448))), entry = e4m3(x' / s)
//
// The operator moves bytes: 2 read per element of q, k and v, 2 written per element of q, 1 per element of k and v.  One pass
// needs the largest value of a whole page and head before anything can be written, so one CTA takes a page of one head and one
// side (keys or values), keeps what it has read in registers, and writes after one reduction: no atomics, nothing is read twice.
// Queries have no such tie and are spread over further CTAs of the same launch.
#pragma once

#include "kv_common.cuh"

namespace ot {

struct KvAppend {
    KvShape shape;
    KvStep step;
    KvRows q, k, v, q_out;
    uint8_t *kc, *vc;                    // this layer's pages [num_pages][kv_heads][page][D]
    float *ks, *vs;                      // [num_pages][kv_heads]
    const int32_t* table;
    const float* cos_sin;                // [positions][rot_dim]: cosines, then sines
    int positions, rot_dim, interleaved;
    const uint16_t *q_norm, *k_norm;
    float eps;
    int wide_q, wide_k, wide_v, wide_out, wide_w;   // rows on 16-byte boundaries
    int page_slots;                      // most pages a sequence's step can touch
    int page_blocks;                     // CTAs that take pages; the others take queries
    FixedDiv by_heads, by_slots, by_q_heads, by_T;
    int* status;
};

constexpr int kAppendQueryRows = 4;      // row groups a warp of a query CTA has in flight

template <class T> __device__ __forceinline__ T rsqrt_of(T x);
template <> __device__ __forceinline__ float rsqrt_of<float>(float x) { return rsqrtf(x); }
template <> __device__ __forceinline__ double rsqrt_of<double>(double x) { return 1.0 / sqrt(x); }

// Norm and rotation of one row: a lane holds eight consecutive elements, D/8 consecutive lanes a row.  F: float, or double where
// the largest value lies so near a border of the scale that single precision could take the other side.
template <int D, class T, class F>
__device__ __forceinline__ void turn_row(const KvAppend& a, const uint16_t* w, int pos, const float (&in)[8], F (&x)[8]) {
    constexpr int kLanes = D / 8;
    const int sub = threadIdx.x & (kLanes - 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (F)in[i];
    if (w) {
        F sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const F r = rsqrt_of<F>(sum / (F)D + (F)a.eps);
        float wf[8];
        unpack8<T>(load8(w + sub * 8, a.wide_w), wf);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (F)wf[i];
    }
    if (a.rot_dim == 0) return;
    const float* cs = a.cos_sin + (long long)pos * a.rot_dim;
    const int half = a.rot_dim >> 1, at = sub * 8;
    if (a.interleaved) {
        if (at >= a.rot_dim) return;
        float c[4], s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { c[i] = cs[at / 2 + i]; s[i] = cs[half + at / 2 + i]; }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F p = x[2 * i], q = x[2 * i + 1];
            x[2 * i] = p * (F)c[i] - q * (F)s[i];
            x[2 * i + 1] = q * (F)c[i] + p * (F)s[i];
        }
    } else {
        const bool low = at < half;
        const int partner = at >= a.rot_dim ? sub : (low ? sub + half / 8 : sub - half / 8);
        const int lane = (threadIdx.x & 31 & ~(kLanes - 1)) + partner;
        F other[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl_sync(0xFFFFFFFFu, x[i], lane);
        if (at >= a.rot_dim) return;
        const float* c = cs + (low ? at : at - half);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const F cc = (F)c[i], ss = (F)c[half + i];
            x[i] = low ? x[i] * cc - other[i] * ss : x[i] * cc + other[i] * ss;
        }
    }
}

__device__ __forceinline__ int kv_position(const KvAppend& a, int b, int j, int len) {
    if (a.rot_dim == 0) return 0;
    const int base = a.step.base_pos ? a.step.base_pos[b] : len;
    const int pos = j == 0 || !a.step.position_ids ? base + j : a.step.position_ids[(long long)b * (a.step.T - 1) + j - 1];
    if ((unsigned)pos >= (unsigned)a.positions) {
        set_status(a.status, kErrInternal);
        return pos < 0 ? 0 : a.positions - 1;
    }
    return pos;
}

// The queries: rows (sequence, token, head) in that order.
template <int D, class T>
__device__ __forceinline__ void append_queries(const KvAppend& a, int block) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    const int lane = threadIdx.x & 31, sub = lane & (kLanes - 1);
    const unsigned rows = (unsigned)a.step.B * a.step.T * a.shape.q_heads;
    const long long first = ((long long)block * (blockDim.x >> 5) + (threadIdx.x >> 5)) * (kRows * kAppendQueryRows) + lane / kLanes;
    uint4 raw[kAppendQueryRows];
    int pos[kAppendQueryRows];
    long long to[kAppendQueryRows];
#pragma unroll
    for (int i = 0; i < kAppendQueryRows; ++i) {
        const long long r = first + i * kRows;
        to[i] = -1; pos[i] = 0;
        raw[i] = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            const unsigned bt = a.by_q_heads.div((unsigned)r), h = (unsigned)r - bt * a.shape.q_heads;
            const unsigned b = a.by_T.div(bt), j = bt - b * a.step.T;
            int len, tokens;
            if (kv_sequence(a.shape, a.step, b, len, tokens, a.status) && (int)j < tokens) {
                raw[i] = load8(a.q.data + b * a.q.batch + j * a.q.token + h * a.q.head + sub * 8, a.wide_q);
                to[i] = b * a.q_out.batch + j * a.q_out.token + h * a.q_out.head + sub * 8;
                pos[i] = kv_position(a, b, j, len);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kAppendQueryRows; ++i) {
        float in[8], x[8];
        unpack8<T>(raw[i], in);
        turn_row<D, T, float>(a, a.q_norm, pos[i], in, x);
        if (to[i] >= 0) {
            const uint4 o = make_uint4(from_float2<T>(x[0], x[1]), from_float2<T>(x[2], x[3]), from_float2<T>(x[4], x[5]), from_float2<T>(x[6], x[7]));
            store8(const_cast<uint16_t*>(a.q_out.data) + to[i], o, a.wide_out);
        }
    }
}

__device__ __forceinline__ float finite_abs(float x) {      // infinities saturate and NaN stays NaN: neither sets the scale
    const float m = fabsf(x);
    return m <= 3.402823466e38f ? m : 0.f;
}
__device__ __forceinline__ double finite_abs(double x) {
    const double m = fabs(x);
    return m <= 3.402823466e38 ? m : 0.0;
}

// kPasses: row groups per warp that cover a page.
template <int D, class T, int kThreadsN, int kPasses>
__global__ void __launch_bounds__(kThreadsN) kv_append_kernel(const __grid_constant__ KvAppend a) {
    grid_dependency_wait();
    if ((int)blockIdx.x >= a.page_blocks) {
        append_queries<D, T>(a, blockIdx.x - a.page_blocks);
        return;
    }
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kWarpsN = kThreadsN / 32;
    __shared__ uint32_t warp_max[kWarpsN];
    __shared__ unsigned long long warp_max64[kWarpsN];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane & (kLanes - 1);
    unsigned item = blockIdx.x >> 1;
    const bool values = blockIdx.x & 1;
    const unsigned bp = a.by_heads.div(item), h = item - bp * a.shape.kv_heads;
    const unsigned b = a.by_slots.div(bp), slot = bp - b * a.page_slots;
    int len, tokens;
    if (!kv_sequence(a.shape, a.step, b, len, tokens, a.status)) return;
    const int page = a.shape.page, at = (len >> a.shape.page_shift) + slot;
    const int start = at << a.shape.page_shift;                              // first slot of the page
    const int lo = max(len, start), hi = min(len + tokens, start + page);    // the step's slots in it
    if (lo >= hi) return;
    const int id = kv_page(a.shape, a.table, b, at, a.status);
    if (id < 0) return;
    const long long head = (long long)id * a.shape.kv_heads + h;
    uint8_t* codes = (values ? a.vc : a.kc) + head * page * D;
    float* scale = (values ? a.vs : a.ks) + head;
    const bool older = lo > start;
    const float was = older ? *scale : 0.f;
    const KvRows& src = values ? a.v : a.k;
    const uint16_t* from = src.data + b * src.batch + h * src.head + sub * 8;
    const bool wide = values ? a.wide_v : a.wide_k;

    float x[kPasses][8];
    float most = 0.f;
    const int n = hi - lo;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (r < n) raw = load8(from + (long long)(lo - len + r) * src.token, wide);
        unpack8<T>(raw, x[i]);
    }
    if (!values) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            if ((i * kWarpsN + warp) * kRows >= n) break;                    // the same for the whole warp
            const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
            const int pos = r < n ? kv_position(a, b, lo - len + r, len) : 0;
            float in[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) in[e] = x[i][e];
            turn_row<D, T, float>(a, a.k_norm, pos, in, x[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_abs(x[i][e]));
    most = warp_max_f32(most);
    if (lane == 0) warp_max[warp] = __float_as_uint(most);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarpsN; ++w) most = fmaxf(most, __uint_as_float(warp_max[w]));
    // Single precision is off by less than 1e-6; nearer than 1e-5 to a border the largest value is found again in double
    // precision, so that the scale, which is a whole power of two, does not hang on a rounding.
    const uint32_t frac = __float_as_uint(most) & 0x7FFFFFu;
    int e = scale_exponent(__float_as_uint(most));
    if (!values && (a.k_norm || a.rot_dim) && frac > 0x600000u - 147u && frac < 0x600000u + 147u) {
        double exact = 0.0;
        for (int i = 0; i < kPasses; ++i) {
            if ((i * kWarpsN + warp) * kRows >= n) break;
            const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (r < n) raw = load8(from + (long long)(lo - len + r) * src.token, wide);
            float in[8];
            double y[8];
            unpack8<T>(raw, in);
            turn_row<D, T, double>(a, a.k_norm, r < n ? kv_position(a, b, lo - len + r, len) : 0, in, y);
#pragma unroll
            for (int c = 0; c < 8; ++c) exact = fmax(exact, finite_abs(y[c]));
        }
        const unsigned long long bits = warp_max_u64((unsigned long long)__double_as_longlong(exact));
        if (lane == 0) warp_max64[warp] = bits;
        __syncthreads();
        unsigned long long all = 0;
        for (int w = 0; w < kWarpsN; ++w) all = warp_max64[w] > all ? warp_max64[w] : all;
        // 1.75 in the fraction of a double
        e = (int)(all >> 52) - 1023 - 8 + ((all & 0xFFFFFFFFFFFFFull) > 0xC000000000000ull ? 1 : 0);
        e = e < kLeastScaleExp ? kLeastScaleExp : e;
    }
    const float now = fmaxf(was, power_of_two(e)), inv = 1.f / now;
    if (older && now > was) {                                                // the page's older entries to the larger scale
        const float ratio = was * inv;
        uint4* rows = reinterpret_cast<uint4*>(codes);
        for (int c = threadIdx.x; c < (lo - start) * (D / 16); c += kThreadsN) rows[c] = recode16(rows[c], ratio);
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
        if (r < n) {
            uint2 o;
            o.x = to_e4m3x4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv);
            o.y = to_e4m3x4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv);
            *reinterpret_cast<uint2*>(codes + (long long)(lo - start + r) * D + sub * 8) = o;
        }
    }
    if (threadIdx.x == 0) *scale = now;
}

}  // namespace ot
