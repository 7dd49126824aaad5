// Keys and values of a step into the paged 8-bit cache; queries and keys normed per head and rotated on the way.
//
//   x' = x * rsqrt(mean(x^2) + eps) * w        (where a weight is given)
//   (a, b) -> (a cos - b sin, b cos + a sin)   for the pairs of the rotated part
//   page scale s = max(s of the page's older entries, 2^ceil(log2(max |x'| / 448))), entry = e4m3(x' / s)
//
// The operator moves bytes: 2 read per element of q, k and v, 2 written per element of q, 1 per element of k and v.  One pass
// needs the largest value of a whole page and head before anything can be written, so one CTA takes a page of one head and one
// side (keys or values), keeps what it has read in registers, and writes after one reduction: no atomics, nothing is read twice.
// Queries have no such tie and are spread over further CTAs of the same launch, a warp for up to 16 heads (of 128 elements) of one token, so that
// positions, angles and weights are looked up and folded once (a row at a time: 211 us, now 118 us, for 4 x 4096 tokens of 32 / 8 heads of
// 128, normed and rotated; 54 us would be the bytes at 6.5 TB/s).  What bounds it now: a CTA's life is a chain of loads (lengths, rows and
// table, angles, scale) around little work, and the arithmetic of norm, rotation and conversion takes 58 % of the issue slots.  Pages
// alone (a call without queries) take 67 us of the 118.

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
    int wide_q, wide_k, wide_v, wide_out, wide_w, wide_cs;   // rows on 16-byte boundaries
    int page_slots;                      // most pages a sequence's step can touch
    int page_blocks;                     // CTAs that take pages; the others take queries
    int query_parts;                     // warps that share a token's query heads
    FixedDiv by_heads, by_slots, by_parts, by_T;
    int* status;
};

constexpr int kAppendRows = 8;           // row groups a warp of a query CTA takes, all of one token: positions and angles are looked up once

// A lane holds eight consecutive elements of a row, D / 8 consecutive lanes a row.  Rotation is x' = x c + y s with y the other element of
// the pair, which another lane (`partner`) or this one holds, and the sign in s; elements that are not rotated have c = 1, s = 0.  (An
// infinity there makes NaN of that; rows with such a result are taken again without it.)
struct KvAngles {
    float c[8], s[8];
};
__device__ __forceinline__ int kv_partner(const KvAppend& a, int sub) {
    const int half = a.rot_dim >> 4;                         // in lanes
    return a.interleaved || sub >= 2 * half ? sub : (sub < half ? sub + half : sub - half);
}
__device__ __forceinline__ void load4(const float* p, int wide, float* x) {
    if (wide) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = p[i];
    }
}
__device__ __forceinline__ void kv_angles(const KvAppend& a, int sub, int pos, KvAngles& g) {
    const int half = a.rot_dim >> 1, at = sub * 8;
    const float* cs = a.cos_sin + (long long)pos * a.rot_dim;
    if (at >= a.rot_dim) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { g.c[i] = 1.f; g.s[i] = 0.f; }
    } else if (a.interleaved) {
        float c[4], s[4];
        load4(cs + at / 2, a.wide_cs, c);
        load4(cs + half + at / 2, a.wide_cs, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) { g.c[2 * i] = g.c[2 * i + 1] = c[i]; g.s[2 * i] = -s[i]; g.s[2 * i + 1] = s[i]; }
    } else {
        const float* from = cs + (at < half ? at : at - half);
        load4(from, a.wide_cs, g.c); load4(from + 4, a.wide_cs, g.c + 4);
        load4(from + half, a.wide_cs, g.s); load4(from + half + 4, a.wide_cs, g.s + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) g.s[i] = at < half ? -g.s[i] : g.s[i];
    }
}
// Largest magnitude; NaN if any is.
__device__ __forceinline__ float max_abs8(const float (&x)[8]) {
    float m = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 7; i += 2) asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(x[i])), "f"(fabsf(x[i + 1])));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(x[7])));
    return m;
}
// Norm and rotation with what does not depend on the row folded together, in packed pairs: x' = r (x (w c) + y (w_y s)), r the norm's factor.
// true: weights so large that products may pass single precision's range on the way to a result within it.
struct KvFold {
    unsigned long long c[4], s[4];
};
template <class T>
__device__ __forceinline__ bool kv_fold(const KvAppend& a, const uint16_t* weights, const KvAngles& g, int sub, int partner, KvFold& f) {
    float c[8], s[8];
    bool large = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = a.rot_dim ? g.c[i] : 1.f; s[i] = a.rot_dim ? g.s[i] : 0.f; }
    if (weights) {
        float w[8], y[8];
        unpack8<T>(load8(weights + sub * 8, a.wide_w), w);
        large = max_abs8(w) > 0x1p60f;
        unpack8<T>(load8(weights + partner * 8, a.wide_w), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] *= w[i]; s[i] *= a.interleaved ? y[i ^ 1] : y[i]; }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { f.c[i] = pack2(c[2 * i], c[2 * i + 1]); f.s[i] = pack2(s[2 * i], s[2 * i + 1]); }
    return large;
}
// true: the norm's factor cannot be relied on, because the mean square is so large or small that squares or products may have passed single precision's
// range (the same for all lanes of a row).  Such rows are taken again in double precision; that they may come costs 5 % of a call without any
// (112 -> 118 us for the chunk above).
template <int D, class T>
__device__ __forceinline__ bool turn_fast(const KvAppend& a, bool norm, const KvFold& f, int partner, uint4 raw, float (&out)[8]) {
    constexpr int kLanes = D / 8;
    constexpr uint32_t kLeast = (127u - 40u) << 23, kMost = (127u + 100u) << 23;           // mean squares, as bits
    bool wild = false;
    unsigned long long x[4];
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 v = to_float2<T>(w[i]); x[i] = pack2(v.x, v.y); }
    float r = 1.f;
    if (norm) {
        unsigned long long s2 = mul2(x[0], x[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) s2 = fma2(x[i], x[i], s2);
        float lo, hi;
        unpack2(s2, lo, hi);
        float sum = lo + hi;
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const float mean = sum * (1.f / D) + a.eps;
        r = rsqrtf(mean);
        wild = __float_as_uint(mean) - kLeast > kMost - kLeast;
    }
    const int lane = (threadIdx.x & 31 & ~(kLanes - 1)) + partner;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned long long z = mul2(x[i], f.c[i]);
        if (a.rot_dim) {
            unsigned long long y;
            if (a.interleaved) {
                float lo, hi;
                unpack2(x[i], lo, hi);
                y = pack2(hi, lo);
            } else {
                const float2 v = to_float2<T>(__shfl_sync(0xFFFFFFFFu, w[i], lane));
                y = pack2(v.x, v.y);
            }
            z = fma2(y, f.s[i], z);
        }
        if (norm) z = mul2(z, pack2(r, r));
        unpack2(z, out[2 * i], out[2 * i + 1]);
    }
    return wild;
}
// The same of one row in double precision, for what single precision cannot be relied on: where the largest value lies so near a border of the
// scale, or any so near the middle between two codes, that it could take the other side, and where squares, products or sums pass its range.
template <int D, class T>
__device__ __forceinline__ void turn_exact(const KvAppend& a, const uint16_t* weights, const KvAngles& g, int sub, int partner, uint4 raw, double (&x)[8]) {
    constexpr int kLanes = D / 8;
    float in[8];
    unpack8<T>(raw, in);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = in[i];
    if (weights) {
        double sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const double r = rsqrt(sum * (1.0 / D) + (double)a.eps);
        unpack8<T>(load8(weights + sub * 8, a.wide_w), in);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * in[i];
    }
    if (a.rot_dim == 0) return;
    const int lane = (threadIdx.x & 31 & ~(kLanes - 1)) + partner;
    double y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = a.interleaved ? x[i ^ 1] : __shfl_sync(0xFFFFFFFFu, x[i], lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = sub * 8 < a.rot_dim ? x[i] * g.c[i] + y[i] * g.s[i] : x[i];
}

// A double as the float that rounds to the same code or 16-bit number: cut off, with the last bit set if anything was.
__device__ __forceinline__ float round_to_odd(double x) {
    const float f = __double2float_rz(x);
    return (double)f == x ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// base: the sequence's base_pos, loaded by the caller together with its lengths (kv_base).
__device__ __forceinline__ int kv_base(const KvAppend& a, int b) { return a.rot_dim && a.step.base_pos ? a.step.base_pos[b] : 0; }
__device__ __forceinline__ int kv_position(const KvAppend& a, int b, int j, int len, int base) {
    if (a.rot_dim == 0) return 0;
    if (!a.step.base_pos) base = len;
    const int pos = j == 0 || !a.step.position_ids ? base + j : a.step.position_ids[(long long)b * (a.step.T - 1) + j - 1];
    if ((unsigned)pos >= (unsigned)a.positions) {
        set_status(a.status, kErrInternal);
        return pos < 0 ? 0 : a.positions - 1;
    }
    return pos;
}

// The rows in the bits of `mine` (one bit a group of heads, the same for the lanes of a row), in double precision.  Other rows of the group have been
// written, perhaps to where they came from.  A function of its own, so that it takes no registers where it is not called.
template <int D, class T>
__device__ __noinline__ void append_queries_again(const KvAppend& a, int b, int j, int h0, int pos, unsigned mine) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    const int sub = threadIdx.x & (kLanes - 1), partner = kv_partner(a, sub);
    KvAngles g;
    if (a.rot_dim) kv_angles(a, sub, pos, g);
    for (unsigned again = __reduce_or_sync(0xFFFFFFFFu, mine); again; again &= again - 1) {
        const int i = __ffs(again) - 1, h = h0 + i * kRows;
        const bool on = (mine >> i & 1) && h < a.shape.q_heads;
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (on) raw = load8(a.q.data + b * a.q.batch + j * a.q.token + h * a.q.head + sub * 8, a.wide_q);
        double y[8];
        turn_exact<D, T>(a, a.q_norm, g, sub, partner, raw, y);
        if (on) {
            const uint4 o = make_uint4(from_float2<T>(round_to_odd(y[0]), round_to_odd(y[1])), from_float2<T>(round_to_odd(y[2]), round_to_odd(y[3])),
                                       from_float2<T>(round_to_odd(y[4]), round_to_odd(y[5])), from_float2<T>(round_to_odd(y[6]), round_to_odd(y[7])));
            store8(const_cast<uint16_t*>(a.q_out.data) + b * a.q_out.batch + j * a.q_out.token + h * a.q_out.head + sub * 8, o, a.wide_out);
        }
    }
}

// The queries: a warp takes kAppendRows groups of heads of one token.
template <int D, class T>
__device__ __forceinline__ void append_queries(const KvAppend& a, unsigned block) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    const int lane = threadIdx.x & 31, sub = lane & (kLanes - 1);
    const unsigned item = block * (blockDim.x >> 5) + (threadIdx.x >> 5), bt = a.by_parts.div(item), part = item - bt * a.query_parts;
    const unsigned b = a.by_T.div(bt);
    const int j = (int)(bt - b * a.step.T), h0 = (int)part * kAppendRows * kRows + lane / kLanes;
    if (b >= (unsigned)a.step.B) return;
    // what is certain to be needed is on its way before the lengths are known (rows of padding may be read, but are not used)
    const uint16_t* from = a.q.data + b * a.q.batch + j * a.q.token + sub * 8;
    uint16_t* to = const_cast<uint16_t*>(a.q_out.data) + b * a.q_out.batch + j * a.q_out.token + sub * 8;
    uint4 raw[kAppendRows];
#pragma unroll
    for (int i = 0; i < kAppendRows; ++i) {
        raw[i] = make_uint4(0, 0, 0, 0);
        if (h0 + i * kRows < a.shape.q_heads) raw[i] = load8(from + (h0 + i * kRows) * a.q.head, a.wide_q);
    }
    const int base = kv_base(a, b);
    int len, tokens;
    if (!kv_sequence(a.shape, a.step, b, len, tokens, a.status) || j >= tokens) return;
    KvAngles g;
    KvFold f;
    const int partner = kv_partner(a, sub), pos = kv_position(a, b, j, len, base);
    if (a.rot_dim) kv_angles(a, sub, pos, g);
    const bool large = __any_sync(0xFFFFFFFFu, kv_fold<T>(a, a.q_norm, g, sub, partner, f));
    const bool partly = a.rot_dim > 0 && a.rot_dim < D;
    unsigned again = 0;                                      // this lane's rows that single precision cannot be relied on for
#pragma unroll
    for (int i = 0; i < kAppendRows; ++i) {
        if (part * kAppendRows * kRows + i * kRows >= (unsigned)a.shape.q_heads) break;    // the same for the whole warp
        float x[8];
        bool wild = turn_fast<D, T>(a, a.q_norm != nullptr, f, partner, raw[i], x) || large;
        if (partly) wild = __any_sync(0xFFFFFFFFu, wild || !(max_abs8(x) < INFINITY));
        if (wild) again |= 1u << i;
        if (!wild && h0 + i * kRows < a.shape.q_heads) {     // (rows that are taken again are read again, perhaps from where they are written to)
            const uint4 o = make_uint4(from_float2<T>(x[0], x[1]), from_float2<T>(x[2], x[3]), from_float2<T>(x[4], x[5]), from_float2<T>(x[6], x[7]));
            store8(to + (h0 + i * kRows) * a.q_out.head, o, a.wide_out);
        }
    }
    if ((!a.q_norm && !partly) || !__any_sync(0xFFFFFFFFu, again != 0)) return;
    append_queries_again<D, T>(a, (int)b, j, h0, pos, again);
}

__device__ __forceinline__ float finite_abs(float x) {      // infinities saturate and NaN stays NaN: neither sets the scale
    const float m = fabsf(x);
    return m < INFINITY ? m : 0.f;
}
__device__ __forceinline__ double finite_abs(double x) {
    const double m = fabs(x);
    return m < (double)INFINITY ? m : 0.0;
}

// kPasses: row groups per warp that cover a page.
template <int D, class T, int kThreadsN, int kPasses>
__global__ void __launch_bounds__(kThreadsN, kThreadsN == 512 ? 1 : kThreadsN == 128 ? 6 : 3) kv_append_kernel(const __grid_constant__ KvAppend a) {
    grid_dependency_wait();
    if ((int)blockIdx.x >= a.page_blocks) {
        append_queries<D, T>(a, blockIdx.x - (unsigned)a.page_blocks);
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
    const int base = values ? 0 : kv_base(a, b);
    int len, tokens;
    if (!kv_sequence(a.shape, a.step, b, len, tokens, a.status)) return;
    const int page = a.shape.page, at = (len >> a.shape.page_shift) + slot;
    const int start = at << a.shape.page_shift;                              // first slot of the page
    const int lo = max(len, start), hi = min(len + tokens, start + page);    // the step's slots in it
    if (lo >= hi) return;
    const KvRows& src = values ? a.v : a.k;
    const uint16_t* from = src.data + b * src.batch + h * src.head + sub * 8;
    const bool wide = values ? a.wide_v : a.wide_k;
    const int n = hi - lo;
    uint4 raw[kPasses];                                                      // on their way while the page is looked up
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
        raw[i] = make_uint4(0, 0, 0, 0);
        if (r < n) raw[i] = load8(from + (long long)(lo - len + r) * src.token, wide);
    }
    const int id = kv_page(a.shape, a.table, b, at, a.status);
    if (id < 0) return;
    const long long head = (long long)id * a.shape.kv_heads + h;
    uint8_t* codes = (values ? a.vc : a.kc) + head * page * D;
    float* scale = (values ? a.vs : a.ks) + head;
    const bool older = lo > start;
    const float was = older ? *scale : 0.f;
    const bool turns = !values && (a.k_norm || a.rot_dim);
    const int partner = kv_partner(a, sub);

    float x[kPasses][8];
    float most = 0.f;                                                        // an infinity: has to be found in double precision
    unsigned again = 0;                                                      // passes of this warp that are taken again in double precision
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        if (turns && (i * kWarpsN + warp) * kRows < n) {                     // the same for the whole warp
            const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
            KvAngles g;
            KvFold f;
            if (a.rot_dim) kv_angles(a, sub, kv_position(a, b, lo - len + min(r, n - 1), len, base), g);
            kv_fold<T>(a, a.k_norm, g, sub, partner, f);
            const bool wild = turn_fast<D, T>(a, a.k_norm != nullptr, f, partner, raw[i], x[i]);
            const float top = max_abs8(x[i]);
            const bool doubt = (wild || !(top < INFINITY)) && r < n;
            if (doubt) again |= 1u << i;
            most = fmaxf(most, doubt ? INFINITY : top);
        } else {
            unpack8<T>(raw[i], x[i]);
            const float top = max_abs8(x[i]);
            if (top < INFINITY) {
                most = fmaxf(most, top);
            } else {
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                    const uint32_t w = e < 2 ? raw[i].x : e < 4 ? raw[i].y : e < 6 ? raw[i].z : raw[i].w;
                    const float2 two = to_float2<T>(w);
                    most = fmaxf(most, finite_abs(e & 1 ? two.y : two.x));
                }
            }
        }
    }
    again = __reduce_or_sync(0xFFFFFFFFu, again);
    most = warp_max_f32(most);
    if (lane == 0) warp_max[warp] = __float_as_uint(most);
    __syncthreads();
#pragma unroll
    for (int w1 = 0; w1 < kWarpsN; ++w1) most = fmaxf(most, __uint_as_float(warp_max[w1]));
    // Single precision is off by less than 1e-6; nearer than 1e-5 to a border, or where it cannot be relied on, the largest value is found again in
    // double precision, so that the scale, which is a whole power of two, does not hang on a rounding.
    const uint32_t frac = __float_as_uint(most) & 0x7FFFFFu;
    int e = scale_exponent(__float_as_uint(most));
    if (turns && (most == INFINITY || (frac > 0x600000u - 147u && frac < 0x600000u + 147u))) {
        double exact = 0.0;
#pragma unroll 1
        for (int i = 0; i < kPasses; ++i) {
            if ((i * kWarpsN + warp) * kRows >= n) break;
            const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
            uint4 again = make_uint4(0, 0, 0, 0);
            if (r < n) again = load8(from + (long long)(lo - len + r) * src.token, wide);
            double y[8];
            KvAngles g;
            if (a.rot_dim) kv_angles(a, sub, kv_position(a, b, lo - len + min(r, n - 1), len, base), g);
            turn_exact<D, T>(a, a.k_norm, g, sub, partner, again, y);
#pragma unroll
            for (int c = 0; c < 8; ++c) exact = fmax(exact, finite_abs(y[c]));
        }
        const unsigned long long bits = warp_max_u64((unsigned long long)__double_as_longlong(exact));
        if (lane == 0) warp_max64[warp] = bits;
        __syncthreads();
        unsigned long long all = 0;
        for (int w1 = 0; w1 < kWarpsN; ++w1) all = warp_max64[w1] > all ? warp_max64[w1] : all;
        // 1.75 in the fraction of a double
        e = (int)(all >> 52) - 1023 - 8 + ((all & 0xFFFFFFFFFFFFFull) > 0xC000000000000ull ? 1 : 0);
        e = e < kLeastScaleExp ? kLeastScaleExp : min(e, 127);
    }
    const float now = fmaxf(was, power_of_two(e)), inv = 1.f / now;
    if (older && now > was) {                                                // the page's older entries to the larger scale
        const float ratio = was * inv;
        uint4* rows = reinterpret_cast<uint4*>(codes);
        for (int c = threadIdx.x; c < (lo - start) * (D / 16); c += kThreadsN) rows[c] = recode16(rows[c], ratio);
    }
    // Single precision is off by less than 1.2e-6 of a pair's larger element (norm's sum and factor, folded weights, rotation; 4e-7 without
    // a norm).  Rows with a value that near the middle between two codes are taken again in double precision below, so that what is
    // stored is the rounding of the exact value.
    const float tol = (a.k_norm ? 1.2e-6f : 4e-7f) * inv;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int r = (i * kWarpsN + warp) * kRows + lane / kLanes;
        if (turns && (i * kWarpsN + warp) * kRows < n) {                     // the same for the whole warp
            float own = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c) own = fmaxf(own, fabsf(x[i][c]));
            own = tol * fmaxf(own, __shfl_sync(0xFFFFFFFFu, own, (lane & ~(kLanes - 1)) + partner));
            float low[8];                                                    // rounding is monotone: codes of both ends tell
#pragma unroll
            for (int c = 0; c < 8; ++c) { low[c] = fmaf(x[i][c], inv, -own); x[i][c] = fmaf(x[i][c], inv, own); }
            const uint2 under = make_uint2(to_e4m3x4(low[0], low[1], low[2], low[3]), to_e4m3x4(low[4], low[5], low[6], low[7]));
            const uint2 over = make_uint2(to_e4m3x4(x[i][0], x[i][1], x[i][2], x[i][3]), to_e4m3x4(x[i][4], x[i][5], x[i][6], x[i][7]));
            const bool near = ((under.x ^ over.x) | (under.y ^ over.y)) != 0;
            again |= (__any_sync(0xFFFFFFFFu, near && r < n) ? 1u : 0u) << i;
            if (r < n) *reinterpret_cast<uint2*>(codes + (long long)(lo - start + r) * D + sub * 8) = over;
        } else if (r < n) {
            uint2 o;
            o.x = to_e4m3x4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv);
            o.y = to_e4m3x4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv);
            *reinterpret_cast<uint2*>(codes + (long long)(lo - start + r) * D + sub * 8) = o;
        }
    }
    while (again) {
        const int i = __ffs(again) - 1, r = (i * kWarpsN + warp) * kRows + lane / kLanes;
        again &= again - 1;
        uint4 raw2 = make_uint4(0, 0, 0, 0);
        if (r < n) raw2 = load8(from + (long long)(lo - len + r) * src.token, wide);
        double y[8];
        KvAngles g;
        if (a.rot_dim) kv_angles(a, sub, kv_position(a, b, lo - len + min(r, n - 1), len, base), g);
        turn_exact<D, T>(a, a.k_norm, g, sub, partner, raw2, y);
        if (r < n) {
            const double by = 1.0 / (double)now;
            uint2 o;
            o.x = to_e4m3x4(round_to_odd(y[0] * by), round_to_odd(y[1] * by), round_to_odd(y[2] * by), round_to_odd(y[3] * by));
            o.y = to_e4m3x4(round_to_odd(y[4] * by), round_to_odd(y[5] * by), round_to_odd(y[6] * by), round_to_odd(y[7] * by));
            *reinterpret_cast<uint2*>(codes + (long long)(lo - start + r) * D + sub * 8) = o;
        }
    }
    if (threadIdx.x == 0) *scale = now;
}

}  // namespace ot
