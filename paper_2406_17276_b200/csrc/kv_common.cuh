// Shared pieces of the cache operators (append, attend, compact): argument blocks, 8-bit conversions, 16-bit loads.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace ot {

// A page's entries are e4m3 values times one power of two per page, head and side (keys, values).  A power of two makes bringing
// an entry to a larger scale exact as long as the entry stays a normal e4m3 number, so that entries can be moved between pages, and
// pages can take larger newcomers, without rounding again.
constexpr float kE4m3Max = 448.f;
constexpr int kLeastScaleExp = -64;      // of an all-zero page; smaller values than 2^-74 round to zero

struct KvShape {
    int q_heads, kv_heads, page, num_pages, max_pages;
    int page_shift;                      // page = 1 << page_shift
};
struct KvStep {
    int B, T;
    const int32_t *kv_len, *nodes, *base_pos, *position_ids;
    const uint64_t* mask;
};
struct KvRows {                          // 16-bit rows [batch][token][head][head_dim], strides in elements
    const uint16_t* data;
    long long batch, token, head;
};

// A sequence of the step: its cached tokens and the step's tokens.  false: takes no part (no tokens, or sizes out of range, which
// are recorded).
__device__ __forceinline__ bool kv_sequence(const KvShape& s, const KvStep& st, int b, int& len, int& tokens, int* status) {
    len = st.kv_len[b];
    const int nodes = st.nodes ? st.nodes[b] : st.T - 1;
    tokens = nodes + 1;
    if (nodes < 0) { tokens = 0; return false; }
    if (len < 0 || tokens > st.T || (long long)len + tokens > (long long)s.max_pages << s.page_shift) {
        set_status(status, kErrInternal);
        tokens = 0;
        return false;
    }
    return true;
}
// A page of a sequence's table; a page that does not exist is recorded and answered with -1.
__device__ __forceinline__ int kv_page(const KvShape& s, const int32_t* table, int b, int at, int* status) {
    const int id = table[(long long)b * s.max_pages + at];
    if ((unsigned)id >= (unsigned)s.num_pages) { set_status(status, kErrInternal); return -1; }
    return id;
}

// --- 16-bit inputs and outputs ---
template <class T> __device__ __forceinline__ float2 to_float2(uint32_t two);
template <> __device__ __forceinline__ float2 to_float2<__nv_bfloat16>(uint32_t two) {
    return make_float2(__uint_as_float(two << 16), __uint_as_float(two & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 to_float2<__half>(uint32_t two) { return __half22float2(*reinterpret_cast<__half2*>(&two)); }
template <class T> __device__ __forceinline__ uint32_t from_float2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t from_float2<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <> __device__ __forceinline__ uint32_t from_float2<__half>(float lo, float hi) {
    const __half2 r = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Eight consecutive elements; `wide`: the address is on a 16-byte boundary.  (The other way is a loop: it stands in many places, and code
// that hardly ever runs should not fill the instruction cache.)
__device__ __forceinline__ uint4 load8(const uint16_t* p, bool wide) {
    uint4 r;
    if (wide) return *reinterpret_cast<const uint4*>(p);
    r = make_uint4(0, 0, 0, 0);
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        r.x = __funnelshift_r(r.x, r.y, 16); r.y = __funnelshift_r(r.y, r.z, 16); r.z = __funnelshift_r(r.z, r.w, 16);
        r.w = r.w >> 16 | (uint32_t)p[i] << 16;
    }
    return r;
}
__device__ __forceinline__ void store8(uint16_t* p, uint4 v, bool wide) {
    if (wide) { *reinterpret_cast<uint4*>(p) = v; return; }
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        p[i] = (uint16_t)v.x;
        v.x = __funnelshift_r(v.x, v.y, 16); v.y = __funnelshift_r(v.y, v.z, 16); v.z = __funnelshift_r(v.z, v.w, 16); v.w >>= 16;
    }
}
template <class T> __device__ __forceinline__ void unpack8(uint4 v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = to_float2<T>(w[i]);
        x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
}

__device__ __forceinline__ uint4 ld_nc_v4(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// --- e4m3 ---
// Two values to two codes (round to nearest even, saturating, NaN stays NaN), `lo` in the low byte.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) { return to_e4m3x2(a, b) | to_e4m3x2(c, d) << 16; }
// Two codes to two half-precision values (exact).
__device__ __forceinline__ uint32_t from_e4m3x2(uint16_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
    return r;
}
// Four codes brought to another scale: value * ratio, rounded once.
__device__ __forceinline__ uint32_t recode4(uint32_t four, float ratio) {
    const uint32_t a = from_e4m3x2((uint16_t)four), b = from_e4m3x2((uint16_t)(four >> 16));
    const float2 x = to_float2<__half>(a), y = to_float2<__half>(b);
    return to_e4m3x4(x.x * ratio, x.y * ratio, y.x * ratio, y.y * ratio);
}
__device__ __forceinline__ uint4 recode16(uint4 v, float ratio) {
    return make_uint4(recode4(v.x, ratio), recode4(v.y, ratio), recode4(v.z, ratio), recode4(v.w, ratio));
}
// Orders this thread's accesses to shared memory before later asynchronous copies into it (and stores before tensor-core reads).
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The exponent of the smallest power of two that brings amax to 448 (1.75 * 2^8) or below.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < kLeastScaleExp ? kLeastScaleExp : e;
}

}  // namespace ot
