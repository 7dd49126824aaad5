// Attention of few query rows (at most 16 per sequence and key head: plain decoding, and the smallest trees): bound by the cache's bytes.
//
// A warp takes 16 keys at a time with all the rows, by mma.sync m16n8k16 in half precision: e4m3 codes are exact there, and
// 16 rows would leave seven eighths of a tcgen05 tile empty while its operands would still have to be converted and stored
// again.  Operands go from the codes in shared memory to fragments without any transposition: the order of the summed index is
// free, so a lane takes 16 consecutive codes of a key as its share of four k-steps; for P V the lane takes the codes of four keys
// at 16 consecutive elements and pairs them by byte permutation.
// Each warp has a ring of its own, filled by bulk copies that its first lane issues (a page's rows of one head are contiguous): nothing in
// the loop waits for another warp.  Values come as four rows a copy, 32 bytes apart, so that the four lanes that read
// the same element of keys 4t ... 4t+3 hit different banks.
#pragma once

#include <type_traits>

#include "copy_ring.cuh"
#include "kv_attend.cuh"

namespace ot {

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Probabilities are rounded to half precision (2^-11 of each at most) for the product with the values; they are held times 2^12 and times the
// page's scale over the largest so far, so that pages with scales down to 2^-24 of the largest keep that accuracy.
constexpr float kProbUnit = 4096.f;

// NT: row groups of eight.  Two CTAs an SM where registers allow (one of 16 warps: 13.8 us against 12.5 for one token over 1500, 175 against
// 170 for 32 over 16384).
template <int D, int NT> struct FewLayout {
    static constexpr int kWarps = 8, kThreads = kWarps * 32, kKeys = kWarps * 16, kPerSm = NT == 1 ? 2 : 1;
    static constexpr int kStages = (D == 128 ? 6 : 12) / kPerSm;
    static constexpr int kKBytes = 16 * D, kVGroup = 4 * D + 32, kStage = kKBytes + 4 * kVGroup;
    static constexpr int kRows = 8 * NT;
    static constexpr int kRing = kWarps * kStages * kStage;
    static constexpr int kMerge = kWarps * (kRows * D + 2 * kRows) * 4;   // the warps' parts, over the ring
    static constexpr int kBig = kRing > kMerge ? kRing : kMerge;
    static constexpr int kBars = kBig, kWord = kBars + kWarps * kStages * 8;
    static constexpr int kBytes = kWord + 16;
};

template <int D, int NT, class T>
__global__ void __launch_bounds__(FewLayout<D, NT>::kThreads, FewLayout<D, NT>::kPerSm) kv_attend_few_kernel(const __grid_constant__ KvAttend a) {
    using L = FewLayout<D, NT>;
    using Ring = CopyRing<L::kStages>;
    constexpr int kRows = L::kRows, kStages = L::kStages, kKeys = L::kKeys, kChunks = D / 64, kSteps = D / 16, kVWords = D / 32;
    extern __shared__ __align__(128) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    unsigned char* ring = smem + warp * kStages * L::kStage;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + L::kBars) + warp * kStages;
    int* word = reinterpret_cast<int*>(smem + L::kWord);
    if (lane == 0)
        for (int s = 0; s < kStages; ++s) mbar_init(bars + s, 1);
    mbar_fence_init();
    __syncwarp();
    grid_dependency_wait();
    KvWalk<kRows, kKeys, false> walk;
    if (!walk.begin(a, blockIdx.x, gridDim.x)) return;
    KvRun r;
    uint32_t count = 0;                                      // blocks this warp has consumed: its place in the ring
    bool dead = false;                                       // a wait ran out: nothing more is loaded
    while (walk.next(a, r)) {
        const int rows = min(kRows, r.tokens * a.group - r.rt * kRows);
        // this warp's blocks of 16 keys: one a tile
        const int key0 = (r.k0 * L::kWarps + warp) * 16;
        const int blocks = key0 < r.keys ? min(r.k1 - r.k0, (r.keys - key0 + L::kKeys - 1) / L::kKeys) : 0;
        // queries: rows g and g + 8, elements in the order in which the lanes hold keys.  bf16 rows are brought to half precision by
        // a power of two of their own (exact but for elements below 2^-25 of the row's largest)
        uint4 raw[NT][kChunks * 2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = n * 8 + g, full = r.rt * kRows + row;
#pragma unroll
            for (int i = 0; i < kChunks * 2; ++i) raw[n][i] = make_uint4(0, 0, 0, 0);
            if (row < rows) {
                const int token = (int)a.by_group.div((unsigned)full), hq = r.h * a.group + full - token * a.group;
                const uint16_t* q = a.q.data + r.b * a.q.batch + token * a.q.token + hq * a.q.head;
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int i = 0; i < 2; ++i) raw[n][c * 2 + i] = load8(q + c * 64 + t * 16 + i * 8, a.wide_q);
            }
        }
        // pages and scales of 32 blocks at a time, a lane each; the next 32 are fetched while these are in use
        int id[2];
        float ks[2], vs[2];
        auto look = [&](int chunk) {
            const int at = chunk * 32 + lane;
            return at < blocks ? max(0, kv_page(a.shape, a.table, r.b, (key0 + at * L::kKeys) >> a.shape.page_shift, a.status)) : -1;
        };
        auto scales = [&](int i, float& k, float& v) {
            k = v = 0.f;
            if (i >= 0) {
                const long long head = (long long)i * a.shape.kv_heads + r.h;
                k = a.ks[head]; v = a.vs[head];
            }
        };
        id[0] = look(0);
        id[1] = blocks > 32 ? look(1) : -1;
        auto fetch = [&](int i, int page_id) {               // lane 0: block i of this run into its stage
            const uint32_t at = count + i;
            unsigned char* stage = ring + Ring::stage(at) * L::kStage;
            unsigned long long* bar = bars + Ring::stage(at);
            const long long row = ((long long)page_id * a.shape.kv_heads + r.h) * a.shape.page + ((key0 + i * L::kKeys) & (a.shape.page - 1));
            mbar_expect_tx(bar, 32 * D);
            bulk_load(stage, a.kc + row * D, 16 * D, bar);
#pragma unroll
            for (int q = 0; q < 4; ++q) bulk_load(stage + L::kKBytes + q * L::kVGroup, a.vc + (row + 4 * q) * D, 4 * D, bar);
        };
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            const int p = __shfl_sync(0xFFFFFFFFu, id[0], i);
            if (lane == 0 && i < blocks && !dead) fetch(i, p);
        }
        scales(id[0], ks[0], vs[0]);
        scales(id[1], ks[1], vs[1]);
        uint32_t qa[NT][kSteps][2];
        float qf[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float f = 1.f, unit = 1.f;
            if (!std::is_same<T, __half>::value) {
                uint32_t top = 0;                            // largest magnitude, by its bits
#pragma unroll
                for (int i = 0; i < kChunks * 2; ++i) {
                    const uint32_t w[4] = {raw[n][i].x, raw[n][i].y, raw[n][i].z, raw[n][i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7FFFu, w[e] >> 16 & 0x7FFFu));
                }
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const int e = min(max((int)(top >> 7) - 127, -112), 120);
                f = power_of_two(8 - e > 127 ? 127 : 8 - e);
                unit = power_of_two(e - 8);
            }
            qf[n] = unit * a.scale;
#pragma unroll
            for (int i = 0; i < kChunks * 2; ++i) {
                const uint32_t w[4] = {raw[n][i].x, raw[n][i].y, raw[n][i].z, raw[n][i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 x = to_float2<T>(w[e]);
                    qa[n][i * 2 + e / 2][e & 1] = from_float2<__half>(x.x * f, x.y * f);
                }
            }
        }
        float o[NT][kSteps][4], m[NT], l[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = -INFINITY; l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
        }
        float ref = 0.f;                                     // largest scale of values so far: the outputs' unit
        uint32_t nan = 0;
        for (int i = 0; i < blocks; ++i) {
            if (i && (i & 31) == 0) {
                id[0] = id[1]; ks[0] = ks[1]; vs[0] = vs[1];
                id[1] = look((i >> 5) + 1);
                scales(id[1], ks[1], vs[1]);
            }
            const float kscale = __shfl_sync(0xFFFFFFFFu, ks[0], i & 31), vscale = __shfl_sync(0xFFFFFFFFu, vs[0], i & 31);
            const int ahead = i + kStages;
            const int p = (ahead >> 5) == (i >> 5) ? __shfl_sync(0xFFFFFFFFu, id[0], ahead & 31) : __shfl_sync(0xFFFFFFFFu, id[1], ahead & 31);
            const uint32_t at = count + i;
            const unsigned char* stage = ring + Ring::stage(at) * L::kStage;
            if (!dead && !mbar_wait_warp(bars + Ring::stage(at), Ring::parity(at), a.status)) {
                dead = true;                                 // what is in flight lands before anything else uses the ring
                Ring::drain(at, count + min(blocks, i + kStages), [&](uint32_t st, uint32_t parity) { mbar_wait_warp(bars + st, parity, a.status); });
            }
            const int s0 = key0 + i * L::kKeys;              // first slot of the block
            // scores: rows x keys, key 4 (n >> 1) + 2 half + (n & 1) as column n of each half
            float s[2][4];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[half][e] = 0.f;
                const unsigned char* k = stage + (4 * (g >> 1) + 2 * half + (g & 1)) * D + t * 16;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const uint4 x = *reinterpret_cast<const uint4*>(k + c * 64);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        mma_f16(s[half], qa[0][c * 4 + e][0], NT == 2 ? qa[NT - 1][c * 4 + e][0] : 0u, qa[0][c * 4 + e][1], NT == 2 ? qa[NT - 1][c * 4 + e][1] : 0u,
                                from_e4m3x2((uint16_t)w[e]), from_e4m3x2((uint16_t)(w[e] >> 16)));
                }
            }
            const bool edge = s0 + 16 > r.len;               // some keys are the step's own, or behind them
            float top[NT], x[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float f = qf[n] * kscale;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[n][e] = s[e >> 1][n * 2 + (e & 1)] * f;      // key 4t + e
                if (edge) {
                    const int token = (int)a.by_group.div((unsigned)min(r.rt * kRows + n * 8 + g, r.tokens * a.group - 1));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = s0 + 4 * t + e - r.len;
                        if (j >= r.tokens || (j >= 0 && !kv_sees(a.step, r.b, token, j))) x[n][e] = -INFINITY;
                    }
                }
                top[n] = fmaxf(fmaxf(x[n][0], x[n][1]), fmaxf(x[n][2], x[n][3]));
                top[n] = fmaxf(top[n], __shfl_xor_sync(0xFFFFFFFFu, top[n], 1));
                top[n] = fmaxf(top[n], __shfl_xor_sync(0xFFFFFFFFu, top[n], 2));
            }
            bool grows = vscale > ref;
#pragma unroll
            for (int n = 0; n < NT; ++n) grows = grows || top[n] > m[n];
            if (__any_sync(0xFFFFFFFFu, grows)) {
                const float now = fmaxf(ref, vscale), unit = ref > 0.f ? ref / now : 1.f;
                ref = now;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float was = m[n];
                    m[n] = fmaxf(m[n], top[n]);
                    const float fade = was == -INFINITY ? 1.f : ex2_approx(was - m[n]);       // nothing to fade before the first key
                    l[n] *= fade;
                    const float lo = unit * __shfl_sync(0xFFFFFFFFu, fade, 8 * t), hi = unit * __shfl_sync(0xFFFFFFFFu, fade, 8 * t + 4);
#pragma unroll
                    for (int d = 0; d < kSteps; ++d) { o[n][d][0] *= lo; o[n][d][1] *= hi; o[n][d][2] *= lo; o[n][d][3] *= hi; }
                }
            }
            uint32_t pb[NT][2];
            const float pv = kProbUnit * (ref > 0.f ? vscale / ref : 0.f);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float base = m[n] == -INFINITY ? 0.f : m[n];
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = ex2_approx(x[n][e] - base);
                l[n] += (p[0] + p[1]) + (p[2] + p[3]);
                pb[n][0] = from_float2<__half>(p[0] * pv, p[1] * pv);
                pb[n][1] = from_float2<__half>(p[2] * pv, p[3] * pv);
            }
            // values: keys 4t ... 4t+3 at this lane's D/8 elements
            const unsigned char* v = stage + L::kKBytes + t * L::kVGroup + g * (D / 8);
            uint32_t w[4][kVWords];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (kVWords == 4) {
                    const uint4 y = *reinterpret_cast<const uint4*>(v + j * D);
                    w[j][0] = y.x; w[j][1] = y.y; w[j][2 % kVWords] = y.z; w[j][3 % kVWords] = y.w;
                } else {
                    const uint2 y = *reinterpret_cast<const uint2*>(v + j * D);
                    w[j][0] = y.x; w[j][1] = y.y;
                }
                if (edge) {
                    const int step = s0 + 4 * t + j - r.len;
                    if (step >= r.tokens) {
#pragma unroll
                        for (int c = 0; c < kVWords; ++c) w[j][c] = 0;
                    } else if (step >= 0) {
#pragma unroll
                        for (int c = 0; c < kVWords; ++c) w[j][c] = drop_nan(w[j][c], nan);
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < kVWords; ++c) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x01 = __byte_perm(w[0][c], w[1][c], e ? 0x7362 : 0x5140), x23 = __byte_perm(w[2][c], w[3][c], e ? 0x7362 : 0x5140);
                    const uint32_t a0 = from_e4m3x2((uint16_t)x01), a1 = from_e4m3x2((uint16_t)(x01 >> 16));
                    const uint32_t a2 = from_e4m3x2((uint16_t)x23), a3 = from_e4m3x2((uint16_t)(x23 >> 16));
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_f16(o[n][c * 2 + e], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                }
            }
            __syncwarp();                                    // the stage has been read by all lanes
            if (lane == 0 && ahead < blocks && !dead) fetch(ahead, p);
        }
        count += blocks;
        __syncthreads();                                     // every warp is done with its ring: the parts go over it
        float* mo = reinterpret_cast<float*>(smem) + warp * (kRows * D + 2 * kRows);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] += __shfl_xor_sync(0xFFFFFFFFu, l[n], 1);
            l[n] += __shfl_xor_sync(0xFFFFFFFFu, l[n], 2);
            if (t == 0) { mo[kRows * D + n * 8 + g] = m[n]; mo[kRows * D + kRows + n * 8 + g] = l[n]; }
            const float over = l[n] > 0.f ? 1.f / l[n] : 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {                    // row 2t + e: this lane's D/8 consecutive elements
                const float unit = ref * (1.f / kProbUnit) * __shfl_sync(0xFFFFFFFFu, over, 8 * t + 4 * e);
                float* to = mo + (n * 8 + 2 * t + e) * D + g * (D / 8);
#pragma unroll
                for (int d = 0; d < kSteps; d += 2)
                    *reinterpret_cast<float4*>(to + d * 2) = make_float4(o[n][d][e] * unit, o[n][d][2 + e] * unit, o[n][d + 1][e] * unit, o[n][d + 1][2 + e] * unit);
            }
        }
        const bool any_nan = __syncthreads_or(nan != 0);
        const bool cut = r.first != r.last;
        float* part = a.parts + (long long)kv_slot(r, blockIdx.x) * kv_part_floats<kRows, D>();
        constexpr int kStride = kRows * D + 2 * kRows;
        const float* all = reinterpret_cast<const float*>(smem);
        for (int at = threadIdx.x; at < kRows * D / 4; at += L::kThreads) {
            const int row = at / (D / 4), d = at % (D / 4) * 4;
            if (row >= rows) break;
            float mm = -INFINITY;
#pragma unroll
            for (int w = 0; w < L::kWarps; ++w) mm = fmaxf(mm, all[w * kStride + kRows * D + row]);
            const float base = mm == -INFINITY ? 0.f : mm;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            float ll = 0.f, share[L::kWarps];
#pragma unroll
            for (int w = 0; w < L::kWarps; ++w) {
                share[w] = ex2_approx(all[w * kStride + kRows * D + row] - base) * all[w * kStride + kRows * D + kRows + row];
                ll += share[w];
            }
            const float over = ll > 0.f ? 1.f / ll : 0.f;
#pragma unroll
            for (int w = 0; w < L::kWarps; ++w) {
                const float f = share[w] * over;
                const float4 y = *reinterpret_cast<const float4*>(all + w * kStride + row * D + d);
                sum.x += f * y.x; sum.y += f * y.y; sum.z += f * y.z; sum.w += f * y.w;
            }
            if (cut) {
                *reinterpret_cast<float4*>(part + (d / 4 * kRows + row) * 4) = sum;
                if (d == 0) { part[kRows * D + row] = mm; part[kRows * D + kRows + row] = ll; }
            } else {
                const float x[4] = {sum.x, sum.y, sum.z, sum.w};
                kv_store<D, 4, T>(a, r, r.rt * kRows + row, d, x, any_nan);
                if (d == 0) kv_store_lse(a, r, r.rt * kRows + row, mm, ll);
            }
        }
        if (cut) {
            if (threadIdx.x == 0) reinterpret_cast<int*>(part)[kRows * D + 2 * kRows] = any_nan;
            if (kv_last_part<0, L::kThreads>(a.arrived + r.first, r.last - r.first + 1, word))
                kv_join<kRows, D, T>(a, r, a.parts, 1, r.rt * kRows, rows, warp, L::kWarps);
        }
        proxy_fence();                                       // the ring is free again, for copies too
        __syncthreads();
    }
}

}  // namespace ot
