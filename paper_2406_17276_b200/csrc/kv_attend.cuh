// Attention of a step's tokens over the paged 8-bit cache: what its kernels share.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(x_ij - m_i) / l_i,  x_ij = scale * q_i . k_j   over the slots j that token i sees
//
// All query rows of a sequence that read one key head (tokens x query heads per key head, token-major) are taken together, so that
// a page is read and converted once for them.  Work is cut by the clock and not by sequence: the tiles (sequence, key head, row
// tile, tile of keys) are numbered in that order and every CTA takes an equal run of them, whatever the lengths; a row tile that is cut
// leaves its parts (maximum, sum, unnormalised output) in the workspace, and the CTA that finishes last joins them in order, so
// results do not depend on who that is.
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
    float scale;                         // times log2 e: scores are kept in powers of two
    int group;                           // query heads per key head
    FixedDiv by_group;
    int wide_q, wide_out;
    float* parts;                        // [2 * grid][part_floats]
    int* arrived;                        // [grid], zero between calls
    int* status;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Whether token i of a step sees token j of it.
__device__ __forceinline__ bool kv_sees(const KvStep& st, int b, int i, int j) {
    if (j == i || j == 0) return true;
    if (!st.mask) return j < i;
    if (i == 0) return false;
    const int W = (st.T - 1 + 63) >> 6;
    return (st.mask[((long long)b * (st.T - 1) + i - 1) * W + ((j - 1) >> 6)] >> ((j - 1) & 63)) & 1ull;
}

// One run of key tiles of one (sequence, key head, row tile).
struct KvRun {
    int b, h, rt;
    int len, tokens;
    int keys;                            // slots that any row of the tile sees
    int k0, k1;                          // tiles [k0, k1) of them
    int first, last;                     // CTAs that hold the row tile's first and last tile: more than one if it is cut
};

// Walks the run of tiles of one CTA of a grid.  kRows rows and kKeys keys a tile.  Every warp keeps its own copy (no shared memory, no
// barrier); the lengths come from the cache after the first warp.
template <int kRows, int kKeys>
struct KvWalk {
    long long total, pos, end, base;     // tiles; base: first tile of sequence b
    int cta, grid, b;

    __device__ __forceinline__ static int row_tiles(const KvAttend& a, int tokens) { return (tokens * a.group + kRows - 1) / kRows; }
    // In a chain a row tile sees no further than its last token.
    __device__ __forceinline__ static int keys_of(const KvAttend& a, int len, int tokens, int rt) {
        if (a.step.mask) return len + tokens;
        const int last = (int)a.by_group.div((unsigned)(rt + 1) * kRows - 1u);
        return len + min(tokens, last + 1);
    }
    __device__ __forceinline__ static int tiles_of(const KvAttend& a, int len, int tokens, int rt) { return (keys_of(a, len, tokens, rt) + kKeys - 1) / kKeys; }
    // Tiles of one key head of a sequence.
    __device__ __forceinline__ static long long head_tiles(const KvAttend& a, int len, int tokens) {
        const int n = row_tiles(a, tokens);
        if (n == 0) return 0;
        if (a.step.mask) return (long long)n * tiles_of(a, len, tokens, 0);
        long long s = 0;
        for (int rt = 0; rt < n; ++rt) s += tiles_of(a, len, tokens, rt);
        return s;
    }
    __device__ __forceinline__ static long long sequence_tiles(const KvAttend& a, int b) {
        int len, tokens;
        if (b >= a.step.B || !kv_sequence(a.shape, a.step, b, len, tokens, a.status)) return 0;
        return head_tiles(a, len, tokens) * a.shape.kv_heads;
    }
    __device__ __forceinline__ static long long warp_scan(long long v) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xFFFFFFFFu, v, o);
            if (lane >= o) v += u;
        }
        return v;
    }
    // false: nothing for this CTA.
    __device__ bool begin(const KvAttend& a, int which, int ctas) {
        const int lane = threadIdx.x & 31;
        total = 0;
        long long incl = 0;
        for (int b0 = 0; b0 < a.step.B; b0 += 32) {
            incl = warp_scan(sequence_tiles(a, b0 + lane));
            total += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
        cta = which;
        grid = (int)min((long long)ctas, total);
        if (cta >= grid) return false;
        pos = total * cta / grid;
        end = total * (cta + 1) / grid;
        find(a, incl);
        return true;
    }
    // Sets b and base to the sequence that holds tile pos; incl: this lane's inclusive count where all sequences fit in a warp.
    __device__ void find(const KvAttend& a, long long incl) {
        const int lane = threadIdx.x & 31;
        base = 0;
        b = 0;
        for (int b0 = 0; b0 < a.step.B; b0 += 32) {
            if (a.step.B > 32) incl = warp_scan(sequence_tiles(a, b0 + lane));
            const unsigned over = __ballot_sync(0xFFFFFFFFu, base + incl > pos);
            if (over) {
                const int l = __ffs(over) - 1;
                const long long before = __shfl_sync(0xFFFFFFFFu, incl, l > 0 ? l - 1 : 0);
                b = b0 + l;
                base += l > 0 ? before : 0;
                break;
            }
            base += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
    }
    // The row tile of this CTA's last key tile (k0, k1: that tile alone).
    __device__ bool last(const KvAttend& a, KvRun& r) {
        pos = end - 1;
        find(a, a.step.B <= 32 ? warp_scan(sequence_tiles(a, threadIdx.x & 31)) : 0);
        return next(a, r);
    }
    __device__ __forceinline__ int owner(long long tile) const { return (int)(((tile + 1) * grid - 1) / total); }
    // The next run; false at the end.
    __device__ bool next(const KvAttend& a, KvRun& r) {
        if (pos >= end) return false;
        int len, tokens;
        long long per_head;
        for (;; ++b) {
            if (b >= a.step.B) return false;                 // (cannot happen: the tiles were counted)
            per_head = kv_sequence(a.shape, a.step, b, len, tokens, a.status) ? head_tiles(a, len, tokens) : 0;
            if (pos < base + per_head * a.shape.kv_heads) break;
            base += per_head * a.shape.kv_heads;
        }
        long long off = pos - base;
        r.h = (int)(off / per_head);
        off -= r.h * per_head;
        r.rt = 0;
        int n = tiles_of(a, len, tokens, 0);
        if (a.step.mask) { r.rt = (int)(off / n); off -= (long long)r.rt * n; }
        else while (off >= n) { off -= n; n = tiles_of(a, len, tokens, ++r.rt); }
        r.b = b; r.len = len; r.tokens = tokens;
        r.keys = keys_of(a, len, tokens, r.rt);
        r.k0 = (int)off;
        r.k1 = (int)min((long long)n, off + (end - pos));
        const bool whole = r.k0 == 0 && r.k1 == n;
        r.first = whole ? cta : owner(pos - off);
        r.last = whole ? cta : owner(pos - off + n - 1);
        pos += r.k1 - r.k0;
        return true;
    }
};

// NaN codes of a step's values are taken as zero by the tensor-core kernels, which would otherwise spread them to rows that do not
// see the token (0 * NaN); outputs that do see one are made NaN here, after they have been stored: elements [d, d + n) of query row
// `row`.
template <int D, class T>
__device__ __noinline__ void kv_mark_nan(const KvAttend& a, const KvRun& r, int row, int d, int n) {
    const int token = (int)a.by_group.div((unsigned)row), hq = r.h * a.group + row - token * a.group;
    uint16_t* to = const_cast<uint16_t*>(a.out.data) + r.b * a.out.batch + token * a.out.token + hq * a.out.head;
#pragma unroll 1
    for (int j = 0; j < r.tokens; ++j) {
        if (!kv_sees(a.step, r.b, token, j)) continue;
        const int s = r.len + j, id = max(0, kv_page(a.shape, a.table, r.b, s >> a.shape.page_shift, a.status));
        const uint8_t* v = a.vc + (((long long)id * a.shape.kv_heads + r.h) * a.shape.page + (s & (a.shape.page - 1))) * D;
#pragma unroll 1
        for (int e = d; e < d + n; ++e)
            if ((v[e] & 0x7F) == 0x7F) to[e] = (uint16_t)from_float2<T>(__int_as_float(0x7FC00000), 0.f);
    }
}
// Clears NaN codes and reports them.
__device__ __forceinline__ uint32_t drop_nan(uint32_t four, uint32_t& seen) {
    const uint32_t nan = __vcmpeq4(four & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
    seen |= nan;
    return four & ~nan;
}

// A cut row tile's part: kRows x D unnormalised outputs (values' scales applied), then maxima, sums and a word that says whether
// NaN values were met.
template <int kRows, int D> __host__ __device__ constexpr int kv_part_floats() { return kRows * D + 2 * kRows + 4; }

// A row's outputs at elements [d, d + N) of query row `row` of the run (row tile included).
template <int D, int N, class T>
__device__ __forceinline__ void kv_store(const KvAttend& a, const KvRun& r, int row, int d, const float (&x)[N], bool nan) {
    const int token = (int)a.by_group.div((unsigned)row), hq = r.h * a.group + row - token * a.group;
    uint16_t* to = const_cast<uint16_t*>(a.out.data) + r.b * a.out.batch + token * a.out.token + hq * a.out.head + d;
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = from_float2<T>(x[2 * i], x[2 * i + 1]);
    if (!a.wide_out) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) { to[2 * i] = (uint16_t)w[i]; to[2 * i + 1] = (uint16_t)(w[i] >> 16); }
    } else if (N % 8 == 0) {
#pragma unroll
        for (int i = 0; i + 3 < N / 2; i += 4) *reinterpret_cast<uint4*>(to + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    } else if (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i + 1 < N / 2; i += 2) *reinterpret_cast<uint2*>(to + 2 * i) = make_uint2(w[i], w[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) *reinterpret_cast<uint32_t*>(to + 2 * i) = w[i];
    }
    if (nan) kv_mark_nan<D, T>(a, r, row, d, N);
}
__device__ __forceinline__ void kv_store_lse(const KvAttend& a, const KvRun& r, int row, float m, float l) {
    if (!a.lse) return;
    const int token = (int)a.by_group.div((unsigned)row), hq = r.h * a.group + row - token * a.group;
    a.lse[((long long)r.b * a.step.T + token) * a.shape.q_heads + hq] = (m + log2f(l)) * kLn2;
}

// Slot of CTA c's part of a cut row tile: 2c for the tile with which it begins, 2c + 1 for the one with which it ends (which began
// in c).
__device__ __forceinline__ int kv_slot(const KvRun& r, int cta) { return cta == r.first ? 2 * cta + 1 : 2 * cta; }

// Counts this CTA's part of a cut row tile as written; true to all kThreadsN threads of the one group that is the last.  They are
// the threads of named barrier kBarrier and call this together after their stores.
template <int kBarrier, int kThreadsN>
__device__ __forceinline__ bool kv_last_part(int* arrived, int pieces, int* word /* shared */) {
    __threadfence();                     // this thread's stores before the arrival
    asm volatile("bar.sync %0, %1;" ::"n"(kBarrier), "n"(kThreadsN) : "memory");
    if (threadIdx.x % kThreadsN == 0) {
        const bool last = atomicAdd(arrived, 1) == pieces - 1;
        if (last) *arrived = 0;          // for the next call
        *word = last;
        __threadfence();
    }
    asm volatile("bar.sync %0, %1;" ::"n"(kBarrier), "n"(kThreadsN) : "memory");
    return *word != 0;
}
// Joins a cut row tile's parts in the order of the keys: a warp a row, for the rows warp, warp + warps, ... of it.  kStep: parts from one
// slot to the next.  row0: the tile's first row.
template <int kRows, int D, class T>
__device__ __forceinline__ void kv_join(const KvAttend& a, const KvRun& r, const float* parts, int kStep, int row0, int rows, int warp, int warps) {
    constexpr int kFloats = kv_part_floats<kRows, D>(), N = D / 32;
    const int lane = threadIdx.x & 31, pieces = r.last - r.first + 1;
    const long long step = (long long)kStep * kFloats;
    auto part = [&](int i) { return parts + kv_slot(r, r.first + i) * step; };
    int seen = 0;
    for (int i = lane; i < pieces; i += 32) seen |= __ldcg(reinterpret_cast<const int*>(part(i)) + kRows * D + 2 * kRows);
    const bool nan = __any_sync(0xFFFFFFFFu, seen != 0);
    for (int row = warp; row < rows; row += warps) {
        float top = -INFINITY, l = 0.f, x[N];
        for (int i = lane; i < pieces; i += 32) top = fmaxf(top, __ldcg(part(i) + kRows * D + row));
        top = warp_max_f32(top);
        if (top == -INFINITY) top = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = 0.f;
        for (int i0 = 0; i0 < pieces; i0 += 32) {
            float w = 0.f;
            if (i0 + lane < pieces) {
                w = ex2_approx(__ldcg(part(i0 + lane) + kRows * D + row) - top);
                l += w * __ldcg(part(i0 + lane) + kRows * D + kRows + row);
            }
            const int n = min(32, pieces - i0);
#pragma unroll 8
            for (int i = 0; i < n; ++i) {
                const float f = __shfl_sync(0xFFFFFFFFu, w, i);
                const float* at = part(i0 + i) + row * D + lane * N;
                if (N == 4) {
                    const float4 y = __ldcg(reinterpret_cast<const float4*>(at));
                    x[0] += f * y.x; x[1] += f * y.y; x[2 % N] += f * y.z; x[3 % N] += f * y.w;
                } else {
                    const float2 y = __ldcg(reinterpret_cast<const float2*>(at));
                    x[0] += f * y.x; x[1] += f * y.y;
                }
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
        const float f = 1.f / l;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] *= f;
        kv_store<D, N, T>(a, r, row0 + row, lane * N, x, nan);
        if (lane == 0) kv_store_lse(a, r, row0 + row, top, l);
    }
}

}  // namespace ot
