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

// Walks the run of tiles of this CTA.  kRows rows and kKeys keys a tile.  Every warp keeps its own copy (no shared memory, no
// barrier); the lengths come from the cache after the first warp.
template <int kRows, int kKeys>
struct KvWalk {
    long long total, pos, end, base;     // tiles; base: first tile of sequence b
    int grid, b;

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
    __device__ bool begin(const KvAttend& a) {
        const int lane = threadIdx.x & 31;
        total = 0;
        long long incl = 0;
        for (int b0 = 0; b0 < a.step.B; b0 += 32) {
            incl = warp_scan(sequence_tiles(a, b0 + lane));
            total += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
        grid = (int)min((long long)gridDim.x, total);
        if ((int)blockIdx.x >= grid) return false;
        pos = total * blockIdx.x / grid;
        end = total * (blockIdx.x + 1) / grid;
        base = 0;
        b = 0;
        for (int b0 = 0; b0 < a.step.B; b0 += 32) {          // the sequence that holds tile pos
            const long long mine = a.step.B <= 32 ? 0 : sequence_tiles(a, b0 + lane);
            if (a.step.B > 32) incl = warp_scan(mine);
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
        return true;
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
        r.first = whole ? (int)blockIdx.x : owner(pos - off);
        r.last = whole ? (int)blockIdx.x : owner(pos - off + n - 1);
        pos += r.k1 - r.k0;
        return true;
    }
};

// NaN codes of a step's values are taken as zero by the tensor-core kernels, which would otherwise spread them to rows that do not
// see the token (0 * NaN); rows that do see it get their NaN here.  x: one output of row `token`, element d.
__device__ __noinline__ float kv_with_nan(const KvAttend& a, const KvRun& r, int token, int d, int D, float x) {
    for (int j = 0; j < r.tokens; ++j) {
        if (!kv_sees(a.step, r.b, token, j)) continue;
        const int s = r.len + j, id = max(0, kv_page(a.shape, a.table, r.b, s >> a.shape.page_shift, a.status));
        const uint8_t c = a.vc[(((long long)id * a.shape.kv_heads + r.h) * a.shape.page + (s & (a.shape.page - 1))) * D + d];
        if ((c & 0x7F) == 0x7F) return __int_as_float(0x7FC00000);
    }
    return x;
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

// Four outputs of one row to memory; `factor` normalises.
template <class T>
__device__ __forceinline__ void kv_store4(const KvAttend& a, const KvRun& r, int row, int d, int D, float4 x, bool nan) {
    const int token = (int)a.by_group.div((unsigned)row), hq = r.h * a.group + row - token * a.group;
    if (nan) {
        x.x = kv_with_nan(a, r, token, d, D, x.x); x.y = kv_with_nan(a, r, token, d + 1, D, x.y);
        x.z = kv_with_nan(a, r, token, d + 2, D, x.z); x.w = kv_with_nan(a, r, token, d + 3, D, x.w);
    }
    uint16_t* to = const_cast<uint16_t*>(a.out.data) + r.b * a.out.batch + token * a.out.token + hq * a.out.head + d;
    const uint32_t lo = from_float2<T>(x.x, x.y), hi = from_float2<T>(x.z, x.w);
    if (a.wide_out) *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
    else { to[0] = (uint16_t)lo; to[1] = (uint16_t)(lo >> 16); to[2] = (uint16_t)hi; to[3] = (uint16_t)(hi >> 16); }
}
__device__ __forceinline__ void kv_store_lse(const KvAttend& a, const KvRun& r, int row, float m, float l) {
    if (!a.lse) return;
    const int token = (int)a.by_group.div((unsigned)row), hq = r.h * a.group + row - token * a.group;
    a.lse[((long long)r.b * a.step.T + token) * a.shape.q_heads + hq] = (m + log2f(l)) * kLn2;
}

// Called by all threads of a CTA after they have written their part of a cut row tile (slot: see below): the CTA that arrives last
// joins the parts in the order of the keys.  Slots: 2c for the part with which CTA c begins, 2c + 1 for the one with which it ends
// (a row tile that begins in c).  weights: kRows * grid floats at most are needed in parts; a chunk of pieces at a time is staged.
__device__ __forceinline__ int kv_slot(const KvRun& r, int cta) { return cta == r.first ? 2 * cta + 1 : 2 * cta; }

constexpr int kJoinChunk = 32;           // parts whose weights are staged together

template <int kRows, int D, int kThreadsN, class T>
__device__ void kv_join(const KvAttend& a, const KvRun& r, float* weights /* [kJoinChunk + 2][kRows] shared */, int* word /* shared */) {
    __threadfence();                     // this thread's part of the part is visible before the arrival is
    __syncthreads();
    if (threadIdx.x == 0) {
        const int pieces = r.last - r.first + 1;
        const int before = atomicAdd(a.arrived + r.first, 1);
        *word = before == pieces - 1;
        if (before == pieces - 1) a.arrived[r.first] = 0;    // for the next call
        __threadfence();
    }
    __syncthreads();
    if (!*word) return;
    constexpr int kFloats = kv_part_floats<kRows, D>();
    constexpr int kPer = kRows * D / 4, kMine = (kPer + kThreadsN - 1) / kThreadsN;
    const int rows = min(kRows, r.tokens * a.group - r.rt * kRows);
    float* top = weights + kJoinChunk * kRows;
    float* sum = top + kRows;
    for (int row = threadIdx.x; row < rows; row += kThreadsN) {
        float m = -INFINITY;
        for (int c = r.first; c <= r.last; ++c) m = fmaxf(m, __ldcg(a.parts + (long long)kv_slot(r, c) * kFloats + kRows * D + row));
        m = m == -INFINITY ? 0.f : m;
        top[row] = m;
        sum[row] = 0.f;
    }
    __syncthreads();
    float4 acc[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    bool nan = false;
    for (int c0 = r.first; c0 <= r.last; c0 += kJoinChunk) {
        const int n = min(kJoinChunk, r.last + 1 - c0);
        for (int i = threadIdx.x; i < n * kRows; i += kThreadsN) {
            const int row = i % kRows;
            if (row < rows) weights[i] = exp2f(__ldcg(a.parts + (long long)kv_slot(r, c0 + i / kRows) * kFloats + kRows * D + row) - top[row]);
        }
        __syncthreads();
        for (int row = threadIdx.x; row < rows; row += kThreadsN) {
            float s = sum[row];
            for (int i = 0; i < n; ++i) s += weights[i * kRows + row] * __ldcg(a.parts + (long long)kv_slot(r, c0 + i) * kFloats + kRows * D + kRows + row);
            sum[row] = s;
        }
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const float* part = a.parts + (long long)kv_slot(r, c0 + i) * kFloats;
            nan = nan || __ldcg(reinterpret_cast<const int*>(part) + kRows * D + 2 * kRows) != 0;
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int at = (int)threadIdx.x + k * kThreadsN, row = at / (D / 4);
                if (row >= rows) continue;
                const float4 x = __ldcg(reinterpret_cast<const float4*>(part) + at);
                const float w = weights[i * kRows + row];
                acc[k].x += w * x.x; acc[k].y += w * x.y; acc[k].z += w * x.z; acc[k].w += w * x.w;
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int at = (int)threadIdx.x + k * kThreadsN, row = at / (D / 4), d = at % (D / 4) * 4;
        if (row >= rows) continue;
        const float f = 1.f / sum[row];
        kv_store4<T>(a, r, r.rt * kRows + row, d, D, make_float4(acc[k].x * f, acc[k].y * f, acc[k].z * f, acc[k].w * f), nan);
    }
    for (int row = threadIdx.x; row < rows; row += kThreadsN) kv_store_lse(a, r, r.rt * kRows + row, top[row], sum[row]);
    __syncthreads();
}

}  // namespace ot
