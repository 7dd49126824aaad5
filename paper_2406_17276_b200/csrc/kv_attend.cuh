// Attention of a step's tokens over the paged 8-bit cache: what its kernels share.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(x_ij - m_i) / l_i,  x_ij = scale * q_i . k_j   over the slots j that token i sees
//
// All query rows of a sequence that read one key head (tokens x query heads per key head, token-major) are taken together, so that
// a page is read and converted once for them.  Work is cut by the clock and not by sequence: the tiles (sequence, key head, row
// tile, tile of keys) are numbered in that order and every CTA takes an equal run of them, whatever the lengths; a row tile that is cut
// leaves its parts (maximum, sum, output) in the workspace.  Few rows: the CTA that finishes last joins them; many rows: a kernel of its own does.
// Either joins them in the order of the keys, so results do not depend on who finishes when.
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
    struct KvRun* cuts;                  // [grid]: the cut row tile that began in each CTA, or b < 0
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

// Walks the run of tiles of one CTA of a grid.  kRows rows and kKeys keys a tile.  kHalves: a row tile of at most kRows / 2 rows costs half
// of the others.  A run is an equal share of the cost; a key tile belongs to the CTA in whose share it begins (shares are no smaller than a
// tile, so none is empty).  Every warp keeps its own copy (no shared memory, no barrier); the lengths come from the cache after the
// first warp.
template <int kRows, int kKeys, bool kHalves>
struct KvWalk {
    static constexpr int kMost = kHalves ? 2 : 1;            // cost of a key tile of a full row tile
    static constexpr int kAhead = 4;                         // groups of 32 sequences whose lengths are loaded together
    // Cost of everything, share of each CTA (and what is left over), next, end of the share; base: where sequence b begins.  The host has
    // seen to it that costs fit (see kv_cost_bound); with 32 bits there are no long divisions.
    unsigned total, share, left, pos, end, base;
    int cta, grid, b;

    __device__ __forceinline__ static int row_tiles(const KvAttend& a, int tokens) { return (tokens * a.group + kRows - 1) / kRows; }
    __device__ __forceinline__ static int cost_of(const KvAttend& a, int tokens, int rt) {
        return kHalves && tokens * a.group - rt * kRows > kRows / 2 ? 2 : 1;
    }
    // In a chain a row tile sees no further than its last token.
    __device__ __forceinline__ static int keys_of(const KvAttend& a, int len, int tokens, int rt) {
        if (a.step.mask) return len + tokens;
        const int last = (int)a.by_group.div((unsigned)(rt + 1) * kRows - 1u);
        return len + min(tokens, last + 1);
    }
    __device__ __forceinline__ static int tiles_of(const KvAttend& a, int len, int tokens, int rt) { return (keys_of(a, len, tokens, rt) + kKeys - 1) / kKeys; }
    // Cost of one key head of a sequence.
    __device__ __forceinline__ static unsigned head_cost(const KvAttend& a, int len, int tokens) {
        const int n = row_tiles(a, tokens);
        if (n == 0) return 0;
        if (a.step.mask || n == 1) return (unsigned)tiles_of(a, len, tokens, 0) * (kMost * (n - 1) + cost_of(a, tokens, n - 1));
        unsigned s = 0;
#pragma unroll 1
        for (int rt = 0; rt < n; ++rt) s += tiles_of(a, len, tokens, rt) * cost_of(a, tokens, rt);
        return s;
    }
    __device__ __forceinline__ static unsigned sequence_cost(const KvAttend& a, int b) {
        int len, tokens;
        if (b >= a.step.B || !kv_sequence(a.shape, a.step, b, len, tokens, a.status)) return 0;
        return head_cost(a, len, tokens) * a.shape.kv_heads;
    }
    __device__ __forceinline__ static unsigned warp_scan(unsigned v) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned u = __shfl_up_sync(0xFFFFFFFFu, v, o);
            if (lane >= o) v += u;
        }
        return v;
    }
    __device__ __forceinline__ unsigned begins(int c) const { return share * c + min((unsigned)c, left); }        // the first `left` CTAs have one more
    // false: nothing for this CTA.
    __device__ __forceinline__ bool begin(const KvAttend& a, int which, int ctas) {
        unsigned incl[kAhead];
        total = 0;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) incl[k] = k * 32 < a.step.B ? sequence_cost(a, k * 32 + (threadIdx.x & 31)) : 0u;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (k * 32 >= a.step.B) break;
            incl[k] = warp_scan(incl[k]);
            total += __shfl_sync(0xFFFFFFFFu, incl[k], 31);
        }
#pragma unroll 1
        for (int b0 = kAhead * 32; b0 < a.step.B; b0 += 32) total += __shfl_sync(0xFFFFFFFFu, warp_scan(sequence_cost(a, b0 + (threadIdx.x & 31))), 31);
        cta = which;
        grid = min(ctas, (int)((total + kMost - 1) / kMost));
        if (cta >= grid) return false;
        share = total / grid;
        if (kMost > 1 && grid > 1 && share < kMost) share = total / --grid;
        if (cta >= grid) return false;
        left = total - share * grid;
        pos = begins(cta);
        end = begins(cta + 1);
        // the sequence that holds pos
        base = 0;
        b = 0;
        bool found = false;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (!found && k * 32 < a.step.B) found = within(incl[k], k * 32);
#pragma unroll 1
        for (int b0 = kAhead * 32; !found && b0 < a.step.B; b0 += 32) found = within(warp_scan(sequence_cost(a, b0 + (threadIdx.x & 31))), b0);
        return true;
    }
    __device__ __forceinline__ bool within(unsigned incl, int b0) {
        const unsigned over = __ballot_sync(0xFFFFFFFFu, base + incl > pos);
        if (over) {
            const int l = __ffs(over) - 1;
            const unsigned before = __shfl_sync(0xFFFFFFFFu, incl, l > 0 ? l - 1 : 0);
            b = b0 + l;
            base += l > 0 ? before : 0;
            return true;
        }
        base += __shfl_sync(0xFFFFFFFFu, incl, 31);
        return false;
    }
    // The CTA in whose share `at` lies.
    __device__ __forceinline__ int owner(unsigned at) const {
        const unsigned more = left * (share + 1);
        return at < more ? (int)(at / (share + 1)) : (int)(left + (at - more) / share);
    }
    // The row tile that holds pos: its run but for [k0, k1), its cost, its key tiles, and where it begins.
    __device__ __forceinline__ bool row_tile(const KvAttend& a, KvRun& r, int& cost, int& n, unsigned& from) {
        int len, tokens;
        unsigned per_head;
#pragma unroll 1
        for (;; ++b) {
            if (b >= a.step.B) return false;                 // (pos is the end of everything)
            per_head = kv_sequence(a.shape, a.step, b, len, tokens, a.status) ? head_cost(a, len, tokens) : 0;
            if (pos < base + per_head * a.shape.kv_heads) break;
            base += per_head * a.shape.kv_heads;
        }
        unsigned off = pos - base;
        r.h = (int)(off / per_head);
        off -= r.h * per_head;
        r.rt = 0;
        n = tiles_of(a, len, tokens, 0);
        if (a.step.mask) {
            r.rt = min((int)(off / (unsigned)(kMost * n)), row_tiles(a, tokens) - 1);
            off -= (unsigned)r.rt * (kMost * n);
            cost = cost_of(a, tokens, r.rt);
        } else {
#pragma unroll 1
            for (cost = cost_of(a, tokens, 0); off >= (unsigned)(n * cost); cost = cost_of(a, tokens, r.rt)) {
                off -= n * cost;
                n = tiles_of(a, len, tokens, ++r.rt);
            }
        }
        from = pos - off;
        r.b = b; r.len = len; r.tokens = tokens;
        r.keys = keys_of(a, len, tokens, r.rt);
        const unsigned last = from + (n - 1) * cost;
        r.first = from >= begins(cta) ? cta : owner(from);
        r.last = last < end ? cta : owner(last);
        return true;
    }
    // The next run; false at the end.
    __device__ __forceinline__ bool next(const KvAttend& a, KvRun& r) {
#pragma unroll 1
        while (pos < end) {
            int cost, n;
            unsigned from;
            if (!row_tile(a, r, cost, n, from)) return false;
            r.k0 = kHalves && cost == 2 ? (int)(pos - from + 1) >> 1 : (int)(pos - from);
            r.k1 = min(n, kHalves && cost == 2 ? (int)(end - from + 1) >> 1 : (int)(end - from));
            pos = from + n * cost;
            if (r.k0 < r.k1) return true;
        }
        return false;
    }
};
// What a call's costs stay below; the host refuses calls for which this does not fit in 31 bits.
inline long long kv_cost_bound(const KvShape& s, int B, int T, int rows, int keys) {
    const long long tiles = (((long long)s.max_pages << s.page_shift) + keys - 1) / keys, row_tiles = ((long long)T * (s.q_heads / s.kv_heads) + rows - 1) / rows;
    return 2 * B * s.kv_heads * tiles * row_tiles;
}

// NaN codes of a step's values are taken as zero by the tensor-core kernels, which would otherwise spread them to rows that do not
// see the token (0 * NaN); outputs that do see one are made NaN here, after they have been stored: elements [d, d + n) of query row
// `row`.
template <int D, class T>
__device__ __forceinline__ void kv_mark_nan(const KvAttend& a, const KvRun& r, int row, int d, int n) {
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

// A cut row tile's part: kRows x D outputs over the part's keys alone (divided by its sum, so that large values stay within single precision however
// many keys there are), then maxima, sums and a word that says whether NaN values were met.  Outputs lie in chunks of four elements, [D / 4][kRows][4], so that threads with a row each write and read whole
// lines (row after row, each store of a warp touched 32 lines, and writing a tile's part took as long as four key tiles).
template <int kRows, int D> __host__ __device__ constexpr int kv_part_floats() { return kRows * D + 2 * kRows + 4; }

template <int D, class T>
__device__ __noinline__ void kv_mark_nan_call(const KvAttend& a, const KvRun& r, int row, int d, int n) { kv_mark_nan<D, T>(a, r, row, d, n); }
// A row's outputs at elements [d, d + N) of query row `row` of the run (row tile included).  kCalls: the kernel may call functions.
template <int D, int N, class T, bool kCalls = true>
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
    if (nan) {
        if (kCalls) kv_mark_nan_call<D, T>(a, r, row, d, N);
        else kv_mark_nan<D, T>(a, r, row, d, N);
    }
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
// Joins a cut row tile's parts in the order of the keys: a lane a row, a chunk of four elements at a time.  kStep: parts from one slot to
// the next.  row0: the tile's first row.  Of the tile's groups of rows times chunks this warp does warp, warp + warps, ...  kAtOnce: parts in flight.
template <int kRows, int D, class T, int kAtOnce>
__device__ __forceinline__ void kv_join_by(const KvAttend& a, const KvRun& r, const float* parts, int kStep, int row0, int rows, int warp, int warps) {
    constexpr int kFloats = kv_part_floats<kRows, D>(), kChunks = D / 4;
    constexpr int kLaneRows = kRows < 32 ? kRows : 32, kLaneChunks = 32 / kLaneRows;
    const int lane = threadIdx.x & 31, pieces = r.last - r.first + 1;
    const long long step = (long long)kStep * kFloats;
    auto part = [&](int i) { return parts + kv_slot(r, r.first + min(i, pieces - 1)) * step; };
    int seen = 0;
    for (int i = lane; i < pieces; i += 32) seen |= reinterpret_cast<const int*>(part(i))[kRows * D + 2 * kRows];
    const bool nan = __any_sync(0xFFFFFFFFu, seen != 0);
    constexpr int kItems = (kRows / kLaneRows) * (kChunks / kLaneChunks);
#pragma unroll 1
    for (int item = warp; item < kItems; item += warps) {
        const int row = item / (kChunks / kLaneChunks) * kLaneRows + lane % kLaneRows, chunk = item % (kChunks / kLaneChunks) * kLaneChunks + lane / kLaneRows;
        if (item / (kChunks / kLaneChunks) * kLaneRows >= rows) break;
        float top = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int i = 0; i < pieces; i += kAtOnce) {
            float m[kAtOnce], s[kAtOnce];
            float4 y[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {                        // (parts behind the last are read again, with weight 0)
                const float* at = part(i + k);
                m[k] = at[kRows * D + row];
                s[k] = at[kRows * D + kRows + row];
                y[k] = *reinterpret_cast<const float4*>(at + (chunk * kRows + row) * 4);
            }
            const float was = top;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, m[k]);
            const float bottom = top == -INFINITY ? 0.f : top, before = l * ex2_approx(was - bottom);
            l = before;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                s[k] = i + k < pieces ? s[k] * ex2_approx(m[k] - bottom) : 0.f;
                l += s[k];
            }
            const float over = l == 0.f ? 0.f : 1.f / l, keep = before * over;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] *= keep;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (i + k < pieces) {
                    const float f = s[k] * over;
                    x[0] += f * y[k].x; x[1] += f * y[k].y; x[2] += f * y[k].z; x[3] += f * y[k].w;
                }
        }
        if (top == -INFINITY) top = 0.f;
        if (row < rows) {
            kv_store<D, 4, T>(a, r, row0 + row, chunk * 4, x, nan);
            if (chunk == 0) kv_store_lse(a, r, row0 + row, top, l);
        }
    }
}

// (Two parts are the rule where there is much to do, many where there is little.)
template <int kRows, int D, class T>
__device__ __forceinline__ void kv_join(const KvAttend& a, const KvRun& r, const float* parts, int kStep, int row0, int rows, int warp, int warps) {
    if (r.last - r.first < 2) kv_join_by<kRows, D, T, 2>(a, r, parts, kStep, row0, rows, warp, warps);
    else kv_join_by<kRows, D, T, kRows < 32 ? 16 : 8>(a, r, parts, kStep, row0, rows, warp, warps);
}

}  // namespace ot
