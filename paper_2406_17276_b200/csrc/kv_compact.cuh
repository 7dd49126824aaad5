// The accepted path's cache entries moved to the end of the prefix: slot len + gather[j] -> slot len + j, for all layers.
//
// A page that takes entries of pages with larger scales is brought to the largest of them first (a power of two: exact but for
// entries that become subnormal).  gather ascends, so entry j comes from slot len + j or later: pages are done in order, and within a
// page the rows in order, each group of rows read before it is written; nothing that is still to be read is overwritten.
//
// A few kilobytes per sequence and layer: the chain of dependent loads (lengths and kept entries, page table, scales, entries) is what
// costs.  One CTA looks a sequence's indices up once for a layer, what does not depend on one another together, and its warps share them,
// a warp per head with keys and values side by side.

#pragma once

#include "kv_common.cuh"

namespace ot {

constexpr int kCompactThreads = 256;
constexpr int kCompactMost = 1024;       // entries kept per sequence

struct KvCompact {
    KvShape shape;
    uint8_t *kc, *vc;                    // [layers][num_pages][kv_heads][page][D]
    float *ks, *vs;
    const int32_t *table, *kv_len, *gather, *keep;
    int G;
    int32_t* new_len;
    int* status;
};

template <int D>
__global__ void __launch_bounds__(kCompactThreads) kv_compact_kernel(const __grid_constant__ KvCompact a) {
    grid_dependency_wait();
    __shared__ int src_page[kCompactMost];
    __shared__ short src_row[kCompactMost];
    __shared__ int dst_page[kCompactMost / 16 + 1];          // pages of 16 slots at least
    const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int shift = a.shape.page_shift, page = a.shape.page;
    const long long slots = (long long)a.shape.max_pages << shift;
    const int32_t* gather = a.gather + (long long)b * a.G;
    // this thread's first entry, before it is known whether it is kept
    int g = tid < a.G ? gather[tid] : 0, before = tid > 0 && tid < a.G ? gather[tid - 1] : -1;
    const int len = a.kv_len[b], keep = a.keep[b];
    bool bad = keep < 0 || keep > a.G || len < 0 || (long long)len + keep > slots;
    const int first = len >> shift, last = (len + keep - 1) >> shift;
    if (!bad && keep > 0) {
        for (int p = first + tid; p <= last; p += kCompactThreads) dst_page[p - first] = kv_page(a.shape, a.table, b, p, a.status);
        for (int j = tid; j < keep; j += kCompactThreads) {
            if (j != tid) { g = gather[j]; before = gather[j - 1]; }
            if (g <= before || (long long)len + g >= slots) { bad = true; continue; }
            const int id = kv_page(a.shape, a.table, b, (len + g) >> shift, a.status);
            bad = bad || id < 0;
            src_page[j] = id;
            src_row[j] = (short)((len + g) & (page - 1));
        }
    }
    bad = __syncthreads_or(bad);
    if (layer == 0 && tid == 0 && a.new_len) a.new_len[b] = bad ? len : len + keep;
    if (bad && tid == 0) set_status(a.status, kErrInternal);               // the sequence stays as it is
    if (bad || keep == 0) return;
    constexpr int kLanes = D / 16, kRows = 32 / kLanes;      // 16 bytes a lane
    const int sub = lane & (kLanes - 1), mine = lane / kLanes;
    uint8_t* const codes[2] = {a.kc, a.vc};
    float* const scales[2] = {a.ks, a.vs};
    for (int h = warp; h < a.shape.kv_heads; h += kCompactThreads / 32) {
        const long long heads = (long long)layer * a.shape.num_pages * a.shape.kv_heads + h;
        for (int p = first; p <= last; ++p) {
            const int start = p << shift, id = dst_page[p - first];
            const int j0 = max(len, start) - len, j1 = min(len + keep, start + page) - len;
            if (id < 0) continue;
            const long long to = heads + (long long)id * a.shape.kv_heads;
            float was[2], now[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) now[s] = was[s] = scales[s][to];
            for (int j = j0 + lane; j < j1; j += 32) {
                const long long from = heads + (long long)src_page[j] * a.shape.kv_heads;
#pragma unroll
                for (int s = 0; s < 2; ++s) now[s] = fmaxf(now[s], scales[s][from]);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) now[s] = warp_max_f32(now[s]);
            for (int j = j0; j < j1; j += kRows) {
                const int jj = j + mine;
                uint4 v[2];
                bool on[2];
                long long from = 0;
                if (jj < j1) from = heads + (long long)src_page[jj] * a.shape.kv_heads;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    on[s] = jj < j1 && !(src_page[jj] == id && src_row[jj] == len + jj - start && now[s] == was[s]);
                    if (on[s]) v[s] = *reinterpret_cast<const uint4*>(codes[s] + (from * page + src_row[jj]) * D + sub * 16);
                }
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (on[s]) {
                        const float own = scales[s][from];
                        if (own != now[s]) v[s] = recode16(v[s], own / now[s]);
                    }
                __syncwarp();                                // the group's rows are read before any is written
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (on[s]) *reinterpret_cast<uint4*>(codes[s] + (to * page + len + jj - start) * D + sub * 16) = v[s];
                __syncwarp();
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (now[s] == was[s]) continue;              // the same for the whole warp
                for (int r = mine; r < page; r += kRows) {   // the page's other rows
                    const int j = start + r - len;
                    if (j >= j0 && j < j1) continue;
                    uint4* at = reinterpret_cast<uint4*>(codes[s] + (to * page + r) * D + sub * 16);
                    *at = recode16(*at, was[s] / now[s]);
                }
                if (lane == 0) scales[s][to] = now[s];
            }
            __syncwarp();
        }
    }
}

}  // namespace ot
