// The accepted path's cache entries moved to the end of the prefix: slot len + gather[j] -> slot len + j, for all layers.
//
// A page that takes entries of pages with larger scales is brought to the largest of them first (a power of two: exact but for
// entries that become subnormal).  gather ascends, so entry j comes from slot len + j or later: pages are done in order, and within a
// page the rows in order, each group of rows read before it is written; nothing that is still to be read is overwritten.
//
// A few kilobytes per sequence and layer: the chain of dependent loads (length, kept entries, page table, scales, entries) is what
// costs.  One CTA looks a sequence's indices up once for a layer and its warps share them, a warp per head and side.
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
    __shared__ int bad;
    const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int len = a.kv_len[b], keep = a.keep[b], shift = a.shape.page_shift, page = a.shape.page;
    const long long slots = (long long)a.shape.max_pages << shift;
    if (tid == 0) bad = keep < 0 || keep > a.G || len < 0 || (long long)len + keep > slots;
    __syncthreads();
    if (!bad) {
        for (int j = tid; j < keep; j += kCompactThreads) {
            const int g = a.gather[(long long)b * a.G + j];
            const int before = j ? a.gather[(long long)b * a.G + j - 1] : -1;
            if (g <= before || (long long)len + g >= slots) { bad = 1; continue; }
            const int id = kv_page(a.shape, a.table, b, (len + g) >> shift, a.status);
            if (id < 0) bad = 1;
            src_page[j] = id;
            src_row[j] = (short)((len + g) & (page - 1));
        }
    }
    __syncthreads();
    if (bad) {                           // the sequence stays as it is
        if (tid == 0) {
            set_status(a.status, kErrInternal);
            if (layer == 0 && a.new_len) a.new_len[b] = len;
        }
        return;
    }
    if (layer == 0 && tid == 0 && a.new_len) a.new_len[b] = len + keep;
    if (keep == 0) return;
    constexpr int kLanes = D / 16, kRows = 32 / kLanes;      // 16 bytes a lane
    const int sub = lane & (kLanes - 1), mine = lane / kLanes;
    const int first = len >> shift, last = (len + keep - 1) >> shift;
    for (int item = warp; item < 2 * a.shape.kv_heads; item += kCompactThreads / 32) {
        const int h = item >> 1;
        const long long heads = (long long)layer * a.shape.num_pages * a.shape.kv_heads + h;
        uint8_t* codes = (item & 1 ? a.vc : a.kc);
        float* scales = (item & 1 ? a.vs : a.ks);
        for (int p = first; p <= last; ++p) {
            const int start = p << shift;
            const int j0 = max(len, start) - len, j1 = min(len + keep, start + page) - len;
            const int id = kv_page(a.shape, a.table, b, p, a.status);
            if (id < 0) continue;
            const long long to = heads + (long long)id * a.shape.kv_heads;
            const float was = scales[to];
            float now = was;
            for (int j = j0 + lane; j < j1; j += 32) now = fmaxf(now, scales[heads + (long long)src_page[j] * a.shape.kv_heads]);
            now = warp_max_f32(now);
            const float inv = 1.f / now;
            uint8_t* rows = codes + to * page * D;
            for (int j = j0; j < j1; j += kRows) {
                const int jj = j + mine;
                const bool on = jj < j1 && !(src_page[jj] == id && src_row[jj] == len + jj - start && now == was);
                uint4 v = make_uint4(0, 0, 0, 0);
                if (on) {
                    const long long from = heads + (long long)src_page[jj] * a.shape.kv_heads;
                    v = *reinterpret_cast<const uint4*>(codes + (from * page + src_row[jj]) * D + sub * 16);
                    const float s = scales[from];
                    if (s != now) v = recode16(v, s * inv);
                }
                __syncwarp();
                if (on) *reinterpret_cast<uint4*>(rows + (long long)(len + jj - start) * D + sub * 16) = v;
                __syncwarp();
            }
            if (now != was) {            // the page's other rows
                for (int r = mine; r < page; r += kRows) {
                    const int j = start + r - len;
                    if (j >= j0 && j < j1) continue;
                    uint4* at = reinterpret_cast<uint4*>(rows + (long long)r * D + sub * 16);
                    *at = recode16(*at, was * inv);
                }
                if (lane == 0) scales[to] = now;
            }
            __syncwarp();
        }
    }
}

}  // namespace ot
