// Host side of the cache operators (include/opt_tree.h: opt_tree_kv_*).
#include <cstring>
#include <new>

#include "../../include/opt_tree.h"
#include "kv_append.cuh"
#include "kv_attend_few.cuh"
#include "kv_attend_tiles.cuh"
#include "kv_compact.cuh"
#include "launch.cuh"

struct opt_tree_kv {
    opt_tree_kv_config cfg;
    ot::KvShape shape;
    void* base;                          // status word, arrival counters, parts
    int* status;
    int* arrived;
    ot::KvRun* cuts;
    float* parts;
    int device, sms;
    int64_t launches;
};

namespace {

bool valid_cfg(const opt_tree_kv_config* c) {
    return c && c->q_heads >= 1 && c->kv_heads >= 1 && c->head_dim >= 1 && c->page >= 1 && c->num_pages >= 1 && c->max_pages >= 1 &&
           c->max_batch >= 1 && c->max_step >= 1 && c->layers >= 1 && c->q_heads % c->kv_heads == 0 &&
           (c->dtype == OPT_TREE_BF16 || c->dtype == OPT_TREE_FP16);
}
bool supported_cfg(const opt_tree_kv_config* c) {
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return false;
    if (c->max_batch > 32767 || c->layers > 32767 || c->q_heads > 32767) return false;
    if ((long long)c->max_pages * c->page > 1ll << 30 || c->max_step > 1 << 30) return false;         // slots of a sequence, of which a step's tokens take some
    if ((long long)c->max_batch * c->max_step * c->q_heads > 0x7FFFFFFFll - 512) return false;         // rows of a step, with a tile's padding
    const long long touched = (c->max_step + c->page - 2) / c->page + 1;
    if ((long long)c->max_batch * touched * c->kv_heads * 2 > 0x3FFFFFFFll) return false;              // CTAs of an append
    return true;
}
int check_launch() { return cudaGetLastError() == cudaSuccess ? OPT_TREE_OK : OPT_TREE_ERR_CUDA; }
bool on_device(const opt_tree_kv* kv) {
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == kv->device;
}
// Whether an address is off a boundary (loads from there would fault).
bool off(const void* p, uintptr_t boundary) { return (reinterpret_cast<uintptr_t>(p) & (boundary - 1)) != 0; }
bool bad_cache(const opt_tree_kv_cache* c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->block_table) return true;
    return off(c->k, 16) || off(c->v, 16) || off(c->k_scale, 4) || off(c->v_scale, 4) || off(c->block_table, 4);
}
bool bad_step(const opt_tree_kv* kv, const opt_tree_kv_step* s) {
    return !s || s->B < 1 || s->B > kv->cfg.max_batch || s->T < 1 || s->T > kv->cfg.max_step || !s->kv_len || off(s->kv_len, 4) || off(s->nodes, 4) ||
           off(s->base_pos, 4) || off(s->position_ids, 4) || off(s->mask, 8);
}
ot::KvStep step_of(const opt_tree_kv_step* s) { return ot::KvStep{s->B, s->T, s->kv_len, s->nodes, s->base_pos, s->position_ids, s->mask}; }
ot::KvRows rows_of(const opt_tree_kv_rows* r) {
    return ot::KvRows{static_cast<const uint16_t*>(r->data), (long long)r->batch, (long long)r->token, (long long)r->head};
}
bool bad_rows(const opt_tree_kv_rows* r) { return !r || !r->data || off(r->data, 2); }
bool overlap(const int32_t* a, size_t n, const int32_t* b, size_t m) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + m * sizeof(int32_t) && y < x + n * sizeof(int32_t);
}
int wide(const opt_tree_kv_rows* r) {
    return ((reinterpret_cast<uintptr_t>(r->data) & 15u) == 0 && r->batch % 8 == 0 && r->token % 8 == 0 && r->head % 8 == 0) ? 1 : 0;
}

using AppendKernel = void (*)(ot::KvAppend);
// A CTA takes a page of one head and side: rows of head_dim / 8 lanes, so page * head_dim / 8 lanes in all, in at most four passes.
template <int D, class T> AppendKernel append_variant(int page, int* threads) {
    switch (page * D) {
        case 1024: *threads = 128; return ot::kv_append_kernel<D, T, 128, 1>;
        case 2048: *threads = 256; return ot::kv_append_kernel<D, T, 256, 1>;
        case 4096: *threads = 256; return ot::kv_append_kernel<D, T, 256, 2>;
        case 8192: *threads = 256; return ot::kv_append_kernel<D, T, 256, 4>;
        default: *threads = 512; return ot::kv_append_kernel<D, T, 512, 4>;
    }
}

using AttendKernel = void (*)(ot::KvAttend);
using JoinKernel = void (*)(ot::KvAttend);
struct AttendVariant { AttendKernel kernel; size_t smem; int per_sm, threads, rows, keys; JoinKernel join; };
template <int D, int NT, class T> AttendVariant few_variant() {
    using L = ot::FewLayout<D, NT>;
    return AttendVariant{ot::kv_attend_few_kernel<D, NT, T>, (size_t)L::kBytes, L::kPerSm, L::kThreads, L::kRows, L::kKeys, nullptr};
}
template <int D, class T> AttendVariant attend_variant(int rows, bool brief) {
    if (rows <= 8) return few_variant<D, 1, T>();
    if (rows <= 16 || (brief && rows <= 64)) return few_variant<D, 2, T>();
    return AttendVariant{ot::kv_attend_tiles_kernel<D, T>, (size_t)ot::TileLayout<D>::kBytes, 1, ot::kTileThreads, 2 * ot::kTileRows, ot::kTileKeys,
                         ot::kv_join_kernel<D, T>};
}
// The kernel for `rows` query rows per sequence and key head at most.  brief: with 16 rows at a time an SM has no more than two key tiles
// to do even if every page is full; up to 64 rows that is quicker than the tensor cores' tiles, which take longer to start (16.4 us
// against 20.7 for 44 rows over 900 slots, 8 key heads; over 8000 slots 35.6 against 31.3).  It goes by what a block table can hold, since only the
// device knows the lengths: short contexts under wide tables take the tiles (the same 44 rows: 16.4 us under a table of 57 pages of 16, 20.9 under one
// of 256).
AttendVariant attend_for(const opt_tree_kv_config& c, int rows, bool brief) {
    const bool bf16 = c.dtype == OPT_TREE_BF16;
    if (c.head_dim == 64) return bf16 ? attend_variant<64, __nv_bfloat16>(rows, brief) : attend_variant<64, __half>(rows, brief);
    return bf16 ? attend_variant<128, __nv_bfloat16>(rows, brief) : attend_variant<128, __half>(rows, brief);
}
const int kVariantRows[] = {1, 16, 17};  // one row count for each variant
constexpr size_t kMaxTiles = 2;          // CTAs of an SM, and row tiles of a CTA, at most

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
// Bytes of the two parts that each CTA may leave of cut row tiles, per SM: two CTAs with 16 rows each, or one with two tiles of 128.
template <int D> size_t part_bytes(long long rows) {
    const size_t few = (size_t)2 * 2 * ot::kv_part_floats<16, D>() * sizeof(float), tiles = (size_t)2 * 2 * ot::kv_part_floats<ot::kTileRows, D>() * sizeof(float);
    return rows <= 16 ? few : tiles;
}
size_t parts_per_sm(const opt_tree_kv_config& c) {
    const long long rows = (long long)c.max_step * (c.q_heads / c.kv_heads);
    return c.head_dim == 64 ? part_bytes<64>(rows) : part_bytes<128>(rows);
}

}  // namespace

extern "C" {

size_t opt_tree_kv_workspace_bytes(const opt_tree_kv_config* cfg) {
    if (!valid_cfg(cfg) || !supported_cfg(cfg)) return 0;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        sms = 148;                                   // no device here: the size on a B200
    }
    return 256 + align256(sms * kMaxTiles * sizeof(int)) + align256(sms * sizeof(ot::KvRun)) + sms * parts_per_sm(*cfg);
}

int opt_tree_kv_create(opt_tree_kv** out, const opt_tree_kv_config* cfg) {
    if (!out) return OPT_TREE_ERR_INVALID_ARG;
    *out = nullptr;
    if (!valid_cfg(cfg)) return OPT_TREE_ERR_INVALID_ARG;
    if (!supported_cfg(cfg)) return OPT_TREE_ERR_UNSUPPORTED;
    opt_tree_kv* kv = new (std::nothrow) opt_tree_kv();
    if (!kv) return OPT_TREE_ERR_CUDA;
    kv->cfg = *cfg;
    int shift = 0;
    while ((1 << shift) < cfg->page) ++shift;
    kv->shape = ot::KvShape{cfg->q_heads, cfg->kv_heads, cfg->page, cfg->num_pages, cfg->max_pages, shift};
    const size_t bytes = opt_tree_kv_workspace_bytes(cfg);
    if (cudaGetDevice(&kv->device) != cudaSuccess || cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, kv->device) != cudaSuccess ||
        cudaMalloc(&kv->base, bytes) != cudaSuccess) {
        cudaGetLastError();
        delete kv;
        return OPT_TREE_ERR_CUDA;
    }
    // (calls may come on streams that do not wait for the one that clears the workspace)
    if (cudaMemset(kv->base, 0, bytes) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        cudaFree(kv->base);
        delete kv;
        return OPT_TREE_ERR_CUDA;
    }
    for (int rows : kVariantRows) {
        const AttendVariant v = attend_for(*cfg, rows, false);
        cudaFuncAttributes got;
        if (cudaFuncGetAttributes(&got, v.kernel) != cudaSuccess || (v.join && got.numRegs != ot::kRegsLaunch) || cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)v.smem) != cudaSuccess) {
            cudaGetLastError();
            cudaFree(kv->base);
            delete kv;
            return OPT_TREE_ERR_CUDA;
        }
    }
    char* at = static_cast<char*>(kv->base);
    kv->status = reinterpret_cast<int*>(at);
    kv->arrived = reinterpret_cast<int*>(at + 256);
    at += 256 + align256(kv->sms * kMaxTiles * sizeof(int));
    kv->cuts = reinterpret_cast<ot::KvRun*>(at);
    kv->parts = reinterpret_cast<float*>(at + align256(kv->sms * sizeof(ot::KvRun)));
    *out = kv;
    return OPT_TREE_OK;
}

int opt_tree_kv_destroy(opt_tree_kv* kv) {
    if (!kv) return OPT_TREE_ERR_INVALID_ARG;
    const cudaError_t e = cudaFree(kv->base);
    delete kv;
    return e == cudaSuccess ? OPT_TREE_OK : OPT_TREE_ERR_CUDA;
}

int opt_tree_kv_append(opt_tree_kv* kv, const opt_tree_kv_cache* cache, int32_t layer, const opt_tree_kv_rows* q, const opt_tree_kv_rows* k,
                       const opt_tree_kv_rows* v, const opt_tree_kv_rows* q_out, const opt_tree_kv_step* step, const opt_tree_kv_turn* turn,
                       void* stream) {
    if (!kv || bad_cache(cache) || layer < 0 || layer >= kv->cfg.layers || bad_rows(k) || bad_rows(v) || bad_step(kv, step)) return OPT_TREE_ERR_INVALID_ARG;
    if ((q != nullptr) != (q_out != nullptr) || (q && (bad_rows(q) || bad_rows(q_out)))) return OPT_TREE_ERR_INVALID_ARG;
    opt_tree_kv_turn none;
    memset(&none, 0, sizeof none);
    if (!turn) turn = &none;
    const int D = kv->cfg.head_dim;
    if (turn->rot_dim < 0 || turn->rot_dim > D || turn->rot_dim % 16 || (turn->rot_dim && (!turn->cos_sin || turn->positions < 1)) ||
        ((turn->q_norm || turn->k_norm) && !(turn->eps >= 0.f)) || off(turn->cos_sin, 4) || off(turn->q_norm, 2) || off(turn->k_norm, 2))
        return OPT_TREE_ERR_INVALID_ARG;
    if (!on_device(kv)) return OPT_TREE_ERR_INVALID_ARG;
    ot::KvAppend a;
    memset(&a, 0, sizeof a);
    a.shape = kv->shape;
    a.step = step_of(step);
    a.k = rows_of(k); a.v = rows_of(v);
    a.wide_k = wide(k); a.wide_v = wide(v);
    if (q) { a.q = rows_of(q); a.q_out = rows_of(q_out); a.wide_q = wide(q); a.wide_out = wide(q_out); }
    const long long layer_pages = (long long)layer * kv->cfg.num_pages * kv->cfg.kv_heads;
    a.kc = cache->k + layer_pages * kv->cfg.page * D; a.vc = cache->v + layer_pages * kv->cfg.page * D;
    a.ks = cache->k_scale + layer_pages; a.vs = cache->v_scale + layer_pages;
    a.table = cache->block_table;
    a.cos_sin = turn->cos_sin; a.positions = turn->positions; a.rot_dim = turn->rot_dim; a.interleaved = turn->interleaved ? 1 : 0;
    a.q_norm = static_cast<const uint16_t*>(turn->q_norm); a.k_norm = static_cast<const uint16_t*>(turn->k_norm);
    a.eps = turn->eps;
    a.wide_cs = (reinterpret_cast<uintptr_t>(turn->cos_sin) & 15u) == 0;
    a.wide_w = ((reinterpret_cast<uintptr_t>(turn->q_norm) | reinterpret_cast<uintptr_t>(turn->k_norm)) & 15u) == 0;
    a.page_slots = (step->T + kv->cfg.page - 2) / kv->cfg.page + 1;
    a.page_blocks = step->B * a.page_slots * kv->cfg.kv_heads * 2;
    a.by_heads = ot::FixedDiv::by((unsigned)kv->cfg.kv_heads); a.by_slots = ot::FixedDiv::by((unsigned)a.page_slots);
    a.by_T = ot::FixedDiv::by((unsigned)step->T);
    a.status = kv->status;
    int threads = 0;
    const bool bf16 = kv->cfg.dtype == OPT_TREE_BF16;
    const AppendKernel kernel = D == 64 ? (bf16 ? append_variant<64, __nv_bfloat16>(kv->cfg.page, &threads) : append_variant<64, __half>(kv->cfg.page, &threads))
                                        : (bf16 ? append_variant<128, __nv_bfloat16>(kv->cfg.page, &threads) : append_variant<128, __half>(kv->cfg.page, &threads));
    const int per_warp = ot::kAppendRows * (256 / D);
    a.query_parts = (kv->cfg.q_heads + per_warp - 1) / per_warp;
    a.by_parts = ot::FixedDiv::by((unsigned)a.query_parts);
    const long long warps = q ? (long long)step->B * step->T * a.query_parts : 0, per_block = threads / 32;
    const long long blocks = a.page_blocks + (warps + per_block - 1) / per_block;
    launch_after(kernel, dim3((unsigned)blocks), dim3(threads), 0, static_cast<cudaStream_t>(stream), a);
    kv->launches++;
    return check_launch();
}

int opt_tree_kv_attend(opt_tree_kv* kv, const opt_tree_kv_cache* cache, int32_t layer, const opt_tree_kv_rows* q, const opt_tree_kv_step* step,
                       float scale, const opt_tree_kv_rows* out, float* lse, void* stream) {
    if (!kv || bad_cache(cache) || layer < 0 || layer >= kv->cfg.layers || bad_rows(q) || bad_rows(out) || bad_step(kv, step) || !(scale > 0.f) ||
        scale > 1e38f || off(lse, 4))
        return OPT_TREE_ERR_INVALID_ARG;
    if (!on_device(kv)) return OPT_TREE_ERR_INVALID_ARG;
    ot::KvAttend a;
    memset(&a, 0, sizeof a);
    const int D = kv->cfg.head_dim;
    a.shape = kv->shape;
    a.step = step_of(step);
    a.q = rows_of(q); a.out = rows_of(out);
    a.wide_q = wide(q); a.wide_out = wide(out);
    const long long layer_pages = (long long)layer * kv->cfg.num_pages * kv->cfg.kv_heads;
    a.kc = cache->k + layer_pages * kv->cfg.page * D; a.vc = cache->v + layer_pages * kv->cfg.page * D;
    a.ks = cache->k_scale + layer_pages; a.vs = cache->v_scale + layer_pages;
    a.table = cache->block_table;
    a.lse = lse;
    a.scale = scale * ot::kLog2e;
    a.group = kv->cfg.q_heads / kv->cfg.kv_heads;
    a.by_group = ot::FixedDiv::by((unsigned)a.group);
    a.parts = kv->parts;
    a.arrived = kv->arrived;
    a.cuts = kv->cuts;
    a.status = kv->status;
    const long long rows = (long long)step->T * a.group, slots = (long long)kv->cfg.max_pages * kv->cfg.page;
    const bool brief = step->B * kv->cfg.kv_heads * ((rows + 15) / 16) * ((slots + 127) / 128) <= 2ll * kv->sms;
    const AttendVariant v = attend_for(kv->cfg, (int)rows, brief);
    if (ot::kv_cost_bound(kv->shape, step->B, step->T, v.rows, v.keys) > 0x7FFFFFFFll) return OPT_TREE_ERR_UNSUPPORTED;
    const int grid = kv->sms * v.per_sm;
    launch_after(v.kernel, dim3(grid), dim3(v.threads), v.smem, static_cast<cudaStream_t>(stream), a);
    if (v.join) {
        launch_after(v.join, dim3(grid, ot::kJoinBlocks), dim3(256), 0, static_cast<cudaStream_t>(stream), a);
        kv->launches++;
    }
    kv->launches++;
    return check_launch();
}

int opt_tree_kv_compact(opt_tree_kv* kv, const opt_tree_kv_cache* cache, const int32_t* kv_len, const int32_t* kv_gather, const int32_t* kv_keep,
                        int32_t G, int32_t B, int32_t* new_len, void* stream) {
    if (!kv || bad_cache(cache) || !kv_len || !kv_gather || !kv_keep || G < 1 || B < 1 || B > kv->cfg.max_batch || off(kv_len, 4) || off(kv_gather, 4) ||
        off(kv_keep, 4) || off(new_len, 4))
        return OPT_TREE_ERR_INVALID_ARG;
    if (G > ot::kCompactMost) return OPT_TREE_ERR_UNSUPPORTED;
    // (layer 0 writes the new lengths while the others may still read)
    if (new_len && (overlap(new_len, B, kv_len, B) || overlap(new_len, B, kv_keep, B) || overlap(new_len, B, kv_gather, (size_t)B * G))) return OPT_TREE_ERR_INVALID_ARG;
    if (!on_device(kv)) return OPT_TREE_ERR_INVALID_ARG;
    ot::KvCompact a{kv->shape, cache->k, cache->v, cache->k_scale, cache->v_scale, cache->block_table, kv_len, kv_gather, kv_keep, G, new_len, kv->status};
    launch_after(kv->cfg.head_dim == 64 ? ot::kv_compact_kernel<64> : ot::kv_compact_kernel<128>, dim3(B, kv->cfg.layers), dim3(ot::kCompactThreads), 0,
                 static_cast<cudaStream_t>(stream), a);
    kv->launches++;
    return check_launch();
}

int opt_tree_kv_last_device_status(opt_tree_kv* kv, int32_t* status_host) {
    if (!kv || !status_host) return OPT_TREE_ERR_INVALID_ARG;
    if (!on_device(kv)) return OPT_TREE_ERR_INVALID_ARG;
    if (cudaDeviceSynchronize() != cudaSuccess) return OPT_TREE_ERR_CUDA;
    if (cudaMemcpy(status_host, kv->status, 4, cudaMemcpyDeviceToHost) != cudaSuccess) return OPT_TREE_ERR_CUDA;
    if (cudaMemset(kv->status, 0, 4) != cudaSuccess) return OPT_TREE_ERR_CUDA;
    return OPT_TREE_OK;
}

int64_t opt_tree_kv_launch_count(const opt_tree_kv* kv) { return kv ? kv->launches : 0; }

}  // extern "C"
