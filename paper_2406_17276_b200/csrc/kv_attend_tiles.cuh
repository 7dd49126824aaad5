// Attention of many query rows (trees and chunks of prompts): row tiles of 2 x 128 on the tensor cores.
//
// Per tile of 128 keys: S = Q K^T (tcgen05, both operands from shared memory, fp32 in TMEM), softmax by the threads that own the rows, P in
// half precision back to TMEM over S, O += P V with P from TMEM.  Two row tiles of 128 alternate, so that the tensor cores
// work on one while the other's exponentials are taken; a row tile that is alone is shared by both softmax groups, which take its key tiles in turn.
// Keys and values become half precision on their way into shared memory, where e4m3 codes are exact: four warps a side load codes, convert,
// bring them to a common page scale (by powers of two: exact to 2^-15 of it, rounded to 2^-25 of it below) and write the swizzled layout; once
// per 256 rows.  (Eight-bit operands would need queries and probabilities in two parts each: the same tensor time as half precision, and
// twice the conversions per row.)
// What bounds it: the chain of a key tile (codes, conversion, scores, exponentials, values), no unit by itself.  32 trees of 65 tokens over up to 4096
// slots, 32 / 8 heads of 128: 201 us, 464 TFLOP/s; the exponentials alone would take 40 us, the products 56.
//
// Roles: warps 0-3 and 4-7 softmax, one thread a row; warps 8-11 convert keys, 12-15 values; warp 16 issues the products; warp 17 divides the
// work, looks pages up and copies their codes into shared memory a key tile ahead; two warps fill the last warpgroup.  Barriers (all waits bounded;
// a role whose wait ran out waits for nothing more and leaves, and the others' waits run out after it):
//   run[8]     copies -> all            what to do next
//   q          softmax -> products      queries of a run are in shared memory
//   rk, rv     copies <-> conversion    codes of a key tile
//   k, v       conversion <-> products  operands, two stages each
//   s[X][2]    products -> softmax X    scores of half a key tile: one half's are ready while the other's exponentials are taken
//   p[X][2]    softmax X -> products
//   o[X][2]    products -> softmax X    O holds the values of half a key tile (waited for before O is rescaled, and at the end)
// and named barrier 1 between the softmax groups: sums of a shared row tile handed over, and its outputs read.
#pragma once

#include <type_traits>

#include "copy_ring.cuh"
#include "kv_attend.cuh"

namespace ot {

// Registers a thread of each role; together they are what a block of five warpgroups is launched with (kRegsLaunch each, which the host
// checks), or the warps that ask for more would wait for good.  (The kernel calls no function: with calls the compiler cannot keep to them.)
constexpr int kRegsLaunch = 96, kRegsSoftmax = 144, kRegsConvert = 64, kRegsIssue = 64;
static_assert(2 * kRegsSoftmax + 2 * kRegsConvert + kRegsIssue <= 5 * kRegsLaunch, "registers of a block");

constexpr int kTileRows = 128, kTileKeys = 128, kTileThreads = 20 * 32;

// --- tcgen05 ---
__device__ __forceinline__ void tmem_alloc(uint32_t* smem_word, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem_word)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(unsigned long long* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Shared-memory descriptor of a 128-byte-swizzled operand: rows of 128 bytes, eight rows an atom of 1024 bytes.  Along the summed index (K-major)
// or along the other (MN-major, with `block` bytes from one 64-element block of the other index to the next).  The address is in
// the low word, the constant rest in the high one.
__device__ __forceinline__ uint32_t tc_desc(uint32_t smem_address, uint32_t block) { return smem_address >> 4 | (block >> 4) << 16; }
constexpr uint32_t kDescHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
// D (+)= A B, one step of 16 along the summed index.  A from shared memory, and from tensor memory.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "n"(kDescHigh) : "memory");
}
// 32 columns of this warp's lanes, to be used after tmem_wait (which names the registers, so that no use moves before it).
__device__ __forceinline__ void tmem_load(uint32_t at, float (&x)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]),
                 "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]),
                 "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]),
                 "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_wait(float (&x)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]), "+f"(x[9]),
                 "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]), "+f"(x[16]), "+f"(x[17]), "+f"(x[18]),
                 "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]), "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]),
                 "+f"(x[28]), "+f"(x[29]), "+f"(x[30]), "+f"(x[31])
                 :: "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const float (&x)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(at), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "f"(x[8]), "f"(x[9]),
                   "f"(x[10]), "f"(x[11]), "f"(x[12]), "f"(x[13]), "f"(x[14]), "f"(x[15]), "f"(x[16]), "f"(x[17]), "f"(x[18]), "f"(x[19]),
                   "f"(x[20]), "f"(x[21]), "f"(x[22]), "f"(x[23]), "f"(x[24]), "f"(x[25]), "f"(x[26]), "f"(x[27]), "f"(x[28]), "f"(x[29]),
                   "f"(x[30]), "f"(x[31]) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&x)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]),
                   "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]) : "memory");
}
// The same of 16 columns, and a store of eight.
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&x)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]),
                   "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_wait16(float (&x)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]), "+f"(x[9]),
                   "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15])
                 :: "memory");
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&x)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
}
// One lane of a converged warp, always the same one.  (Asked by elect.sync and not by the lane's number, the compiler knows that a single
// thread is left, and hands the tensor instructions their operands without asking every lane for its own.)
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// fp32 accumulators, half-precision operands, M = 128; mn: the second operand is MN-major.
__host__ __device__ constexpr uint32_t tc_idesc(int n, bool mn) { return 1u << 4 | (mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(128 >> 4) << 24; }

// What the copying warp finds out about a key tile.  A scale is taken as a power of two, which the operands are brought to in half precision
// without a rounding, times a fraction, which scores and probabilities are multiplied by in single precision (half precision's rounding of a scale
// would shift all scores of a page alike).  Fractions other than 1 are dealt with apart, in loops that are not unrolled: that they may come at all
// takes 3 % of a call without any (195 -> 201 us, 296 -> 304 us for the batches below); multiplied in where the scores are in registers, 8 to 18 %.  Keys of a tile are brought to the tile's largest power, values to one reference that
// outputs are kept in: the first tile's largest power, or a later one's that is over 64 times the reference so far (64 * 448 is within
// half precision).
struct alignas(16) TileHead {
    float kmax, ref;                     // largest power of the keys, reference of the values
    int odd, pad;                        // fractions other than 1: of keys (1), of values (2)
};
struct TileInfo {
    uint32_t kratio[8], vratio[8];       // of each 16 keys: the power over the tile's, twice in half precision
    float kfrac[8], vfrac[8];            // of each 16 keys: the fraction
    TileHead head;
};
// The smallest power of two that is no smaller than a scale (2^127 above it, 2^-126 for subnormal scales; 0 for 0).
__device__ __forceinline__ float scale_power(float s) { return __uint_as_float(min((__float_as_uint(s) + 0x7FFFFFu) & 0x7F800000u, 0x7F000000u)); }
// Slots of TileInfo, by tile, and of the runs and their NaN words, by run.  The copying warp writes those of tile t (of run r) once the codes
// of keys of tile t - 2 at least have been taken.  Then keys of t - 3 have been written, so the scores of t - 5 are complete; those were
// issued after the values of tile t - 7 (t - 6 with two row tiles) had been added up.  So both softmax groups, and the conversion of values, are done with tile
// t - 7, and the groups with the run before that tile's.  (A run is published a tile earlier than that: its slot was taken at the start of the run that
// used it, which has to be over by t - 8.)
constexpr int kTileSlots = 8;

template <int D> struct TileLayout {
    static constexpr int kOperand = 128 * D * 2;             // one half-precision operand of 128 rows
    static constexpr int kCodes = 128 * D, kRaw = D == 128 ? 1 : 2;          // codes of one side of a key tile; stages of them
    static constexpr int kQ = 0, kK = 2 * kOperand, kV = kK + 2 * kOperand, kRawK = kV + 2 * kOperand, kRawV = kRawK + kRaw * kCodes;
    static constexpr int kBars = kRawV + kRaw * kCodes;
    enum { kBarQ, kBarKFull, kBarKFree = kBarKFull + 2, kBarVFull = kBarKFree + 2, kBarVFree = kBarVFull + 2, kBarS = kBarVFree + 2, kBarP = kBarS + 4,
           kBarO = kBarP + 4, kBarRKFull = kBarO + 4, kBarRKFree = kBarRKFull + kRaw, kBarRVFull = kBarRKFree + kRaw, kBarRVFree = kBarRVFull + kRaw,
           kBarRun = kBarRVFree + kRaw, kBarEnd = kBarRun + kTileSlots, kBarCount };
    static constexpr int kInfo = (kBars + kBarCount * 8 + 15) & ~15, kNan = kInfo + kTileSlots * (int)sizeof(TileInfo), kWord = kNan + kTileSlots * 4, kMerge = kWord + 16,
                         kRuns = kMerge + 1024 + 16;
    static constexpr int kBytes = kRuns + kTileSlots * (int)sizeof(KvRun);
    static constexpr uint32_t kColumns = 512, kColS = 0, kColO = 256;
};
static_assert(TileLayout<128>::kBytes <= 227 * 1024, "shared memory of a CTA");
// 1 / p of a power of two of scale_power (2^-126 ... 2^127); something finite for 0.
__device__ __forceinline__ float power_inverse(float p) { return __uint_as_float(max(0x7F000000u - __float_as_uint(p), 0x00400000u)); }

// Bits of the slots that token i of a run's sequence sees among the step's tokens [j0, j0 + 64) (negative j: the prefix).
__device__ __forceinline__ uint64_t kv_sees64(const KvStep& st, int b, int i, int tokens, int j0) {
    const int end = tokens - j0;                             // bits at or beyond are behind the last slot
    const uint64_t inside = end >= 64 ? ~0ull : (end <= 0 ? 0ull : (1ull << end) - 1ull);
    if (!st.mask) {
        const int n = i + 1 - j0;
        return inside & (n >= 64 ? ~0ull : (n <= 0 ? 0ull : (1ull << n) - 1ull));
    }
    uint64_t v = 0;
    if (j0 <= 0) v = j0 <= -64 ? ~0ull : (2ull << -j0) - 1ull;                     // the prefix and the root (j <= 0)
    if (i > 0 && j0 > -64) {
        const int W = (st.T - 1 + 63) >> 6, at = j0 - 1;
        const uint64_t* m = st.mask + ((long long)b * (st.T - 1) + i - 1) * W;
        if (at < 0) v |= -at < 64 ? m[0] << -at : 0ull;
        else {
            const int w = at >> 6, s = at & 63;
            if (w < W) v |= m[w] >> s;
            if (s > 0 && w + 1 < W) v |= m[w + 1] << (64 - s);
        }
    }
    if (i >= j0 && i < j0 + 64) v |= 1ull << (i - j0);
    return v & inside;
}

// A row's sums are kept relative to a reference 2^5 below the largest score at the time; the largest may grow by another 2^10 before they
// are brought to a new reference.  So probabilities of up to 2^15 use the range of half precision (rounded by 2^-11 of each down to 2^-19
// of the largest, by 2^-30 of the largest below; relative to the largest alone, small ones would lose bits that matter where the large
// ones' values cancel).
constexpr float kLift = 5.f, kGrowth = 10.f;

__device__ __forceinline__ float max3_nan(float a, float b, float c) {         // NaN if any is
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
template <int D, class T>
__global__ void __launch_bounds__(kTileThreads, 1) kv_attend_tiles_kernel(const __grid_constant__ KvAttend a) {
    using L = TileLayout<D>;
    extern __shared__ __align__(1024) unsigned char tile_smem[];
    unsigned char* smem = tile_smem;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + L::kBars);
    TileInfo* infos = reinterpret_cast<TileInfo*>(smem + L::kInfo);
    int* nans = reinterpret_cast<int*>(smem + L::kNan);
    KvRun* runs = reinterpret_cast<KvRun*>(smem + L::kRuns);
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + L::kWord);
    if (smem_u32(smem) & 1023u) {                            // (swizzled operands need it; nothing has been started yet)
        if (threadIdx.x == 0) set_status(a.status, kErrInternal);
        return;
    }
    if (warp == 16) {
        if (lane == 0) {
            mbar_init(bars + L::kBarQ, 8);
            for (int i = 0; i < 2; ++i) {
                mbar_init(bars + L::kBarKFull + i, 4); mbar_init(bars + L::kBarKFree + i, 1);
                mbar_init(bars + L::kBarVFull + i, 4); mbar_init(bars + L::kBarVFree + i, 1);
                for (int k = 0; k < 2; ++k) {
                    mbar_init(bars + L::kBarS + 2 * i + k, 1); mbar_init(bars + L::kBarP + 2 * i + k, 4); mbar_init(bars + L::kBarO + 2 * i + k, 1);
                }
            }
            for (int i = 0; i < L::kRaw; ++i) {
                mbar_init(bars + L::kBarRKFull + i, 1); mbar_init(bars + L::kBarRKFree + i, 4);
                mbar_init(bars + L::kBarRVFull + i, 1); mbar_init(bars + L::kBarRVFree + i, 4);
            }
            for (int i = 0; i < kTileSlots; ++i) mbar_init(bars + L::kBarRun + i, 1);
            mbar_init(bars + L::kBarEnd, 1);
            mbar_fence_init();
        }
        __syncwarp();
        tmem_alloc(words, L::kColumns);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_wait();
    // A wait that runs out is recorded; this warp waits for nothing more then and leaves at the end of its run (softmax: of all runs; conversion: at once).
    bool dead = false;
    auto wait = [&](int bar, uint32_t parity) { dead = dead || !mbar_wait_warp(bars + bar, parity, a.status); };
    KvRun r;
    // the next run of this CTA, from the copying warp; false at the end
    int runs_taken = 0;
    auto next_run = [&](auto&& waits) {
        const int slot = runs_taken & (kTileSlots - 1);
        waits(L::kBarRun + slot, runs_taken / kTileSlots & 1);
        ++runs_taken;
        r = runs[slot];
        return !dead && r.b >= 0;
    };
    if (warp < 8) {
        // ---- softmax: a thread a row ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const int X = warp >> 2, in_tile = threadIdx.x & 127;
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) * 32u << 16);
        const uint32_t ts = lanes + L::kColS + X * 128, to = lanes + L::kColO + X * D;
        uint32_t tiles = 0, at = 0;                          // key tiles of this group, and of the runs before
        int run = 0;
        // Both groups go through all runs, also when a wait has run out (it is the last one then), so that neither misses the other at the
        // named barrier; the copying warp gives the last run out in any case, later by a wait of its own at most.
        auto next = [&] {
            const int slot = runs_taken & (kTileSlots - 1);
            const bool there = mbar_wait_warp(bars + L::kBarRun + slot, runs_taken / kTileSlots & 1, a.status, 8 * kWaitCycles);
            ++runs_taken;
            r = runs[slot];
            return there && r.b >= 0;
        };
        while (next()) {
            const bool single = r.tokens * a.group - r.rt * 2 * kTileRows <= kTileRows;
            const int row0 = r.rt * 2 * kTileRows + (single ? 0 : X * kTileRows), rows = min(kTileRows, r.tokens * a.group - row0);
            const int row = row0 + in_tile;
            const bool mine = in_tile < rows, busy = (warp & 3) * 32 < rows;       // this thread, this warp
            const int token = (int)a.by_group.div((unsigned)min(row, r.tokens * a.group - 1));
            // Queries to shared memory, D / 8 lanes a row, all of a warp's 32 rows in flight.  bf16 numbers from 2^-17 on to 2^15 are half-precision
            // numbers too, and smaller ones are rounded by up to 2^-25 (2^-19 of the row's largest at most): rows whose largest lies between 2^-6 and 2^15
            // are taken as they are, which spares a second pass over them.  Where a row is larger or smaller, the warp's
            // rows are brought there by powers of two of their own (exact but for elements below 2^-25 of the row's largest).
            float qf = a.scale;
            {
                constexpr int kRowLanes = D / 8, kAt = 32 / kRowLanes, kLoads = 32 / kAt;
                constexpr uint32_t kRowMask = kRowLanes == 16 ? 0xFFFFu : 0xFFu;
                const int sub = lane & (kRowLanes - 1), low = (warp & 3) * 32;
                unsigned char* to_q = smem + L::kQ + X * L::kOperand + (sub >> 3) * (128 * 128);
                auto fetch = [&](int i) {
                    const int at_row = low + i * kAt + lane / kRowLanes;
                    if (at_row >= rows) return make_uint4(0, 0, 0, 0);
                    const int tok = (int)a.by_group.div((unsigned)(row0 + at_row)), hq = r.h * a.group + row0 + at_row - tok * a.group;
                    return load8(a.q.data + r.b * a.q.batch + tok * a.q.token + hq * a.q.head + sub * 8, a.wide_q);
                };
                auto magnitude = [&](const uint4& q) {       // largest of the lane's eight, as a bf16 pattern
                    const uint32_t m2 = max_bf16x2(max_bf16x2(q.x & 0x7FFF7FFFu, q.y & 0x7FFF7FFFu), max_bf16x2(q.z & 0x7FFF7FFFu, q.w & 0x7FFF7FFFu));
                    return max(m2 & 0xFFFFu, m2 >> 16);
                };
                auto keep = [&](int i, const uint4& q, float f) {
                    const int at_row = low + i * kAt + lane / kRowLanes;
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                    uint32_t h[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 y = to_float2<T>(w[k]);
                        h[k] = std::is_same<T, __half>::value ? w[k] : from_float2<__half>(y.x * f, y.y * f);
                    }
                    if (!single || X == 0) *reinterpret_cast<uint4*>(to_q + at_row * 128 + (((sub & 7) ^ (at_row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                };
                uint4 q[kLoads];
                bool fits = true;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) q[i] = fetch(i);
                if (!std::is_same<T, __half>::value) {
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) {
                        const uint32_t top = magnitude(q[i]);
                        const unsigned big = __ballot_sync(0xFFFFFFFFu, top >= (127u + 15u) << 7), some = __ballot_sync(0xFFFFFFFFu, top >= (127u - 6u) << 7);
                        bool rows_fit = big == 0;
#pragma unroll
                        for (int k = 0; k < kAt; ++k) rows_fit = rows_fit && (some >> k * kRowLanes & kRowMask || low + i * kAt + k >= rows);
                        fits = fits && rows_fit;
                    }
                }
                if (fits) {
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) keep(i, q[i], 1.f);
                } else {
#pragma unroll 1
                    for (int i = 0; i < kLoads; ++i) {
                        const uint4 y = fetch(i);
                        uint32_t top = magnitude(y);
#pragma unroll
                        for (int o = kRowLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                        const int e = min(max((int)(top >> 7) - 127, -112), 120) - 8;
                        const int own = __shfl_sync(0xFFFFFFFFu, e, lane % kAt * kRowLanes);       // this thread's row, if it is among these
                        if (lane / kAt == i) qf = a.scale * power_of_two(own);
                        keep(i, y, power_of_two(-e));
                    }
                }
            }
            proxy_fence();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + L::kBarQ);
            float m = -INFINITY, l = 0.f, ref = 1.f;
            const int first = r.k0 + (single ? X : 0), step = single ? 2 : 1;      // this group's key tiles
            for (int kt = first; kt < r.k1; kt += step, ++tiles) {
                const TileInfo& info = infos[(at + kt - r.k0) & (kTileSlots - 1)];
                for (int half = 0; half < 2; ++half) {
                    const int j0 = kt * kTileKeys + half * 64 - r.len;             // the first slot, as a token of the step
                    const bool edge = j0 + 64 > 0;
                    const uint64_t see = edge && busy ? kv_sees64(a.step, r.b, token, r.tokens, j0) : 0ull;
                    wait(L::kBarS + 2 * X + half, tiles & 1);
                    tc_fence_after();
                    if (busy) {
                        const uint32_t from = ts + half * 64;
                        const TileHead head = info.head;
                        const float f = fmaxf(qf * head.kmax, 1.2e-38f);
                        const float unit = ref == head.ref ? 1.f : ref / head.ref;
                        ref = head.ref;
                        float x[2][32];
                        tmem_load(from, x[0]);
                        tmem_load(from + 32, x[1]);
                        tmem_wait(x[0]);
                        tmem_wait(x[1]);
                        if (__builtin_expect(head.odd & 1, 0)) {               // fractions of key scales
#pragma unroll 1
                            for (int g = 0; g < 4; ++g) {
                                float y[16];
                                tmem_load16(from + g * 16, y);
                                tmem_wait16(y);
                                uint32_t z[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) z[i] = __float_as_uint(y[i] * info.kfrac[half * 4 + g]);
                                tmem_store16(from + g * 16, z);
                            }
                            tmem_wait_stores();
                            tmem_load(from, x[0]);
                            tmem_load(from + 32, x[1]);
                            tmem_wait(x[0]);
                            tmem_wait(x[1]);
                        }
                        if (edge) {
#pragma unroll
                            for (int c = 0; c < 2; ++c)
#pragma unroll
                                for (int i = 0; i < 32; ++i) x[c][i] = (uint32_t)(see >> c * 32) >> i & 1 ? x[c][i] : -INFINITY;
                        }
                        float top4[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const float* y = x[c >> 1] + (c & 1) * 16;
                            top4[c] = max3_nan(y[0], y[1], y[2]);
#pragma unroll
                            for (int i = 3; i < 15; i += 2) top4[c] = max3_nan(top4[c], y[i], y[i + 1]);
                            top4[c] = max3_nan(top4[c], y[15], y[15]);
                        }
                        const float top = max3_nan(max3_nan(top4[0], top4[1], top4[2]), top4[3], top4[3]) * f;
                        const float was = m;
                        const bool grows = top > m + (kLift + kGrowth);      // (the first score that is seen, too)
                        if (grows) m = top - kLift;
                        if ((kt > first || half) && (unit != 1.f || __any_sync(0xFFFFFFFFu, grows))) {
                            // S being there, the products of two halves ago are complete; those of the half before are waited for
                            wait(L::kBarO + 2 * X + (half ^ 1), half ? tiles & 1 : (tiles - 1) & 1);
                            tc_fence_after();
                            float fade = grows ? ex2_approx(was - m) : 1.f;
                            l *= fade;
                            fade *= unit;
#pragma unroll 1
                            for (int c = 0; c < D / 32; ++c) {
                                float o[32];
                                tmem_load(to + c * 32, o);
                                tmem_wait(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] *= fade;
                                tmem_store32(to + c * 32, o);
                            }
                        }
                        // a row that sees a NaN or an infinite score is NaN
                        const float base = !(top < INFINITY) ? __int_as_float(0x7FC00000) : (m == -INFINITY ? 0.f : m);
                        const unsigned long long f2 = pack2(f, f), base2 = pack2(-base, -base);
                        unsigned long long sum[2] = {0ull, 0ull};
                        if (__builtin_expect(!(head.odd & 2), 1)) {
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                uint32_t p[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    float e0, e1;
                                    unpack2(fma2(pack2(x[c][2 * i], x[c][2 * i + 1]), f2, base2), e0, e1);
                                    e0 = ex2_approx(e0); e1 = ex2_approx(e1);
                                    sum[i & 1] = add2(sum[i & 1], pack2(e0, e1));
                                    p[i] = from_float2<__half>(e0, e1);
                                }
                                tmem_store16(from + c * 16, p);
                            }
                        } else {                             // fractions of value scales: 16 scores at a time, read again (P(g) only covers scores that have been)
#pragma unroll 1
                            for (int g = 0; g < 4; ++g) {
                                const float vfrac = info.vfrac[half * 4 + g];
                                float y[16];
                                tmem_load16(from + g * 16, y);
                                tmem_wait16(y);
                                uint32_t p[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    float e0, e1;
                                    unpack2(fma2(pack2(y[2 * i], y[2 * i + 1]), f2, base2), e0, e1);
                                    e0 = ex2_approx(!edge || see >> (g * 16 + 2 * i) & 1 ? e0 : -INFINITY);
                                    e1 = ex2_approx(!edge || see >> (g * 16 + 2 * i + 1) & 1 ? e1 : -INFINITY);
                                    sum[i & 1] = add2(sum[i & 1], pack2(e0, e1));
                                    p[i] = from_float2<__half>(e0 * vfrac, e1 * vfrac);
                                }
                                tmem_store8(from + g * 8, p);
                            }
                        }
                        float s0, s1;
                        unpack2(add2(sum[0], sum[1]), s0, s1);
                        l += s0 + s1;
                        tmem_wait_stores();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bars + L::kBarP + 2 * X + half);
                }
            }
            at += r.k1 - r.k0;
            const bool has = first < r.k1;                   // (a single row tile with one key tile has none for X = 1)
            if (has) {
                wait(L::kBarO + 2 * X, (tiles - 1) & 1);
                wait(L::kBarO + 2 * X + 1, (tiles - 1) & 1);
            }
            tc_fence_after();
            const bool cut = r.first != r.last;
            constexpr int kFloats = kv_part_floats<kTileRows, D>();
            float* part = a.parts + ((long long)kv_slot(r, blockIdx.x) * 2 + (single ? 0 : X)) * kFloats;
            // a single row tile: the first group takes the second's sums, and reads its outputs from TMEM
            const bool both = single && r.k1 - r.k0 > 1;
            float mine_f = ref, other_f = 0.f;
            float* hand = reinterpret_cast<float*>(smem + L::kMerge);              // [2][128], and one
            if (single) {
                if (X == 1) {
                    hand[in_tile] = m; hand[128 + in_tile] = l;
                    if (in_tile == 0) hand[256] = ref;
                    tc_fence_before();
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                tc_fence_after();
                if (both && X == 0) {
                    const float m1 = hand[in_tile], mm = fmaxf(m, m1), base = mm == -INFINITY ? 0.f : mm;
                    const float w0 = ex2_approx(m - base), w1 = ex2_approx(m1 - base);
                    l = l * w0 + hand[128 + in_tile] * w1;
                    mine_f = ref * w0;
                    other_f = hand[256] * w1;
                    m = mm;
                }
            }
            // (behind the barrier: of a single row tile, the run's last values may be the second group's, which has waited for their products)
            const bool nan = nans[run & (kTileSlots - 1)] != 0;
            ++run;
            const float norm = l == 0.f ? 0.f : 1.f / l;
            mine_f *= norm; other_f *= norm;
            if (busy && (!single || X == 0)) {
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    float x[32];
                    tmem_load(to + c * 32, x);
                    tmem_wait(x);
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] *= mine_f;
                    if (both) {
                        float y[32];
                        tmem_load(to + D + c * 32, y);
                        tmem_wait(y);
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = fmaf(y[i], other_f, x[i]);
                    }
                    if (!mine) continue;
                    if (cut) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<float4*>(part + ((c * 8 + i) * kTileRows + in_tile) * 4) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    } else {
                        kv_store<D, 32, T, false>(a, r, row, c * 32, x, nan);
                    }
                }
                if (mine && cut) { part[kTileRows * D + in_tile] = m; part[kTileRows * D + kTileRows + in_tile] = l; }
                if (mine && !cut) kv_store_lse(a, r, row, m, l);
                if (cut && in_tile == 0) reinterpret_cast<int*>(part)[kTileRows * D + 2 * kTileRows] = nan;
            }
            tc_fence_before();
            if (single) asm volatile("bar.sync 1, 256;" ::: "memory");             // the second group's outputs have been read
        }
    } else if (warp < 16) {
        // ---- conversion: codes to half precision, in the layout of the products; four warps a side ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConvert));
        constexpr int kLanes = D / 16, kAtOnce = 128 / kLanes, kIter = 128 / kAtOnce;   // 16 codes a lane; keys at once
        const int tid = threadIdx.x & 127, side = warp >= 12, sub = tid & (kLanes - 1), key = tid / kLanes;
        uint32_t done = 0;                                   // key tiles converted so far
        int run = 0;
        // where this lane's two chunks of eight elements go in a row; lanes of the second 64 elements begin with the other one, whose banks
        // are free
        const int block = sub >> 2, chunk = (sub & 3) * 2;
        while (next_run(wait)) {
            const int end = r.len + r.tokens;                // slots at or beyond it are not the sequence's
            for (int kt = r.k0; kt < r.k1; ++kt, ++done) {
                const uint32_t stage = done & 1, phase = done >> 1 & 1, st = done % L::kRaw, raw_phase = done / L::kRaw & 1;
                const TileInfo& info = infos[done & (kTileSlots - 1)];
                {                                            // (the same code for both sides)
                    const int raw_full = side ? L::kBarRVFull : L::kBarRKFull, raw_free = side ? L::kBarRVFree : L::kBarRKFree;
                    const int full = side ? L::kBarVFull : L::kBarKFull, free_ = side ? L::kBarVFree : L::kBarKFree;
                    const unsigned char* from = smem + (side ? L::kRawV : L::kRawK) + st * L::kCodes + tid * 16;
                    unsigned char* to = smem + (side ? L::kV : L::kK) + stage * L::kOperand + block * (128 * 128);
                    const uint32_t* ratios = side ? info.vratio : info.kratio;
                    const bool edge = side && (kt + 1) * kTileKeys > r.len;        // NaN codes of the step's own values, and what lies behind them
                    uint32_t seen = 0;
                    wait(raw_full + st, raw_phase);
                    uint4 codes[kIter];                      // all of them, so that the next tile's may come in
#pragma unroll
                    for (int i = 0; i < kIter; ++i) codes[i] = *reinterpret_cast<const uint4*>(from + i * 2048);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bars + raw_free + st);
                    wait(free_ + stage, phase ^ 1);
                    if (dead) break;                         // (no stage is handed back any more, so the copying warp gets no further ahead)
#pragma unroll
                    for (int i = 0; i < kIter; ++i) {
                        const int row = i * kAtOnce + key;
                        uint4 x = codes[i];
                        if (edge) {
                            const int s = kt * kTileKeys + row;
                            if (s >= end) x = make_uint4(0, 0, 0, 0);
                            else if (s >= r.len) { x.x = drop_nan(x.x, seen); x.y = drop_nan(x.y, seen); x.z = drop_nan(x.z, seen); x.w = drop_nan(x.w, seen); }
                        }
                        const __half2 f = *reinterpret_cast<const __half2*>(ratios + (row >> 4));
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                        uint32_t h[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t two = from_e4m3x2((uint16_t)(w[e >> 1] >> (e & 1) * 16));
                            const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&two), f);
                            h[e] = *reinterpret_cast<const uint32_t*>(&y);
                        }
                        const uint4 c0 = make_uint4(h[0], h[1], h[2], h[3]), c1 = make_uint4(h[4], h[5], h[6], h[7]);
                        *reinterpret_cast<uint4*>(to + row * 128 + (((chunk + block) ^ (row & 7)) << 4)) = block ? c1 : c0;
                        *reinterpret_cast<uint4*>(to + row * 128 + (((chunk + 1 - block) ^ (row & 7)) << 4)) = block ? c0 : c1;
                    }
                    if (seen) atomicOr(nans + (run & (kTileSlots - 1)), 1);
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bars + full + stage);
                }
            }
            ++run;
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == 17) {
        // ---- copies: pages of a key tile, a lane for each 16 keys; four tiles are looked up at a time, four ahead ----
        uint32_t done = 0, issued_k = 0, issued_v = 0;       // key tiles, and those of which keys and values were copied
        int run = 0;
        const int shift = a.shape.page_shift, inside = a.shape.page - 1;
        const int copy_rows = min(a.shape.page, kTileKeys);
        KvWalk<2 * kTileRows, kTileKeys, true> walk;
        KvRun before{-1};
        bool more = walk.begin(a, blockIdx.x, gridDim.x);
        for (int given = 0;; ++given) {
            more = more && walk.next(a, r) && !dead;
            if (!more) r.b = -1;
            if (lane == 0) {
                runs[given & (kTileSlots - 1)] = r;
                mbar_arrive(bars + L::kBarRun + (given & (kTileSlots - 1)));
            }
            __syncwarp();
            if (!more) break;
            before = r;
            const int end = r.len + r.tokens;
            int id[2];
            float ks[2], vs[2];
            auto look = [&](int batch, int& i, float& k, float& v) {
                const int s = (r.k0 + batch * 4) * kTileKeys + lane * 16;
                i = -1; k = v = 0.f;
                if (s < min(end, r.k1 * kTileKeys)) {
                    i = max(0, kv_page(a.shape, a.table, r.b, s >> shift, a.status));
                    const long long head = (long long)i * a.shape.kv_heads + r.h;
                    k = __ldg(a.ks + head); v = __ldg(a.vs + head);
                }
            };
            look(0, id[0], ks[0], vs[0]);
            look(1, id[1], ks[1], vs[1]);
            float ref = 0.f;
            for (int kt = r.k0; kt < r.k1; ++kt, ++done) {
                const int n = kt - r.k0;
                if (n && (n & 3) == 0) {
                    id[0] = id[1]; ks[0] = ks[1]; vs[0] = vs[1];
                    look((n >> 2) + 1, id[1], ks[1], vs[1]);
                }
                // lanes 0 to 7: this tile's groups of 16 keys
                const int from = (n & 3) * 8 + (lane & 7);
                const int mine = __shfl_sync(0xFFFFFFFFu, id[0], from);
                const float kscale = __shfl_sync(0xFFFFFFFFu, ks[0], from), vscale = __shfl_sync(0xFFFFFFFFu, vs[0], from);
                const float k = scale_power(kscale), v = scale_power(vscale);
                const float kfrac = kscale * power_inverse(k), vfrac = vscale * power_inverse(v);
                const int odd = (__any_sync(0xFFFFFFFFu, kscale != k) ? 1 : 0) | (__any_sync(0xFFFFFFFFu, vscale != v) ? 2 : 0);
                const float kmax = warp_max_f32(k), vmax = warp_max_f32(v);
                if (n == 0 || vmax > 64.f * ref) ref = vmax;
                const int s = kt * kTileKeys + lane * 16;
                const bool copies = lane < 8 && mine >= 0 && (s & (copy_rows - 1)) == 0;
                const uint32_t bytes = __popc(__ballot_sync(0xFFFFFFFFu, copies)) * copy_rows * D;
                const uint32_t st = done % L::kRaw, phase = done / L::kRaw & 1;
                const long long row = ((long long)mine * a.shape.kv_heads + r.h) * a.shape.page + (s & inside);
                wait(L::kBarRKFree + st, phase ^ 1);
                if (lane < 8) {
                    TileInfo& info = infos[done & (kTileSlots - 1)];
                    const __half2 kr = __float2half2_rn(k * power_inverse(kmax)), vr = __float2half2_rn(v * power_inverse(ref));
                    info.kratio[lane] = *reinterpret_cast<const uint32_t*>(&kr);
                    info.vratio[lane] = *reinterpret_cast<const uint32_t*>(&vr);
                    info.kfrac[lane] = kfrac; info.vfrac[lane] = vfrac;
                    if (lane == 0) {
                        info.head = TileHead{kmax, ref, odd, 0};
                        if (n == 0) nans[run & (kTileSlots - 1)] = 0;
                    }
                }
                __syncwarp();
                if (dead) continue;                          // (nobody takes codes any more)
                if (lane == 0) mbar_expect_tx(bars + L::kBarRKFull + st, bytes);
                __syncwarp();
                if (copies) bulk_load(smem + L::kRawK + st * L::kCodes + lane * 16 * D, a.kc + row * D, copy_rows * D, bars + L::kBarRKFull + st);
                ++issued_k;
                wait(L::kBarRVFree + st, phase ^ 1);
                if (dead) continue;
                if (lane == 0) mbar_expect_tx(bars + L::kBarRVFull + st, bytes);
                __syncwarp();
                if (copies) bulk_load(smem + L::kRawV + st * L::kCodes + lane * 16 * D, a.vc + row * D, copy_rows * D, bars + L::kBarRVFull + st);
                ++issued_v;
            }
            ++run;
        }
        // the cut row tile that begins here, for the kernel that joins the parts
        if (lane == 0) {
            if (before.first == before.last || before.first != (int)blockIdx.x) before.b = -1;
            a.cuts[blockIdx.x] = before;
        }
        // copies in flight land before the CTA ends, also where their reader has given up
        using Ring = CopyRing<L::kRaw>;
        Ring::drain(Ring::oldest(issued_k), issued_k, [&](uint32_t st, uint32_t parity) { mbar_wait_warp(bars + L::kBarRKFull + st, parity, a.status); });
        Ring::drain(Ring::oldest(issued_v), issued_v, [&](uint32_t st, uint32_t parity) { mbar_wait_warp(bars + L::kBarRVFull + st, parity, a.status); });
    } else if (warp == 16) {
        // ---- products: one lane issues ----
        if (elect_one()) {
            constexpr uint32_t kScores = tc_idesc(64, false), kOutputs = tc_idesc(D, true), kHalf = 64 * 128 >> 4, kStageStep = L::kOperand >> 4;
            const uint32_t dq = tc_desc(smem_u32(smem + L::kQ), 16), dk = tc_desc(smem_u32(smem + L::kK), 16), dv = tc_desc(smem_u32(smem + L::kV), 128 * 128);
            auto wait1 = [&](int bar, uint32_t parity) { dead = dead || !mbar_wait_thread(bars + bar, parity, a.status); };
            uint32_t done = 0, nrun = 0, tiles[2] = {0, 0};
            auto scores = [&](int X, int Q, uint32_t stage, int half) {
                const uint32_t d = tmem + L::kColS + X * 128 + half * 64, q = dq + Q * kStageStep, k0 = dk + stage * kStageStep + half * kHalf;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t at = ((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4;
                    tc_mma_ss(d, q + at, k0 + at, kScores, k > 0);
                }
                tc_commit(bars + L::kBarS + 2 * X + half);
            };
            auto outputs = [&](int X, uint32_t stage, int half, bool add) {
                wait1(L::kBarP + 2 * X + half, tiles[X] & 1);
                tiles[X] += half;
                tc_fence_after();
                const uint32_t d = tmem + L::kColO + X * D, p = tmem + L::kColS + X * 128 + half * 64, v = dv + stage * kStageStep + half * kHalf;
#pragma unroll
                for (int k = 0; k < 4; ++k) tc_mma_ts(d, p + k * 8, v + k * (2048 >> 4), kOutputs, add || k > 0);
                tc_commit(bars + L::kBarO + 2 * X + half);
            };
            while (next_run(wait1)) {
                // Two row tiles in turn, each with its own scores; or one, whose key tiles the two groups take in turn.  A key tile's scores are
                // issued `ahead` tiles before its values; both stand here once for all cases, for the sake of the instruction cache.
                const bool single = r.tokens * a.group - r.rt * 2 * kTileRows <= kTileRows;
                const int n = r.k1 - r.k0, ahead = single ? 2 : 1, pieces = single ? 2 : 4;
                wait1(L::kBarQ, nrun & 1);
                ++nrun;
#pragma unroll 1
                for (int i = -ahead; i < n; ++i) {
                    const uint32_t now = (done + i) & 1, tile = done + i + ahead, next = tile & 1;
                    const bool more = i + ahead < n;
                    if (i >= 0) wait1(L::kBarVFull + now, (done + i) >> 1 & 1);
#pragma unroll 1
                    for (int k = 0; k < pieces; ++k) {
                        const int half = single ? k : k >> 1, X = single ? i & 1 : k & 1;
                        if (i >= 0) outputs(X, now, half, i >= ahead || half);
                        if (more) {
                            if (k == 0) {
                                wait1(L::kBarKFull + next, tile >> 1 & 1);
                                tc_fence_after();
                            }
                            scores(X, single ? 0 : X, next, half);
                        }
                    }
                    if (i >= 0) tc_commit(bars + L::kBarVFree + now);
                    if (more) tc_commit(bars + L::kBarKFree + next);
                }
                done += n;
            }
            // everything issued is complete before TMEM is given back, also after a wait that ran out
            tc_commit(bars + L::kBarEnd);
            mbar_wait_thread(bars + L::kBarEnd, 0, a.status);
        }
        __syncwarp();
    }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 16) tmem_free(tmem, L::kColumns);
}

// Joins the parts of the row tiles that the kernel above has cut: block (c, j) takes eight rows of every 8 * kJoinBlocks of the tile that began
// in CTA c, if it is one.  A kernel of its own, because there is much to read (64 KB a part at D = 128) and the CTA that finished last would be
// alone with it.
constexpr int kJoinBlocks = 16;

template <int D, class T>
__global__ void __launch_bounds__(256) kv_join_kernel(const __grid_constant__ KvAttend a) {
    grid_dependency_wait();
    const KvRun r = a.cuts[blockIdx.x];
    if (r.b < 0) return;
    constexpr int kFloats = kv_part_floats<kTileRows, D>();
    const int warp = threadIdx.x >> 5;
    for (int X = 0; X < 2; ++X) {
        const int row0 = r.rt * 2 * kTileRows + X * kTileRows, rows = min(kTileRows, r.tokens * a.group - row0);
        kv_join<kTileRows, D, T>(a, r, a.parts + (long long)X * kFloats, 2, row0, rows, blockIdx.y * 8 + warp, kJoinBlocks * 8);
    }
}

}  // namespace ot
