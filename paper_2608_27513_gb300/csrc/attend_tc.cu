// attend_tc.cu -- attention over the 8-bit cache for many rows (drafts, prompts) on tcgen05.
//
// An item has R = 128 SUB rows (attend.cuh): one or two blocks of 128 (query token, query head) pairs of a
// KV head, which are the lanes of tensor memory.  Per key tile of 128 tokens (4 pages; 64 at d = 256) and block
//     S = Q K^T            Q in shared memory, FP16         128 x 128 x D
//     P = 2^(S f + a - R)  a thread per row; over S in tensor memory, FP16
//     O += P V             in two halves of the tokens      128 x D x 128
// One CTA per SM walks over an equal range of the items' key tiles.  Items that lie in one range are written at
// once; parts are joined by a second launch, as for single tokens, unless ranges end with items (attend_tc_whole).
//
// Warps.  Softmax: 4 per block of rows.  Codes to FP16: 4 (SUB = 1: 4 for K, 4 for V); a 16-byte chunk of codes
// becomes two 16-byte rows of core matrices (8 rows of 8 FP16), which serve K as a K-major and V as an MN-major
// operand without another layout.  Pages: one warp copies a tile's records in bulk, K and V apart, and notes the
// scales.  Products: a warp per block of rows, which issues from descriptors in uniform registers in loops of few
// instructions.  With two blocks a token goes back and forth between the issuing warps, a tile's P V and the next
// tile's Q K^T at a time, so that one block's products run under the other's softmax: left alone both fall into
// step (a piece of 4096 queries at the end of 32768 tokens, 32 heads, 8 KV heads, d = 128: 1.96 ms; with it, at
// that state of the kernel, 1.58).  With one block S has two buffers, and the next tile's Q K^T runs under the
// softmax.  Scores are read from tensor memory twice, half of a tile at a time, once for the maximum and once for
// the weights: 64 in registers, at 128 registers a thread, and little code (all roles share the instruction caches;
// all 128 scores held, with registers moved between warps, spilled and was no faster).
//
// Queries arrive and outputs leave as whole rows by bulk copies, and a warp transposes 32 of them between rows and
// core matrices in place along diagonals, without bank conflicts: 16-byte accesses by threads took 5000 clocks an item.
// Columns that a row does not see are overwritten in tensor memory, in the border tiles of an item alone.
//
// Rounding.  Codes - 128 are exact in FP16; BF16 queries are scaled by a power of two per row (exact
// down to 2^-39 of the row's largest).  The value scales enter the weights: P = p s_v / 2^e 2^10 with
// the running power of two 2^e above those of the pages that the row has seen, in FP16 (2^-11 relative, a BF16 output is
// rounded by 2^-8).  2^e is of the row, not of its block: what a row does not see changes no bit of its output.
// The row sum takes the unrounded p in FP32.  The reference R of the exponents is a maximum that may lag
// behind by 2^5.9 (2^10 2^5.9 is below the largest FP16), so that O is rescaled, from tensor memory and back,
// only where it moves by more.
//
// Measured (GPU alone).  That piece: 1.523 ms, 1.35 PFLOP/s, 71 % of a large BF16 matrix product.  A block's chain
// S, softmax, P V, Q K^T takes 3700 clocks a tile; the products of both blocks 2080 of them, the exponentials 1024
// per block.  16 rows of up to 1000 queries in up to 1500 tokens, 32 heads, 16 KV heads, window 512: 249 us, where an
// item is 6 tiles, 3 of them with borders, and 16 000 clocks of start and end.  61 rows of 5 queries in up to 2048
// tokens, 16 heads, 2 KV heads, d = 256: 44 us; 40 of 128 rows are used, a tile of 64 tokens is a chain of 2500 clocks.
#include "attend.cuh"
#include "prefill_tc.cuh"

#include <algorithm>

namespace damp {

static __device__ uint32_t g_status_attend_tc;

namespace {

constexpr int kAtThreads = 15 * 32;
constexpr uint32_t kAtCols = 512;
constexpr uint32_t kAtO = 256;  // S blocks at columns 0 and 128, O from here on
constexpr float kAtLag = 5.9f;  // 2^10 2^5.9 is below the largest FP16; half of the rescalings that 4 makes
// A score S (below 2^30) times its factor f is taken off the reference in one fused operation, and so is off by half a unit of
// the product: nothing below 2^20, but beyond FP16's range from 2^21 on.  Scores of rows with factors from kAtFar on become
// S f / kAtLeast, rounded, where they are; their factor then is kAtLeast, as it is of key scales of 0 (2^-20 at most).
constexpr float kAtFar = 9.765625e-4f;                 // 2^-10
constexpr float kAtLeast = 8.8817841970012523e-16f;    // 2^-50
constexpr float kAtMost = 1.5845632502852868e29f;      // 2^97: of f / kAtLeast, which leaves S finite
constexpr int kAtNotes = 8;
constexpr int kAtMaxPages = 4;  // of a key tile
constexpr int kAtNoScale = -1000;  // below every exponent field
constexpr float kAtLowest = -60.f;  // weights of value scales further below a row's unit: under 2^-54, 0 in FP16

struct AtNote {  // of a key tile: what the softmax needs of its pages
    float factor[kAtMaxPages];  // key scale
    float weight[kAtMaxPages];  // log2 of 2^10 times value scale over the tile's unit, a multiple of 2^-15
    int e[kAtMaxPages];         // exponent field of the power of two above the value scale; kAtNoScale for 0
    int top;                    // the largest e: the tile's unit
    int hidden;                 // bit i: page i is bad or missing
    float reach;                // the largest key scale
    int unused;
};

template <int D, int SUB>
struct AtSmem {
    static constexpr int tokens = D == 256 ? 64 : 128;  // of a key tile
    static constexpr int pages = tokens / kCachePage;
    static constexpr int q_tile = 128 * D * 2, tile = tokens * D * 2;
    static constexpr int buffers = 2;                 // of K and of V
    static constexpr int codes = tokens * D;          // of K or of V
    static constexpr int stages = D == 64 ? 4 : D == 128 && SUB == 1 ? 2 : 1;  // of codes
    static constexpr int q = 0, k = SUB * q_tile, v = k + buffers * tile;
    static constexpr int kc = v + buffers * tile, vc = kc + stages * codes;
    static constexpr int note = vc + stages * codes;
    static constexpr int bar = note + kAtNotes * (int)sizeof(AtNote);
    static constexpr int bytes = bar + 448;
    static constexpr int before = k;  // until the roles begin
    static_assert(SUB * q_tile + 4 * (kCacheMaxBatch + 1) <= kc, "before");
    static constexpr int sm_warps = 4 * SUB, turn_warps = 4;  // SUB = 1: four for K, four for V
};
// mbarriers
enum {
    kBarQ = 0, kBarDone = 2,  // of blocks of rows
    kBarKFull = 4, kBarKFree = 6, kBarVFull = 8, kBarVFree = 10,  // operands, two buffers
    kBarS = 12, kBarP = 14, kBarPV = 18,  // P: halves of two buffers
    kBarTurn = 19, kBarNote = 21,
    kBarKcFull = kBarNote + kAtNotes, kBarKcFree = kBarKcFull + 4, kBarVcFull = kBarKcFree + 4, kBarVcFree = kBarVcFull + 4,  // codes, up to 4 stages
    kBarRows = kBarVcFree + 4, kBarCount = kBarRows + 8  // of softmax warps
};
static_assert(kBarCount * 8 <= 448, "barriers");

// instruction descriptor: f16 x f16 -> FP32, M = 128, N columns, B MN-major if set
__host__ __device__ constexpr uint32_t at_idesc(int n, bool b_mn) {
    return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// Products are issued by a whole warp in step, one elected lane each, from descriptors whose words are
// in uniform registers (a reduction's result is).
__device__ __forceinline__ uint32_t at_uniform(uint32_t x) { return __reduce_max_sync(kFull, x); }
// four K steps: the descriptors' low words advance by a_step and b_step each
template <int A, int B>
__device__ __forceinline__ void at_mma4(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p, e;\n.reg .b64 da, db;\nelect.sync _|e, 0xffffffff;\nsetp.ne.u32 p, %6, 0;\n"
                 "mov.b64 da, {%1, %2};\nmov.b64 db, {%3, %4};\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n"
                 "add.s64 da, da, %7;\nadd.s64 db, db, %8;\nsetp.ne.u32 p, %5, 0;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n"
                 "add.s64 da, da, %7;\nadd.s64 db, db, %8;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n"
                 "add.s64 da, da, %7;\nadd.s64 db, db, %8;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n}" ::"r"(d),
                 "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc), "n"(A), "n"(B)
                 : "memory");
}
template <int A, int B>
__device__ __forceinline__ void at_mma4_ta(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p, e;\n.reg .b64 db;\n.reg .b32 ta;\nelect.sync _|e, 0xffffffff;\nsetp.ne.u32 p, %5, 0;\n"
                 "mov.b32 ta, %1;\nmov.b64 db, {%2, %3};\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], db, %4, p;\n"
                 "add.s32 ta, ta, %6;\nadd.s64 db, db, %7;\nsetp.ne.u32 p, %4, 0;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], db, %4, p;\n"
                 "add.s32 ta, ta, %6;\nadd.s64 db, db, %7;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], db, %4, p;\n"
                 "add.s32 ta, ta, %6;\nadd.s64 db, db, %7;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], db, %4, p;\n}" ::"r"(d),
                 "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc), "n"(A), "n"(B)
                 : "memory");
}
template <int A, int B>
__device__ __forceinline__ void at_mma2_ta(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p, e;\n.reg .b64 db;\n.reg .b32 ta;\nelect.sync _|e, 0xffffffff;\nsetp.ne.u32 p, %5, 0;\n"
                 "mov.b32 ta, %1;\nmov.b64 db, {%2, %3};\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], db, %4, p;\n"
                 "add.s32 ta, ta, %6;\nadd.s64 db, db, %7;\nsetp.ne.u32 p, %4, 0;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], db, %4, p;\n}" ::"r"(d),
                 "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc), "n"(A), "n"(B)
                 : "memory");
}
__device__ __forceinline__ void at_commit(uint32_t bar) {
    asm volatile("{\n.reg .pred e;\nelect.sync _|e, 0xffffffff;\n"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar)
                 : "memory");
}
__device__ __forceinline__ void at_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// 16 columns of a thread's lane, to be used after at_ld_wait on them
__device__ __forceinline__ void at_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void at_ld_wait(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ void at_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void at_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// An item of the sequence, the same in all lanes of a warp.
struct AtItem {
    int b, rt, h, first, pages, tiles, begin;
    AttRow row;
};
__device__ __forceinline__ void at_set(AtItem &it, const AttendArgs &p, int R, int unit) {
    const AttItem x = att_item(p, it.row, it.rt, R);
    it.first = x.first;
    it.pages = x.pages;
    it.tiles = att_units(x.pages, unit);
}
// the item that unit x < total lies in
__device__ __forceinline__ AtItem at_seek(const AttendArgs &p, const int32_t *before, int x, int R, int unit) {
    AtItem it;
    int lo = 0, hi = p.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] * p.Hk <= x) lo = mid;
        else hi = mid;
    }
    it.b = lo;
    it.row = att_row(p, lo);
    int at = before[lo] * p.Hk;
    it.rt = 0;
    const int lane = threadIdx.x & 31;
    for (;; it.rt += 32) {  // 32 tiles of rows at a time
        const int rt = it.rt + lane;
        int n = rt < att_tiles(it.row.n, R, p.group) ? att_units(att_item(p, it.row, rt, R).pages, unit) * p.Hk : 0;
        int sum = n;
#pragma unroll
        for (int i = 1; i < 32; i <<= 1) {
            const int y = __shfl_up_sync(kFull, sum, i);
            if (lane >= i) sum += y;
        }
        const unsigned past = __ballot_sync(kFull, at + sum > x);
        if (past) {
            const int l = __ffs(past) - 1;
            it.rt += l;
            at += __shfl_sync(kFull, sum - n, l);
            break;
        }
        at += __shfl_sync(kFull, sum, 31);
        if (it.rt > att_tiles(it.row.n, R, p.group)) break;  // (not reached: x lies in this row)
    }
    at_set(it, p, R, unit);
    it.h = it.tiles ? (x - at) / it.tiles : 0;
    it.begin = at + it.h * it.tiles;
    return it;
}
// the item after `it`, given that there is one
__device__ __forceinline__ void at_next(AtItem &it, const AttendArgs &p, int R, int unit) {
    it.begin += it.tiles;
    if (++it.h < p.Hk) return;
    it.h = 0;
    do {
        if (++it.rt * R >= it.row.n * p.group) {
            it.rt = 0;
            if (++it.b >= p.batch) return;
            it.row = att_row(p, it.b);
        }
        at_set(it, p, R, unit);
    } while (it.tiles == 0);
}

// suspended for up to a millisecond at a time, so that a waiting warp leaves the issue slots to others
__device__ __forceinline__ bool at_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity), "r"(1000000u)
                 : "memory");
    return ok != 0;
}
template <bool TEST>
struct AtWait {  // bounded waits, all of which give up once one has
    volatile uint32_t *dead;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
        if (at_try_wait(bar, parity)) return true;
        const uint64_t t0 = global_timer_ns();
        for (uint32_t i = 0; !at_try_wait(bar, parity); ++i) {
            if (*dead || global_timer_ns() - t0 > kAttWait<TEST> || i >> 27) {
                *dead = 1;
                return false;
            }
        }
        return true;
    }
};

// What a CTA whose waits have run out does at its end (not inlined: the other code stays as it is).  Copies in flight end
// before the shared memory does; the join finds no part of an item that this range should have left, and makes NaN of it.
template <int STAGES>
__device__ __noinline__ void at_lost(uint32_t *status, float2 *ml, int n, uint32_t rows_bar, uint32_t rows, uint32_t kc_bar, uint32_t vc_bar, uint32_t copied, uint32_t half, uint64_t limit) {
    if (threadIdx.x == 0) atomicOr(status, kDevWaitTimeout);
    if (rows) mbar_wait_bounded(rows_bar, rows - 1, limit);
    for (uint32_t k = copied > STAGES ? copied - STAGES : 0; k < copied + half; ++k) {
        mbar_wait_bounded(kc_bar + 8 * (k % STAGES), (k / STAGES) & 1, limit);
        if (k < copied) mbar_wait_bounded(vc_bar + 8 * (k % STAGES), (k / STAGES) & 1, limit);
    }
    for (int i = threadIdx.x; i < n; i += kAtThreads) ml[i] = make_float2(NAN, NAN);
}

template <int D, int SUB, bool TEST>
__global__ void __launch_bounds__(kAtThreads, 1) attend_tc_kernel(const AttendArgs p) {
    using M = AtSmem<D, SUB>;
    constexpr int R = 128 * SUB, TN = M::tokens, PG = M::pages;
    extern __shared__ __align__(1024) uint8_t sm[];
    __shared__ uint32_t s_dead, s_tmem, s_copied, s_half;  // tiles of codes that were copied, the keys of one more
    __shared__ uint32_t s_rows[4 * SUB];  // 1 + the phase of a softmax warp's queries that it has given up
    __shared__ AtItem s_next[4 * SUB];  // a softmax warp's next item, kept out of its registers
    const uint32_t sb = smem_u32(sm);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.group;
    auto bar = [&](int i) { return sb + M::bar + 8 * i; };
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the join waits for the end of this grid itself
    if (threadIdx.x == 0) {
        s_dead = s_half = s_copied = 0;
        for (int i = 0; i < 4 * SUB; ++i) s_rows[i] = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(kBarQ + i), 4);
            mbar_init(bar(kBarDone + i), 1);
            mbar_init(bar(kBarKFull + i), M::turn_warps);
            mbar_init(bar(kBarKFree + i), SUB);
            mbar_init(bar(kBarVFull + i), M::turn_warps);
            mbar_init(bar(kBarVFree + i), SUB);
            mbar_init(bar(kBarTurn + i), 1);
            mbar_init(bar(kBarS + i), 1);
            mbar_init(bar(kBarP + 2 * i), 4);
            mbar_init(bar(kBarP + 2 * i + 1), 4);
        }
        mbar_init(bar(kBarPV), 1);
        for (int i = 0; i < M::sm_warps; ++i) mbar_init(bar(kBarRows + i), 1);
        for (int i = 0; i < kAtNotes; ++i) mbar_init(bar(kBarNote + i), 1);
        for (int i = 0; i < M::stages; ++i) {
            mbar_init(bar(kBarKcFull + i), 1);
            mbar_init(bar(kBarKcFree + i), M::turn_warps);
            mbar_init(bar(kBarVcFull + i), 1);
            mbar_init(bar(kBarVcFree + i), M::turn_warps);
        }
        fence_mbar_init();
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kAtCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    int32_t *const before = reinterpret_cast<int32_t *>(sm + M::before);
    att_count(p, R, PG, before);  // (synchronizes)
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    const AttWork work = att_work(p.workspace, gridDim.x, R);
    const int total = before[p.batch] * p.Hk, per = att_per(total, gridDim.x);
    int end = (int)min((int64_t)total, ((int64_t)blockIdx.x + 1) * per);
    int begin = (int)min((int64_t)end, (int64_t)blockIdx.x * per);
    AtItem it{};
    if (p.whole) {  // the range takes the items that start in it, all of them
        if (end < total) {
            it = at_seek(p, before, end, R, PG);
            if (it.begin < end) end = it.begin + it.tiles;
        }
        if (begin < total && begin > 0) {
            it = at_seek(p, before, begin, R, PG);
            if (it.begin < begin) begin = it.begin + it.tiles;
        }
        const int slice = att_clear_slice(p.H, D, 2), blocks = p.batch * ((p.T + slice - 1) / slice);
        for (int i = blockIdx.x; i < blocks; i += gridDim.x) att_clear<D, true>(p, i, slice);
    }
    if (begin < end) it = at_seek(p, before, begin, R, PG);
    __syncthreads();  // `before` is given up
    const AtWait<TEST> wait{&s_dead};
    auto together = [](bool ok) { return __all_sync(kFull, ok) != 0; };
    const uint32_t n_tiles = (uint32_t)(end - begin);  // of this range
    AttSplit split{0, 0, 0, -1, 0, {0, 0, 0}};  // (thread 0)

    if (begin < end && warp < M::sm_warps) {
        // ---- softmax: thread = row of a block ----
        const int x = warp >> 2;            // block of rows
        const int row = threadIdx.x & 127;  // in the block: the lane of tensor memory
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t o_at = lanes + kAtO + x * D;
        // Rows move between global and shared memory 8 at a time, 4 chunks of 16 bytes each: lane = (row, chunk);
        // in shared memory a chunk of 8 rows is a core matrix.
        const uint32_t stage = sb + M::q + x * M::q_tile + (warp & 3) * (64 * D) + (lane & 7) * 16 + (lane >> 3) * 128;
        const uint32_t stage_row = sb + M::q + x * M::q_tile + (row >> 3) * (16 * D) + (row & 7) * 16;
        uint32_t tile = 0, items = 0;
        bool ok = true;
        constexpr int kC = D / 32;  // chunks of a lane in 8 rows
        for (int at = begin; at < end && ok; ++items) {
            if (items) it = s_next[warp];
            const int last = min(end, it.begin + it.tiles);
            const int r = it.rt * R + x * 128 + row, t = att_div(p, r);
            const bool live = t < it.row.n;
            const int limit = live ? it.row.len - it.row.n + t : INT_MAX / 2;  // (what rows of no query hold is not used)
            const int from = p.window && live ? limit - (p.window - 1) : 0;
            const int head = it.h * G + (r - t * G);
            float factor = 0.f;
            {  // q: copied as it is to where its rows go, then scaled by a power of two to below 2^15, 8 rows at a time
                const int64_t mine = live ? ((int64_t)it.b * p.T + t) * p.q_stride + (int64_t)head * D : -1;
                const uint32_t q_bar = bar(kBarRows + warp), rows = sb + M::q + x * M::q_tile + (warp & 3) * (64 * D);
                const unsigned some = __ballot_sync(kFull, live);
                if (lane == 0) mbar_arrive_expect_tx(q_bar, __popc(some) * 2 * D + att_extra<TEST>(p, blockIdx.x, 2));
                __syncwarp();
                if (live) {
                    fence_proxy_async_smem();  // (the item before was staged here)
                    bulk_g2s(rows + lane * 2 * D, static_cast<const __nv_bfloat16 *>(p.q) + mine, 2 * D, q_bar);
                }
                if (last < end) {  // the next item is found and its queries brought into L2 meanwhile
                    AtItem next = it;
                    at_next(next, p, R, PG);
                    __syncwarp();
                    if (lane == 0) s_next[warp] = next;
                    __syncwarp();
                    const int r2 = next.rt * R + x * 128 + row, t2 = att_div(p, r2);
                    if (t2 < next.row.n) {
                        const __nv_bfloat16 *const q = static_cast<const __nv_bfloat16 *>(p.q) + ((int64_t)next.b * p.T + t2) * p.q_stride + (int64_t)(next.h * G + r2 - t2 * G) * D;
#pragma unroll
                        for (int i = 0; i < D; i += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + i));
                    }
                }
                ok = together(wait(q_bar, items & 1));
                if (!ok) {
                    if (lane == 0) s_rows[warp] = 1 + (items & 1);
                    break;
                }
#pragma unroll 1
                for (int g = 0; g < 4; ++g) {
                    // From rows to core matrices in the same 16 D bytes.  Lane = (row j, b = 4 i + its quarter): chunk
                    // (b & ~7) | ((b + j) & 7), so that eight lanes touch eight 16-byte columns on either side.
                    uint4 v[kC];
                    const int j = lane & 7;
                    const bool there = (some >> (8 * g + j)) & 1;
#pragma unroll
                    for (int i = 0; i < kC; ++i) {
                        const int b = 4 * i + (lane >> 3), chunk = (b & ~7) | ((b + j) & 7);
                        v[i] = there ? lds128(rows + (8 * g + j) * 2 * D + chunk * 16) : make_uint4(0, 0, 0, 0);
                    }
                    __syncwarp();
                    uint32_t top = 0;  // largest magnitudes of both halves of the words
#pragma unroll
                    for (int i = 0; i < kC; ++i)
                        top = __vmaxu2(__vmaxu2(__vmaxu2(top, v[i].x & 0x7fff7fffu), __vmaxu2(v[i].y & 0x7fff7fffu, v[i].z & 0x7fff7fffu)), v[i].w & 0x7fff7fffu);
                    top = __vmaxu2(top, __shfl_xor_sync(kFull, top, 8));
                    top = __vmaxu2(top, __shfl_xor_sync(kFull, top, 16));
                    const int e = min(max((int)(max(top >> 16, top & 0xffffu) >> 7), 15), 254);
                    const float up = __uint_as_float((uint32_t)(268 - e) << 23);
                    if ((lane >> 3) == g) factor = p.scale * (kLog2e * __uint_as_float((uint32_t)(e - 14) << 23));  // over up, of this thread's own row
#pragma unroll
                    for (int i = 0; i < kC; ++i) {
                        const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                        uint32_t h[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            h[k] = half_pair(__uint_as_float(u[k] << 16) * up, __uint_as_float(u[k] & 0xffff0000u) * up);
                        const int b = 4 * i + (lane >> 3), chunk = (b & ~7) | ((b + j) & 7);
                        sts128(rows + g * (16 * D) + chunk * 128 + j * 16, make_uint4(h[0], h[1], h[2], h[3]));
                    }
                }
            }
            fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) at_arrive(bar(kBarQ + x));
            float ref = -INFINITY, sum = 0.f;
            int ve = 1;  // exponent field of the row's unit: above the value scales of the pages that it has seen
            const int first_tile = at - it.begin;
            for (; at < last; ++at, ++tile) {
                const int sbuf = SUB == 2 ? x : tile & 1;
                const uint32_t s_at = lanes + sbuf * 128;
                ok = wait(bar(kBarNote + tile % kAtNotes), (tile / kAtNotes) & 1);
                const AtNote *const note = reinterpret_cast<const AtNote *>(sm + M::note) + tile % kAtNotes;
                const int i = at - it.begin;
                const int token = (it.first + i * PG) * kCachePage;  // of column 0
                const int4 about = *reinterpret_cast<const int4 *>(&note->top);  // top, hidden, reach
                const int hidden = about.y;
                int e = max(ve, about.x);
                bool far = factor * __int_as_float(about.z) >= kAtFar;
                ok = together(ok && wait(bar(kBarS + sbuf), (SUB == 2 ? tile : tile >> 1) & 1));
                if (!ok) break;
                tc_fence_after();
                if (__any_sync(kFull, hidden != 0 || limit < token + TN - 1 || from > token || far)) {
                    // A page that a row does not see leaves its unit and its products as they are.
                    auto sees = [&](int c) { return limit >= token + kCachePage * c && from < token + kCachePage * (c + 1); };
                    e = ve;
#pragma unroll
                    for (int c = 0; c < PG; ++c)
                        if (sees(c)) e = max(e, note->e[c]);
                    if (__any_sync(kFull, far)) {
                        far = false;
#pragma unroll 1
                        for (int c = 0; c < PG; ++c) far = far || (sees(c) && factor * note->factor[c] >= kAtFar);
                        const float up = far ? factor * (1.f / kAtLeast) : 0.f;
#pragma unroll 1
                        for (int c = 0; c < 2 * PG; ++c) {
                            const float f = far ? fminf(up * note->factor[c >> 1], kAtMost) : 1.f;
                            uint32_t y[16];
                            at_ld16(s_at + 16 * c, y);
                            at_ld_wait(y);
#pragma unroll
                            for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * f);
                            at_st16(s_at + 16 * c, y);
                        }
                        at_st_wait();
                    }
                    // Columns that a row does not see become -inf where they are, 16 at a time (of the border tiles of an item
                    // only: a small loop, for the instruction caches' sake, which all roles share).
#pragma unroll 1
                    for (int c = 0; c < 2 * PG; ++c) {
                        const int lo = from - (token + 16 * c), hi = limit - (token + 16 * c);  // sees lo .. hi
                        const bool all = (hidden >> (c >> 1)) & 1;
                        if (!all && !__any_sync(kFull, lo > 0 || hi < 15)) continue;
                        const uint32_t seen = hi < 0 || lo > 15 || all ? 0u : (0xffffu >> (15 - min(hi, 15))) & (0xffffu << max(lo, 0));
                        uint32_t y[16];
                        at_ld16(s_at + 16 * c, y);
                        at_ld_wait(y);
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (!(seen & (1u << j))) y[j] = 0xff800000u;
                        at_st16(s_at + 16 * c, y);
                    }
                    at_st_wait();
                }
                const float over = (float)(about.x - e);  // the tile's unit over the row's
                const float near = far ? 0.f : factor;
                // Half of the columns at a time, in loops: registers hold 64 scores, and the code stays small (the
                // instruction caches are shared by all roles).
                float top = -INFINITY;
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint32_t s[PG][16];
                    float f[PG / 2];  // while the scores are on their way
#pragma unroll
                    for (int c = 0; c < PG / 2; ++c) f[c] = fmaxf(near * note->factor[h * (PG / 2) + c], kAtLeast);  // not 0: times a hidden -inf
#pragma unroll
                    for (int c = 0; c < PG; ++c) at_ld16(s_at + (16 * PG) * h + 16 * c, s[c]);
#pragma unroll
                    for (int c = 0; c < PG; ++c) at_ld_wait(s[c]);
#pragma unroll
                    for (int c = 0; c < PG / 2; ++c) {
                        float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int j = 0; j < 32; j += 2)
                            m[(j >> 1) & 3] = fmax3(m[(j >> 1) & 3], __uint_as_float(s[2 * c + (j >> 4)][j & 15]), __uint_as_float(s[2 * c + (j >> 4)][(j & 15) + 1]));
                        top = fmaxf(top, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) * f[c]);
                    }
                }
                const bool moves = top > ref + kAtLag;
                const float ref_new = moves ? top : ref;
                float corr = moves ? ex2(ref - ref_new) : 1.f;
                sum *= corr;
                ref = ref_new;
                if (e != ve) {
                    const int shift = 127 + ve - e;
                    corr *= shift > 0 ? __uint_as_float((uint32_t)shift << 23) : 0.f;
                }
                if (i != first_tile && __any_sync(kFull, moves || e != ve)) {
                    if (SUB == 1) {  // the last product into O may still run
                        ok = together(wait(bar(kBarPV), (tile - 1) & 1));
                        if (!ok) break;
                        tc_fence_after();
                    }
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t y[2][16];
                        at_ld16(o_at + 32 * c, y[0]);
                        at_ld16(o_at + 32 * c + 16, y[1]);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            at_ld_wait(y[k]);
#pragma unroll
                            for (int j = 0; j < 16; ++j) y[k][j] = __float_as_uint(__uint_as_float(y[k][j]) * corr);
                            at_st16(o_at + 32 * c + 16 * k, y[k]);
                        }
                    }
                }
                ve = e;
                const float base = ref == -INFINITY ? 0.f : -ref;
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint32_t s[PG][16];
                    float f[PG / 2], weight[PG / 2], a[PG / 2];  // while the scores are on their way
#pragma unroll
                    for (int c = 0; c < PG / 2; ++c) {
                        f[c] = fmaxf(near * note->factor[h * (PG / 2) + c], kAtLeast);
                        weight[c] = fmaxf(over + note->weight[h * (PG / 2) + c], kAtLowest);  // (exact)
                        a[c] = __fadd_rd(base, weight[c]);  // (to the nearest, 10 could become 16)
                    }
#pragma unroll
                    for (int c = 0; c < PG; ++c) at_ld16(s_at + (16 * PG) * h + 16 * c, s[c]);
#pragma unroll
                    for (int c = 0; c < PG; ++c) at_ld_wait(s[c]);
#pragma unroll
                    for (int c = 0; c < PG / 2; ++c) {
                        const int page = h * (PG / 2) + c;
                        const float2 f2 = splat2(f[c]), a2 = splat2(a[c]);
                        float2 z[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            z[j] = fma2(make_float2(__uint_as_float(s[2 * c + (j >> 3)][2 * (j & 7)]), __uint_as_float(s[2 * c + (j >> 3)][2 * (j & 7) + 1])), f2, a2);
                        float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                        uint32_t w[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] = make_float2(ex2(z[j].x), ex2(z[j].y));
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            part[j & 1] = add2(part[j & 1], z[j]);
                            w[j] = half_pair(z[j].x, z[j].y);
                        }
                        at_st16(s_at + 16 * page, w);
                        const float2 both = add2(part[0], part[1]);
                        sum = fmaf(both.x + both.y, ex2(-weight[c]), sum);
                    }
                    at_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) at_arrive(bar(kBarP + 2 * sbuf + h));
                }
            }
            if (!ok) break;
            const bool whole = it.begin >= begin && it.begin + it.tiles <= end, starts = it.begin >= begin;
            const int64_t mine = live ? (((int64_t)it.b * p.T + t) * p.H + head) * D : -1;
            if (threadIdx.x == 0 && starts && !whole)
                split = AttSplit{it.b, it.rt, it.h, (it.begin + it.tiles - 1) / per, min(R, it.row.n * G - it.rt * R), {0, 0, 0}};
            ok = together(wait(bar(kBarDone + x), items & 1));  // the item's products into O
            if (!ok) break;
            tc_fence_after();
            const float unit = __uint_as_float((uint32_t)ve << 23) * (1.f / 1024.f);
            if (whole) {
                const float y = sum == 0.f ? 0.f : unit / sum;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[2][16];
                    at_ld16(o_at + 32 * c, o[0]);
                    at_ld16(o_at + 32 * c + 16, o[1]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if ((k & 1) == 0) at_ld_wait(o[k >> 1]);
                        uint32_t h[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const __nv_bfloat162 z = __floats2bfloat162_rn(__uint_as_float(o[k >> 1][8 * (k & 1) + 2 * j]) * y,
                                                                           __uint_as_float(o[k >> 1][8 * (k & 1) + 2 * j + 1]) * y);
                            memcpy(&h[j], &z, 4);
                        }
                        sts128(stage_row + (4 * c + k) * 128, make_uint4(h[0], h[1], h[2], h[3]));
                    }
                }
                __syncwarp();
                // core matrices to rows, as the queries came, and the rows out
                const uint32_t rows = sb + M::q + x * M::q_tile + (warp & 3) * (64 * D);
#pragma unroll 1
                for (int g = 0; g < 4; ++g) {
                    uint4 v[kC];
                    const int j = lane & 7;
#pragma unroll
                    for (int i = 0; i < kC; ++i) {
                        const int b = 4 * i + (lane >> 3), chunk = (b & ~7) | ((b + j) & 7);
                        v[i] = lds128(rows + g * (16 * D) + chunk * 128 + j * 16);
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < kC; ++i) {
                        const int b = 4 * i + (lane >> 3), chunk = (b & ~7) | ((b + j) & 7);
                        sts128(rows + (8 * g + j) * 2 * D + chunk * 16, v[i]);
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (live) {
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(static_cast<__nv_bfloat16 *>(p.o) + mine), "r"(rows + lane * 2 * D), "r"(2 * D) : "memory");
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                }
                __syncwarp();
            } else {
                const int64_t slot = (int64_t)(2 * blockIdx.x + (starts ? 1 : 0)) * R + x * 128 + row;
                if (live) work.ml[slot] = make_float2(ref, sum);
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[2][16];
                    at_ld16(o_at + 32 * c, o[0]);
                    at_ld16(o_at + 32 * c + 16, o[1]);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        at_ld_wait(o[k]);
                        float z[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] = __uint_as_float(o[k][j]) * unit;
                        if (live) store_out<false, 16>(work.o + slot * D, 32 * c + 16 * k, z);
                    }
                }
            }
            tc_fence_before();
        }
    } else if (begin < end && warp < 12) {
        // ---- codes into operands: by four warps, with one block of rows by four for K and four for V ----
        constexpr int kQuads = D / 64;                             // 4 chunks of 16 codes
        constexpr int kUnits = (TN / 8) * kQuads / M::turn_warps;  // of 8 tokens x 4 chunks, of a warp
        const int w = (warp - M::sm_warps) & 3;
        const bool keys = SUB == 2 || warp < 8, values = SUB == 2 || warp >= 8;
        const int tok = lane & 7, mi = lane >> 3;
        auto turn = [&](uint32_t from, uint32_t free, uint32_t to, uint32_t to_free, bool wait_free, uint32_t parity, uint32_t full) {
            uint4 c[kUnits];
#pragma unroll
            for (int j = 0; j < kUnits; ++j) {
                const int u = w + j * M::turn_warps, tg = u / kQuads, mq = u % kQuads;
                c[j] = lds128(from + tg * 8 * D + cache_chunk(tok, mq * 4 + mi, D));
            }
            __syncwarp();
            if (lane == 0) at_arrive(free);
            if (wait_free && !together(wait(to_free, parity))) return false;
#pragma unroll
            for (int j = 0; j < kUnits; ++j) {
                const int u = w + j * M::turn_warps, tg = u / kQuads, mq = u % kQuads;
                const uint32_t at = to + tg * (16 * D) + (mq * 4 + mi) * 256 + tok * 16;
                sts128(at, make_uint4(half_codes(c[j].x, 0x4140u), half_codes(c[j].x, 0x4342u), half_codes(c[j].y, 0x4140u), half_codes(c[j].y, 0x4342u)));
                sts128(at + 128, make_uint4(half_codes(c[j].z, 0x4140u), half_codes(c[j].z, 0x4342u), half_codes(c[j].w, 0x4140u), half_codes(c[j].w, 0x4342u)));
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) at_arrive(full);
            return true;
        };
        for (uint32_t i = 0; i < n_tiles; ++i) {
            const uint32_t buf = i & 1, use = i >> 1;
            const uint32_t st = i % M::stages, lap = i / M::stages;
            if (keys && !(together(wait(bar(kBarKcFull + st), lap & 1)) &&
                          turn(sb + M::kc + st * M::codes, bar(kBarKcFree + st), sb + M::k + buf * M::tile, bar(kBarKFree + buf), use != 0,
                               (use - 1) & 1, bar(kBarKFull + buf))))
                break;
            if (values && !(together(wait(bar(kBarVcFull + st), lap & 1)) &&
                            turn(sb + M::vc + st * M::codes, bar(kBarVcFree + st), sb + M::v + buf * M::tile, bar(kBarVFree + buf), use != 0,
                                 (use - 1) & 1, bar(kBarVFull + buf))))
                break;
        }
    } else if (begin < end) {
        if (warp == 14) {
        // ---- the pages' copies, and what the softmax needs of them: lane = page of a tile ----
        bool there_next;  // lane is a page of the tile
        auto entry = [&](int x) {  // of tile x, which lies in `it`
            const int i = (x - it.begin) * PG + lane;
            there_next = lane < PG && i < it.pages;
            return there_next ? p.pages[(int64_t)it.b * p.table + it.first + i] : -1;
        };
        int32_t next = entry(begin);
        int h_next = it.h;
        uint32_t i = 0;
        bool ok = true;
        for (; i < n_tiles; ++i) {
            const int32_t e = next;
            const int h = h_next;
            const bool there = there_next;
            if (i + 1 < n_tiles) {
                const int x = begin + (int)i + 1;
                if (x >= it.begin + it.tiles) {
                    at_next(it, p, R, PG);
                    h_next = it.h;
                }
                next = entry(x);
            }
            const int64_t slot = cache_page(e, p.num_pages);
            const uint8_t *const record = p.pool + (slot * p.Hk + h) * cache_record_bytes(D);
            if (there && slot < 0) atomicOr(p.status, kDevBadSlot);
            const bool here = there && slot >= 0;
            const unsigned shown = __ballot_sync(kFull, here);
            float2 scales = make_float2(0.f, 0.f);
            if (here) scales = *reinterpret_cast<const float2 *>(record + 2 * cache_rows_bytes(D));
            const uint32_t st = i % M::stages, lap = i / M::stages;
            const uint32_t bytes = __popc(shown) * cache_rows_bytes(D) + att_extra<TEST>(p, blockIdx.x, 1);
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const uint32_t full = bar((which ? kBarVcFull : kBarKcFull) + st);
                if (lap) ok = together(wait(bar((which ? kBarVcFree : kBarKcFree) + st), (lap - 1) & 1));
                if (!ok) {
                    if (lane == 0) s_half = which;
                    break;
                }
                if (lane == 0) mbar_arrive_expect_tx(full, bytes);
                __syncwarp();
                if (here) {
                    fence_proxy_async_smem();
                    bulk_g2s(sb + (which ? M::vc : M::kc) + st * M::codes + lane * cache_rows_bytes(D), record + which * cache_rows_bytes(D),
                             cache_rows_bytes(D), full);
                }
            }
            if (!ok) break;
            AtNote *const note = reinterpret_cast<AtNote *>(sm + M::note) + i % kAtNotes;
            // A scale of 0 stands for zeros whatever the codes are: scores of 0 (times kAtLeast in the softmax, so that hidden
            // columns stay -inf), weights that are 0 in FP16 (at kAtLowest) but count in the sum.
            const int ve = scales.y > 0.f ? (int)min((__float_as_uint(scales.y) >> 23) + 1u, 253u) : kAtNoScale;
            const int top = __reduce_max_sync(kFull, ve);
            const uint32_t reach = __reduce_max_sync(kFull, __float_as_uint(fmaxf(scales.x, 0.f)));  // not negative: ordered as integers
            if (lane < PG) {
                const float m = scales.y > 0.f ? __log2f(scales.y * __uint_as_float((uint32_t)(254 - ve) << 23)) : 0.f;
                note->factor[lane] = scales.x;
                note->weight[lane] = rintf(m * 32768.f) * (1.f / 32768.f) + (float)(10 + ve - top);
                note->e[lane] = ve;
            }
            if (lane == 0) {
                note->top = top;
                note->reach = __uint_as_float(reach);
                note->hidden = (int)(~shown & ((1u << PG) - 1u));
            }
            __syncwarp();
            if (lane == 0) at_arrive(bar(kBarNote + i % kAtNotes));
        }
        if (lane == 0) s_copied = i;
        } else if (warp - 12 < SUB) {
        // ---- the products: a warp per block of rows; with two blocks they take turns, a tile's P V and the next tile's
        // Q K^T at a time, so that one block's softmax runs under the other's products ----
        constexpr uint32_t kIdS = at_idesc(TN, false), kIdO = at_idesc(D, true);
        const int x = warp - 12;
        auto key_buf = [&](uint32_t t) { return t & 1u; };
        auto key_use = [&](uint32_t t) { return (t >> 1) & 1u; };
        const uint64_t dq = tc_desc(sb + M::q + x * M::q_tile, 128, 16 * D), dk = tc_desc(sb + M::k, 128, 16 * D), dv = tc_desc(sb + M::v, 16 * D, 128);
        const uint32_t q_lo = at_uniform((uint32_t)dq), k_lo = at_uniform((uint32_t)dk), v_lo = at_uniform((uint32_t)dv);
        const uint32_t k_hi = at_uniform((uint32_t)(dk >> 32)), v_hi = at_uniform((uint32_t)(dv >> 32)), tm = at_uniform(tmem);
        const uint32_t tm_o = at_uniform(tmem + kAtO + x * D);
        auto s_buf = [&](uint32_t t) { return SUB == 2 ? (uint32_t)x : t & 1u; };
        auto s_use = [&](uint32_t t) { return (SUB == 2 ? t : t >> 1) & 1u; };
        auto scores = [&](uint32_t t) {  // S = Q_x K_t^T
            const uint32_t d = tm + 128 * at_uniform(s_buf(t)), b = k_lo + at_uniform(key_buf(t)) * (M::tile >> 4);
#pragma unroll 1
            for (int k = 0; k < D / 16; k += 4) at_mma4<16, 16>(d, q_lo + 16 * k, k_hi, b + 16 * k, k_hi, kIdS, k != 0);
            at_commit(bar(kBarS + s_buf(t)));
            at_commit(bar(kBarKFree + key_buf(t)));
        };
        auto keys = [&](uint32_t t) { return wait(bar(kBarKFull + key_buf(t)), key_use(t)); };
        uint32_t items = 0;
        bool ok = together(wait(bar(kBarQ + x), 0) && keys(0)), first = true;
        if (ok) {
            tc_fence_after();
            scores(0);
        }
        for (uint32_t t = 0; t < n_tiles && ok; ++t) {
            const bool more = t + 1 < n_tiles;
            const bool last = begin + (int)t + 1 == min(end, it.begin + it.tiles);  // of the item
            ok = (last || keys(t + 1)) && wait(bar(kBarVFull + key_buf(t)), key_use(t));
            if (SUB == 2) ok = ok && (x ? wait(bar(kBarTurn), t & 1) : t == 0 || wait(bar(kBarTurn + 1), (t - 1) & 1));
            if (SUB == 1 && !last) {
                if (!together(ok)) break;
                tc_fence_after();
                scores(t + 1);
            }
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {  // O_x += P V_t, half of the tokens
                ok = together(ok && wait(bar(kBarP + 2 * s_buf(t) + half), s_use(t)));
                if (!ok) break;
                tc_fence_after();
                constexpr int kSteps = TN / 32;
                const uint32_t h = at_uniform(half);
                const uint32_t a = tm + 128 * at_uniform(s_buf(t)) + 8 * kSteps * h;
                const uint32_t b = v_lo + at_uniform(key_buf(t)) * (M::tile >> 4) + 2 * D * kSteps * h;
                const uint32_t add = at_uniform(first && half == 0 ? 0u : 1u);
                if constexpr (kSteps == 4)
                    at_mma4_ta<8, 2 * D>(tm_o, a, b, v_hi, kIdO, add);
                else
                    at_mma2_ta<8, 2 * D>(tm_o, a, b, v_hi, kIdO, add);
            }
            if (!ok) break;
            if (SUB == 2 && !last) scores(t + 1);
            at_commit(bar(kBarVFree + key_buf(t)));
            if (SUB == 1) at_commit(bar(kBarPV));
            if (last) at_commit(bar(kBarDone + x));
            if (SUB == 2 && lane == 0) at_arrive(bar(kBarTurn + x));
            first = last;
            if (last && more) {
                at_next(it, p, R, PG);
                ++items;
                ok = together(wait(bar(kBarQ + x), items & 1) && keys(t + 1));
                if (!ok) break;
                tc_fence_after();
                scores(t + 1);
            }
        }
        if (!ok)  // what was issued ends by itself; no other product is issued
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
    }
    if (threadIdx.x == 0 && !p.whole) work.split[blockIdx.x] = split;  // (a range starts one such item at most, its last)
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (s_dead)
        at_lost<M::stages>(p.status, att_work(p.workspace, gridDim.x, R).ml + (int64_t)2 * blockIdx.x * R, p.whole ? 0 : 2 * R, bar(kBarRows + warp),
                           warp < M::sm_warps ? s_rows[warp] : 0, bar(kBarKcFull), bar(kBarVcFull), warp == 14 ? s_copied : 0, warp == 14 ? s_half : 0,
                           kAttWait<TEST>);
    if (warp == 12)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kAtCols) : "memory");
}

template <int D, int SUB, bool TEST>
cudaError_t launch_tc(const AttendArgs &a, int grid, cudaStream_t s) {
    using M = AtSmem<D, SUB>;
    const int smem = M::bytes;
    const cudaError_t e = ensure_smem_limit(reinterpret_cast<const void *>(attend_tc_kernel<D, SUB, TEST>), smem);
    if (e != cudaSuccess) return e;
    attend_tc_kernel<D, SUB, TEST><<<grid, kAtThreads, smem, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

bool attend_tc_takes(const AttendArgs &a) { return a.in_bf16 && (int64_t)a.T * (a.H / a.Hk) > 16; }

int attend_tc_rows(const AttendArgs &a) { return a.d <= 128 && (int64_t)a.T * (a.H / a.Hk) > 128 ? 256 : 128; }

// Ranges end with items, no parts and one launch, where no item can be long: 4 key tiles, or twice as many as there are
// items per SM (8 at least), so that the longest adds little to what an SM has anyway.  The lengths are not known here: a
// table's width and the window bound an item.  Whole items against parts, even lengths and ragged ones, us: 16 rows of
// 1000 queries, 32 heads, 16 KV, window 512 273 / 328 and 278 / 338; 10 of 256 in 1000 tokens 65 / 66 and 71 / 73;
// 320 of 5 in 1000, 32 heads, 8 KV 265 / 252 and 269 / 250, in 4000 822 / 562 and 840 / 543; but 256 rows of 5, one in
// 131072 tokens and the others in 1000: 1376 and 329.  256 rows of 5 in 1000 tokens each under a table of 4096 pages, which
// could hold such a row, pay for it: 222 and 244.
bool attend_tc_whole(const AttendArgs &a) {
    const int64_t G = a.H / a.Hk, R = attend_tc_rows(a), items = (int64_t)a.batch * (((int64_t)a.T * G + R - 1) / R) * a.Hk;
    const int64_t keys = a.window ? (int64_t)a.window + R / G + 1 : 32 * (int64_t)a.table;  // of an item
    const int64_t tile = a.d == 256 ? 2 : 4, pages = std::min<int64_t>(a.table, (keys + kCachePage - 2) / kCachePage + 1);
    const int64_t tiles = (pages + tile - 1) / tile;
    return tiles <= 4 || (items >= 8 * (int64_t)sm_count() && tiles * sm_count() <= 2 * items);
}

cudaError_t launch_attend_tc(AttendArgs a, int grid, cudaStream_t s) {
    a.whole = attend_tc_whole(a);
    static std::atomic<uint32_t *> cache[64];
    const cudaError_t e = symbol_address_cached(&g_status_attend_tc, cache, &a.status);
    if (e != cudaSuccess) return e;
    const bool two = attend_tc_rows(a) == 256;
    if (a.test) return a.d != 128 ? cudaErrorNotSupported : two ? launch_tc<128, 2, true>(a, grid, s) : launch_tc<128, 1, true>(a, grid, s);
    if (a.d == 64) return two ? launch_tc<64, 2, false>(a, grid, s) : launch_tc<64, 1, false>(a, grid, s);
    if (a.d == 128) return two ? launch_tc<128, 2, false>(a, grid, s) : launch_tc<128, 1, false>(a, grid, s);
    return launch_tc<256, 1, false>(a, grid, s);
}

cudaError_t take_status_attend_tc(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_attend_tc, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_attend_tc, &zero, sizeof(uint32_t));
}

}  // namespace damp
