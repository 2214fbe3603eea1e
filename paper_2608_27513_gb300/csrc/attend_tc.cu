// attend_tc.cu -- attention over the 8-bit cache for many rows (drafts, prompts) on tcgen05.
//
// An item has R = 128 SUB rows (attend.cuh): one or two blocks of 128 (query token, query head) pairs of a
// KV head, which are the lanes of tensor memory.  Per key tile of 128 tokens (4 pages) and block
//     S = Q K^T   (Q in shared memory, FP16)          128 x 128 x D
//     P = 2^(S f + a - R)                              a thread per row
//     O += P V    (P in tensor memory over S, FP16)    128 x D x 128
// One CTA per SM walks over an equal range of the items' key tiles.  Items that lie in one range are
// written at once, parts are joined by a second launch, as for single tokens.
//
// Warps: 4 per block of rows for the softmax (SUB = 2: warps 0-7; SUB = 1: 0-3), 4 (8) that turn codes
// into FP16 operands, one that issues the products.  With two blocks one's products run while the
// other's softmax does; with one, S has two buffers and the next tile's Q K^T runs under the softmax.
// The warps that turn codes hold the next tile's codes in registers (loaded a tile ahead), so no copy
// waits in shared memory; a 16-byte chunk of codes becomes two 16-byte rows of core matrices (8 rows of
// 8 FP16), which serve K as a K-major and V as an MN-major operand without another layout.
//
// Rounding.  Codes - 128 are exact in FP16; BF16 queries are scaled by a power of two per row (exact
// down to 2^-39 of the row's largest).  The value scales enter the weights: P = p s_v / 2^e 2^10 with
// the running power of two 2^e above them, in FP16 (2^-12 relative, a BF16 output is rounded to 2^-9).
// The row sum takes the unrounded p in FP32.  The reference R of the exponents is a maximum that may lag
// behind by 2^4, so that O is rescaled (from tensor memory and back) only where it moves by more.
#include "attend.cuh"
#include "prefill_tc.cuh"

#include <algorithm>

namespace damp {

static __device__ uint32_t g_status_attend_tc;

namespace {

constexpr int kAtThreads = 13 * 32;
constexpr int kAtTile = 128;  // tokens of a key tile
constexpr uint32_t kAtCols = 512;
constexpr uint32_t kAtO = 256;  // S blocks at columns 0 and 128, O from here on
constexpr float kAtLag = 4.f;
constexpr int kAtNotes = 4;

struct AtNote {  // of a key tile: what the softmax needs of its pages
    float factor[kTcUnit];  // key scale
    float weight[kTcUnit];  // log2 of 2^10 times value scale over 2^e
    float back[kTcUnit];    // 2^-weight, exactly what the sums divide by
    int e;                  // exponent field of 2^e
    int hidden;             // bit i: page i is bad or missing
    int unused[2];
};

template <int D, int SUB>
struct AtSmem {
    static constexpr int tile = kAtTile * D * 2;
    static constexpr int buffers = D == 256 ? 1 : 2;  // of K and of V
    static constexpr int q = 0, k = SUB * tile, v = k + buffers * tile;
    static constexpr int note = v + buffers * tile;
    static constexpr int bar = note + kAtNotes * (int)sizeof(AtNote);
    static constexpr int before = bar + 256;
    static constexpr int sm_warps = 4 * SUB, turn_warps = 12 - sm_warps;
};
// mbarriers
enum { kBarQ = 0, kBarKFull = 1, kBarKFree = 3, kBarVFull = 5, kBarVFree = 7, kBarS = 9, kBarP = 11, kBarNote = 13, kBarDone = 17, kBarPV = 18, kBarCount = 19 };

// instruction descriptor: f16 x f16 -> FP32, M = 128, N columns, B MN-major if set
__host__ __device__ constexpr uint32_t at_idesc(int n, bool b_mn) {
    return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// Products are issued by a whole warp in step, one elected lane each.
__device__ __forceinline__ void at_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p, e;\nelect.sync _|e, 0xffffffff;\nsetp.ne.u32 p, %4, 0;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
}
__device__ __forceinline__ void at_mma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p, e;\nelect.sync _|e, 0xffffffff;\nsetp.ne.u32 p, %4, 0;\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
                 "r"(a), "l"(b), "r"(idesc), "r"(acc)
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
// 32 columns of a thread's lane, to be used after at_ld_wait on them
__device__ __forceinline__ void at_ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
                   "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
                   "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
                   "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(taddr));
}
__device__ __forceinline__ void at_ld_wait(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                   "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                   "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]),
                   "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}
__device__ __forceinline__ void at_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void at_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
                 "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
                 "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}
__device__ __forceinline__ void at_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t at_half2(float a, float b) {  // a in the low half
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// bytes of w that `sel` names as FP16 codes minus 128
__device__ __forceinline__ uint32_t at_codes(uint32_t w, uint32_t sel) {
    const uint32_t h = prmt(w, 0x64646464u, sel);
    const __half2 y = __hadd2(*reinterpret_cast<const __half2 *>(&h), __half2(__ushort_as_half(0xE480), __ushort_as_half(0xE480)));
    return *reinterpret_cast<const uint32_t *>(&y);
}

// An item of the sequence, the same in all lanes of a warp.
struct AtItem {
    int b, rt, h, first, pages, tiles, begin;
    AttRow row;
};
__device__ __forceinline__ void at_set(AtItem &it, const AttendArgs &p, int R, int G) {
    const AttItem x = att_item(p, it.row, it.rt, R, G);
    it.first = x.first;
    it.pages = x.pages;
    it.tiles = att_units(x.pages, kTcUnit);
}
// the item that unit x < total lies in
__device__ __forceinline__ AtItem at_seek(const AttendArgs &p, const int32_t *before, int x, int R, int G) {
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
        int n = rt < att_tiles(it.row.n, R, G) ? att_units(att_item(p, it.row, rt, R, G).pages, kTcUnit) * p.Hk : 0;
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
        if (it.rt > att_tiles(it.row.n, R, G)) break;  // (not reached: x lies in this row)
    }
    at_set(it, p, R, G);
    it.h = it.tiles ? (x - at) / it.tiles : 0;
    it.begin = at + it.h * it.tiles;
    return it;
}
// the item after `it`, given that there is one
__device__ __forceinline__ void at_next(AtItem &it, const AttendArgs &p, int R, int G) {
    it.begin += it.tiles;
    if (++it.h < p.Hk) return;
    it.h = 0;
    do {
        if (++it.rt >= att_tiles(it.row.n, R, G)) {
            it.rt = 0;
            if (++it.b >= p.batch) return;
            it.row = att_row(p, it.b);
        }
        at_set(it, p, R, G);
    } while (it.tiles == 0);
}

struct AtWait {  // bounded waits, all of which give up once one has
    volatile uint32_t *dead;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
        if (mbar_try_wait(bar, parity)) return true;
        const uint64_t t0 = global_timer_ns();
        for (uint32_t i = 0; i < (1u << 26); ++i) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((i & 255u) == 255u && (*dead || global_timer_ns() - t0 > 2000000000ull)) break;
        }
        *dead = 1;
        return false;
    }
};

template <int D, int SUB>
__global__ void __launch_bounds__(kAtThreads, 1) attend_tc_kernel(const AttendArgs p) {
    using M = AtSmem<D, SUB>;
    constexpr int R = 128 * SUB;
    extern __shared__ __align__(1024) uint8_t sm[];
    __shared__ uint32_t s_dead, s_tmem;
    int32_t *const before = reinterpret_cast<int32_t *>(sm + M::before);
    const uint32_t sb = smem_u32(sm);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.H / p.Hk;
    auto bar = [&](int i) { return sb + M::bar + 8 * i; };
    if (threadIdx.x == 0) {
        s_dead = 0;
        mbar_init(bar(kBarQ), 128 * SUB);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(kBarKFull + i), M::turn_warps);
            mbar_init(bar(kBarKFree + i), 1);
            mbar_init(bar(kBarVFull + i), M::turn_warps);
            mbar_init(bar(kBarVFree + i), 1);
            mbar_init(bar(kBarS + i), 1);
            mbar_init(bar(kBarP + i), 128);
        }
        for (int i = 0; i < kAtNotes; ++i) mbar_init(bar(kBarNote + i), 1);
        mbar_init(bar(kBarDone), 1);
        mbar_init(bar(kBarPV), 1);
        fence_mbar_init();
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kAtCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    att_count(p, R, G, kTcUnit, before);  // (synchronizes)
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    const AttWork work = att_work(p.workspace, p.batch, gridDim.x, R, D);
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= p.batch; b += kAtThreads) work.before[b] = before[b];
    const int total = before[p.batch] * p.Hk, per = att_per(total, gridDim.x);
    const int end = (int)min((int64_t)total, ((int64_t)blockIdx.x + 1) * per);
    const int begin = (int)min((int64_t)end, (int64_t)blockIdx.x * per);
    const AtWait wait{&s_dead};

    if (begin < end && warp < M::sm_warps) {
        // ---- softmax: thread = row of a block ----
        const int x = warp >> 2;                 // block of rows
        const int row = threadIdx.x & 127;       // in the block: the lane of tensor memory
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t o_at = lanes + kAtO + x * D;
        AtItem it = at_seek(p, before, begin, R, G);
        uint32_t tile = 0;  // of this range
        uint32_t items = 0;
        bool ok = true;
        for (int at = begin; at < end && ok; ++items) {
            if (items) at_next(it, p, R, G);
            const int last = min(end, it.begin + it.tiles);
            const int r = it.rt * R + x * 128 + row, t = r / G;
            const bool live = t < it.row.n;
            const int limit = live ? it.row.len - it.row.n + t : kNoRow;
            const int from = p.window && live ? limit - (p.window - 1) : 0;
            const int head = it.h * G + (r - t * G);
            // q, scaled by a power of two to below 2^15
            float factor;
            {
                const uint4 *const q = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) +
                                                                       ((int64_t)it.b * p.T + t) * p.q_stride + (int64_t)head * D);
                uint32_t top = 0;  // largest magnitude of the bf16 values, both halves
                constexpr int kC = D / 8;
                constexpr int kHold = D == 256 ? 1 : kC;  // chunks kept between the passes
                uint4 hold[kHold];
#pragma unroll
                for (int i = 0; i < kC; ++i) {
                    const uint4 w = live ? q[i] : make_uint4(0, 0, 0, 0);
                    if (kHold == kC) hold[i < kHold ? i : 0] = w;
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) top = __vmaxu2(top, u[k] & 0x7fff7fffu);
                }
                const uint32_t most = max(top >> 16, top & 0xffffu);
                const int e = min(max((int)(most >> 7), 15), 254);
                const float up = __uint_as_float((uint32_t)(268 - e) << 23);
                factor = p.scale * kLog2e / up;
                const uint32_t to = sb + M::q + x * M::tile + (row >> 3) * (16 * D) + (row & 7) * 16;
#pragma unroll
                for (int i = 0; i < kC; ++i) {
                    const uint4 w = kHold == kC ? hold[i < kHold ? i : 0] : live ? q[i] : make_uint4(0, 0, 0, 0);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                    uint32_t h[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        h[k] = at_half2(__uint_as_float(u[k] << 16) * up, __uint_as_float(u[k] & 0xffff0000u) * up);
                    sts128(to + i * 128, make_uint4(h[0], h[1], h[2], h[3]));
                }
                fence_proxy_async_smem();
                tc_fence_before();
                at_arrive(bar(kBarQ));
            }
            float ref = -INFINITY, sum = 0.f;
            int ve = 0;
            const int first_tile = at - it.begin;
            for (; at < last; ++at, ++tile) {
                const int sbuf = SUB == 2 ? x : tile & 1;
                const uint32_t s_at = lanes + sbuf * 128;
                const uint32_t n_bar = bar(kBarNote + tile % kAtNotes);
                ok = wait(n_bar, (tile / kAtNotes) & 1) && wait(bar(kBarS + sbuf), (SUB == 2 ? tile : tile >> 1) & 1);
                if (!__all_sync(kFull, ok)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const AtNote *const note = reinterpret_cast<const AtNote *>(sm + M::note) + tile % kAtNotes;
                const int i = at - it.begin;
                const int token = (it.first + i * kTcUnit) * kCachePage;  // of column 0
                const int hidden = note->hidden, e = note->e;
                float f[kTcUnit];
#pragma unroll
                for (int c = 0; c < kTcUnit; ++c) f[c] = fmaxf(factor * note->factor[c], FLT_MIN);  // not 0: times a hidden -inf
                const bool masked = __any_sync(kFull, hidden != 0 || (limit != kNoRow && (limit < token + kAtTile - 1 || from > token)));
                auto hide = [&](uint32_t (&s)[32], int c) {
                    const int lo = from - (token + 32 * c), hi = limit - (token + 32 * c);
                    const bool all = (hidden >> c) & 1;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j > hi || j < lo || all) s[j] = 0xff800000u;
                };
                uint32_t s[2][32];
                float top = -INFINITY;
                at_ld32(s_at, s[0]);
#pragma unroll
                for (int c = 0; c < kTcUnit; ++c) {
                    at_ld_wait(s[c & 1]);
                    if (c + 1 < kTcUnit) at_ld32(s_at + 32 * (c + 1), s[(c + 1) & 1]);
                    if (masked) hide(s[c & 1], c);
                    float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        m[0] = fmax3(m[0], __uint_as_float(s[c & 1][j]), __uint_as_float(s[c & 1][j + 1]));
                        m[1] = fmax3(m[1], __uint_as_float(s[c & 1][j + 2]), __uint_as_float(s[c & 1][j + 3]));
                    }
                    top = fmaxf(top, fmaxf(m[0], m[1]) * f[c]);
                }
                at_ld32(s_at, s[0]);
                const bool moves = top > ref + kAtLag || (ref == -INFINITY && top > ref);
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
                        ok = wait(bar(kBarPV), (tile - 1) & 1);
                        if (!__all_sync(kFull, ok)) {
                            at_ld_wait(s[0]);
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                    }
                    at_ld_wait(s[0]);
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        at_ld32(o_at + 32 * c, s[1]);
                        at_ld_wait(s[1]);
#pragma unroll
                        for (int j = 0; j < 32; ++j) s[1][j] = __float_as_uint(__uint_as_float(s[1][j]) * corr);
                        at_st32(o_at + 32 * c, s[1]);
                    }
                }
                ve = e;
                const float base = ref == -INFINITY ? 0.f : -ref;
#pragma unroll
                for (int c = 0; c < kTcUnit; ++c) {
                    at_ld_wait(s[c & 1]);
                    if (c + 1 < kTcUnit) at_ld32(s_at + 32 * (c + 1), s[(c + 1) & 1]);
                    if (masked) hide(s[c & 1], c);
                    const float2 f2 = splat2(f[c]), a2 = splat2(base + note->weight[c]);
                    float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 y = fma2(make_float2(__uint_as_float(s[c & 1][2 * j]), __uint_as_float(s[c & 1][2 * j + 1])), f2, a2);
                        const float2 z = make_float2(ex2(y.x), ex2(y.y));
                        part[j & 1] = add2(part[j & 1], z);
                        w[j] = at_half2(z.x, z.y);
                    }
                    at_st16(s_at + 16 * c, w);
                    const float2 both = add2(part[0], part[1]);
                    sum = fmaf(both.x + both.y, note->back[c], sum);
                }
                at_st_wait();
                tc_fence_before();
                at_arrive(bar(kBarP + sbuf));
            }
            if (!ok) break;
            // the item's products are done
            ok = wait(bar(kBarDone), items & 1);
            if (!__all_sync(kFull, ok)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const bool whole = it.begin >= begin && it.begin + it.tiles <= end;
            const int slot = 2 * blockIdx.x + (it.begin >= begin ? 1 : 0);
            const float unit = __uint_as_float((uint32_t)ve << 23) * (1.f / 1024.f);
            const float y = whole ? (sum == 0.f ? 0.f : unit / sum) : unit;
            const int64_t to = (((int64_t)it.b * p.T + t) * p.H + head) * D;
            float *const part = work.o + ((int64_t)slot * R + x * 128 + row) * D;
            if (live && !whole) work.ml[(int64_t)slot * R + x * 128 + row] = make_float2(ref, sum);
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t s[32];
                at_ld32(o_at + 32 * c, s);
                at_ld_wait(s);
                if (live) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float z[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] = __uint_as_float(s[16 * k + j]) * y;
                        if (whole)
                            store_out<true, 16>(p.o, to + 32 * c + 16 * k, z);
                        else
                            store_out<false, 16>(part, 32 * c + 16 * k, z);
                    }
                }
            }
            tc_fence_before();
        }
    } else if (begin < end && warp < 12) {
        // ---- codes into operands ----
        constexpr int kQuads = D / 64;                             // 4 chunks of 16 codes
        constexpr int kUnits = 16 * kQuads / M::turn_warps;        // of 8 tokens x 4 chunks, of a warp
        const int w = warp - M::sm_warps;
        const int tok = lane & 7, mi = lane >> 3;
        AtItem it = at_seek(p, before, begin, R, G);
        int lt = begin;  // the tile that is loaded next
        int ve = 0;
        uint4 kreg[kUnits], vreg[kUnits];
        // lane c < 4: page c of the tile that is loaded next, and of the one at hand
        int slot = -1, slot_now = -1, h_now = 0, h_next = 0;
        bool fresh_next = true, fresh_now = true;  // starts an item
        bool bad_next = false, bad_now = false;
        auto find = [&]() {  // the pages of tile lt
            if (lt >= it.begin + it.tiles) {
                at_next(it, p, R, G);
                fresh_next = true;
            }
            const int i = (lt - it.begin) * kTcUnit + lane;
            slot = -1;
            bad_next = false;
            if (lane < kTcUnit && i < it.pages) {
                const int32_t e = p.pages[(int64_t)it.b * p.table + it.first + i];
                slot = (int)cache_page(e, p.num_pages);
                bad_next = slot < 0;
            }
            h_next = it.h;
        };
        auto load = [&](uint4 (&r)[kUnits], int which) {
#pragma unroll
            for (int j = 0; j < kUnits; ++j) {
                const int u = w + j * M::turn_warps, tg = u / kQuads, mq = u % kQuads;
                const int s = __shfl_sync(kFull, slot_now, tg >> 2);
                const int t = (tg & 3) * 8 + tok, m = mq * 4 + mi;
                r[j] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);  // zeros
                if (s >= 0)
                    r[j] = __ldg(reinterpret_cast<const uint4 *>(p.pool + ((int64_t)s * p.Hk + h_now) * cache_record_bytes(D) +
                                                                which * cache_rows_bytes(D) + cache_chunk(t, m, D)));
            }
        };
        auto turn = [&](const uint4 (&r)[kUnits], uint32_t to) {
#pragma unroll
            for (int j = 0; j < kUnits; ++j) {
                const int u = w + j * M::turn_warps, tg = u / kQuads, mq = u % kQuads;
                const uint32_t at = to + tg * (16 * D) + (mq * 4 + mi) * 256 + tok * 16;
                const uint4 c = r[j];
                sts128(at, make_uint4(at_codes(c.x, 0x4140u), at_codes(c.x, 0x4342u), at_codes(c.y, 0x4140u), at_codes(c.y, 0x4342u)));
                sts128(at + 128, make_uint4(at_codes(c.z, 0x4140u), at_codes(c.z, 0x4342u), at_codes(c.w, 0x4140u), at_codes(c.w, 0x4342u)));
            }
        };
        float2 scales = make_float2(0.f, 0.f);
        auto step = [&]() {  // the tile that was next is at hand
            slot_now = slot;
            h_now = h_next;
            fresh_now = fresh_next;
            bad_now = bad_next;
            fresh_next = false;
            scales = make_float2(0.f, 0.f);
            if (w == 0 && slot_now >= 0)
                scales = *reinterpret_cast<const float2 *>(p.pool + ((int64_t)slot_now * p.Hk + h_now) * cache_record_bytes(D) + 2 * cache_rows_bytes(D));
        };
        find();
        step();
        load(kreg, 0);
        load(vreg, 1);
        ++lt;
        if (lt < end) find();
        bool ok = true;
        const int tiles = end - begin;
        for (int i = 0; i < tiles; ++i) {
            const int buf = M::buffers == 2 ? i & 1 : 0, use = M::buffers == 2 ? i >> 1 : i;
            if (use) ok = wait(bar(kBarKFree + buf), (use - 1) & 1);
            if (!__all_sync(kFull, ok)) break;
            if (w == 0) {
                AtNote *const note = reinterpret_cast<AtNote *>(sm + M::note) + i % kAtNotes;
                if (fresh_now) ve = 0;
                int e = scales.y > 0.f ? min((int)(__float_as_uint(scales.y) >> 23) + 1, 253) : 0;
                e = max(e, __shfl_xor_sync(kFull, e, 1));
                e = max(e, __shfl_xor_sync(kFull, e, 2));
                ve = max(max(ve, 1), __shfl_sync(kFull, e, 0));
                const float rel = fmaxf(scales.y * __uint_as_float((uint32_t)(254 - ve) << 23), 9.0949470177292824e-13f);  // 2^-40
                const unsigned hidden = __ballot_sync(kFull, slot_now < 0) & ((1u << kTcUnit) - 1u);
                if (lane < kTcUnit) {
                    // a block of zeros stands for zeros at any scale
                    const float u = scales.y > 0.f ? rel * 1024.f : 1024.f;
                    note->factor[lane] = scales.x > 0.f ? scales.x : 1.f;
                    note->weight[lane] = __log2f(u);
                    note->back[lane] = 1.f / u;
                }
                if (lane == 0) {
                    note->e = ve;
                    note->hidden = (int)hidden;
                }
                if (bad_now) atomicOr(p.status, kDevBadSlot);
                __syncwarp();
                if (lane == 0) at_arrive(bar(kBarNote + i % kAtNotes));
            }
            turn(kreg, sb + M::k + buf * M::tile);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) at_arrive(bar(kBarKFull + buf));
            const bool more = i + 1 < tiles;
            if (more) {
                step();
                load(kreg, 0);
            }
            if (use) ok = wait(bar(kBarVFree + buf), (use - 1) & 1);
            if (!__all_sync(kFull, ok)) break;
            turn(vreg, sb + M::v + buf * M::tile);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) at_arrive(bar(kBarVFull + buf));
            if (more) {
                load(vreg, 1);
                ++lt;
                if (lt < end) find();
            }
        }
    } else if (begin < end) {
        // ---- the products ----
        constexpr uint32_t kIdS = at_idesc(kAtTile, false), kIdO = at_idesc(D, true);
        AtItem it = at_seek(p, before, begin, R, G);
        uint32_t tile = 0, items = 0;
        bool ok = true;
        auto key_buf = [&](uint32_t t) { return M::buffers == 2 ? t & 1u : 0u; };
        auto key_use = [&](uint32_t t) { return (M::buffers == 2 ? t >> 1 : t) & 1u; };
        auto scores = [&](uint32_t t, int x) {  // Q_x K_t^T; SUB = 1: into the buffer of the tile
            const uint32_t d = tmem + 128 * (SUB == 2 ? x : t & 1);
            const uint64_t a = tc_desc(sb + M::q + x * M::tile, 128, 16 * D), b = tc_desc(sb + M::k + key_buf(t) * M::tile, 128, 16 * D);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) at_mma(d, a + 16 * k, b + 16 * k, kIdS, k != 0);
            at_commit(bar(kBarS + (SUB == 2 ? x : t & 1)));
        };
        auto outputs = [&](uint32_t t, int x, bool first) {  // O_x += P V_t
            const uint32_t a = tmem + 128 * (SUB == 2 ? x : t & 1);
            const uint64_t b = tc_desc(sb + M::v + key_buf(t) * M::tile, 16 * D, 128);
#pragma unroll
            for (int k = 0; k < kAtTile / 16; ++k) at_mma_ta(tmem + kAtO + x * D, a + 8 * k, b + 2 * D * k, kIdO, !(first && k == 0));
        };
        for (int at = begin; at < end && ok; ++items) {
            if (items) at_next(it, p, R, G);
            const int last = min(end, it.begin + it.tiles), n = last - at;
            ok = wait(bar(kBarQ), items & 1) && wait(bar(kBarKFull + key_buf(tile)), key_use(tile));
            if (!__all_sync(kFull, ok)) break;
            tc_fence_after();
            for (int x = 0; x < SUB; ++x) scores(tile, x);
            at_commit(bar(kBarKFree + key_buf(tile)));
            for (int i = 0; i < n && ok; ++i, ++tile) {
                const bool more = i + 1 < n;
                if (SUB == 1 && more) {
                    ok = wait(bar(kBarKFull + key_buf(tile + 1)), key_use(tile + 1));
                    if (!__all_sync(kFull, ok)) break;
                    tc_fence_after();
                    scores(tile + 1, 0);
                    at_commit(bar(kBarKFree + key_buf(tile + 1)));
                }
                for (int x = 0; x < SUB && ok; ++x) {
                    const int s = SUB == 2 ? x : (int)(tile & 1);
                    ok = wait(bar(kBarP + s), (SUB == 2 ? tile : tile >> 1) & 1) && wait(bar(kBarVFull + key_buf(tile)), key_use(tile));
                    if (SUB == 2 && more && ok) ok = wait(bar(kBarKFull + key_buf(tile + 1)), key_use(tile + 1));
                    if (!__all_sync(kFull, ok)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    outputs(tile, x, i == 0);
                    if (x == SUB - 1) at_commit(bar(kBarVFree + key_buf(tile)));
                    if (SUB == 1) at_commit(bar(kBarPV));
                    if (SUB == 2 && more) {
                        scores(tile + 1, x);
                        if (x == 1) at_commit(bar(kBarKFree + key_buf(tile + 1)));
                    }
                }
            }
            if (!ok) break;
            at_commit(bar(kBarDone));
            at = last;
        }
        if (!ok) {  // what was issued ends by itself; no other product is issued
            at_commit(bar(kBarDone));
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && s_dead) atomicOr(p.status, kDevWaitTimeout);
    if (warp == 12)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kAtCols) : "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <int D, int SUB>
cudaError_t launch_tc(const AttendArgs &a, int grid, cudaStream_t s) {
    using M = AtSmem<D, SUB>;
    const int smem = M::before + (a.batch + 1) * 4;
    const cudaError_t e = ensure_smem_limit(reinterpret_cast<const void *>(attend_tc_kernel<D, SUB>), smem);
    if (e != cudaSuccess) return e;
    attend_tc_kernel<D, SUB><<<grid, kAtThreads, smem, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

bool attend_tc_takes(const AttendArgs &a) { return a.in_bf16 && (int64_t)a.T * (a.H / a.Hk) > 16; }

int attend_tc_rows(const AttendArgs &a) { return a.d <= 128 && (int64_t)a.T * (a.H / a.Hk) > 128 ? 256 : 128; }

cudaError_t launch_attend_tc(AttendArgs a, int grid, cudaStream_t s) {
    static std::atomic<uint32_t *> cache[64];
    const cudaError_t e = symbol_address_cached(&g_status_attend_tc, cache, &a.status);
    if (e != cudaSuccess) return e;
    const bool two = attend_tc_rows(a) == 256;
    if (a.d == 64) return two ? launch_tc<64, 2>(a, grid, s) : launch_tc<64, 1>(a, grid, s);
    if (a.d == 128) return two ? launch_tc<128, 2>(a, grid, s) : launch_tc<128, 1>(a, grid, s);
    return launch_tc<256, 1>(a, grid, s);
}

cudaError_t take_status_attend_tc(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_attend_tc, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_attend_tc, &zero, sizeof(uint32_t));
}

}  // namespace damp
