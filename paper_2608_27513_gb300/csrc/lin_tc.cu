// lin_tc.cu -- a chunk of linear attention with a decay per head on the tensor cores.
//
// A piece of C = 64 tokens, with G_i = g_0 + ... + g_i inside it (base-2 logs below):
//     o_i = e^{G_i} S_0^T q_i + sum_{j<=i} e^{G_i - G_j} (q_i.k_j) v_j
//     S_C = e^{G_C} S_0 + sum_j (e^{G_C - G_j} k_j) v_j^T
// as four tcgen05.mma products, all transposed so that the value column is the tensor-
// memory lane and an output row is stored by 32 lanes of a warp as one line:
//     Q K^T                                        (lanes 0-63 of 128)
//     S_0^T Q^T                                    -> O1 (A from tensor memory)
//     V^T (K~ = e^{G_C - G_j} k_j)                 -> what the piece adds to S^T
//     V^T P^T, P = (e^{G_i - G_j} q_i.k_j)_{j<=i}  -> O2;  o_i = O2_i + e^{G_i} O1_i
// One CTA per SM walks over items of 128 value columns of a (slot, head); a last block of 64
// columns leaves zeros in the upper lanes.  An item's state stays with its threads in FP32
// (thread = value column and half the key channels); only its operand copy is split.
//
// Rounding.  q, k and v are bf16 inputs and enter exactly.  The FP32 operands (S_0, K~, P)
// enter as three bf16 parts that hold them exactly.  Accumulation and the state are FP32.  G
// is summed as pairs of floats, so that G_i - G_j keeps its digits where both are large
// (fast decays).  Measured against 64 bits: 2e-7 of o.  Two parts instead of three (half the
// tensor memory, two CTAs per SM) took 204 and 255 us where three took 209 and 263 (64
// ragged prompts of up to 256 tokens, one of 16381; 32 heads, d = 128), at 2.9e-6.
//
// Values that are not finite.  The products are masked by zeros in P, and 0 times a v_j that is
// not finite is a NaN in the outputs before token j: blocks of outputs with such a value are
// summed plainly (lt_outputs; 350 us a piece: 64 prompts of 256 tokens take 19 ms if every
// piece has one).  Everything else is causal as it stands.  A part split off an infinity is a
// NaN, so an infinite state gives NaN outputs; in the registers it stays infinite.
//
// Sixteen warps in two groups that meet only at mbarriers.  Warps 0-7 hold the state: they
// add what a piece adds and write the next operand parts to tensor memory.  Warps 8-15 turn
// Q K^T into P and k into K~, one piece ahead of the outputs that they combine and store;
// warp 12, which has no part in P and K~, issues the products, warp 13 the copies (TMA,
// 128-byte swizzle, three stages) and warp 9 sums the gates.
//
// Bound by latency along two chains (d = 128, 32 heads, 250 rows: 53 items per SM; 1.94 GHz).
// A further piece of an item takes 3.2 us, 6200 clocks (rows of 256 and 512 tokens: 880 and
// 1559 us): a product takes 45 clocks with 64 columns and 59 with 128, which makes 2700 for the
// piece's 56, the splits about 2000 in each group (9 operations per pair of values), and the two
// wait for each other in turn; DRAM would need 1.8 us.  The border of two items takes another 3
// to 5 us (rows of 64 tokens, one piece: 437 us, 8.2 us an item; of 128: 506, 9.5), more than
// half of the time of short rows: warps 0-7 store 64 values per thread, load 64 and split them
// while the products wait; DRAM would need 2.9 us for the 128 KB.  The next states are brought
// into L2 ahead by warp 13 (61 slots of 128 tokens: 139 us without, 131 with; of 17: 105 and 88).
// At d = 128 the 128 registers of a thread do not hold a role's values all the time: 372 bytes
// of spill stores and 372 of loads (`-Xptxas -v`; d = 64: 12 and 4).
//
// Few (slot, head) pairs and many tokens: the tokens are split into segments.  A first
// launch computes what each segment adds to the state (k and v only), a second one joins the
// additions to states, a third one starts every segment from its own.
#include <cuda.h>

#include "damp_internal.h"
#include "prefill_tc.cuh"

#include <algorithm>
#include <cfloat>

namespace damp {

static __device__ uint32_t g_status_lin_tc;

namespace {

constexpr int kLtC = 64;
constexpr int kLtThreads = 512;
constexpr int kLtBox = 64 * 128;  // bytes of a copied box: 64 tokens x 64 bf16
constexpr uint32_t kLtCols = 512;
// tensor-memory columns: Q K^T | O1 | O2 | what the piece adds to S | S_0 as three bf16 parts
constexpr uint32_t kLtG = 0, kLtO1 = 64, kLtO2 = 128, kLtD = 192, kLtS = 320;
constexpr int kLtStages = 3;
constexpr int kLtGates = 4;  // a piece's sums may be read while the copies of the third piece after it start

constexpr int kLtSorted = 256;  // rows at most that are taken by length

template <int DK, bool STATE>
struct LtSmem {  // bytes from the base of the dynamic shared memory
    static constexpr int tile = kLtC * DK * 2;
    // a stage: the 64-column boxes of q (not for the state alone), k and v.  Q K^T takes 128 rows from q
    // on: the upper 64 are other boxes of the stage, and their products are not used.
    static constexpr int q = 0, k = STATE ? 0 : tile, v = STATE ? tile : 2 * tile;
    static constexpr int stage = v + 2 * kLtBox;
    static constexpr int kdn = STATE ? 2 : 1;     // buffers of K~
    static constexpr int kd = kLtStages * stage;  // K~, three parts
    static constexpr int p = kd + kdn * 3 * tile; // P, three parts: columns 0-31 of 64 rows, columns 32-63 of rows 32-63
    static constexpr int ppart = 64 * 64 + 32 * 64;
    static constexpr int g = p + (STATE ? 0 : 3 * ppart);  // per piece: (hi, lo) of G in base 2, 64 pairs, and e^{G_i}
    static constexpr int gbuf = 512 + 256;
    static constexpr int bar = g + kLtGates * gbuf;  // mbarriers, the tensor-memory address
    static constexpr int zero = bar + 160;  // 512 bytes: an output row past a row's length
    static constexpr int order = zero + 512;  // rows by falling length: 16 bits each
    static constexpr int bytes = order + (STATE ? 0 : 2 * kLtSorted);
    static_assert(STATE || 4 * kLtSorted <= 3 * ppart, "pieces of the rows");
};

struct LinTcParams {
    float *state;
    int64_t num_slots;
    const int32_t *slot_idx, *lengths;
    const float *g;
    float *o;
    float *part;      // [batch * H * nc][nseg][DK][128]: states and additions of the segments
    float *part_dec;  // [batch * H * nc][nseg]: the decay of segment s - 1
    int32_t H, Hqk, dv, nc, T, g_per_head;
    int32_t nseg, seg_len, items;  // items: with their segments
    int32_t sorted;                // rows to take by length (0: in their order)
    uint32_t *status;
};
// the inputs of the tensor maps, for the outputs of pieces with a value of v that is not finite
struct LinTcInputs {
    const __nv_bfloat16 *q, *k, *v;
};

__device__ __forceinline__ float lt_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the boxes of 64 tokens of a head of a [batch][token][head][channel] tensor, from 64-channel group
// `group` on, into shared memory
__device__ __forceinline__ void lt_copy_boxes(uint32_t dst, const CUtensorMap *map, int group, int head, int t, int b, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(map), "r"(0), "r"(head), "r"(t), "r"(group), "r"(b), "r"(bar)
        : "memory");
}
// descriptor of an operand in 128-byte swizzled boxes.  K-major: rows of 128 bytes, 8 rows `sbo`
// apart, a K step of 16 is 32 bytes.  MN-major: 64 columns per box, boxes `lbo` apart, 8 rows of K
// `sbo` apart.
__device__ __forceinline__ uint64_t lt_desc_sw(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return tc_desc(addr, lbo, sbo) | (2ull << 61);
}
__device__ __forceinline__ void lt_ld16(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void lt_ld8(uint32_t taddr, float (&v)[8]) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\ntcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ float lt_ld1(uint32_t taddr) {
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\ntcgen05.wait::ld.sync.aligned;" : "=r"(r) : "r"(taddr) : "memory");
    return __uint_as_float(r);
}
__device__ __forceinline__ void lt_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void lt_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Products are issued by whole warps in step, one elected lane each, from descriptors in uniform
// registers.
struct LtDesc {  // a shared-memory descriptor whose low word is the same in all lanes
    uint32_t lo, hi;
};
__device__ __forceinline__ LtDesc lt_uniform(uint64_t d) {
    return LtDesc{__reduce_max_sync(kFull, (uint32_t)d), __reduce_max_sync(kFull, (uint32_t)(d >> 32))};
}
__device__ __forceinline__ LtDesc lt_at(LtDesc d, uint32_t off) { return LtDesc{d.lo + (off >> 4), d.hi}; }  // `off` bytes further
__device__ __forceinline__ void lt_mma(uint32_t d, LtDesc a, LtDesc b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p, e;\n.reg .b64 da, db;\nelect.sync _|e, 0xffffffff;\nsetp.ne.u32 p, %6, 0;\n"
                 "mov.b64 da, {%1, %2};\nmov.b64 db, {%3, %4};\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n}" ::"r"(d),
                 "r"(a.lo), "r"(a.hi), "r"(b.lo), "r"(b.hi), "r"(idesc), "r"(acc)
                 : "memory");
}
// A from tensor memory (K-major: two bf16 per column)
__device__ __forceinline__ void lt_mma_ta(uint32_t d, uint32_t a, LtDesc b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p, e;\n.reg .b64 db;\nelect.sync _|e, 0xffffffff;\nsetp.ne.u32 p, %5, 0;\n"
                 "mov.b64 db, {%2, %3};\n"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}" ::"r"(d),
                 "r"(a), "r"(b.lo), "r"(b.hi), "r"(idesc), "r"(acc)
                 : "memory");
}
__device__ __forceinline__ void lt_commit(uint32_t bar) {
    asm volatile("{\n.reg .pred e;\nelect.sync _|e, 0xffffffff;\n"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar)
                 : "memory");
}

// x = hi + mid + lo as bf16 parts, two values per word: each part cuts off eight significant bits of
// what is left, so that the three hold x exactly
__device__ __forceinline__ void lt_split(float2 x, uint32_t &h, uint32_t &m, uint32_t &l) {
    auto minus_upper = [](float2 y) {
        return make_float2(-__uint_as_float(__float_as_uint(y.x) & 0xffff0000u), -__uint_as_float(__float_as_uint(y.y) & 0xffff0000u));
    };
    auto uppers = [](float2 y) { return prmt(__float_as_uint(y.x), __float_as_uint(y.y), 0x7632u); };
    h = uppers(x);
    x = add2(x, minus_upper(x));
    m = uppers(x);
    x = add2(x, minus_upper(x));
    l = uppers(x);
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// a sum of two floats, hi + lo
struct Pair {
    float hi, lo;
};
// 2^x within an ulp (ex2.approx is within three): 2^round(x) times the Taylor series of 2^f, |f| <= 1/2,
// whose ninth term is below 6e-9.  For the factors that a state meets again and again; P takes lt_ex2.
__device__ __forceinline__ float lt_exp2(Pair x) {
    const float n = rintf(fminf(fmaxf(x.hi, -160.f), 160.f));
    const float f = (x.hi - n) + x.lo;
    float y = 1.525273381e-5f;  // ln2^7 / 7!
    y = fmaf(y, f, 1.540353039e-4f);
    y = fmaf(y, f, 1.333355815e-3f);
    y = fmaf(y, f, 9.618129108e-3f);
    y = fmaf(y, f, 5.550410866e-2f);
    y = fmaf(y, f, 2.402265070e-1f);
    y = fmaf(y, f, 6.931471806e-1f);
    y = fmaf(y, f, 1.f);
    const float n1 = rintf(0.5f * n);  // 2^n in two factors: n may be below -126
    const float r = y * __uint_as_float((uint32_t)((int)n1 + 127) << 23) * __uint_as_float((uint32_t)((int)(n - n1) + 127) << 23);
    return x.hi < -160.f ? 0.f : x.hi != x.hi ? x.hi : r;
}
__device__ __forceinline__ Pair add_pair(Pair a, Pair b) {
    const float s = a.hi + b.hi, t = s - a.hi;
    const float e = ((a.hi - (s - t)) + (b.hi - t)) + (a.lo + b.lo);  // the rounding of s, and the low parts
    const float h = s + e;
    return Pair{h, e - (h - s)};
}

// o_i = e^{G_i} O1_i + sum_{j<=i} e^{G_i - G_j} (q_i.k_j) v_j of tokens i = i0 .. i1-1 of a piece, a
// sum per lane's value column and no term after i: for pieces with a v_j that is not finite, which the
// product V^T P^T takes times zero into the outputs before it.  A lane takes the dot products of keys
// `lane` and 32 + lane.  o: the piece's token 0 in the lane's column `row` of outputs o0.
template <int DK>
__device__ __noinline__ void lt_outputs(const LinTcInputs in, int H, int Hqk, int dv, const float *o0, float *o, int row, uint32_t sg,
                                        uint32_t o1, int i0, int i1, bool on) {
    const int64_t v_step = (int64_t)H * dv, at = o - o0 - row, t0 = at / v_step;  // token 0 of the piece
    const int64_t qk_step = (int64_t)Hqk * DK, qk = t0 * qk_step + (at - t0 * v_step) / dv * Hqk / H * DK;
    const __nv_bfloat16 *const q = in.q + qk, *const k = in.k + qk, *const v = in.v + (o - o0);
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        const float gih = ldsf(sg + 8 * i), gil = ldsf(sg + 8 * i + 4);
        float sum = ldsf(sg + 512 + 4 * i) * lt_ld1(o1 + i);
#pragma unroll 1
        for (int j0 = 0; j0 <= i; j0 += 32) {
            const int j = min(j0 + lane, i);
            const uint4 *const qi = reinterpret_cast<const uint4 *>(q + i * qk_step), *const kj = reinterpret_cast<const uint4 *>(k + j * qk_step);
            float2 dot = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int c = 0; c < DK / 8; ++c) {
                const uint4 a = qi[c], b = kj[c];
                const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    dot = fma2(make_float2(__uint_as_float(aw[e] << 16), __uint_as_float(aw[e] & 0xffff0000u)),
                               make_float2(__uint_as_float(bw[e] << 16), __uint_as_float(bw[e] & 0xffff0000u)), dot);
            }
            const float p = (dot.x + dot.y) * lt_ex2((gih - ldsf(sg + 8 * j)) + (gil - ldsf(sg + 8 * j + 4)));
            const int n = min(32, i + 1 - j0);
#pragma unroll 4
            for (int e = 0; e < n; ++e) {
                const float pe = __shfl_sync(kFull, p, e);
                if (on) sum = fmaf(pe, __bfloat162float(v[(j0 + e) * v_step]), sum);
            }
        }
        if (on) o[i * v_step] = sum;
    }
}

// A piece of work: one segment of one row, head and 128 value columns
struct LtItem {
    int b, h, c, seg, len, t_begin, t_end;
    int64_t slot, index;  // index: of the row, head and columns
    bool live;            // has tokens (and, for the state alone, a live segment after it)
};

// STATE: only what the segment adds to the state and its decay
// FULL: d_v is a multiple of 128 (no block of 64 columns)
template <int DK, bool STATE, bool FULL>
__global__ void __launch_bounds__(kLtThreads, 1)
    lin_tc_kernel(const LinTcParams p, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                  const __grid_constant__ CUtensorMap vmap, const LinTcInputs in) {
    extern __shared__ __align__(1024) uint8_t smem[];
    using M = LtSmem<DK, STATE>;
    constexpr int CELLS = DK / 8;
    constexpr int NR = DK / 2;  // state rows of a thread
    constexpr uint32_t kIdG = tc_idesc(64, false, false), kIdO2 = tc_idesc(64, true, false), kIdO2b = tc_idesc(32, true, false),
                       kIdS = tc_idesc(DK, true, true);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = 32 * (warp & 3) + lane, half = (warp >> 2) & 1;
    const uint32_t sb = smem_u32(smem);
    // Barriers, one phase per piece (`full` and `free`: per piece of a stage; `ds` and `kd`: two each, of
    // even and odd pieces, as a phase can be told from the next one only).  Copies landed and gates summed;
    // all products of the stage done; products done: Q K^T, O1, the addition to S, O2; written: K~, P, the
    // parts of S; read: the addition, the outputs.
    const uint32_t bar_full = sb + M::bar, bar_free = bar_full + 24, bar_qk = bar_full + 48, bar_o1 = bar_qk + 8,
                   bar_ds = bar_qk + 16, bar_o2 = bar_qk + 32, bar_kd = bar_qk + 40, bar_p = bar_qk + 56, bar_sp = bar_qk + 64,
                   bar_dsr = bar_qk + 72, bar_or = bar_qk + 80, s_taddr = bar_qk + 88;
    constexpr int kKdWarps = STATE ? 6 : 4;  // warps 10, 11, 14, 15 (the state alone: all of 8-15 but 12 and 13)
    if (tid == 0) {
        for (int i = 0; i < kLtStages; ++i) {
            mbar_init(bar_full + 8 * i, 2);
            mbar_init(bar_free + 8 * i, 1);
        }
        mbar_init(bar_qk, 1);
        mbar_init(bar_o1, 1);
        mbar_init(bar_ds, 1);
        mbar_init(bar_ds + 8, 1);
        mbar_init(bar_o2, 1);
        mbar_init(bar_kd, 32 * kKdWarps);
        mbar_init(bar_kd + 8, 32 * kKdWarps);
        mbar_init(bar_p, 96);
        mbar_init(bar_sp, 256);
        mbar_init(bar_dsr, 256);
        mbar_init(bar_or, 32 * 7);  // warps 8-15 but 12
        fence_mbar_init();
    }
    // Rows of different lengths: the long ones first, and every other round of items backwards, so that
    // the CTAs end together.
    if (!STATE && p.sorted) {
        uint32_t *const pieces = reinterpret_cast<uint32_t *>(smem + M::p);  // of the rows, where P will be
        if (tid < p.sorted) pieces[tid] = (uint32_t)(min(max(p.lengths[tid], 0), p.T) + kLtC - 1) / kLtC;
        __syncthreads();
        if (tid < p.sorted) {
            const uint32_t own = pieces[tid];
            int before = 0;
#pragma unroll 4
            for (int r = 0; r < p.sorted; ++r) before += pieces[r] > own || (pieces[r] == own && r < tid);
            reinterpret_cast<uint16_t *>(smem + M::order)[before] = (uint16_t)tid;
        }
    }
    if (tid >= 480) {
        sts128(sb + M::zero + 16 * (tid - 480), make_uint4(0u, 0u, 0u, 0u));
        fence_proxy_async_smem();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_taddr), "r"(kLtCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = lds32(s_taddr);
    const uint32_t tl = tmem + ((uint32_t)(32 * (warp & 3)) << 16);  // this warp's lanes

    const bool bulk_clear = (reinterpret_cast<uintptr_t>(p.o) & 15) == 0;  // warp 13 clears the rows of live items
    const int T = p.T, segs = STATE ? p.nseg - 1 : p.nseg;
    // The items of this CTA in order.  A cursor holds the next one's row values, fetched an item ahead.
    struct Cursor {
        int i, step, slot, len;
    };
    auto row_of = [&](int b) { return !STATE && p.sorted ? (int)reinterpret_cast<const uint16_t *>(smem + M::order)[b] : b; };
    auto fetch_row = [&](Cursor &c) {
        if (c.i >= p.items) return;
        const int b = row_of(c.i / segs / p.nc / p.H);
        c.slot = b;
        c.len = T;
        if (p.slot_idx) asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(c.slot) : "l"(p.slot_idx + b));
        if (p.lengths) asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(c.len) : "l"(p.lengths + b));
    };
    auto first_item = [&]() {
        Cursor c{(int)blockIdx.x, 2 * (int)(gridDim.x - blockIdx.x) - 1, 0, 0};
        fetch_row(c);
        return c;
    };
    auto item_at = [&](const Cursor &c) {
        LtItem x;
        const int index = c.i / segs, row = index / p.nc;
        x.seg = c.i - index * segs;
        x.index = index;
        x.c = index - row * p.nc;
        const int b = row / p.H;
        x.b = row_of(b);
        x.h = row - b * p.H;
        x.slot = c.slot;
        x.len = min(max(c.len, 0), T);
        x.t_begin = x.seg * p.seg_len;
        x.t_end = min(min(x.t_begin + p.seg_len, T), x.len);
        x.live = x.slot >= 0 && x.slot < p.num_slots && x.t_begin < x.len && !(STATE && x.t_end == x.len);
        return x;
    };
    auto step_item = [&](Cursor &c) {
        c.i += c.step;
        c.step = 2 * (int)gridDim.x - c.step;
        fetch_row(c);
    };
    auto to_live = [&](Cursor &c) {  // to the next item with work; false: there is none
        for (; c.i < p.items; step_item(c))
            if (item_at(c).live) return true;
        return false;
    };
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t phase) {  // the warp's lanes agree
        if (ok) ok = __all_sync(kFull, mbar_wait_bounded(bar, phase & 1u));
        return ok;
    };
    auto wait_ds = [&](uint32_t w) { return wait(bar_ds + 8 * (w & 1u), w >> 1); };
    auto stage_of = [&](uint32_t u) { return sb + (u % kLtStages) * M::stage; };
    auto gates_of = [&](uint32_t u) { return sb + M::g + (u % kLtGates) * M::gbuf; };
    uint32_t u = 0;  // pieces so far: the stage and the phases of a piece

    if (warp < 8) {
        // ---- the state: value column `row`, key channels NR half .. ----
        const uint32_t tD = tl + kLtD + (uint32_t)(NR * half), tS = tl + kLtS + (uint32_t)(3 * NR / 2 * half);
        auto clear_rows = [&](const LtItem &x) {  // past the length
            if (STATE || (x.live && bulk_clear) || !(FULL || x.c * 128 + row < p.dv)) return;
            const int64_t ostep = (int64_t)p.H * p.dv;
            float *const o = p.o + ((int64_t)x.b * T * p.H + x.h) * p.dv + x.c * 128 + row;
            for (int t = max(x.len, x.t_begin) + half; t < min(x.t_begin + p.seg_len, T); t += 2) o[t * ostep] = 0.f;
        };
        for (Cursor cur = first_item(); cur.i < p.items && ok;) {
            const LtItem x = item_at(cur);
            step_item(cur);
            if (!x.live) {
                if (x.slot < 0 || x.slot >= p.num_slots) {
                    if (tid == 0) atomicOr(p.status, (uint32_t)kDevBadSlot);
                } else {
                    clear_rows(x);
                }
                continue;
            }
            float2 S[NR / 2];
            const bool on = FULL || x.c * 128 + row < p.dv;
            float *const st = p.state + ((x.slot * p.H + x.h) * DK + NR * half) * (int64_t)p.dv + x.c * 128 + (on ? row : 0);
            float *const part0 = p.part + (x.index * p.nseg * DK + NR * half) * 128 + row;
            auto load_state = [&](const float *src, int64_t ld) {
#pragma unroll
                for (int r = 0; r < NR / 2; ++r) S[r] = make_float2(src[(2 * r) * ld], src[(2 * r + 1) * ld]);
            };
            auto store_state = [&](float *dst, int64_t ld) {
#pragma unroll
                for (int r = 0; r < NR / 2; ++r) {
                    dst[(2 * r) * ld] = S[r].x;
                    dst[(2 * r + 1) * ld] = S[r].y;
                }
            };
            // Parts of a split row: 0 the state before it (the last segment overwrites the pool's while
            // others may still start), 1 the state after segment 0, s what segment s - 1 adds; joined
            // between the launches to the state before segment s.
            if (STATE && x.seg > 0) {
#pragma unroll
                for (int r = 0; r < NR / 2; ++r) S[r] = make_float2(0.f, 0.f);
            } else if (STATE || (x.seg == 0 && x.t_end == x.len)) {
                load_state(st, p.dv);
                if (!on) {
#pragma unroll
                    for (int r = 0; r < NR / 2; ++r) S[r] = make_float2(0.f, 0.f);
                }
                if (STATE) store_state(part0, 128);
            } else {
                load_state(part0 + (int64_t)x.seg * DK * 128, 128);
            }
            // S as three bf16 parts: the half's hi words, mid words, lo words
            auto write_parts = [&]() {
#pragma unroll
                for (int r8 = 0; r8 < NR / 16; ++r8) {  // 16 rows
                    uint32_t hw[8], mw[8], lw[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) lt_split(S[8 * r8 + e], hw[e], mw[e], lw[e]);
                    lt_st8(tS + 8 * r8, hw);
                    lt_st8(tS + NR / 2 + 8 * r8, mw);
                    lt_st8(tS + NR + 8 * r8, lw);
                }
                lt_wait_st();
                tc_fence_before();
                mbar_arrive(bar_sp);
            };
            if (!STATE) {
                if (u > 0 && !wait(bar_o1, u - 1)) break;
                write_parts();
                clear_rows(x);
            }
#pragma unroll 1
            for (int t0 = x.t_begin; t0 < x.t_end; t0 += kLtC, ++u) {
                if (!wait_ds(u)) break;
                tc_fence_after();
                const float2 eC = splat2(ldsf(gates_of(u) + 512 + 4 * 63));
#pragma unroll
                for (int r8 = 0; r8 < NR / 16; ++r8) {
                    float d[16];
                    lt_ld16(tD + 16 * r8, d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) S[8 * r8 + e] = fma2(S[8 * r8 + e], eC, make_float2(d[2 * e], d[2 * e + 1]));
                }
                tc_fence_before();
                mbar_arrive(bar_dsr);
                if (!STATE && t0 + kLtC < x.t_end) {
                    if (!wait(bar_o1, u)) break;
                    write_parts();
                }
            }
            if (!ok) break;
            if (STATE) store_state(part0 + (int64_t)(x.seg + 1) * DK * 128, 128);
            else if (x.t_end == x.len && on) store_state(st, p.dv);
        }
    } else if (warp == 12) {
        // ---- products (the small parts first: a sum is cut off at its own size after every step) ----
        const LtDesc dp = lt_uniform(tc_desc(sb + M::p, 128, 512));
        const uint32_t tm = __reduce_max_sync(kFull, tmem);
        auto landed = [&](uint32_t w) { return wait(bar_full + 8 * (w % kLtStages), w / kLtStages); };
        for (Cursor cur = first_item(); ok && to_live(cur);) {
            const LtItem x = item_at(cur);
            step_item(cur);
#pragma unroll 1
            for (int t0 = x.t_begin; t0 < x.t_end; t0 += kLtC, ++u) {
                const uint32_t at = stage_of(u), vt = at + M::v;
                const LtDesc dv = lt_uniform(lt_desc_sw(vt, kLtBox, 1024));
                if (!landed(u)) break;
                const int n = x.t_end - t0;
                if (n < kLtC) {  // v past the row's length may hold anything: zero, as 0 times it has to be
                    for (int e = lane; e < (kLtC - n) * 16; e += 32)
                        sts128(vt + (uint32_t)((e & 1) * kLtBox + (n + (e >> 4)) * 128 + ((e >> 1) & 7) * 16), make_uint4(0u, 0u, 0u, 0u));
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                // K step ks of the products Q K^T
                auto mma_qk = [&](LtDesc q, LtDesc k, int ks) {
                    const uint32_t off = (uint32_t)(kLtBox * (ks / 4) + 32 * (ks % 4));
                    lt_mma(tm + kLtG, lt_at(q, off), lt_at(k, off), kIdG, ks != 0);
                };
                if (!STATE && u == 0) {
                    const LtDesc q = lt_uniform(lt_desc_sw(at + M::q, 16, 1024)), k = lt_uniform(lt_desc_sw(at + M::k, 16, 1024));
#pragma unroll
                    for (int ks = 0; ks < DK / 16; ++ks) mma_qk(q, k, ks);
                    lt_commit(bar_qk);
                }
                // what the piece adds to S
                if (!wait(bar_kd + 8 * (u & 1u), u >> 1) || (u > 0 && !wait(bar_dsr, u - 1))) break;
                tc_fence_after();
                {
                    const LtDesc kd = lt_uniform(tc_desc(sb + M::kd + (STATE ? (u & 1u) * 3 * M::tile : 0u), 16 * DK, 128));
#pragma unroll 1
                    for (int part = 2; part >= 0; --part)
#pragma unroll
                        for (int ks = 0; ks < kLtC / 16; ++ks)
                            lt_mma(tm + kLtD, lt_at(dv, 2048 * ks), lt_at(kd, M::tile * part + 32 * DK * ks), kIdS, part != 2 || ks != 0);
                    lt_commit(bar_ds + 8 * (u & 1u));
                }
                if (!STATE) {
                    // the next piece's Q K^T first: its conversion is next
                    if (!wait(bar_p, u)) break;
                    const LtDesc q = lt_uniform(lt_desc_sw(at + M::q, 16, 1024));
                    if (t0 + kLtC < x.t_end || to_live(cur)) {
                        if (!landed(u + 1)) break;
                        tc_fence_after();
                        const uint32_t to = stage_of(u + 1);
                        const LtDesc q1 = lt_uniform(lt_desc_sw(to + M::q, 16, 1024)), k1 = lt_uniform(lt_desc_sw(to + M::k, 16, 1024));
#pragma unroll
                        for (int ks = 0; ks < DK / 16; ++ks) mma_qk(q1, k1, ks);
                        lt_commit(bar_qk);
                    }
                    if (!wait(bar_sp, u) || (u > 0 && !wait(bar_or, u - 1))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int part = 2; part >= 0; --part)
#pragma unroll
                        for (int ks = 0; ks < DK / 16; ++ks) {
                            constexpr int HS = DK / 32;  // K steps per half
                            lt_mma_ta(tm + kLtO1, tm + kLtS + (uint32_t)(3 * NR / 2 * (ks / HS) + NR / 2 * part + 8 * (ks % HS)),
                                      lt_at(q, kLtBox * (ks / 4) + 32 * (ks % 4)), kIdG, part != 2 || ks != 0);
                        }
                    lt_commit(bar_o1);
#pragma unroll 1
                    for (int part = 2; part >= 0; --part)
#pragma unroll
                        for (int ks = 0; ks < kLtC / 16; ++ks) {
                            if (ks < 2) lt_mma(tm + kLtO2, lt_at(dv, 2048 * ks), lt_at(dp, M::ppart * part + 256 * ks), kIdO2, part != 2 || ks != 0);
                            else lt_mma(tm + kLtO2 + 32, lt_at(dv, 2048 * ks), lt_at(dp, M::ppart * part + 4096 + 256 * (ks - 2)), kIdO2b, 1);
                        }
                    lt_commit(bar_o2);
                }
                lt_commit(bar_free + 8 * (u % kLtStages));
            }
        }
        if (!ok) {  // products that did not complete in time get one more bounded wait
            mbar_wait_bounded(bar_ds + 8 * (u & 1u), (u >> 1) & 1u);
            if (!STATE) mbar_wait_bounded(bar_o2, u & 1u);
        }
        __syncwarp();
    } else {
        // ---- K~ and P of a piece, then the outputs of the piece before; warp 13 copies, warp 9 sums ----
        // The next piece to copy (warp 13) or to sum the gates of (warp 9; the state alone: warp 13 too)
        struct Next {
            Cursor cur;
            bool live;
            int t;
            LtItem x;
            uint32_t u;
        } nx;
        nx.cur = first_item();
        nx.u = 0;
        auto find_live = [&]() {
            nx.live = to_live(nx.cur);
            if (!nx.live) return;
            nx.x = item_at(nx.cur);
            nx.t = nx.x.t_begin;
            step_item(nx.cur);
        };
        auto advance = [&]() {
            ++nx.u;
            nx.t += kLtC;
            if (nx.t >= nx.x.t_end) find_live();
        };
        auto copy_piece = [&]() {
            const LtItem &x = nx.x;
            const uint32_t full = bar_full + 8 * (nx.u % kLtStages), at = stage_of(nx.u);
            if (lane == 0) {
                const int hq = (int)((int64_t)x.h * p.Hqk / p.H);
                mbar_arrive_expect_tx(full, ((STATE ? 1 : 2) * (DK / 64) + 2) * kLtBox);
                if (!STATE) lt_copy_boxes(at + M::q, &qmap, 0, hq, nx.t, x.b, full);
                lt_copy_boxes(at + M::k, &kmap, 0, hq, nx.t, x.b, full);
                lt_copy_boxes(at + M::v, &vmap, 2 * x.c, x.h, nx.t, x.b, full);
            }
            __syncwarp();
        };
        float gate_a = 0.f, gate_b = 0.f;   // tokens 2 lane and 2 lane + 1 of the next piece
        Pair dec_total{0.f, 0.f};           // base-2 log of the segment's decay (the state alone)
        auto fetch_gates = [&]() {          // a piece ahead of their use
            if (!nx.live) return;
            const LtItem &x = nx.x;
            const float *const g0 = p.g_per_head ? p.g + x.h : p.g + (int64_t)x.b * T * p.H + x.h;
            const int64_t gstep = p.g_per_head ? 0 : p.H;
            const int t = nx.t + 2 * lane;
            gate_a = gate_b = 0.f;
            if (t < x.t_end) gate_a = __ldg(g0 + (int64_t)t * gstep);
            if (t + 1 < x.t_end) gate_b = __ldg(g0 + (int64_t)(t + 1) * gstep);
        };
        // inclusive sums of a piece's gates in base 2 as pairs of floats; `full` waits for them too
        auto sum_gates = [&]() {
            const LtItem &x = nx.x;
            const uint32_t sg = gates_of(nx.u);
            constexpr float kLog2eF = 1.4426950408889634f;
            const float ga = gate_a < -200.f ? -200.f : gate_a;  // e^-200 is 0 in FP32 (-inf: a reset)
            const float gb = gate_b < -200.f ? -200.f : gate_b;
            const Pair x0{ga * kLog2eF, 0.f};
            Pair s = add_pair(x0, Pair{gb * kLog2eF, 0.f});
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) {
                const Pair y{__shfl_up_sync(kFull, s.hi, m), __shfl_up_sync(kFull, s.lo, m)};
                if (lane >= m) s = add_pair(s, y);
            }
            Pair before{__shfl_up_sync(kFull, s.hi, 1), __shfl_up_sync(kFull, s.lo, 1)};
            if (lane == 0) before = Pair{0.f, 0.f};
            const Pair first = add_pair(before, x0);
            sts128(sg + 16 * lane, make_uint4(__float_as_uint(first.hi), __float_as_uint(first.lo), __float_as_uint(s.hi), __float_as_uint(s.lo)));
            sts32(sg + 512 + 8 * lane, __float_as_uint(lt_exp2(first)));
            sts32(sg + 512 + 8 * lane + 4, __float_as_uint(lt_exp2(s)));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_full + 8 * (nx.u % kLtStages));
            if (STATE) {
                dec_total = add_pair(dec_total, Pair{__shfl_sync(kFull, s.hi, 31), __shfl_sync(kFull, s.lo, 31)});
                if (nx.t + kLtC >= x.t_end) {
                    if (lane == 0) p.part_dec[x.index * p.nseg + x.seg + 1] = lt_exp2(dec_total);
                    dec_total = Pair{0.f, 0.f};
                }
            }
        };
        // the piece after the last of warp 13 or 9, once its stage is free (warp 9: its buffer of sums is,
        // with the outputs of three pieces before)
        auto next_piece = [&]() {
            if (!nx.live) return;
            if (warp == 13) {
                if (nx.u >= kLtStages && !wait(bar_free + 8 * (nx.u % kLtStages), nx.u / kLtStages - 1)) return;
                if (!STATE && bulk_clear && nx.t == nx.x.t_begin) {  // output rows past the row's length
                    const LtItem &x = nx.x;
                    const int t1 = min(x.t_begin + p.seg_len, T);
                    float *const o = p.o + ((int64_t)x.b * T * p.H + x.h) * p.dv + x.c * 128;
                    for (int t = x.len + lane; t < t1; t += 32)
                        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(o + (int64_t)t * p.H * p.dv),
                                     "r"(sb + M::zero), "r"(4 * min(128, p.dv - x.c * 128))
                                     : "memory");
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    __syncwarp();
                }
                copy_piece();
                // its state into L2, up to three items ahead of its use (a segment's is there from the join)
                if (!STATE && nx.t == nx.x.t_begin && p.nseg == 1) {
                    const LtItem &x = nx.x;
                    const float *const from = p.state + ((x.slot * p.H + x.h) * DK + (lane >> 2)) * (int64_t)p.dv + x.c * 128 + 32 * (lane & 3);
                    if (FULL || x.c * 128 + 32 * (lane & 3) < p.dv) {
#pragma unroll 4
                        for (int r = 0; r < DK; r += 8) asm volatile("prefetch.global.L2 [%0];" ::"l"(from + (int64_t)r * p.dv));
                    }
                }
            }
            if (STATE || warp == 9) sum_gates();
            advance();
            if (STATE || warp == 9) fetch_gates();
        };
        auto convert = [&](int n) {
            const uint32_t sg = gates_of(u), ks = stage_of(u) + M::k;
            if (!wait(bar_full + 8 * (u % kLtStages), u / kLtStages)) return;
            if (STATE || (warp & 3) >= 2) {  // K~ = e^{G_C - G_j} k_j
                if (u >= M::kdn && !wait_ds(u - M::kdn)) return;
                const uint32_t kd = sb + M::kd + (STATE ? (u & 1u) * 3 * M::tile : 0u);
                const float Ch = ldsf(sg + 8 * 63), Cl = ldsf(sg + 8 * 63 + 4);
                // Small loop bodies here and below: the roles run different code at the same time, and what is
                // unrolled whole misses the instruction caches.
                auto fetch = [&](int t, int c) { return lds128(ks + (uint32_t)(kLtBox * (c >> 3) + t * 128 + ((c ^ t) & 7) * 16)); };
                auto cell = [&](uint4 w4, int t, int c, float2 f) {
                    if (t >= n) w4 = make_uint4(0u, 0u, 0u, 0u);  // past the row's length
                    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
                    uint32_t hw[4], mw[4], lw[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        lt_split(mul2(make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u)), f), hw[e], mw[e], lw[e]);
                    const uint32_t dst = kd + (uint32_t)((t >> 3) * CELLS * 128 + c * 128 + (t & 7) * 16);
                    sts128(dst, make_uint4(hw[0], hw[1], hw[2], hw[3]));
                    sts128(dst + M::tile, make_uint4(mw[0], mw[1], mw[2], mw[3]));
                    sts128(dst + 2 * M::tile, make_uint4(lw[0], lw[1], lw[2], lw[3]));
                };
                auto factor = [&](int t) { return splat2(lt_exp2(Pair{Ch - ldsf(sg + 8 * t), Cl - ldsf(sg + 8 * t + 4)})); };
                if (STATE) {
                    const int first = 32 * (warp < 12 ? warp - 8 : warp - 10) + lane;
                    static_assert(32 * kKdWarps % kLtC == 0 || !STATE, "a thread's cells are of one token");
                    const int t = first % kLtC;
                    const float2 f = factor(t);
                    uint4 w = fetch(t, first / kLtC);
#pragma unroll 1
                    for (int e = first; e < kLtC * CELLS; e += 32 * kKdWarps) {
                        const uint4 w1 = fetch(t, min(e + 32 * kKdWarps, kLtC * CELLS - 1) / kLtC);
                        cell(w, t, e / kLtC, f);
                        w = w1;
                    }
                } else {
                    const int t = (warp & 1) * 32 + lane, c0 = CELLS / 2 * half;
                    const float2 f = factor(t);
                    uint4 w = fetch(t, c0);
#pragma unroll 1
                    for (int i = 0; i < CELLS / 2; ++i) {
                        const uint4 w1 = fetch(t, c0 + min(i + 1, CELLS / 2 - 1));
                        cell(w, t, c0 + i, f);
                        w = w1;
                    }
                }
                fence_proxy_async_smem();
                mbar_arrive(bar_kd + 8 * (u & 1u));
            } else {  // P: rows 0-31; rows 32-63, columns 0-31 and 32-63
                if (!wait(bar_qk, u) || (u > 0 && !wait(bar_o2, u - 1))) return;
                tc_fence_after();
                const float gih = ldsf(sg + 8 * row), gil = ldsf(sg + 8 * row + 4);
                const uint32_t prow = sb + M::p + (half ? 4096u + (uint32_t)(((row - 32) >> 3) * 512) : (uint32_t)((row >> 3) * 512)) +
                                      (uint32_t)((row & 7) * 16);
#pragma unroll 1
                for (int g8 = 0; g8 < 4; ++g8) {
                    const int j8 = 32 * half + 8 * g8;
                    float x[8];
                    lt_ld8(tl + kLtG + j8, x);
                    uint4 gates[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) gates[e] = lds128(sg + 8 * (j8 + 2 * e));
                    uint32_t hw[4], mw[4], lw[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = j8 + 2 * e;
                        const float d0 = (gih - __uint_as_float(gates[e].x)) + (gil - __uint_as_float(gates[e].y));
                        const float d1 = (gih - __uint_as_float(gates[e].z)) + (gil - __uint_as_float(gates[e].w));
                        lt_split(make_float2(j <= row ? x[2 * e] * lt_ex2(d0) : 0.f, j + 1 <= row ? x[2 * e + 1] * lt_ex2(d1) : 0.f),
                                 hw[e], mw[e], lw[e]);
                    }
                    const uint32_t at = prow + (uint32_t)(g8 * 128);
                    sts128(at, make_uint4(hw[0], hw[1], hw[2], hw[3]));
                    sts128(at + M::ppart, make_uint4(mw[0], mw[1], mw[2], mw[3]));
                    sts128(at + 2 * M::ppart, make_uint4(lw[0], lw[1], lw[2], lw[3]));
                }
                tc_fence_before();  // Q K^T is read
                fence_proxy_async_smem();
                mbar_arrive(bar_p);
            }
        };
        // o_i = O2_i + e^{G_i} O1_i of piece w: this warp's value columns and 32 tokens (warp 8: all 64,
        // those of warp 12 too)
        const int64_t ostep = (int64_t)p.H * p.dv;
        auto output = [&](uint32_t w, float *dst, int n, bool on) {
            if (!wait(bar_o2, w)) return;
            tc_fence_after();
            const int j_end = warp == 8 ? 64 : 32 * half + 32;
            const uint32_t eg = gates_of(w) + 512;
            float *oj = dst + (int64_t)(32 * half) * ostep;
#pragma unroll 1
            for (int j = 32 * half; j < j_end; j += 16) {  // 16 tokens
                float o1[16], o2[16];
                lt_ld16(tl + kLtO1 + j, o1);
                lt_ld16(tl + kLtO2 + j, o2);
                // a v_j that is not finite is in every output of the product, in the first one too (looked
                // for after the combination, with a jump past the rest, which costs the long prompt 262 -> 270 us;
                // elsewhere in the loop, with d = 64, up to 12 %)
                const bool bad = (FULL || on) && !(fabsf(o2[0]) <= FLT_MAX);
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const uint4 g4 = lds128(eg + 4 * (j + e));
                    o1[e] = fmaf(__uint_as_float(g4.x), o1[e], o2[e]);
                    o1[e + 1] = fmaf(__uint_as_float(g4.y), o1[e + 1], o2[e + 1]);
                    o1[e + 2] = fmaf(__uint_as_float(g4.z), o1[e + 2], o2[e + 2]);
                    o1[e + 3] = fmaf(__uint_as_float(g4.w), o1[e + 3], o2[e + 3]);
                }
                if (!STATE && __any_sync(kFull, bad)) {
                    lt_outputs<DK>(in, p.H, p.Hqk, p.dv, p.o, dst, row, gates_of(w), tl + kLtO1, j, min(j + 16, n), FULL || on);
                    if (j + 16 == j_end) {
                        tc_fence_before();
                        mbar_arrive(bar_or);
                    }
                    oj += 16 * ostep;
                    continue;
                }
                if (j + 16 == j_end) {
                    tc_fence_before();
                    mbar_arrive(bar_or);
                }
                const int nh = FULL || on ? n - j : 0;
#pragma unroll
                for (int e = 0; e < 16; ++e, oj += ostep)
                    if (e < nh) *oj = o1[e];
            }
        };
        if (warp == 13 || (!STATE && warp == 9)) {
            find_live();
            if (STATE || warp == 9) fetch_gates();
            for (int i = 0; i < kLtStages; ++i) next_piece();
            while (STATE && nx.live && ok) next_piece();
        }
        float *before = nullptr;  // the piece whose outputs are due
        int before_n = 0;
        bool before_on = false;
        for (Cursor cur = first_item(); ok && !(STATE && warp == 13) && to_live(cur);) {
            const LtItem x = item_at(cur);
            step_item(cur);
            float *const o = p.o + ((int64_t)x.b * T * p.H + x.h) * p.dv + x.c * 128 + row;
#pragma unroll 1
            for (int t0 = x.t_begin; t0 < x.t_end && ok; t0 += kLtC, ++u) {
                convert(x.t_end - t0);
                if (!STATE) {
                    if (before) {
                        output(u - 1, before, before_n, before_on);
                        if (warp == 13 || warp == 9) next_piece();
                    }
                    before = o + (int64_t)t0 * ostep;
                    before_n = x.t_end - t0;
                    before_on = FULL || x.c * 128 + row < p.dv;
                }
            }
        }
        if (!STATE && before && ok) output(u - 1, before, before_n, before_on);
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        if (!ok && warp == 13) {  // copies that did not land in time get one more bounded wait
            for (uint32_t w = nx.u > kLtStages ? nx.u - kLtStages : 0; w < nx.u; ++w)
                mbar_wait_bounded(bar_full + 8 * (w % kLtStages), (w / kLtStages) & 1u);
        }
    }
    if (!ok && lane == 0) atomicOr(p.status, (uint32_t)kDevWaitTimeout);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kLtCols) : "memory");
    }
}

// part s of every split row, head and columns, from what segment s - 1 adds to the state before segment s
__global__ void __launch_bounds__(256) lin_tc_join_kernel(const LinTcParams p, int dk) {
    const int64_t n = (int64_t)dk * 32, e = (int64_t)blockIdx.x * 256 + threadIdx.x, index = e / n;  // 16 bytes each
    const int b = (int)(index / p.nc / p.H);
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
    float4 *const at = reinterpret_cast<float4 *>(p.part) + index * p.nseg * n + e % n;
    if (2 * (int64_t)p.seg_len >= len) return;  // two segments at most
    const int64_t slot = p.slot_idx ? (int64_t)p.slot_idx[b] : (int64_t)b;
    if (slot < 0 || slot >= p.num_slots) return;  // a skipped row has no parts
    float4 S = at[n];
    for (int s = 2; s < p.nseg && s * (int64_t)p.seg_len < len; ++s) {
        const float d = p.part_dec[index * p.nseg + s];
        const float4 x = at[s * n];
        S = make_float4(fmaf(S.x, d, x.x), fmaf(S.y, d, x.y), fmaf(S.z, d, x.z), fmaf(S.w, d, x.w));
        at[s * n] = S;
    }
}

// Segments of a launch (1: no split) and the tokens of each.  The CTAs (one per SM) take the items
// in rounds; the cost of a choice is its rounds times the pieces of an item and about three more
// for its start and end, and half as much again for the launch that computes the states.
int lin_tc_segments(const LinArgs &a, int *seg_len) {
    const int64_t items = (int64_t)a.batch * a.H * ((a.dv + 127) / 128), sms = sm_count();
    const int pieces = (a.T + kLtC - 1) / kLtC;
    auto cost = [&](int nseg) {
        const int64_t per = (pieces + nseg - 1) / nseg + 3;
        const int64_t main = (items * nseg + sms - 1) / sms * per, states = nseg > 1 ? (items * (nseg - 1) + sms - 1) / sms * per : 0;
        return 2 * main + states;
    };
    int best = 1;
    if (items < 2 * sms)
        for (int nseg = 2; nseg <= std::min(pieces / 4, 64); ++nseg)
            if (cost(nseg) < cost(best)) best = nseg;
    const int per = (pieces + best - 1) / best;  // pieces of a segment
    *seg_len = per * kLtC;
    return (pieces + per - 1) / per;
}

// cuTensorMapEncodeTiled through the runtime (libdamp does not link the driver library)
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
cudaError_t encode_tiled(EncodeTiled *out) {
    static std::atomic<EncodeTiled> cached{nullptr};
    EncodeTiled f = cached.load(std::memory_order_acquire);
    if (!f) {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return e;
        if (found != cudaDriverEntryPointSuccess || !ptr) return cudaErrorNotSupported;
        f = reinterpret_cast<EncodeTiled>(ptr);
        cached.store(f, std::memory_order_release);
    }
    *out = f;
    return cudaSuccess;
}
// boxes of 64 channels x 64 tokens of one head and batch row, `groups` of 64 channels at once (64-channel
// groups are the fourth dimension: a box of one follows the other); tokens past T read as zeros
cudaError_t lin_tc_map(CUtensorMap *map, const void *base, int channels, int heads, int T, int batch, int groups) {
    EncodeTiled encode;
    const cudaError_t e = encode_tiled(&encode);
    if (e != cudaSuccess) return e;
    const cuuint64_t dims[5] = {64, (cuuint64_t)heads, (cuuint64_t)T, (cuuint64_t)channels / 64, (cuuint64_t)batch};
    const cuuint64_t row = (cuuint64_t)channels * 2;
    const cuuint64_t strides[4] = {row, row * (cuuint64_t)heads, 128, row * (cuuint64_t)heads * (cuuint64_t)T};
    const cuuint32_t box[5] = {64, 1, kLtC, (cuuint32_t)groups, 1}, steps[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(base), dims, strides, box, steps,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

struct LinTcMaps {
    CUtensorMap q, k, v;
    LinTcInputs in;
};

template <int DK, bool STATE, bool FULL>
cudaError_t lin_tc_launch_one(const LinTcParams &p, const LinTcMaps &m, int64_t items, cudaStream_t s) {
    const void *const kern = reinterpret_cast<const void *>(lin_tc_kernel<DK, STATE, FULL>);
    const cudaError_t e = ensure_smem_limit(kern, LtSmem<DK, STATE>::bytes);
    if (e != cudaSuccess) return e;
    LinTcParams q = p;
    q.items = (int32_t)items;
    lin_tc_kernel<DK, STATE, FULL><<<(unsigned)std::min<int64_t>(items, sm_count()), kLtThreads, LtSmem<DK, STATE>::bytes, s>>>(q, m.q, m.k, m.v, m.in);
    return cudaGetLastError();
}

template <bool STATE>
cudaError_t lin_tc_launch(const LinTcParams &p, const LinTcMaps &m, int dk, int64_t items, cudaStream_t s) {
    if (p.dv % 128 == 0) return dk == 64 ? lin_tc_launch_one<64, STATE, true>(p, m, items, s) : lin_tc_launch_one<128, STATE, true>(p, m, items, s);
    return dk == 64 ? lin_tc_launch_one<64, STATE, false>(p, m, items, s) : lin_tc_launch_one<128, STATE, false>(p, m, items, s);
}

}  // namespace

// From 17 tokens on (61 rows of 32 heads, d = 128: 84 us token by token against 87 at T = 16, 118
// against 89 at T = 24; two rows: 9.3 against 9.5 at T = 16).
bool lin_tc_takes(const LinArgs &a) {
    return a.in_bf16 && (a.dk == 64 || a.dk == 128) && a.dv % 64 == 0 && a.T > 16;
}

size_t lin_tc_workspace(const LinArgs &a) {
    int seg_len;
    const int64_t nseg = lin_tc_segments(a, &seg_len);
    const int64_t parts = nseg > 1 ? (int64_t)a.batch * a.H * ((a.dv + 127) / 128) * nseg : 0;
    return (size_t)(parts * (a.dk * 128 + 1) * 4);
}

cudaError_t launch_lin_tc(LinArgs a, void *workspace, cudaStream_t s) {
    LinTcParams p{};
    static std::atomic<uint32_t *> cache[64];
    cudaError_t e = symbol_address_cached(&g_status_lin_tc, cache, &p.status);
    if (e != cudaSuccess) return e;
    p.state = a.state;
    p.num_slots = a.num_slots;
    p.slot_idx = a.slot_idx;
    p.lengths = a.lengths;
    LinTcMaps m;
    m.in = LinTcInputs{static_cast<const __nv_bfloat16 *>(a.q), static_cast<const __nv_bfloat16 *>(a.k), static_cast<const __nv_bfloat16 *>(a.v)};
    if ((e = lin_tc_map(&m.q, a.q, a.dk, a.Hqk, a.T, a.batch, a.dk / 64)) != cudaSuccess) return e;
    if ((e = lin_tc_map(&m.k, a.k, a.dk, a.Hqk, a.T, a.batch, a.dk / 64)) != cudaSuccess) return e;
    if ((e = lin_tc_map(&m.v, a.v, a.dv, a.H, a.T, a.batch, 2)) != cudaSuccess) return e;
    p.g = a.g;
    p.o = a.o;
    p.H = a.H;
    p.Hqk = a.Hqk;
    p.dv = a.dv;
    p.nc = (a.dv + 127) / 128;
    p.T = a.T;
    p.g_per_head = a.g_per_head;
    p.nseg = lin_tc_segments(a, &p.seg_len);
    const int64_t items = (int64_t)a.batch * a.H * p.nc;
    // Rows by length where a CTA has a few items (16 rows of 250 to 1000 tokens, 32 heads: 189 us in
    // their order, 183 by length; 4 rows, 48 heads: 95 and 89; but 24 rows of 128 to 512 tokens, 32 heads:
    // 144 and 151).  With many items the lengths even out by themselves (200 rows of 75 to 300 tokens, 16 heads: 350 in their order, 357 by length).
    const int64_t sms = sm_count();
    p.sorted = a.lengths && p.nseg == 1 && a.batch <= kLtSorted && items > sms && items <= 8 * sms ? (int32_t)a.batch : 0;
    if (p.nseg > 1) {
        p.part = static_cast<float *>(workspace);
        p.part_dec = p.part + items * p.nseg * a.dk * 128;
        e = lin_tc_launch<true>(p, m, a.dk, items * (p.nseg - 1), s);
        if (e != cudaSuccess) return e;
        if (p.nseg > 2) lin_tc_join_kernel<<<(unsigned)(items * a.dk / 8), 256, 0, s>>>(p, a.dk);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    return lin_tc_launch<false>(p, m, a.dk, items * p.nseg, s);
}

cudaError_t take_status_lin_tc(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_lin_tc, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_lin_tc, &zero, sizeof(uint32_t));
}

}  // namespace damp
