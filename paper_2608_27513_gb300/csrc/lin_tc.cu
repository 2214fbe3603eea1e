// lin_tc.cu -- a chunk of linear attention with a decay per head on the tensor cores.
//
// A piece of C = 64 tokens, with G_i = g_0 + ... + g_i inside it (base-2 logs below):
//     o_i = e^{G_i} S_0^T q_i + sum_{j<=i} e^{G_i - G_j} (q_i.k_j) v_j
//     S_C = e^{G_C} S_0 + sum_j (e^{G_C - G_j} k_j) v_j^T
// as four tcgen05.mma products, all transposed so that the value column is the tensor-
// memory lane and an output row is stored by 32 lanes of a warp as one line:
//     [Q; K] K^T          -> Q K^T in lanes 0-63 (the other rows are not used)
//     S_0^T Q^T           -> O1 (A from tensor memory)
//     V^T (K~ = e^{G_C - G_j} k_j)    -> what the piece adds to S^T
//     V^T P^T, P = (e^{G_i - G_j} q_i.k_j)_{j<=i}  -> O2;  o_i = O2_i + e^{G_i} O1_i
// One CTA owns 128 value columns of a (slot, head).  The state stays in registers in FP32
// (thread = value column and half the key channels); only its operand copy is rounded.
//
// Rounding.  q, k and v are bf16 inputs and enter exactly.  The FP32 operands (S_0, K~, P)
// enter as two bf16 parts hi + lo, which leaves at most 2^-16 of a value (2.4e-6 in the
// mean): one part alone would leave 2^-8, a third part costs half as much tensor time
// again and 48 KB.  Accumulation and the state are FP32.  G is summed in FP64 and kept as
// two floats, so that G_i - G_j keeps its digits where both are large (fast decays).
//
// q, k and v come by tensor copies (TMA, 128-byte swizzle), issued as soon as the products that
// read the tile before are done.  Warp 4, which has no part in P and K~, issues copies and
// products and sums the next piece's gates meanwhile.  Two CTAs per SM (110 KB of shared memory,
// 256 of the 512 tensor-memory columns each) overlap one's products with the other's
// conversions.  Bound by the conversions, with the bytes of q, k, v and o next.
//
// Few (slot, head) pairs and many tokens: the tokens are split into segments.  A first
// launch computes what each segment adds to the state (k and v only), a second one starts
// every segment from the joined state before it.
#include <cuda.h>

#include "damp_internal.h"
#include "prefill_tc.cuh"

#include <algorithm>

namespace damp {

static __device__ uint32_t g_status_lin_tc;

namespace {

constexpr int kLtC = 64;
constexpr int kLtThreads = 256;
constexpr int kLtBox = 64 * 128;  // bytes of a copied box: 64 tokens x 64 bf16
constexpr uint32_t kLtCols = 256;
// tensor-memory columns: Q K^T, then O2 | O1 | S_0 as bf16 parts, then what the piece adds
constexpr uint32_t kLtG = 0, kLtO1 = 64, kLtS = 128;

template <int DK>
struct LtSmem {  // bytes from the base of the dynamic shared memory
    static constexpr int tile = kLtC * DK * 2;
    static constexpr int vtile = kLtC * 128 * 2;
    // 64-column boxes: [q box 0][k box 0][q box 1][k box 1], so that [Q; K] is one operand of 128 rows
    static constexpr int q = 0, k = kLtBox;
    static constexpr int v = 2 * tile;        // two buffers of two boxes
    static constexpr int kd = v + 2 * vtile;  // K~ hi, lo
    static constexpr int p = kd + 2 * tile;   // P hi, lo: columns 0-31 of 64 rows, columns 32-63 of rows 32-63
    static constexpr int ppart = 64 * 64 + 32 * 64;
    static constexpr int g = p + 2 * ppart;   // two buffers: (hi, lo) of G in base 2, 64 pairs, and e^{G_i}
    static constexpr int gbuf = 512 + 256;
    static constexpr int bar = g + 2 * gbuf;  // seven mbarriers, the tensor-memory address
    static constexpr int bytes = bar + 64;
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
    int32_t nseg, seg_len;
    uint32_t *status;
};

__device__ __forceinline__ float lt_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// one box of a [batch][token][head][channel] tensor at (channel, head, token, row) into shared memory
__device__ __forceinline__ void lt_copy_box(uint32_t dst, const CUtensorMap *map, int ch, int head, int t, int b, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
                     dst),
                 "l"(map), "r"(ch), "r"(head), "r"(t), "r"(b), "r"(bar)
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
// eight columns at two addresses
__device__ __forceinline__ void lt_ld8x2(uint32_t ta, uint32_t tb, float (&a)[8], float (&b)[8]) {
    uint32_t r[8], s[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%16];\n"
                 "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%8,%9,%10,%11,%12,%13,%14,%15}, [%17];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(s[0]), "=r"(s[1]), "=r"(s[2]), "=r"(s[3]), "=r"(s[4]), "=r"(s[5]), "=r"(s[6]), "=r"(s[7])
                 : "r"(ta), "r"(tb)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        a[i] = __uint_as_float(r[i]);
        b[i] = __uint_as_float(s[i]);
    }
}
__device__ __forceinline__ void lt_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void lt_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// A from tensor memory (K-major: two bf16 per column)
__device__ __forceinline__ void lt_mma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
                 "r"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
}
// x = hi + lo as bf16 parts, two values per word
__device__ __forceinline__ void split2_pair(float2 x, uint32_t &h, uint32_t &l) {
    const __nv_bfloat162 h2 = __floats2bfloat162_rn(x.x, x.y);
    memcpy(&h, &h2, 4);
    const float2 r = add2(x, make_float2(-__uint_as_float(h << 16), -__uint_as_float(h & 0xffff0000u)));  // exact
    const __nv_bfloat162 l2 = __floats2bfloat162_rn(r.x, r.y);
    memcpy(&l, &l2, 4);
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// a sum of two floats, hi + lo
struct Pair {
    float hi, lo;
};
__device__ __forceinline__ Pair add_pair(Pair a, Pair b) {
    const float s = a.hi + b.hi, t = s - a.hi;
    const float e = ((a.hi - (s - t)) + (b.hi - t)) + (a.lo + b.lo);  // the rounding of s, and the low parts
    const float h = s + e;
    return Pair{h, e - (h - s)};
}

// STATE: only what the segment adds to the state and its decay
template <int DK, bool STATE>
__global__ void __launch_bounds__(kLtThreads, 2)
    lin_tc_kernel(const LinTcParams p, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                  const __grid_constant__ CUtensorMap vmap) {
    extern __shared__ __align__(1024) uint8_t smem[];
    using M = LtSmem<DK>;
    constexpr int CELLS = DK / 8;
    constexpr int NR = DK / 2;  // state rows of a thread
    constexpr uint32_t kIdG = tc_idesc(64, false, false), kIdO2 = tc_idesc(64, true, false), kIdO2b = tc_idesc(32, true, false),
                       kIdS = tc_idesc(DK, true, true);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool issuer = warp == 4;
    const int row = 32 * (warp & 3) + lane, half = warp >> 2;
    const uint32_t sb = smem_u32(smem);
    // copies landed; products done: Q K^T, O1, the addition to S, O2; operands written: K~, P
    const uint32_t bar_full = sb + M::bar, bar_qk = bar_full + 8, bar_o1 = bar_full + 16, bar_ds = bar_full + 24,
                   bar_o2 = bar_full + 32, bar_kd = bar_full + 40, bar_p = bar_full + 48, s_taddr = bar_full + 56;

    const int seg = (int)(blockIdx.x % (STATE ? p.nseg - 1 : p.nseg));
    const int item = (int)(blockIdx.x / (STATE ? p.nseg - 1 : p.nseg));
    const int c = item % p.nc, h = (item / p.nc) % p.H, b = item / p.nc / p.H;
    const int64_t slot = p.slot_idx ? (int64_t)p.slot_idx[b] : (int64_t)b;
    if (slot < 0 || slot >= p.num_slots) {
        if (tid == 0) atomicOr(p.status, (uint32_t)kDevBadSlot);
        return;
    }
    const int T = p.T;
    const int len = p.lengths ? min(max(p.lengths[b], 0), T) : T;
    const int t_begin = seg * p.seg_len, t_stop = min(t_begin + p.seg_len, T), t_end = min(t_stop, len);
    const int64_t ostep = (int64_t)p.H * p.dv;
    float *const o = p.o + ((int64_t)b * T * p.H + h) * p.dv + c * 128 + row;
    if (!STATE) {  // rows past the length
        for (int t = max(len, t_begin) + half; t < t_stop; t += 2) o[(int64_t)t * ostep] = 0.f;
    }
    if (t_begin >= len) return;
    if (STATE && t_end == len) return;  // no live segment follows

    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_taddr), "r"(kLtCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    constexpr int kKdWarps = STATE ? 8 : 4, kPWarps = 3;
    if (tid == 0) {
        mbar_init(bar_full, 1);
        mbar_init(bar_qk, 1);
        mbar_init(bar_o1, 1);
        mbar_init(bar_ds, 1);
        mbar_init(bar_o2, 1);
        mbar_init(bar_kd, 32 * kKdWarps);
        mbar_init(bar_p, 32 * kPWarps);
        fence_mbar_init();
    }
    const int hq = (int)((int64_t)h * p.Hqk / p.H);
    constexpr int QKBOX = DK / 64;  // boxes of q or k
    auto copy_qk = [&](int t) {  // one thread
#pragma unroll
        for (int j = 0; j < QKBOX; ++j) {
            if (!STATE) lt_copy_box(sb + M::q + 2 * kLtBox * j, &qmap, 64 * j, hq, t, b, bar_full);
            lt_copy_box(sb + M::k + 2 * kLtBox * j, &kmap, 64 * j, hq, t, b, bar_full);
        }
    };
    auto copy_v = [&](int t, uint32_t buf) {  // one thread; the bytes of the piece's q and k too
        mbar_arrive_expect_tx(bar_full, ((STATE ? 1 : 2) * QKBOX + 2) * kLtBox);
#pragma unroll
        for (int j = 0; j < 2; ++j) lt_copy_box(sb + M::v + buf * M::vtile + kLtBox * j, &vmap, c * 128 + 64 * j, h, t, b, bar_full);
    };
    // Gates of a piece (the issuing warp; lane l holds tokens 2l and 2l + 1): inclusive sums in base 2
    // as pairs of floats, so that G_i - G_j keeps its digits where both are large.
    const float *const g0 = p.g_per_head ? p.g + h : p.g + (int64_t)b * T * p.H + h;
    const int64_t gstep = p.g_per_head ? 0 : p.H;
    float ga = 0.f, gb = 0.f;
    Pair dec_total{0.f, 0.f};  // base-2 log of the segment's decay
    auto fetch_gates = [&](int t) {  // used a piece later
        t += 2 * lane;
        ga = t < t_end ? g0[(int64_t)t * gstep] : 0.f;
        gb = t + 1 < t_end ? g0[(int64_t)(t + 1) * gstep] : 0.f;
    };
    auto sum_gates = [&](int buf) {
        constexpr float kLog2eF = 1.4426950408889634f;
        // below -200, e^g is 0 in FP32 (-inf: a reset)
        const Pair x0{(ga < -200.f ? -200.f : ga) * kLog2eF, 0.f}, x1{(gb < -200.f ? -200.f : gb) * kLog2eF, 0.f},
            own = add_pair(x0, x1);
        Pair x = own;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const Pair y{__shfl_up_sync(kFull, x.hi, m), __shfl_up_sync(kFull, x.lo, m)};
            if (lane >= m) x = add_pair(x, y);
        }
        Pair before{__shfl_up_sync(kFull, x.hi, 1), __shfl_up_sync(kFull, x.lo, 1)};
        if (lane == 0) before = Pair{0.f, 0.f};
        const Pair first = add_pair(before, x0);
        const uint32_t at = sb + M::g + (uint32_t)(buf * M::gbuf);
        sts128(at + 16 * lane, make_uint4(__float_as_uint(first.hi), __float_as_uint(first.lo), __float_as_uint(x.hi), __float_as_uint(x.lo)));
        sts32(at + 512 + 8 * lane, __float_as_uint(lt_ex2(first.hi)));
        sts32(at + 512 + 8 * lane + 4, __float_as_uint(lt_ex2(x.hi)));
        if (STATE) dec_total = add_pair(dec_total, Pair{__shfl_sync(kFull, x.hi, 31), __shfl_sync(kFull, x.lo, 31)});
    };

    // the state before the segment, transposed: value column `row`, key channels NR half ..
    float2 S[NR / 2];
    float *const st = p.state + ((slot * p.H + h) * DK + NR * half) * (int64_t)p.dv + c * 128 + row;
    float *const part0 = p.part + ((int64_t)item * p.nseg * DK + NR * half) * 128 + row;
    const float *const dec0 = p.part_dec + (int64_t)item * p.nseg;
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
    if (issuer) {
        fetch_gates(t_begin);
        sum_gates(0);
        fetch_gates(t_begin + kLtC);
    }
    {
        // Parts of a split row: 0 the state before it (the last segment overwrites the pool's while
        // others may still start), 1 the state after segment 0, s what segment s - 1 adds.
        const bool whole = seg == 0 && t_end == len;  // the row is one segment
        if (STATE && seg > 0) {
#pragma unroll
            for (int r = 0; r < NR / 2; ++r) S[r] = make_float2(0.f, 0.f);
        } else if (STATE || whole) {
            load_state(st, p.dv);
            if (STATE) store_state(part0, 128);
        } else {
            load_state(part0 + (seg > 0 ? DK * 128 : 0), 128);
            for (int s = 2; s <= seg; ++s) {
                const float2 d2 = splat2(dec0[s]);
                const float *const ps = part0 + (int64_t)s * DK * 128;
#pragma unroll
                for (int r = 0; r < NR / 2; ++r) S[r] = fma2(S[r], d2, make_float2(ps[(2 * r) * 128], ps[(2 * r + 1) * 128]));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (tid == 128) {
        copy_v(t_begin, 0);
        copy_qk(t_begin);
    }
    const uint32_t tmem = lds32(s_taddr);
    const uint32_t tl = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const uint32_t tS = tl + kLtS + (uint32_t)(NR * half);  // this thread's columns of both uses

    // S as two bf16 parts: the half's hi words, then its lo words
    auto store_parts = [&]() {
#pragma unroll
        for (int r8 = 0; r8 < NR / 16; ++r8) {  // 16 rows
            uint32_t hw[8], lw[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) split2_pair(S[8 * r8 + i], hw[i], lw[i]);
            lt_st8(tS + 8 * r8, hw);
            lt_st8(tS + NR / 2 + 8 * r8, lw);
        }
        lt_wait_st();
    };
    if (!STATE) store_parts();

    bool ok = true;
    uint32_t buf = 0;  // buffers and the phase of every barrier
#pragma unroll 1
    for (int t0 = t_begin; t0 < t_end; t0 += kLtC, buf ^= 1) {
        const bool more = t0 + kLtC < t_end;
        const uint32_t vt = sb + M::v + buf * M::vtile, sg = sb + M::g + buf * M::gbuf;
        ok &= mbar_wait_bounded(bar_full, buf);
        const int n = t_end - t0;  // tokens of the piece (64 or more: all)
        if (n < kLtC) {  // v past the row's length may hold anything: zero, as 0 times it has to be
            for (int i = tid; i < (kLtC - n) * 16; i += kLtThreads)
                sts128(vt + (uint32_t)((i & 1) * kLtBox + (n + (i >> 4)) * 128 + ((i >> 1) & 7) * 16), make_uint4(0u, 0u, 0u, 0u));
            fence_proxy_async_smem();
        }
        tc_fence_before();
        ok = __syncthreads_and(ok);
        tc_fence_after();
        if (!ok) break;
        auto issue_add = [&]() {  // what the piece adds to S
            if (!STATE) ok &= mbar_wait_bounded(bar_o1, buf);  // it goes over O1's operand
            ok &= mbar_wait_bounded(bar_kd, buf);
            tc_fence_after();
            if (lane == 0) {
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int ks = 0; ks < kLtC / 16; ++ks)
                        tc_mma(tmem + kLtS, lt_desc_sw(vt + 2048 * ks, kLtBox, 1024),
                               tc_desc(sb + M::kd + M::tile * part + 32 * DK * ks, 16 * DK, 128), kIdS, (part | ks) != 0);
                tc_commit(bar_ds);
                if (more) copy_qk(t0 + kLtC);  // q and k are read
            }
            __syncwarp();
        };
        if (issuer) {
            if (lane == 0) {
                if (!STATE) {
#pragma unroll
                    for (int ks = 0; ks < DK / 16; ++ks) {
                        const uint32_t off = (uint32_t)(2 * kLtBox * (ks / 4) + 32 * (ks % 4));
                        tc_mma(tmem + kLtG, lt_desc_sw(sb + M::q + off, 16, 1024), lt_desc_sw(sb + M::k + off, 16, 1024), kIdG, ks != 0);
                    }
                    tc_commit(bar_qk);
#pragma unroll
                    for (int part = 0; part < 2; ++part)
#pragma unroll
                        for (int ks = 0; ks < DK / 16; ++ks) {
                            constexpr int HS = DK / 32;  // K steps per half
                            const uint32_t a = tmem + kLtS + (uint32_t)(NR * (ks / HS) + NR / 2 * part + 8 * (ks % HS));
                            const uint32_t off = (uint32_t)(2 * kLtBox * (ks / 4) + 32 * (ks % 4));
                            lt_mma_ta(tmem + kLtO1, a, lt_desc_sw(sb + M::q + off, 16, 1024), kIdG, (part | ks) != 0);
                        }
                    tc_commit(bar_o1);
                }
                if (more) copy_v(t0 + kLtC, buf ^ 1);
            }
            __syncwarp();
            if (!STATE) {
                if (more) {
                    sum_gates(buf ^ 1);
                    fetch_gates(t0 + 2 * kLtC);
                }
                issue_add();
                ok &= mbar_wait_bounded(bar_p, buf);
                tc_fence_after();
                if (lane == 0) {
#pragma unroll
                    for (int part = 0; part < 2; ++part)
#pragma unroll
                        for (int ks = 0; ks < kLtC / 16; ++ks) {
                            const uint64_t a = lt_desc_sw(vt + 2048 * ks, kLtBox, 1024);
                            const uint32_t pp = sb + M::p + M::ppart * part;
                            if (ks < 2) tc_mma(tmem + kLtG, a, tc_desc(pp + 256 * ks, 128, 512), kIdO2, (part | ks) != 0);
                            else tc_mma(tmem + kLtG + 32, a, tc_desc(pp + 4096 + 256 * (ks - 2), 128, 512), kIdO2b, 1);
                        }
                    tc_commit(bar_o2);
                }
                __syncwarp();
            }
        }
        if (STATE || (warp & 3) >= 2) {  // K~
            constexpr int NC = STATE ? CELLS / 4 : CELLS / 2;  // cells of a thread
            const int kt = STATE ? tid & 63 : (warp & 1) * 32 + lane, c0 = NC * (STATE ? tid >> 6 : half);
            const uint32_t gj = sg + 8 * kt, gC = sg + 8 * 63;
            const float2 f = splat2(lt_ex2((ldsf(gC) - ldsf(gj)) + (ldsf(gC + 4) - ldsf(gj + 4))));
            const uint32_t cell = (uint32_t)((kt >> 3) * CELLS * 128 + (kt & 7) * 16 + c0 * 128);
#pragma unroll 4
            for (int i = 0; i < NC; ++i) {
                const uint32_t off = cell + (uint32_t)(i * 128);
                uint4 w4 = lds128(sb + M::k + (uint32_t)(2 * kLtBox * ((c0 + i) >> 3) + kt * 128 + (((c0 + i) ^ kt) & 7) * 16));
                if (kt >= n) w4 = make_uint4(0u, 0u, 0u, 0u);  // past the row's length
                const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
                uint32_t hw[4], lw[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    split2_pair(mul2(make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u)), f), hw[e], lw[e]);
                sts128(sb + M::kd + off, make_uint4(hw[0], hw[1], hw[2], hw[3]));
                sts128(sb + M::kd + M::tile + off, make_uint4(lw[0], lw[1], lw[2], lw[3]));
            }
            fence_proxy_async_smem();
            mbar_arrive(bar_kd);
        } else if (!issuer) {  // P: rows 0-31; rows 32-63, columns 0-31 and 32-63
            ok &= mbar_wait_bounded(bar_qk, buf);
            tc_fence_after();
            const float gih = ldsf(sg + 8 * row), gil = ldsf(sg + 8 * row + 4);
            const uint32_t prow = sb + M::p + (half ? 4096u + (uint32_t)(((row - 32) >> 3) * 512) : (uint32_t)((row >> 3) * 512)) +
                                  (uint32_t)((row & 7) * 16);
#pragma unroll
            for (int j0 = 0; j0 < 32; j0 += 16) {
                float x[16];
                lt_ld16(tl + kLtG + 32 * half + j0, x);
                const int jb = 32 * half + j0;
#pragma unroll
                for (int g8 = 0; g8 < 2; ++g8) {
                    uint32_t hw[4], lw[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = jb + 8 * g8 + 2 * e;
                        const uint4 gg = lds128(sg + 8 * j);
                        const float d0 = (gih - __uint_as_float(gg.x)) + (gil - __uint_as_float(gg.y));
                        const float d1 = (gih - __uint_as_float(gg.z)) + (gil - __uint_as_float(gg.w));
                        split2_pair(make_float2(j <= row ? x[8 * g8 + 2 * e] * lt_ex2(d0) : 0.f,
                                                j + 1 <= row ? x[8 * g8 + 2 * e + 1] * lt_ex2(d1) : 0.f),
                                    hw[e], lw[e]);
                    }
                    const uint32_t at = prow + (uint32_t)((j0 / 8 + g8) * 128);
                    sts128(at, make_uint4(hw[0], hw[1], hw[2], hw[3]));
                    sts128(at + M::ppart, make_uint4(lw[0], lw[1], lw[2], lw[3]));
                }
            }
            tc_fence_before();  // Q K^T is read: O2 goes over it
            fence_proxy_async_smem();
            mbar_arrive(bar_p);
        }
        if (STATE && issuer) {
            issue_add();
            if (more) {
                sum_gates(buf ^ 1);
                fetch_gates(t0 + 2 * kLtC);
            }
        }
        const float2 eC = splat2(ldsf(sg + 512 + 4 * 63));
        ok &= mbar_wait_bounded(bar_ds, buf);
        tc_fence_after();
#pragma unroll
        for (int r8 = 0; r8 < NR / 16; ++r8) {
            float d[16];
            lt_ld16(tS + 16 * r8, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) S[8 * r8 + i] = fma2(S[8 * r8 + i], eC, make_float2(d[2 * i], d[2 * i + 1]));
        }
        if (!STATE) {
            if (more) store_parts();
            ok &= mbar_wait_bounded(bar_o2, buf);
            tc_fence_after();
            float *const oc = o + (int64_t)(t0 + 32 * half) * ostep;
            const int nh = n - 32 * half;
#pragma unroll
            for (int j0 = 0; j0 < 32; j0 += 8) {
                if (j0 >= nh) break;
                float o1[8], o2[8];
                lt_ld8x2(tl + kLtO1 + 32 * half + j0, tl + kLtG + 32 * half + j0, o1, o2);
                float *oj = oc + j0 * ostep;
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    const uint4 eg = lds128(sg + 512 + 4 * (32 * half + j0 + e));
                    const float ev[4] = {__uint_as_float(eg.x), __uint_as_float(eg.y), __uint_as_float(eg.z), __uint_as_float(eg.w)};
#pragma unroll
                    for (int i = 0; i < 4; ++i, oj += ostep)
                        if (j0 + e + i < nh) *oj = fmaf(ev[i], o1[e + i], o2[e + i]);
                }
            }
        }
    }
    if (ok) ok = __syncthreads_and(ok);
    if (ok) {
        if (STATE) {
            if (tid == 128) p.part_dec[(int64_t)item * p.nseg + seg + 1] = lt_ex2(dec_total.hi);
            store_state(part0 + (int64_t)(seg + 1) * DK * 128, 128);
        } else if (t_end == len) {
            store_state(st, p.dv);
        }
    } else {  // copies and products that did not complete in time get one more bounded wait
        if (tid == 0) atomicOr(p.status, (uint32_t)kDevWaitTimeout);
        mbar_wait_bounded(bar_full, buf);
        mbar_wait_bounded(bar_ds, buf ^ 1);
        if (!STATE) mbar_wait_bounded(bar_o2, buf ^ 1);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kLtCols) : "memory");
    }
}

// segments of a launch (1: no split) and the tokens of each
int lin_tc_segments(const LinArgs &a, int *seg_len) {
    const int64_t items = (int64_t)a.batch * a.H * (a.dv / 128);
    const int pieces = (a.T + kLtC - 1) / kLtC;
    const int64_t room = 2 * (int64_t)sm_count();
    int nseg = (int)std::min<int64_t>(room / std::max<int64_t>(items, 1), pieces / 4);
    if (nseg < 2) nseg = 1;
    const int per = (pieces + nseg - 1) / nseg;  // pieces of a segment
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
// boxes of 64 channels x 64 tokens of one head and batch row; tokens past T read as zeros
cudaError_t lin_tc_map(CUtensorMap *map, const void *base, int channels, int heads, int T, int batch) {
    EncodeTiled encode;
    const cudaError_t e = encode_tiled(&encode);
    if (e != cudaSuccess) return e;
    const cuuint64_t dims[4] = {(cuuint64_t)channels, (cuuint64_t)heads, (cuuint64_t)T, (cuuint64_t)batch};
    const cuuint64_t row = (cuuint64_t)channels * 2;
    const cuuint64_t strides[3] = {row, row * (cuuint64_t)heads, row * (cuuint64_t)heads * (cuuint64_t)T};
    const cuuint32_t box[4] = {64, 1, kLtC, 1}, steps[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, steps,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

struct LinTcMaps {
    CUtensorMap q, k, v;
};

template <int DK, bool STATE>
cudaError_t lin_tc_launch(const LinTcParams &p, const LinTcMaps &m, int64_t ctas, cudaStream_t s) {
    const void *const kern = reinterpret_cast<const void *>(lin_tc_kernel<DK, STATE>);
    const cudaError_t e = ensure_smem_limit(kern, LtSmem<DK>::bytes);
    if (e != cudaSuccess) return e;
    lin_tc_kernel<DK, STATE><<<(unsigned)ctas, kLtThreads, LtSmem<DK>::bytes, s>>>(p, m.q, m.k, m.v);
    return cudaGetLastError();
}

}  // namespace

bool lin_tc_takes(const LinArgs &a) {
    return a.in_bf16 && (a.dk == 64 || a.dk == 128) && a.dv % 128 == 0 && a.T > 16;
}

size_t lin_tc_workspace(const LinArgs &a) {
    int seg_len;
    const int64_t nseg = lin_tc_segments(a, &seg_len);
    const int64_t parts = nseg > 1 ? (int64_t)a.batch * a.H * (a.dv / 128) * nseg : 0;
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
    if ((e = lin_tc_map(&m.q, a.q, a.dk, a.Hqk, a.T, a.batch)) != cudaSuccess) return e;
    if ((e = lin_tc_map(&m.k, a.k, a.dk, a.Hqk, a.T, a.batch)) != cudaSuccess) return e;
    if ((e = lin_tc_map(&m.v, a.v, a.dv, a.H, a.T, a.batch)) != cudaSuccess) return e;
    p.g = a.g;
    p.o = a.o;
    p.H = a.H;
    p.Hqk = a.Hqk;
    p.dv = a.dv;
    p.nc = a.dv / 128;
    p.T = a.T;
    p.g_per_head = a.g_per_head;
    p.nseg = lin_tc_segments(a, &p.seg_len);
    const int64_t items = (int64_t)a.batch * a.H * p.nc;
    if (p.nseg > 1) {
        p.part = static_cast<float *>(workspace);
        p.part_dec = p.part + items * p.nseg * a.dk * 128;
        e = a.dk == 64 ? lin_tc_launch<64, true>(p, m, items * (p.nseg - 1), s) : lin_tc_launch<128, true>(p, m, items * (p.nseg - 1), s);
        if (e != cudaSuccess) return e;
    }
    return a.dk == 64 ? lin_tc_launch<64, false>(p, m, items * p.nseg, s) : lin_tc_launch<128, false>(p, m, items * p.nseg, s);
}

cudaError_t take_status_lin_tc(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_lin_tc, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_lin_tc, &zero, sizeof(uint32_t));
}

}  // namespace damp
