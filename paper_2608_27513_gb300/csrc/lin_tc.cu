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
// Two CTAs per SM (112 KB of shared memory, 256 of the 512 tensor-memory columns each)
// overlap one's products with the other's conversions; the next piece's q, k and v are
// fetched while the current one is finished.  Bound by the bytes of q, k, v and o, with
// the conversions next.
//
// Few (slot, head) pairs and many tokens: the tokens are split into segments.  A first
// launch computes what each segment adds to the state (k and v only), a second one starts
// every segment from the joined state before it.
#include "damp_internal.h"
#include "prefill_tc.cuh"

#include <algorithm>

namespace damp {

static __device__ uint32_t g_status_lin_tc;

namespace {

constexpr int kLtC = 64;
constexpr int kLtThreads = 256;
constexpr uint32_t kLtCols = 256;
// tensor-memory columns: Q K^T, then O2 | O1 | S_0 as bf16 parts, then what the piece adds
constexpr uint32_t kLtG = 0, kLtO1 = 64, kLtS = 128;

template <int DK>
struct LtSmem {  // bytes from the base of the dynamic shared memory
    static constexpr int tile = kLtC * DK * 2;
    static constexpr int vtile = kLtC * 128 * 2;
    static constexpr int q = 0;              // rows 0-63 of [Q; K]
    static constexpr int k = tile;           // rows 64-127
    static constexpr int v = 2 * tile;       // two buffers
    static constexpr int kd = v + 2 * vtile; // K~ hi, lo
    static constexpr int p = kd + 2 * tile;  // P hi, lo
    static constexpr int g = p + 2 * kLtC * kLtC * 2;  // (hi, lo) of G in base 2, 64 pairs
    static constexpr int eg = g + 512;       // e^{G_i}
    static constexpr int bar = eg + 256;     // two mbarriers, the tensor-memory address
    static constexpr int bytes = bar + 32;
};

struct LinTcParams {
    float *state;
    int64_t num_slots;
    const int32_t *slot_idx, *lengths;
    const uint8_t *q, *k, *v;
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
// 16 bytes, or zeros where the row is past the tokens
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void *src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16u : 0u) : "memory");
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

// 64 rows of CELLS 16-byte cells (row stride `ld` bytes in global memory) into the layout of
// the operands: cell c of row t at (t >> 3) CELLS 128 + c 128 + (t & 7) 16.  Eight lanes
// write 128 contiguous bytes and four take 64 contiguous bytes of a row.
template <int CELLS>
__device__ __forceinline__ void lt_load(uint32_t dst, const uint8_t *src, int64_t ld, int n, int warp, int lane) {
    const int t0 = lane & 7, c0 = lane >> 3;
#pragma unroll
    for (int r = 0; r < CELLS / 4; ++r) {
        const int u = r * 8 + warp;
        const int t = (u / (CELLS / 4)) * 8 + t0, c = (u % (CELLS / 4)) * 4 + c0;
        const bool live = t < n;
        cp_async16_or_zero(dst + (uint32_t)((t >> 3) * CELLS * 128 + c * 128 + (t & 7) * 16),
                           src + (int64_t)(live ? t : 0) * ld + 16 * c, live);
    }
}

// STATE: only what the segment adds to the state and its decay
template <int DK, bool STATE>
__global__ void __launch_bounds__(kLtThreads, 2) lin_tc_kernel(const LinTcParams p) {
    extern __shared__ __align__(128) uint8_t smem[];
    using M = LtSmem<DK>;
    constexpr int CELLS = DK / 8;
    constexpr int NR = DK / 2;  // state rows of a thread
    constexpr uint32_t kIdG = tc_idesc(64, false, false), kIdO2 = tc_idesc(64, true, false), kIdS = tc_idesc(DK, true, true);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = 32 * (warp & 3) + lane, half = warp >> 2;
    const uint32_t sb = smem_u32(smem);
    const uint32_t bar1 = sb + M::bar, bar2 = bar1 + 8, s_taddr = bar1 + 16;

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
    if (tid == 0) {
        mbar_init(bar1, 1);
        mbar_init(bar2, 1);
        fence_mbar_init();
    }
    const int64_t qk_ld = (int64_t)p.Hqk * DK * 2, v_ld = (int64_t)p.H * p.dv * 2;
    const int64_t qk_off = ((int64_t)b * T * p.Hqk + (int64_t)h * p.Hqk / p.H) * DK * 2;
    const uint8_t *const q0 = p.q + qk_off, *const k0 = p.k + qk_off;
    const uint8_t *const v0 = p.v + (((int64_t)b * T * p.H + h) * p.dv + c * 128) * 2;
    auto load_qk = [&](int t) {
        if (!STATE) lt_load<CELLS>(sb + M::q, q0 + t * qk_ld, qk_ld, t_end - t, warp, lane);
        lt_load<CELLS>(sb + M::k, k0 + t * qk_ld, qk_ld, t_end - t, warp, lane);
    };
    auto load_v = [&](int t, int buf) {
        lt_load<16>(sb + M::v + buf * M::vtile, v0 + t * v_ld, v_ld, t_end - t, warp, lane);
    };
    load_qk(t_begin);
    load_v(t_begin, 0);
    cp_async_commit();

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
    if (!STATE) {
        // columns 32-63 of rows 0-31 of P are above the diagonal: zero for every piece
        const int part = tid >> 7, r = (tid >> 2) & 31, cell = 4 + (tid & 3);
        sts128(sb + M::p + (uint32_t)(part * 8192 + (r >> 3) * 1024 + cell * 128 + (r & 7) * 16), make_uint4(0u, 0u, 0u, 0u));
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = lds32(s_taddr);
    const uint32_t tl = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const uint32_t tS = tl + kLtS + (uint32_t)(NR * half);  // this thread's columns of both uses

    // S as two bf16 parts: the half's hi words, then its lo words
    auto store_parts = [&](int r8, const float2 *x) {  // 16 rows from 16 r8
        uint32_t hw[8], lw[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) split2_pair(x[i], hw[i], lw[i]);
        lt_st8(tS + 8 * r8, hw);
        lt_st8(tS + NR / 2 + 8 * r8, lw);
    };
    if (!STATE) {
#pragma unroll
        for (int r8 = 0; r8 < NR / 16; ++r8) store_parts(r8, S + 8 * r8);
        lt_wait_st();
    }

    // gates of a piece: lane l holds tokens 2l and 2l + 1
    const float *const g0 = p.g_per_head ? p.g + h : p.g + (int64_t)b * T * p.H + h;
    const int64_t gstep = p.g_per_head ? 0 : p.H;
    auto gate = [&](int t) -> float {
        if (t >= t_end) return 0.f;
        const float x = g0[(int64_t)t * gstep];
        return x < -200.f ? -200.f : x;  // e^-200 is 0 in FP32 (-inf: a reset)
    };
    float ga = 0.f, gb = 0.f;
    if (warp == 0) {
        ga = gate(t_begin + 2 * lane);
        gb = gate(t_begin + 2 * lane + 1);
    }
    double dec_total = 0.0;  // warp 0: base-2 log of the segment's decay
    bool ok = true;
    uint32_t last1 = 0, last2 = 0;  // phases of the last products issued
    int buf = 0;
#pragma unroll 1
    for (int t0 = t_begin; t0 < t_end; t0 += kLtC, buf ^= 1) {
        const int n = min(kLtC, t_end - t0);
        const bool more = t0 + kLtC < t_end;
        const uint32_t vt = sb + M::v + (uint32_t)(buf * M::vtile);
        cp_async_wait_all();
        fence_proxy_async_smem();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (!STATE && tid == 128) {
#pragma unroll
            for (int ks = 0; ks < DK / 16; ++ks) {
                const uint64_t d = tc_desc(sb + M::q + 256 * ks, 128, 16 * DK);
                tc_mma(tmem + kLtG, d, tc_desc(sb + M::k + 256 * ks, 128, 16 * DK), kIdG, ks != 0);
            }
            tc_commit(bar1);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int ks = 0; ks < DK / 16; ++ks) {
                    constexpr int HS = DK / 32;  // K steps per half
                    const uint32_t a = tmem + kLtS + (uint32_t)(NR * (ks / HS) + NR / 2 * part + 8 * (ks % HS));
                    lt_mma_ta(tmem + kLtO1, a, tc_desc(sb + M::q + 256 * ks, 128, 16 * DK), kIdG, (part | ks) != 0);
                }
            tc_commit(bar2);
        }
        last1 = last2 = 0;
        if (more) load_v(t0 + kLtC, buf ^ 1);
        if (warp == 0) {  // inclusive sums of the gates, base 2
            constexpr double kLog2eD = 1.4426950408889634074;
            const double a0 = (double)ga * kLog2eD, a1 = a0 + (double)gb * kLog2eD;
            double x = a1;
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) {
                const double y = __shfl_up_sync(kFull, x, m);
                if (lane >= m) x += y;
            }
            dec_total += __shfl_sync(kFull, x, 31);
            const double x0 = x - a1 + a0;
            const float h0 = (float)x0, h1 = (float)x;
            sts128(sb + M::g + 16 * lane, make_uint4(__float_as_uint(h0), __float_as_uint((float)(x0 - (double)h0)),
                                                     __float_as_uint(h1), __float_as_uint((float)(x - (double)h1))));
            sts32(sb + M::eg + 8 * lane, __float_as_uint(lt_ex2(h0)));
            sts32(sb + M::eg + 8 * lane + 4, __float_as_uint(lt_ex2(h1)));
            if (more) {
                ga = gate(t0 + kLtC + 2 * lane);
                gb = gate(t0 + kLtC + 2 * lane + 1);
            }
        }
        if (!STATE) ok &= mbar_wait_bounded(bar1, 0);
        if (!__syncthreads_and(ok)) break;
        tc_fence_after();
        // warps 0, 1, 5: P (rows 0-31; rows 32-63, columns 0-31 and 32-63);
        // warps 2, 3, 6, 7: K~ (warps 4 and, with the state alone, 0, 1, 5 have none)
        if ((warp & 3) >= 2) {
            const int kt = (warp & 1) * 32 + lane;  // token
            const uint32_t gj = sb + M::g + 8 * kt, gC = sb + M::g + 8 * 63;
            const float2 f = splat2(lt_ex2((ldsf(gC) - ldsf(gj)) + (ldsf(gC + 4) - ldsf(gj + 4))));
            const uint32_t cell = (uint32_t)((kt >> 3) * CELLS * 128 + (kt & 7) * 16);
#pragma unroll 4
            for (int i = 0; i < CELLS / 2; ++i) {
                const uint32_t off = cell + (uint32_t)((CELLS / 2 * half + i) * 128);
                const uint4 w4 = lds128(sb + M::k + off);
                const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
                uint32_t hw[4], lw[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    split2_pair(mul2(make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u)), f), hw[e], lw[e]);
                sts128(sb + M::kd + off, make_uint4(hw[0], hw[1], hw[2], hw[3]));
                sts128(sb + M::kd + M::tile + off, make_uint4(lw[0], lw[1], lw[2], lw[3]));
            }
        } else if (!STATE && warp != 4) {
            const float gih = ldsf(sb + M::g + 8 * row), gil = ldsf(sb + M::g + 8 * row + 4);
#pragma unroll
            for (int j0 = 0; j0 < 32; j0 += 16) {
                float x[16];
                lt_ld16(tl + kLtG + 32 * half + j0, x);
                const int jb = 32 * half + j0;
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const uint4 gg = lds128(sb + M::g + 8 * (jb + e));
                    const float d0 = (gih - __uint_as_float(gg.x)) + (gil - __uint_as_float(gg.y));
                    const float d1 = (gih - __uint_as_float(gg.z)) + (gil - __uint_as_float(gg.w));
                    x[e] = jb + e <= row ? x[e] * lt_ex2(d0) : 0.f;
                    x[e + 1] = jb + e + 1 <= row ? x[e + 1] * lt_ex2(d1) : 0.f;
                }
#pragma unroll
                for (int g8 = 0; g8 < 2; ++g8) {
                    uint32_t hw[4], lw[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) split2_pair(make_float2(x[8 * g8 + 2 * e], x[8 * g8 + 2 * e + 1]), hw[e], lw[e]);
                    const uint32_t off = (uint32_t)((row >> 3) * 1024 + (jb / 8 + g8) * 128 + (row & 7) * 16);
                    sts128(sb + M::p + off, make_uint4(hw[0], hw[1], hw[2], hw[3]));
                    sts128(sb + M::p + 8192 + off, make_uint4(lw[0], lw[1], lw[2], lw[3]));
                }
            }
        }
        fence_proxy_async_smem();
        if (!STATE) ok &= mbar_wait_bounded(bar2, 0);
        tc_fence_before();
        if (!__syncthreads_and(ok)) break;
        tc_fence_after();
        if (tid == 128) {
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int ks = 0; ks < kLtC / 16; ++ks)
                    tc_mma(tmem + kLtS, tc_desc(vt + 4096 * ks, 2048, 128),
                           tc_desc(sb + M::kd + M::tile * part + 32 * DK * ks, 16 * DK, 128), kIdS, (part | ks) != 0);
            tc_commit(bar1);
            if (!STATE) {
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int ks = 0; ks < kLtC / 16; ++ks)
                        tc_mma(tmem + kLtG, tc_desc(vt + 4096 * ks, 2048, 128),
                               tc_desc(sb + M::p + 8192 * part + 256 * ks, 128, 1024), kIdO2, (part | ks) != 0);
                tc_commit(bar2);
            }
        }
        if (more) {
            load_qk(t0 + kLtC);
            cp_async_commit();
        }
        last1 = STATE ? (uint32_t)buf : 1u;
        last2 = 1;
        const float2 eC = splat2(ldsf(sb + M::eg + 4 * 63));
        ok &= mbar_wait_bounded(bar1, last1);
        tc_fence_after();
#pragma unroll
        for (int r8 = 0; r8 < NR / 16; ++r8) {
            float d[16];
            lt_ld16(tS + 16 * r8, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) S[8 * r8 + i] = fma2(S[8 * r8 + i], eC, make_float2(d[2 * i], d[2 * i + 1]));
        }
        if (!STATE && more) {
#pragma unroll
            for (int r8 = 0; r8 < NR / 16; ++r8) store_parts(r8, S + 8 * r8);
        }
        if (!STATE) {
            ok &= mbar_wait_bounded(bar2, 1);
            tc_fence_after();
            float *const oc = o + (int64_t)(t0 + 32 * half) * ostep;
            const int nh = n - 32 * half;
#pragma unroll
            for (int j0 = 0; j0 < 32; j0 += 16) {
                if (j0 < nh) {
                    float o1[16], o2[16];
                    lt_ld16(tl + kLtO1 + 32 * half + j0, o1);
                    lt_ld16(tl + kLtG + 32 * half + j0, o2);
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const uint4 eg = lds128(sb + M::eg + 4 * (32 * half + j0 + e));
                        const float ev[4] = {__uint_as_float(eg.x), __uint_as_float(eg.y), __uint_as_float(eg.z), __uint_as_float(eg.w)};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (j0 + e + i < nh) oc[(j0 + e + i) * ostep] = fmaf(ev[i], o1[e + i], o2[e + i]);
                    }
                }
            }
        }
        lt_wait_st();
    }
    ok = __syncthreads_and(ok);
    if (ok) {
        if (STATE) {
            store_state(part0 + (int64_t)(seg + 1) * DK * 128, 128);
            if (tid == 0) p.part_dec[(int64_t)item * p.nseg + seg + 1] = lt_ex2((float)dec_total);
        } else if (t_end == len) {
            store_state(st, p.dv);
        }
    } else {  // products that did not complete in time get one more bounded wait
        if (tid == 0) atomicOr(p.status, (uint32_t)kDevWaitTimeout);
        mbar_wait_bounded(bar1, last1);
        mbar_wait_bounded(bar2, last2);
    }
    cp_async_commit();
    cp_async_wait_all();
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

template <int DK, bool STATE>
cudaError_t lin_tc_launch(const LinTcParams &p, int64_t ctas, cudaStream_t s) {
    const void *const kern = reinterpret_cast<const void *>(lin_tc_kernel<DK, STATE>);
    const cudaError_t e = ensure_smem_limit(kern, LtSmem<DK>::bytes);
    if (e != cudaSuccess) return e;
    lin_tc_kernel<DK, STATE><<<(unsigned)ctas, kLtThreads, LtSmem<DK>::bytes, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

bool lin_tc_takes(const LinArgs &a) {
    return a.in_bf16 && (a.dk == 64 || a.dk == 128) && a.dv % 128 == 0 && a.T >= 32;
}

size_t lin_tc_workspace(const LinArgs &a) {
    if (!lin_tc_takes(a)) return 0;
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
    p.q = static_cast<const uint8_t *>(a.q);
    p.k = static_cast<const uint8_t *>(a.k);
    p.v = static_cast<const uint8_t *>(a.v);
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
        e = a.dk == 64 ? lin_tc_launch<64, true>(p, items * (p.nseg - 1), s) : lin_tc_launch<128, true>(p, items * (p.nseg - 1), s);
        if (e != cudaSuccess) return e;
    }
    return a.dk == 64 ? lin_tc_launch<64, false>(p, items * p.nseg, s) : lin_tc_launch<128, false>(p, items * p.nseg, s);
}

cudaError_t take_status_lin_tc(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_lin_tc, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_lin_tc, &zero, sizeof(uint32_t));
}

}  // namespace damp
