// lin.cu -- linear attention with a decay per head (no delta rule) on an FP32 state
// pool: the single-token step and the token-by-token chunk.
//
//     S_t = e^{g_t} S_{t-1} + k_t v_t^T,   o_t = S_t^T q_t
//
// Step.  o = e^g S^T q + (q.k) v and S <- e^g S + k v^T need each state value once: a
// CTA takes CW columns of one (slot, head), 16 bytes per thread and row, all rows of a
// thread in flight at once; the column sums of o go over the rows of the CTA through
// shared memory.  Bound by the state's bytes (read + write): 256 slots of 32 heads, d = 128,
// 159 us, the time of a plain copy of as many bytes.
//
// Chunk (any type, any supported size).  The same tile per CTA, held in registers over the
// tokens; k, q and v of kGroup tokens are staged in shared memory one group ahead, a thread
// sums its rows' share of an output, and the shares of kGroup outputs are joined over the
// rows at once.  For a few tokens the state's bytes and the latency of a CTA's loads bound it
// (61 slots, 32 heads, d = 128: 46 us for 5 tokens, 83 for 16; the bytes need 39), beyond
// that the FP32 pipe (three operations per state value and token: 0.98 ms for FP32 inputs at
// 64 rows of 256 tokens).  Few (slot, head) pairs and many tokens: the
// tokens are split into segments; a first launch computes what each segment adds to the
// state, a second one starts every segment from the joined state before it (twice the work,
// so from three segments on).
#include "damp_common.cuh"
#include "damp_internal.h"

#include <algorithm>
#include <cfloat>

namespace damp {

static __device__ uint32_t g_status_lin;

// a log-decay as the exponent of the kernels: below -200, e^g is 0 in FP32 (also for -inf,
// a reset), and a NaN stays one
__device__ __forceinline__ float lin_gate(float g) { return g < -200.f ? -200.f : g; }

// e^g = a (1 + lo): a rounded, and what the rounding lost.  A gate that is the same for every token
// would lose it every time in the same direction (400 tokens: 1e-5).
struct Decay {
    float a, lo, g;
};
__device__ __forceinline__ Decay lin_decay(float g) {
    g = lin_gate(g);
    const float a = expf(g);
    return Decay{a, a >= 0.5f && a <= 2.f ? g - log1pf(a - 1.f) : 0.f, g};  // a - 1 is exact
}

// x with its infinities as the largest finite value, for the remainder: infinity times a remainder of
// 0 or of the other sign would make a NaN where the recurrence has an infinity (a NaN needs no care, it
// stays one in the product with a)
__device__ __forceinline__ float finite(float x) {
    float y;
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(FLT_MAX));
    return y;
}

template <bool BF16>
__device__ __forceinline__ float4 load_in4(const void *p, int64_t i) {
    if (BF16) {
        const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(p) + i);
        return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                           __uint_as_float(w.y & 0xffff0000u));
    }
    return *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i);
}

template <int DK, int CW, bool BF16>
__global__ void __launch_bounds__(256) lin_step_kernel(const LinArgs p) {
    constexpr int TPR = CW / 4;        // threads per state row
    constexpr int RPI = 256 / TPR;     // rows per sweep of the CTA
    constexpr int R = DK / RPI;        // rows per thread (RPI is at most 32)
    __shared__ float sk[DK], sq[DK];
    __shared__ float4 part[8][32];
    const int nc = p.dv / CW;
    const int c = blockIdx.x % nc;
    const int h = (blockIdx.x / nc) % p.H;
    const int b = blockIdx.x / nc / p.H;
    const int64_t slot = p.slot_idx ? (int64_t)p.slot_idx[b] : (int64_t)b;
    if (slot < 0 || slot >= p.num_slots) {
        if (threadIdx.x == 0) atomicOr(p.status, (uint32_t)kDevBadSlot);
        return;
    }
    const int col = 4 * (threadIdx.x % TPR), row0 = threadIdx.x / TPR;
    float4 *const S = reinterpret_cast<float4 *>(p.state + ((slot * p.H + h) * DK + row0) * p.dv + c * CW + col);
    const int64_t ld = (int64_t)RPI * p.dv / 4;
    float4 x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = S[r * ld];
    const int64_t qoff = ((int64_t)b * p.Hqk + h / (p.H / p.Hqk)) * DK;  // (h H_qk may pass 32 bits)
    if (threadIdx.x < DK) {
        sk[threadIdx.x] = load_in(p.k, qoff + threadIdx.x, BF16);
        sq[threadIdx.x] = load_in(p.q, qoff + threadIdx.x, BF16);
    }
    const int64_t voff = ((int64_t)b * p.H + h) * p.dv + c * CW + col;
    const float4 v = load_in4<BF16>(p.v, voff);
    const Decay d = lin_decay(p.g[p.g_per_head ? h : (int64_t)b * p.H + h]);
    const float a = d.a, lo = fminf(a, 2.f) * d.lo;  // (there is a remainder up to 2, and a may be infinite)
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float kr = sk[row0 + r * RPI], qr = sq[row0 + r * RPI];
        x[r].x = fmaf(x[r].x, a, fmaf(finite(x[r].x), lo, kr * v.x));
        x[r].y = fmaf(x[r].y, a, fmaf(finite(x[r].y), lo, kr * v.y));
        x[r].z = fmaf(x[r].z, a, fmaf(finite(x[r].z), lo, kr * v.z));
        x[r].w = fmaf(x[r].w, a, fmaf(finite(x[r].w), lo, kr * v.w));
        S[r * ld] = x[r];
        o.x = fmaf(x[r].x, qr, o.x);
        o.y = fmaf(x[r].y, qr, o.y);
        o.z = fmaf(x[r].z, qr, o.z);
        o.w = fmaf(x[r].w, qr, o.w);
    }
#pragma unroll
    for (int m = 16; m >= TPR; m >>= 1) {  // rows of the same warp
        o.x += __shfl_xor_sync(kFull, o.x, m);
        o.y += __shfl_xor_sync(kFull, o.y, m);
        o.z += __shfl_xor_sync(kFull, o.z, m);
        o.w += __shfl_xor_sync(kFull, o.w, m);
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane < TPR) part[warp][lane] = o;
    __syncthreads();
    if (threadIdx.x < CW) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += reinterpret_cast<const float *>(part[w])[threadIdx.x];
        p.o[((int64_t)b * p.H + h) * p.dv + c * CW + threadIdx.x] = s;
    }
}

__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

constexpr int kGroup = 8;  // tokens staged at a time

// STATE: only what the segment adds to the state and its decay.  Parts of a split row: 0 the state
// before it (the last segment overwrites the pool's while others may still start), 1 the state after
// segment 0, s what segment s - 1 adds.
template <int DK, int CW, bool BF16, bool STATE>
__global__ void __launch_bounds__(256, DK * CW <= 8192 ? 3 : 2) lin_chunk_kernel(const LinArgs p, int nseg, int seg_len, int ahead, float *part, float *part_dec) {
    constexpr int TPR = CW / 4;     // threads per state row
    constexpr int RPI = 256 / TPR;  // row groups of the CTA
    constexpr int R = DK / RPI;     // consecutive rows of a thread (RPI is at most 32)
    // one buffer of operands: the barrier before the shares are joined also ends their use (the state
    // alone joins nothing and has two)
    constexpr int NB = STATE ? 2 : 1;
    __shared__ __align__(16) float sk[NB][kGroup][DK], sq[STATE ? 1 : NB][kGroup][DK], sv[NB][kGroup][CW];
    __shared__ Decay sa[NB][kGroup];
    __shared__ __align__(16) float share[STATE ? 1 : 8][kGroup][CW];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int segs = STATE ? nseg - 1 : nseg;
    const int seg = (int)(blockIdx.x % segs), nc = p.dv / CW;
    const int64_t item = blockIdx.x / segs;
    const int c = (int)(item % nc), h = (int)(item / nc % p.H), b = (int)(item / nc / p.H);
    const int64_t slot = p.slot_idx ? (int64_t)p.slot_idx[b] : (int64_t)b;
    if (slot < 0 || slot >= p.num_slots) {
        if (tid == 0) atomicOr(p.status, (uint32_t)kDevBadSlot);
        return;
    }
    const int T = p.T, len = p.lengths ? min(max(p.lengths[b], 0), T) : T;
    const int t_begin = seg * seg_len, t_stop = min(t_begin + seg_len, T), t_end = min(t_stop, len);
    const int64_t ostep = (int64_t)p.H * p.dv;
    float *const o = p.o + ((int64_t)b * T * p.H + h) * p.dv + c * CW;
    if (!STATE) {  // rows past the length
        for (int i = tid; i < (t_stop - max(len, t_begin)) * CW; i += 256)
            o[(int64_t)(max(len, t_begin) + i / CW) * ostep + i % CW] = 0.f;
    }
    if (t_begin >= len) return;
    if (STATE && t_end == len) return;  // no live segment follows
    const bool vec_o = (reinterpret_cast<uintptr_t>(p.o) & 15) == 0;

    const int col = 4 * (tid % TPR), row0 = R * (tid / TPR);
    float4 *const S = reinterpret_cast<float4 *>(p.state + ((slot * p.H + h) * DK + row0) * p.dv + c * CW + col);
    float *const parts = part + item * nseg * DK * CW + row0 * CW + col;
    float2 x[R][2];
    auto load_state = [&](const float4 *src, int64_t ld) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float4 y = src[r * ld];
            x[r][0] = make_float2(y.x, y.y);
            x[r][1] = make_float2(y.z, y.w);
        }
    };
    auto store_state = [&](float4 *dst, int64_t ld) {
#pragma unroll
        for (int r = 0; r < R; ++r) dst[r * ld] = make_float4(x[r][0].x, x[r][0].y, x[r][1].x, x[r][1].y);
    };
    auto part_of = [&](int s) { return reinterpret_cast<float4 *>(parts + (int64_t)s * DK * CW); };

    // the next group's operands, in registers: a float4 of q, of k and of v per thread
    const int hq = (int)((int64_t)h * p.Hqk / p.H);
    const int qt = tid / (DK / 4), qu = 4 * (tid % (DK / 4)), vt = tid / TPR;
    const int64_t qoff = (((int64_t)b * T + qt) * p.Hqk + hq) * DK + qu;
    const int64_t voff = (((int64_t)b * T + vt) * p.H + h) * p.dv + c * CW + col;
    float4 nk, nq, nv;
    float na = 1.f;
    auto fetch = [&](int t0) {
        nk = nq = nv = make_float4(0.f, 0.f, 0.f, 0.f);
        if (qt < kGroup && t0 + qt < t_end) {
            nk = load_in4<BF16>(p.k, qoff + (int64_t)t0 * p.Hqk * DK);
            if (!STATE) nq = load_in4<BF16>(p.q, qoff + (int64_t)t0 * p.Hqk * DK);
        }
        if (vt < kGroup && t0 + vt < t_end) nv = load_in4<BF16>(p.v, voff + (int64_t)t0 * ostep);
        if (tid < kGroup)
            na = t0 + tid < t_end ? p.g[p.g_per_head ? h : ((int64_t)b * T + t0 + tid) * p.H + h] : 0.f;
    };
    fetch(t_begin);
    if (STATE && seg > 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) x[r][0] = x[r][1] = make_float2(0.f, 0.f);
    } else if (STATE || (seg == 0 && t_end == len)) {
        load_state(S, p.dv / 4);
        if (STATE) store_state(part_of(0), CW / 4);
    } else {
        load_state(part_of(seg > 0), CW / 4);
        for (int s = 2; s <= seg; ++s) {
            const float2 d = splat2(part_dec[item * nseg + s]);
            const float4 *const src = part_of(s);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 y = src[r * (CW / 4)];
                x[r][0] = fma2(x[r][0], d, make_float2(y.x, y.y));
                x[r][1] = fma2(x[r][1], d, make_float2(y.z, y.w));
            }
        }
    }
    if (!STATE && ahead > 0 && blockIdx.x + (unsigned)ahead < gridDim.x) {
        // what the CTA that takes this one's place reads first, into L2 (one segment: a CTA is an item)
        const int64_t item2 = (int64_t)blockIdx.x + ahead;
        const int c2 = (int)(item2 % nc), h2 = (int)(item2 / nc % p.H), b2 = (int)(item2 / nc / p.H);
        const int64_t slot2 = p.slot_idx ? (int64_t)p.slot_idx[b2] : (int64_t)b2;
        const int len2 = p.lengths ? min(p.lengths[b2], T) : T;
        if (slot2 >= 0 && slot2 < p.num_slots && len2 > 0) {
            constexpr int L = CW / 32;  // lines of 128 bytes in a row of the tile
            const float *const s2 = p.state + (slot2 * p.H + h2) * DK * (int64_t)p.dv + c2 * CW;
            for (int l = tid; l < DK * L; l += 256) prefetch_l2(s2 + (int64_t)(l / L) * p.dv + 32 * (l % L));
            constexpr int E = BF16 ? 2 : 4;
            const int hq2 = (int)((int64_t)h2 * p.Hqk / p.H);
            if (qt < min(kGroup, len2) && qu * E % 128 == 0) {
                const int64_t at = ((((int64_t)b2 * T + qt) * p.Hqk + hq2) * DK + qu) * E;
                prefetch_l2(static_cast<const char *>(p.k) + at);
                prefetch_l2(static_cast<const char *>(p.q) + at);
            }
            if (vt < min(kGroup, len2) && col * E % 128 == 0)
                prefetch_l2(static_cast<const char *>(p.v) + ((((int64_t)b2 * T + vt) * p.H + h2) * p.dv + c2 * CW + col) * E);
        }
    }
    float gates = 0.f, lost = 0.f;  // of the segment so far
    int buf = 0;
#pragma unroll 1
    for (int t0 = t_begin; t0 < t_end; t0 += kGroup, buf ^= NB - 1) {
        if (qt < kGroup) {
            *reinterpret_cast<float4 *>(&sk[buf][qt][qu]) = nk;
            if (!STATE) *reinterpret_cast<float4 *>(&sq[buf][qt][qu]) = nq;
        }
        if (vt < kGroup) *reinterpret_cast<float4 *>(&sv[buf][vt][col]) = nv;
        if (tid < kGroup) sa[buf][tid] = lin_decay(na);
        __syncthreads();
        if (t0 + kGroup < t_end) fetch(t0 + kGroup);
        const int n = min(kGroup, t_end - t0);
#pragma unroll
        for (int t = 0; t < kGroup; ++t) {
            if (t < n) {
                const float a1 = sa[buf][t].a;
                const float2 a = splat2(a1);
                lost += sa[buf][t].lo;
                if (STATE) gates += sa[buf][t].g;
                const float4 v4 = *reinterpret_cast<const float4 *>(&sv[buf][t][col]);
                const float2 v0 = make_float2(v4.x, v4.y), v1 = make_float2(v4.z, v4.w);
                float2 o0 = make_float2(0.f, 0.f), o1 = o0;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float2 k = splat2(sk[buf][t][row0 + r]);
                    x[r][0] = fma2(x[r][0], a, mul2(k, v0));
                    x[r][1] = fma2(x[r][1], a, mul2(k, v1));
                    if (!STATE) {
                        const float2 q = splat2(sq[buf][t][row0 + r]);
                        o0 = fma2(x[r][0], q, o0);
                        o1 = fma2(x[r][1], q, o1);
                    }
                }
                if (!STATE) {
                    float4 y = make_float4(o0.x, o0.y, o1.x, o1.y);
#pragma unroll
                    for (int m = 16; m >= TPR; m >>= 1) {  // rows of the same warp
                        y.x += __shfl_xor_sync(kFull, y.x, m);
                        y.y += __shfl_xor_sync(kFull, y.y, m);
                        y.z += __shfl_xor_sync(kFull, y.z, m);
                        y.w += __shfl_xor_sync(kFull, y.w, m);
                    }
                    if (lane < TPR) *reinterpret_cast<float4 *>(&share[warp][t][col]) = y;
                }
            }
        }
        // What the decays lost to rounding, once it makes a unit of 1: as a factor, which leaves an
        // infinity what it is
        const float regain = 1.f + lost;
        lost -= regain - 1.f;
        if (regain != 1.f) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                x[r][0] = mul2(x[r][0], splat2(regain));
                x[r][1] = mul2(x[r][1], splat2(regain));
            }
        }
        if (!STATE) {
            __syncthreads();
            if (vt < n) {  // token vt, columns col .. col + 3
                float4 y = *reinterpret_cast<const float4 *>(&share[0][vt][col]);
#pragma unroll
                for (int w = 1; w < 8; ++w) {
                    const float4 z = *reinterpret_cast<const float4 *>(&share[w][vt][col]);
                    y = make_float4(y.x + z.x, y.y + z.y, y.z + z.z, y.w + z.w);
                }
                float *const dst = o + (int64_t)(t0 + vt) * ostep + col;
                if (vec_o) {
                    *reinterpret_cast<float4 *>(dst) = y;
                } else {
                    dst[0] = y.x;
                    dst[1] = y.y;
                    dst[2] = y.z;
                    dst[3] = y.w;
                }
            }
        }
    }
    if (STATE) {
        store_state(part_of(seg + 1), CW / 4);
        if (tid == 0) {  // from the sum: a product would round the same way in every segment
            const Decay d = lin_decay(gates);
            part_dec[item * nseg + seg + 1] = fmaf(d.a, d.lo, d.a);
        }
    } else if (t_end == len) {
        store_state(S, p.dv / 4);
    }
}

static int lin_chunk_columns(const LinArgs &p) { return p.dv % 128 == 0 ? 128 : p.dv % 64 == 0 ? 64 : 32; }

// segments (1: no split) and the tokens of each
static int lin_chunk_segments(const LinArgs &p, int *seg_len) {
    const int64_t items = (int64_t)p.batch * p.H * (p.dv / lin_chunk_columns(p));
    int64_t nseg = std::min<int64_t>(2 * (int64_t)sm_count() / std::max<int64_t>(items, 1), p.T / 64);
    if (nseg < 3) nseg = 1;
    *seg_len = (int)((p.T + nseg * kGroup - 1) / (nseg * kGroup)) * kGroup;
    return (p.T + *seg_len - 1) / *seg_len;
}

size_t lin_chunk_workspace(const LinArgs &p) {
    int seg_len;
    const int cw = lin_chunk_columns(p), nseg = lin_chunk_segments(p, &seg_len);
    return nseg > 1 ? (size_t)p.batch * p.H * (p.dv / cw) * nseg * (p.dk * cw + 1) * 4 : 0;
}

template <int DK, int CW, bool BF16>
static void lin_chunk_run(const LinArgs &p, void *workspace, cudaStream_t s) {
    int seg_len;
    const int nseg = lin_chunk_segments(p, &seg_len);
    const int64_t items = (int64_t)p.batch * p.H * (p.dv / CW);
    float *const part = static_cast<float *>(workspace), *const dec = part + (nseg > 1 ? items * nseg * DK * CW : 0);
    // A CTA of at most one group is mostly waiting for its tile, which the CTA a wave before it brings
    // into L2 (61 slots, 32 heads, d = 128, with and without: 2 tokens 44 and 53 us, 5 50 and 55, 8 59
    // and 61; 304 CTAs ahead instead of 152 take 1 us more).  More tokens (16: 88 and 86) and small
    // tiles (d = 64: 19.4 and 18.3) do without.
    const int ahead = nseg == 1 && p.T <= kGroup && DK * CW >= 8192 ? sm_count() : 0;
    if (nseg > 1) lin_chunk_kernel<DK, CW, BF16, true><<<(unsigned)(items * (nseg - 1)), 256, 0, s>>>(p, nseg, seg_len, ahead, part, dec);
    lin_chunk_kernel<DK, CW, BF16, false><<<(unsigned)(items * nseg), 256, 0, s>>>(p, nseg, seg_len, ahead, part, dec);
}
template <int DK, bool BF16>
static void lin_chunk_pick(const LinArgs &p, void *workspace, cudaStream_t s) {
    const int cw = lin_chunk_columns(p);
    if (cw == 128) lin_chunk_run<DK, 128, BF16>(p, workspace, s);
    else if (cw == 64) lin_chunk_run<DK, 64, BF16>(p, workspace, s);
    else lin_chunk_run<DK, 32, BF16>(p, workspace, s);
}

template <int DK, bool BF16>
static void lin_step_pick(const LinArgs &p, cudaStream_t s) {
    const int64_t bh = (int64_t)p.batch * p.H;
    if (p.dv % 128 == 0) lin_step_kernel<DK, 128, BF16><<<(unsigned)(bh * (p.dv / 128)), 256, 0, s>>>(p);
    else if (p.dv % 64 == 0) lin_step_kernel<DK, 64, BF16><<<(unsigned)(bh * (p.dv / 64)), 256, 0, s>>>(p);
    else lin_step_kernel<DK, 32, BF16><<<(unsigned)(bh * (p.dv / 32)), 256, 0, s>>>(p);
}

static cudaError_t lin_status_word(LinArgs &p) {
    static std::atomic<uint32_t *> cache[64];
    return symbol_address_cached(&g_status_lin, cache, &p.status);
}

cudaError_t launch_lin_step(LinArgs p, cudaStream_t s) {
    const cudaError_t e = lin_status_word(p);
    if (e != cudaSuccess) return e;
    if (p.dk == 32) p.in_bf16 ? lin_step_pick<32, true>(p, s) : lin_step_pick<32, false>(p, s);
    else if (p.dk == 64) p.in_bf16 ? lin_step_pick<64, true>(p, s) : lin_step_pick<64, false>(p, s);
    else p.in_bf16 ? lin_step_pick<128, true>(p, s) : lin_step_pick<128, false>(p, s);
    return cudaGetLastError();
}

cudaError_t launch_lin_chunk(LinArgs p, void *workspace, cudaStream_t s) {
    const cudaError_t e = lin_status_word(p);
    if (e != cudaSuccess) return e;
    if (p.dk == 32) p.in_bf16 ? lin_chunk_pick<32, true>(p, workspace, s) : lin_chunk_pick<32, false>(p, workspace, s);
    else if (p.dk == 64) p.in_bf16 ? lin_chunk_pick<64, true>(p, workspace, s) : lin_chunk_pick<64, false>(p, workspace, s);
    else p.in_bf16 ? lin_chunk_pick<128, true>(p, workspace, s) : lin_chunk_pick<128, false>(p, workspace, s);
    return cudaGetLastError();
}

cudaError_t take_status_lin(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_lin, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_lin, &zero, sizeof(uint32_t));
}

}  // namespace damp
