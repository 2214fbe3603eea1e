// lin.cu -- linear attention with a decay per head (no delta rule) on an FP32 state
// pool: the single-token step and the token-by-token chunk.
//
//     S_t = e^{g_t} S_{t-1} + k_t v_t^T,   o_t = S_t^T q_t
//
// Step.  o = e^g S^T q + (q.k) v and S <- e^g S + k v^T need each state value once: a
// CTA takes CW columns of one (slot, head), 16 bytes per thread and row, all rows of a
// thread in flight at once; the column sums of o go over the rows of the CTA through
// shared memory.  Bound by the state's bytes (read + write).
//
// Chunk (any type, any supported size).  A lane owns one value column for all d_k rows
// in registers, so both the update and o_t = S_t^T q_t are thread-local; k and q of
// kRecTok tokens at a time are staged in shared memory and read as broadcasts.  Bound by
// the FP32 pipe: 3 d_k operations per token and column.
#include "damp_common.cuh"
#include "damp_internal.h"

namespace damp {

static __device__ uint32_t g_status_lin;

// a log-decay as the exponent of the kernels: below -200, e^g is 0 in FP32 (also for -inf,
// a reset), and a NaN stays one
__device__ __forceinline__ float lin_gate(float g) { return g < -200.f ? -200.f : g; }

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
    const int64_t qoff = ((int64_t)b * p.Hqk + (h * p.Hqk) / p.H) * DK;
    if (threadIdx.x < DK) {
        sk[threadIdx.x] = load_in(p.k, qoff + threadIdx.x, BF16);
        sq[threadIdx.x] = load_in(p.q, qoff + threadIdx.x, BF16);
    }
    const int64_t voff = ((int64_t)b * p.H + h) * p.dv + c * CW + col;
    const float4 v = load_in4<BF16>(p.v, voff);
    const float a = expf(lin_gate(p.g[p.g_per_head ? h : (int64_t)b * p.H + h]));
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float kr = sk[row0 + r * RPI], qr = sq[row0 + r * RPI];
        x[r].x = fmaf(x[r].x, a, kr * v.x);
        x[r].y = fmaf(x[r].y, a, kr * v.y);
        x[r].z = fmaf(x[r].z, a, kr * v.z);
        x[r].w = fmaf(x[r].w, a, kr * v.w);
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

constexpr int kRecTok = 16;   // tokens staged at a time
constexpr int kRecWarps = 4;  // value blocks of 32 columns per CTA

template <int DK, bool BF16>
__global__ void __launch_bounds__(32 * kRecWarps) lin_chunk_kernel(const LinArgs p) {
    __shared__ __align__(16) float sk[kRecTok][DK], sq[kRecTok][DK];
    __shared__ float sa[kRecTok];
    const int V = p.dv / 32;
    const int nc = (V + kRecWarps - 1) / kRecWarps;
    const int c = blockIdx.x % nc;
    const int h = (blockIdx.x / nc) % p.H;
    const int b = blockIdx.x / nc / p.H;
    const int64_t slot = p.slot_idx ? (int64_t)p.slot_idx[b] : (int64_t)b;
    if (slot < 0 || slot >= p.num_slots) {
        if (threadIdx.x == 0) atomicOr(p.status, (uint32_t)kDevBadSlot);
        return;
    }
    const int T = p.T;
    const int len = p.lengths ? min(max(p.lengths[b], 0), T) : T;
    const int lane = threadIdx.x & 31, vb = c * kRecWarps + (threadIdx.x >> 5);
    const bool on = vb < V;
    const int hq = (h * p.Hqk) / p.H;
    const int col = vb * 32 + lane;
    float *const S = p.state + (slot * p.H + h) * DK * (int64_t)p.dv + col;
    float *const o = p.o + ((int64_t)b * T * p.H + h) * p.dv + col;
    const int64_t ostep = (int64_t)p.H * p.dv;
    float2 x[DK / 2];
    if (on && len > 0) {
#pragma unroll
        for (int u = 0; u < DK / 2; ++u) x[u] = make_float2(S[(2 * u) * (int64_t)p.dv], S[(2 * u + 1) * (int64_t)p.dv]);
    }
    for (int t0 = 0; t0 < len; t0 += kRecTok) {
        const int n = min(kRecTok, len - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < n * DK / 4; i += 32 * kRecWarps) {
            const int t = i / (DK / 4), u = 4 * (i % (DK / 4));
            const int64_t off = (((int64_t)b * T + t0 + t) * p.Hqk + hq) * DK + u;
            *reinterpret_cast<float4 *>(&sk[t][u]) = load_in4<BF16>(p.k, off);
            *reinterpret_cast<float4 *>(&sq[t][u]) = load_in4<BF16>(p.q, off);
        }
        if ((int)threadIdx.x < n)
            sa[threadIdx.x] = expf(lin_gate(p.g[p.g_per_head ? h : ((int64_t)b * T + t0 + threadIdx.x) * p.H + h]));
        __syncthreads();
        if (!on) continue;
        float vn[kRecTok];
#pragma unroll
        for (int t = 0; t < kRecTok; ++t)
            vn[t] = t < n ? load_in(p.v, (((int64_t)b * T + t0 + t) * p.H + h) * p.dv + col, BF16) : 0.f;
#pragma unroll 1
        for (int t = 0; t < n; ++t) {
            float vt = 0.f;
#pragma unroll
            for (int i = 0; i < kRecTok; ++i) vt = i == t ? vn[i] : vt;
            const float2 v2 = splat2(vt), a2 = splat2(sa[t]);
            float2 s0 = splat2(0.f), s1 = s0;
#pragma unroll
            for (int u = 0; u < DK / 2; u += 2) {
                const float4 k4 = *reinterpret_cast<const float4 *>(&sk[t][2 * u]);
                const float4 q4 = *reinterpret_cast<const float4 *>(&sq[t][2 * u]);
                x[u] = fma2(x[u], a2, mul2(make_float2(k4.x, k4.y), v2));
                x[u + 1] = fma2(x[u + 1], a2, mul2(make_float2(k4.z, k4.w), v2));
                s0 = fma2(x[u], make_float2(q4.x, q4.y), s0);
                s1 = fma2(x[u + 1], make_float2(q4.z, q4.w), s1);
            }
            const float2 s = add2(s0, s1);
            o[(int64_t)(t0 + t) * ostep] = s.x + s.y;
        }
    }
    if (!on) return;
    if (len > 0) {
#pragma unroll
        for (int u = 0; u < DK / 2; ++u) {
            S[(2 * u) * (int64_t)p.dv] = x[u].x;
            S[(2 * u + 1) * (int64_t)p.dv] = x[u].y;
        }
    }
    for (int t = len; t < T; ++t) o[(int64_t)t * ostep] = 0.f;
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

cudaError_t launch_lin_chunk(LinArgs p, cudaStream_t s) {
    const cudaError_t e = lin_status_word(p);
    if (e != cudaSuccess) return e;
    const int V = p.dv / 32;
    const unsigned grid = (unsigned)((int64_t)p.batch * p.H * ((V + kRecWarps - 1) / kRecWarps));
    const unsigned block = 32 * kRecWarps;
    if (p.dk == 32) p.in_bf16 ? lin_chunk_kernel<32, true><<<grid, block, 0, s>>>(p) : lin_chunk_kernel<32, false><<<grid, block, 0, s>>>(p);
    else if (p.dk == 64) p.in_bf16 ? lin_chunk_kernel<64, true><<<grid, block, 0, s>>>(p) : lin_chunk_kernel<64, false><<<grid, block, 0, s>>>(p);
    else p.in_bf16 ? lin_chunk_kernel<128, true><<<grid, block, 0, s>>>(p) : lin_chunk_kernel<128, false><<<grid, block, 0, s>>>(p);
    return cudaGetLastError();
}

cudaError_t take_status_lin(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_lin, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_lin, &zero, sizeof(uint32_t));
}

}  // namespace damp
