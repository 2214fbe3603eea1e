// verify.cu -- verification of drafted tokens against the target's probabilities, from
// given random numbers (speculative sampling).
//
// For a request with drafts x_0 .. x_{L-1}, p_i = softmax(target_i / T) and
// q_i = softmax(draft_i / T): x_i is accepted iff u_i q_i(x_i) < p_i(x_i), until the first
// rejection at a.  The next token is drawn from r = max(p_a - q_a, 0) (after a rejection)
// or r = p_L (nothing rejected) as argmax_t r_t / e_t with e_t exponential: the first
// arrival of a race with rates r_t, which is t with probability r_t / sum r.  The emitted
// tokens are then distributed as the target's own samples.  T = 0 is greedy: x_i is
// accepted iff it is the target's first maximum, which is also the next token.
//
// Logits: NaN and -inf are excluded tokens, +inf counts as the largest finite value; a row
// with every token excluded accepts nothing and gives no token.  Maximum and sum of a
// softmax are FP32, in one pass with a running maximum per thread.
#include "damp_common.cuh"
#include "damp_internal.h"

#include <cfloat>

namespace damp {

static __device__ uint32_t g_status_verify;

constexpr int kVerThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// an excluded token as -inf, +inf as the largest finite value (fmaxf drops a NaN)
__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }

// maximum m and sum of 2^{(x - m) s} of what was seen
struct Soft {
    float m, s;
};
__device__ __forceinline__ Soft soft_join(Soft a, Soft b, float scale) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return Soft{m, 0.f};
    return Soft{m, a.s * ex2((a.m - m) * scale) + b.s * ex2((b.m - m) * scale)};
}
// the larger value, the lower index on ties (index -1: nothing seen)
struct Best {
    float v;
    int i;
};
__device__ __forceinline__ Best best_of(Best a, Best b) {
    if (b.i < 0) return a;
    if (a.i < 0) return b;
    return b.v > a.v || (b.v == a.v && b.i < a.i) ? b : a;
}

template <bool BF16>
__device__ Soft block_soft(const void *row, int n, float scale, Soft *red) {
    Soft a{-INFINITY, 0.f};
    for (int i = threadIdx.x; i < n; i += kVerThreads) {
        const float x = clean(load_in(row, i, BF16));
        if (x > a.m) {
            a.s = a.m == -INFINITY ? 0.f : a.s * ex2((a.m - x) * scale);
            a.m = x;
        }
        if (x > -INFINITY) a.s += ex2((x - a.m) * scale);
    }
#pragma unroll
    for (int m = 16; m; m >>= 1)
        a = soft_join(a, Soft{__shfl_xor_sync(kFull, a.m, m), __shfl_xor_sync(kFull, a.s, m)}, scale);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
    __syncthreads();
    a = red[0];
    for (int w = 1; w < kVerThreads / 32; ++w) a = soft_join(a, red[w], scale);
    return a;
}

__device__ Best block_best(Best a, Best *red) {
#pragma unroll
    for (int m = 16; m; m >>= 1) a = best_of(a, Best{__shfl_xor_sync(kFull, a.v, m), __shfl_xor_sync(kFull, a.i, m)});
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
    __syncthreads();
    a = red[0];
    for (int w = 1; w < kVerThreads / 32; ++w) a = best_of(a, red[w]);
    return a;
}

template <bool BF16>
__global__ void __launch_bounds__(kVerThreads) verify_kernel(const VerifyArgs p) {
    __shared__ Soft red_s[kVerThreads / 32];
    __shared__ Best red_b[kVerThreads / 32];
    const int b = blockIdx.x, D = p.n_draft, V = p.vocab;
    const int L = p.draft_len ? min(max(p.draft_len[b], 0), D) : D;
    const float temp = p.temperature ? p.temperature[b] : 1.0f;
    const bool greedy = !(temp > 0.f);
    const float scale = greedy ? kLog2e : fminf(fmaxf(1.0f / temp, 1e-30f), 1e37f) * kLog2e;
    const int64_t es = BF16 ? 2 : 4;
    auto trow = [&](int i) { return static_cast<const uint8_t *>(p.target) + ((int64_t)b * (D + 1) + i) * p.row_stride * es; };
    auto drow = [&](int i) { return static_cast<const uint8_t *>(p.draft) + ((int64_t)b * D + i) * p.row_stride * es; };
    int a = 0, token = -1;
    Soft P{}, Q{};
    int point = -1;  // the rejected token of a draft without probabilities (a point mass)
    bool rejected = false;
    for (;; ++a) {
        const bool last = a == L;
        const int x = last ? -1 : p.tokens[(int64_t)b * D + a];
        const bool valid = x >= 0 && x < V;
        if (!last && !valid && threadIdx.x == 0) atomicOr(p.status, (uint32_t)kDevBadToken);
        if (greedy) {
            Best best{0.f, -1};
            for (int i = threadIdx.x; i < V; i += kVerThreads) {
                const float y = clean(load_in(trow(a), i, BF16));
                if (y > -INFINITY) best = best_of(best, Best{y, i});
            }
            best = block_best(best, red_b);
            token = best.i;
            if (last || x != token || !valid) break;
            continue;
        }
        P = block_soft<BF16>(trow(a), V, scale, red_s);
        if (last) break;
        const bool point_mass = p.draft == nullptr;
        if (!point_mass) Q = block_soft<BF16>(drow(a), V, scale, red_s);
        bool ok = false;
        if (valid && P.s > 0.f) {
            const float px = ex2((clean(load_in(trow(a), x, BF16)) - P.m) * scale) / P.s;
            float qx = 1.f;
            if (!point_mass) qx = Q.s > 0.f ? ex2((clean(load_in(drow(a), x, BF16)) - Q.m) * scale) / Q.s : 0.f;
            ok = p.u[(int64_t)b * D + a] * qx < px;
        }
        if (ok) continue;
        rejected = true;
        if (point_mass) point = x;
        break;
    }
    if (!greedy && P.s > 0.f) {
        const float *noise = p.noise + (int64_t)b * V;
        const float ip = 1.f / P.s;
        for (int pass = rejected ? 0 : 1; pass < 2 && token < 0; ++pass) {  // pass 1: no residual is left, or none is due
            const bool minus_q = pass == 0 && point < 0 && p.draft && Q.s > 0.f;
            const float iq = minus_q ? 1.f / Q.s : 0.f;
            Best best{0.f, -1};
            for (int i = threadIdx.x; i < V; i += kVerThreads) {
                const float xt = clean(load_in(trow(a), i, BF16));
                float r = ex2((xt - P.m) * scale) * ip;
                if (minus_q) r -= ex2((clean(load_in(drow(a), i, BF16)) - Q.m) * scale) * iq;
                if (pass == 0 && i == point) r = 0.f;
                const float score = r / noise[i];
                if (r > 0.f && score >= 0.f) best = best_of(best, Best{score, i});
            }
            token = block_best(best, red_b).i;
        }
    }
    if (threadIdx.x == 0) p.count_out[b] = a + (token >= 0 ? 1 : 0);
    for (int i = threadIdx.x; i <= D; i += kVerThreads)
        p.tokens_out[(int64_t)b * (D + 1) + i] = i < a ? p.tokens[(int64_t)b * D + i] : i == a ? token : -1;
}

cudaError_t launch_verify(VerifyArgs p, cudaStream_t s) {
    static std::atomic<uint32_t *> cache[64];
    const cudaError_t e = symbol_address_cached(&g_status_verify, cache, &p.status);
    if (e != cudaSuccess) return e;
    if (p.bf16) verify_kernel<true><<<(unsigned)p.batch, kVerThreads, 0, s>>>(p);
    else verify_kernel<false><<<(unsigned)p.batch, kVerThreads, 0, s>>>(p);
    return cudaGetLastError();
}

cudaError_t take_status_verify(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_verify, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_verify, &zero, sizeof(uint32_t));
}

}  // namespace damp
