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
// with every token excluded accepts nothing and gives no token.
//
// A request is one cluster of CL CTAs, each with a contiguous part of every row.  A round
// takes the softmax maxima and sums (FP32, one pass with a running maximum per thread) of
// the rows of R positions, joins them over the cluster through distributed shared memory
// in one fixed order, so that every CTA comes to the same decisions, and goes on until a
// rejection.  With many requests R = 1: rows after a rejection are not read.  With few, the
// time is latency and all positions share a round.  Within a round the loads of the next
// batch are in flight while one is summed, across rows.  Bound by the bytes of the rows
// needed, with the exponentials (one per logit) next.
//
// The race reads its target row again (from L2) and the noise; p_t >= r_t, so a token whose
// p_t does not reach the best arrival of its warp so far cannot win, and only for the few
// others the draft's probability and the quotient are taken.
#include "damp_common.cuh"
#include "damp_internal.h"

#include <cfloat>

namespace damp {

static __device__ uint32_t g_status_verify;

namespace {

constexpr int kVerThreads = 512;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerBatch = 2;    // 16-byte loads of a thread per batch (two batches in flight)
constexpr int kVerRound = 8;    // positions of a round at most
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// an excluded token as -inf, +inf as the largest finite value (fmaxf drops a NaN)
__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }
// the maximum as a subtrahend: finite, so that -inf minus it is -inf
__device__ __forceinline__ float finite_max(float m) { return fmaxf(m, -FLT_MAX); }

__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// What a thread, a warp, a CTA or the cluster has seen of a row: for a softmax, the maximum
// m and the sum of 2^{(x - m) scale}; for a first maximum, its value and index (-1: nothing).
struct Soft {
    float m, s;
};
struct Best {
    float v;
    int i;
};
__device__ __forceinline__ Soft join(Soft a, Soft b, float scale) {
    const float m = finite_max(fmaxf(a.m, b.m));
    return Soft{fmaxf(a.m, b.m), a.s * ex2((a.m - m) * scale) + b.s * ex2((b.m - m) * scale)};
}
__device__ __forceinline__ Best join(Best a, Best b, float) {
    if (b.i < 0) return a;
    if (a.i < 0) return b;
    return b.v > a.v || (b.v == a.v && b.i < a.i) ? b : a;
}
template <class P>
__device__ __forceinline__ P peer(const P *local, uint32_t rank) {  // the same variable in CTA `rank` of the cluster
    uint32_t a, x, y;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.v2.b32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(a) : "memory");
    P p;
    const uint32_t w[2] = {x, y};
    memcpy(&p, w, 8);
    return p;
}
__device__ __forceinline__ Soft shuffle(Soft a, int m) {
    return Soft{__shfl_xor_sync(kFull, a.m, m), __shfl_xor_sync(kFull, a.s, m)};
}
__device__ __forceinline__ Best shuffle(Best a, int m) {
    return Best{__shfl_xor_sync(kFull, a.v, m), __shfl_xor_sync(kFull, a.i, m)};
}
template <class P>
__device__ __forceinline__ P join_warp(P a, float scale) {
#pragma unroll
    for (int m = 16; m; m >>= 1) a = join(a, shuffle(a, m), scale);
    return a;
}

// Elements [e0, e1) of a row: whole 16-byte vectors, and the elements before and after them
struct Part {
    const uint4 *vec;
    int nv, first;  // vectors; the index of the first vector's first element
};
template <bool BF16>
__device__ __forceinline__ Part part_of(const uint8_t *row, int e0, int e1) {
    constexpr int ES = BF16 ? 2 : 4, VE = 16 / ES;
    const uint8_t *const a = row + (int64_t)e0 * ES;
    const int skip = min(e1 - e0, (int)((16 - (reinterpret_cast<uintptr_t>(a) & 15)) & 15) / ES);
    return Part{reinterpret_cast<const uint4 *>(a + skip * ES), (e1 - e0 - skip) / VE, e0 + skip};
}
__device__ __forceinline__ uint4 ldg_stream(const uint4 *p) {
    uint4 v;
    asm volatile("ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <bool BF16>
__device__ __forceinline__ void load_batch(const Part &r, int batch, uint4 (&x)[kVerBatch]) {
    constexpr uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
#pragma unroll
    for (int u = 0; u < kVerBatch; ++u) {
        const int i = (batch * kVerBatch + u) * kVerThreads + (int)threadIdx.x;
        x[u] = i < r.nv ? ldg_stream(r.vec + i) : make_uint4(none, none, none, none);
    }
}
// the elements of a vector, cleaned
__device__ __forceinline__ void elements(const uint4 &x, float (&f)[8], bool) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const __nv_bfloat162 lo = __nv_bfloat162(__ushort_as_bfloat16(0xff80), __ushort_as_bfloat16(0xff80));
    const __nv_bfloat162 hi = __nv_bfloat162(__ushort_as_bfloat16(0x7f7f), __ushort_as_bfloat16(0x7f7f));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 b;
        memcpy(&b, &w[i], 4);
        b = __hmin2(__hmax2(b, lo), hi);  // __hmax2 drops a NaN
        uint32_t c;
        memcpy(&c, &b, 4);
        f[2 * i] = __uint_as_float(c << 16);
        f[2 * i + 1] = __uint_as_float(c & 0xffff0000u);
    }
}
__device__ __forceinline__ void elements(const uint4 &x, float (&f)[4], bool) {
    f[0] = clean(__uint_as_float(x.x));
    f[1] = clean(__uint_as_float(x.y));
    f[2] = clean(__uint_as_float(x.z));
    f[3] = clean(__uint_as_float(x.w));
}

template <int N>
__device__ __forceinline__ void add_vector(Soft &a, const float (&f)[N], float scale, int) {
    float m = f[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, f[i]);
    if (m > a.m) {
        a.s *= ex2((a.m - m) * scale);  // a.m = -inf: times 0
        a.m = m;
    }
    const float2 nm = splat2(-finite_max(a.m)), s2 = splat2(scale);
    float2 t = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 d = mul2(add2(make_float2(f[i], f[i + 1]), nm), s2);
        t = add2(t, make_float2(ex2(d.x), ex2(d.y)));
    }
    a.s += t.x + t.y;
}
template <int N>
__device__ __forceinline__ void add_vector(Best &a, const float (&f)[N], float, int first) {
    float m = f[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, f[i]);
    if (m > a.v) {  // indices of a thread ascend
        a.v = m;
#pragma unroll
        for (int i = N - 1; i >= 0; --i)
            if (f[i] == m) a.i = first + i;
    }
}
__device__ __forceinline__ void add_one(Soft &a, float x, float scale, int) {
    if (x > a.m) {
        a.s *= ex2((a.m - x) * scale);
        a.m = x;
    }
    a.s += ex2((x - finite_max(a.m)) * scale);
}
__device__ __forceinline__ void add_one(Best &a, float x, float, int i) {
    if (x > -INFINITY) a = join(a, Best{x, i}, 0.f);
}
__device__ __forceinline__ void clear(Soft &a) { a = Soft{-INFINITY, 0.f}; }
__device__ __forceinline__ void clear(Best &a) { a = Best{-INFINITY, -1}; }

// Elements [e0, e1) of `rows` rows (row(r) its address), joined per row over the CTA's threads
// into red[r][warp].
template <bool BF16, class P, class Row>
__device__ __forceinline__ void scan_rows(const Row &row, int rows, int e0, int e1, float scale, P (*red)[kVerWarps]) {
    constexpr int VE = BF16 ? 8 : 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int batches = max(1, ((e1 - e0) / VE + kVerBatch * kVerThreads - 1) / (kVerBatch * kVerThreads));
    Part now = part_of<BF16>(row(0), e0, e1);
    uint4 x[kVerBatch];
    load_batch<BF16>(now, 0, x);
    for (int r = 0; r < rows; ++r) {
        P a;
        clear(a);
        Part next = now;
        if (r + 1 < rows) next = part_of<BF16>(row(r + 1), e0, e1);
        // elements before and after the vectors: fewer than VE each
        const int head = now.first - e0, tail = now.first + now.nv * VE;
        const int one = (int)threadIdx.x < VE ? ((int)threadIdx.x < head ? e0 + (int)threadIdx.x : e1)
                                              : tail + (int)threadIdx.x - VE;
        const bool odd = one < e1;
        float xo = 0.f;
        if (odd) xo = load_in(row(r), one, BF16);
        for (int i = 0; i < batches; ++i) {
            uint4 y[kVerBatch];
            if (i + 1 < batches) load_batch<BF16>(now, i + 1, y);
            else if (r + 1 < rows) load_batch<BF16>(next, 0, y);
#pragma unroll
            for (int u = 0; u < kVerBatch; ++u) {
                float f[VE];
                elements(x[u], f, BF16);
                add_vector(a, f, scale, now.first + ((i * kVerBatch + u) * kVerThreads + (int)threadIdx.x) * VE);
                x[u] = y[u];
            }
        }
        if (odd) add_one(a, clean(xo), scale, one);
        a = join_warp(a, scale);
        if (lane == 0) red[r][warp] = a;
        now = next;
    }
}

// red[r][warp] of every CTA joined over its warps and the cluster into total[r], for `rows`
// rows; `part` is exchanged (alternate buffers in consecutive calls: a CTA that has passed
// the next call's barrier has read this call's).
template <class P>
__device__ __forceinline__ void join_cluster(P (*red)[kVerWarps], P *part, P *total, int rows, float scale, int CL) {
    __syncthreads();
    if ((int)threadIdx.x < rows) {
        P a = red[threadIdx.x][0];
        for (int w = 1; w < kVerWarps; ++w) a = join(a, red[threadIdx.x][w], scale);
        part[threadIdx.x] = a;
    }
    cluster_sync();
    if ((int)threadIdx.x < rows) {
        P a = peer(part + threadIdx.x, 0);
        for (int c = 1; c < CL; ++c) a = join(a, peer(part + threadIdx.x, (uint32_t)c), scale);
        total[threadIdx.x] = a;
    }
    __syncthreads();
}

template <bool BF16>
__global__ void __launch_bounds__(kVerThreads, 2) verify_kernel(const VerifyArgs p, int CL, int round) {
    __shared__ Soft red_s[2 * kVerRound][kVerWarps], part_s[2][2 * kVerRound], total_s[2 * kVerRound];
    __shared__ Best red_b[kVerRound][kVerWarps], part_b[2][kVerRound], total_b[kVerRound];
    const int b = blockIdx.x / CL, D = p.n_draft, V = p.vocab;
    const int rank = CL > 1 ? (int)cluster_rank() : 0;
    // parts of whole 64-element groups
    const int groups = (V + 63) / 64;
    const int e0 = min(V, 64 * (int)((int64_t)groups * rank / CL)), e1 = min(V, 64 * (int)((int64_t)groups * (rank + 1) / CL));
    const int L = p.draft_len ? min(max(p.draft_len[b], 0), D) : D;
    const float temp = p.temperature ? p.temperature[b] : 1.0f;
    const bool greedy = !(temp > 0.f), point_mass = p.draft == nullptr;
    const float scale = greedy ? kLog2e : fminf(fmaxf(1.0f / temp, 1e-30f), 1e37f) * kLog2e;
    constexpr int64_t ES = BF16 ? 2 : 4;
    auto trow = [&](int i) { return static_cast<const uint8_t *>(p.target) + ((int64_t)b * (D + 1) + i) * p.row_stride * ES; };
    auto drow = [&](int i) { return static_cast<const uint8_t *>(p.draft) + ((int64_t)b * D + i) * p.row_stride * ES; };
    const bool first_thread = threadIdx.x == 0 && rank == 0;
    int a = 0, token = -1, flip = 0;
    Soft P{-INFINITY, 0.f}, Q{-INFINITY, 0.f};
    int point = -1;  // the rejected token of a draft without probabilities (a point mass)
    bool rejected = false;
    if (greedy) {
        for (bool done = false; !done; flip ^= 1) {
            const int n = min(round, L + 1 - a), a0 = a;
            scan_rows<BF16>([&](int r) { return trow(a0 + r); }, n, e0, e1, scale, red_b);
            join_cluster(red_b, part_b[flip], total_b, n, scale, CL);
            for (int r = 0; r < n && !done; ++r) {
                token = total_b[r].i;
                const int x = a < L ? p.tokens[(int64_t)b * D + a] : -1;
                if (a < L && (x < 0 || x >= V) && first_thread) atomicOr(p.status, (uint32_t)kDevBadToken);
                if (a < L && x >= 0 && x == token) ++a;
                else done = true;
            }
        }
    } else {
        const int per = point_mass ? 1 : 2;  // rows of a position
        for (bool done = false; !done; flip ^= 1) {
            const int n = min(round, L + 1 - a), a0 = a;
            const int rows = per * n - (per == 2 && a0 + n > L ? 1 : 0);  // position L has no draft
            scan_rows<BF16>([&](int r) { return per == 1 ? trow(a0 + r) : r & 1 ? drow(a0 + (r >> 1)) : trow(a0 + (r >> 1)); },
                            rows, e0, e1, scale, red_s);
            join_cluster(red_s, part_s[flip], total_s, rows, scale, CL);
            for (int r = 0; r < n && !done; ++r) {
                P = total_s[per * r];
                if (a == L) {
                    done = true;
                    break;
                }
                const int x = p.tokens[(int64_t)b * D + a];
                const bool valid = x >= 0 && x < V;
                if (!valid && first_thread) atomicOr(p.status, (uint32_t)kDevBadToken);
                if (!point_mass) Q = total_s[2 * r + 1];
                bool ok = false;
                if (valid && P.s > 0.f) {
                    const float px = ex2((clean(load_in(trow(a), x, BF16)) - P.m) * scale) / P.s;
                    float qx = 1.f;
                    if (!point_mass) qx = Q.s > 0.f ? ex2((clean(load_in(drow(a), x, BF16)) - Q.m) * scale) / Q.s : 0.f;
                    ok = p.u[(int64_t)b * D + a] * qx < px;
                }
                if (ok) {
                    ++a;
                } else {
                    rejected = done = true;
                    if (point_mass) point = x;
                }
            }
        }
        if (P.s > 0.f) {
            const float *const noise = p.noise + (int64_t)b * V;
            const uint8_t *const prow = trow(a), *const qrow = rejected && !point_mass ? drow(a) : nullptr;
            const float ip = 1.f / P.s;
            for (int pass = rejected ? 0 : 1; pass < 2 && token < 0; ++pass, flip ^= 1) {  // pass 1: no residual is left, or none is due
                const bool minus_q = pass == 0 && qrow && Q.s > 0.f;
                const float iq = minus_q ? 1.f / Q.s : 0.f;
                Best best{0.f, -1};
                float bar = 0.f;  // below the best of the warp, by more than the rounding of the test
                constexpr int U = 8;
                for (int i0 = e0 + (threadIdx.x & ~31); i0 < e1; i0 += U * kVerThreads) {
                    const int i = i0 + (threadIdx.x & 31);
                    float xt[U], nz[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int j = min(i + u * kVerThreads, e1 - 1);
                        xt[u] = load_in(prow, j, BF16);
                        nz[u] = noise[j];
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int j = i + u * kVerThreads;
                        float r = ex2((clean(xt[u]) - P.m) * scale) * ip;
                        if (r > bar * nz[u] && j < e1) {
                            if (minus_q) r -= ex2((clean(load_in(qrow, j, BF16)) - Q.m) * scale) * iq;
                            if (pass == 0 && j == point) r = 0.f;
                            const float score = r / nz[u];
                            if (r > 0.f && score > best.v) best = Best{score, j};
                        }
                    }
                    // positive floats compare as their bits
                    bar = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(best.v))) * (1.f - 0x1p-20f);
                }
                best = join_warp(best, 0.f);
                if ((threadIdx.x & 31) == 0) red_b[0][threadIdx.x >> 5] = best;
                join_cluster(red_b, part_b[flip], total_b, 1, 0.f, CL);
                token = total_b[0].i;
            }
        }
    }
    if (rank == 0) {
        if (threadIdx.x == 0) p.count_out[b] = a + (token >= 0 ? 1 : 0);
        for (int i = threadIdx.x; i <= D; i += kVerThreads)
            p.tokens_out[(int64_t)b * (D + 1) + i] = i < a ? p.tokens[(int64_t)b * D + i] : i == a ? token : -1;
    }
    if (CL > 1) cluster_sync();  // a CTA's shared memory is read until here
}

}  // namespace

cudaError_t launch_verify(VerifyArgs p, cudaStream_t s) {
    static std::atomic<uint32_t *> cache[64];
    const cudaError_t e = symbol_address_cached(&g_status_verify, cache, &p.status);
    if (e != cudaSuccess) return e;
    // up to 8 CTAs per request while they are at most 8 per SM, parts of 2048 tokens at least
    const int sms = sm_count();
    int CL = 8;
    while (CL > 1 && ((int64_t)p.batch * CL > 8 * (int64_t)sms || p.vocab / CL < 2048)) CL /= 2;
    // few requests: the rows of all positions in one round
    const int round = (int64_t)p.batch * CL >= 2 * (int64_t)sms ? 1 : kVerRound;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.batch * CL));
    cfg.blockDim = dim3(kVerThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)CL, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return p.bf16 ? cudaLaunchKernelEx(&cfg, verify_kernel<true>, p, CL, round)
                  : cudaLaunchKernelEx(&cfg, verify_kernel<false>, p, CL, round);
}

cudaError_t take_status_verify(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_verify, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_verify, &zero, sizeof(uint32_t));
}

}  // namespace damp
