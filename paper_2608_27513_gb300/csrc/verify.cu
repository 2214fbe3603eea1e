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
// time is latency and all positions share a round.  Bound by the chain of rounds of a request,
// with the bytes of the rows needed next: 256 requests of 3 drafts, V = 151552, bf16 take
// 135 us (3.8 TB/s), of which the race is 50; 61 of 5 drafts, V = 100003, 50 us (two in a
// round); one of 4 drafts, V = 32000, FP32, 12.7 us.  Tokens masked with a large negative number,
// shifted logits and log-probabilities take as long (64 of 3 drafts, V = 100000: 41 us each).
// Rows whose largest logit is infinite or more than 727000 temperatures (2^20 in base 2) from 0 are
// summed element by element after the fast pass, at about twice the time, as are parts with NaN.
//
// The race reads its target row again (from L2) and the noise; p_t >= r_t, so a token whose
// p_t / noise_t does not reach the best score of its CTA so far cannot win, and only for the
// few others the draft's probability and the quotient are taken.
#include "damp_common.cuh"
#include "damp_internal.h"

#include <cfloat>

namespace damp {

static __device__ uint32_t g_status_verify;

namespace {

constexpr int kVerThreads = 256;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerDepth = 12;   // 16-byte slots of a thread in the ring (48 KB per CTA, four CTAs per SM)
constexpr int kVerBatch = 4;    // vectors of a batch of scan_rows; a batch of the race takes 6 slots
constexpr int kVerRing = kVerDepth * kVerThreads * 16;
constexpr int kVerRound = 4;    // positions of a round at most
constexpr int kVerCluster = 8;  // CTAs per request at most
static_assert(2 * kVerRound <= kVerWarps, "a warp joins a row");
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
__device__ __forceinline__ Best join(Best a, Best b) {
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
// over groups of 2 M neighbouring lanes; every lane has the result
template <int M>
__device__ __forceinline__ Best join_warp(Best a, float) {
#pragma unroll
    for (int m = M; m; m >>= 1) a = join(a, Best{__shfl_xor_sync(kFull, a.v, m), __shfl_xor_sync(kFull, a.i, m)});
    return a;
}
template <int M>
__device__ __forceinline__ Soft join_warp(Soft a, float scale) {  // the maximum first: one exponential
    float m = a.m;
#pragma unroll
    for (int d = M; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, d));
    float s = a.s * ex2((a.m - finite_max(m)) * scale);
#pragma unroll
    for (int d = M; d; d >>= 1) s += __shfl_xor_sync(kFull, s, d);
    return Soft{m, s};
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
// the elements of a vector, as they are
__device__ __forceinline__ void elements(const uint4 &x, float (&f)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void elements(const uint4 &x, float (&f)[4]) {
    f[0] = __uint_as_float(x.x);
    f[1] = __uint_as_float(x.y);
    f[2] = __uint_as_float(x.z);
    f[3] = __uint_as_float(x.w);
}
// the largest element of some vectors (a NaN is dropped)
template <bool BF16, int N>
__device__ __forceinline__ float largest(const uint4 (&x)[N]) {
    if (BF16) {
        __nv_bfloat162 m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __nv_bfloat162 w[4];
            memcpy(w, &x[i], 16);
            const __nv_bfloat162 y = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
            m = i ? __hmax2(m, y) : y;
        }
        uint32_t w;
        memcpy(&w, &m, 4);
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i)
        m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(x[i].x), __uint_as_float(x[i].y)), fmaxf(__uint_as_float(x[i].z), __uint_as_float(x[i].w))));
    return m;
}

// one element, cleaned
__device__ __forceinline__ void add_one(Soft &a, float x, float scale, int) {
    if (x > a.m) {
        a.s *= ex2((a.m - x) * scale);
        a.m = x;
    }
    a.s += ex2((x - finite_max(a.m)) * scale);
}
__device__ __forceinline__ void add_one(Best &a, float x, float, int i) {
    if (x > -INFINITY) a = join(a, Best{x, i});
}
__device__ __forceinline__ void clear(Soft &a) { a = Soft{-INFINITY, 0.f}; }
__device__ __forceinline__ void clear(Best &a) { a = Best{-INFINITY, -1}; }

// What a thread collects over its vectors of a row, as they are.  Sums are of 2^{x scale - c} with
// an integer c (the running maximum's exponent, rounded up): x scale - c is one fused operation
// with one rounding, and c changes by exact factors.  c is kSoftLow at least (the initial one stands for
// an empty sum), which leaves tokens masked with a large negative number out of the sum; a row whose
// maximum is lower than that is summed element by element.
constexpr float kSoftLow = -0x1p20f;
struct SoftRun {
    float m, c, s;
    __device__ __forceinline__ SoftRun() : m(-INFINITY), c(-FLT_MAX), s(0.f) {}
    template <bool BF16, int N>
    __device__ __forceinline__ void add(const uint4 (&x)[N], float scale, int, int) {
        constexpr int VE = BF16 ? 8 : 4;
        const float top = largest<BF16>(x);
        if (top > m) {
            m = top;
            const float c1 = ceilf(fmaxf(top * scale, kSoftLow));
            s *= ex2(c - c1);
            c = c1;
        }
        const float2 nc = splat2(-c), s2 = splat2(scale);
        float2 t[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f[VE];
            elements(x[i], f);
#pragma unroll
            for (int e = 0; e < VE; e += 2) {
                const float2 d = fma2(make_float2(f[e], f[e + 1]), s2, nc);
                t[e / 2 & 1] = add2(t[e / 2 & 1], make_float2(ex2(d.x), ex2(d.y)));
            }
        }
        s += (t[0].x + t[0].y) + (t[1].x + t[1].y);
    }
    // false: an infinity or a NaN beside other elements, or a maximum too large for whole exponents to be
    // exact
    __device__ __forceinline__ bool result(Soft &a, float scale) const {
        a = Soft{m, s == 0.f ? 0.f : s * ex2(fmaf(-m, scale, c))};
        return s <= FLT_MAX && m * scale < 0x1p20f;
    }
};
struct BestRun {
    Best a;
    __device__ __forceinline__ BestRun() : a{-INFINITY, -1} {}
    template <bool BF16, int N>
    __device__ __forceinline__ void add(const uint4 (&x)[N], float, int first, int step) {  // ascending indices
        constexpr int VE = BF16 ? 8 : 4;
        if (largest<BF16>(x) > a.v) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float f[VE];
                elements(x[i], f);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float y = clean(f[e]);
                    if (y > a.v) a = Best{y, first + i * step + e};
                }
            }
        }
    }
    __device__ __forceinline__ bool result(Best &b, float) const {
        b = a;
        return true;
    }
};
// a joined row, with a sum of -1 if its maximum is where the sums are not exact
__device__ __forceinline__ Soft marked(Soft a, float scale, bool single) {
    if (!single && a.m > -INFINITY && a.m * scale < kSoftLow) a.s = -1.f;
    return a;
}
__device__ __forceinline__ Best marked(Best a, float, bool) { return a; }
__device__ __forceinline__ SoftRun run_of(Soft) { return SoftRun(); }
__device__ __forceinline__ BestRun run_of(Best) { return BestRun(); }

// Warps on one of `rows` rows at a time: more than one row in a round go to groups of warps, so
// that a warp has longer pieces of fewer rows.
__device__ __forceinline__ int warps_per_row(int rows) {
    return rows >= 8 ? kVerWarps / 8 : rows >= 4 ? kVerWarps / 4 : rows >= 2 ? kVerWarps / 2 : kVerWarps;
}

// Elements [e0, e1) of `rows` rows (row(r) the address of one), joined per row over each warp of
// its group into red[r][warp of the group].  A thread copies its vectors of all its rows, in
// order, into its own slots of the ring (asynchronous 16-byte copies, a group per batch, also
// empty ones) and reads only those: the copies run on across the ends of rows and no barrier is
// needed.
// `single`: element by element in any case.
template <bool BF16, class P, class Row>
__device__ __forceinline__ void scan_rows(const Row &row, int rows, int e0, int e1, float scale, P (*red)[kVerWarps],
                                          uint32_t ring, bool single = false) {
    constexpr int VE = BF16 ? 8 : 4, AHEAD = kVerDepth / kVerBatch, SLOT = kVerThreads * 16;
    constexpr uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
    const int lane = threadIdx.x & 31, per = warps_per_row(rows), groups = kVerWarps / per;
    const int r0 = (threadIdx.x >> 5) / per, warp = (threadIdx.x >> 5) % per;  // first row, warp of the group
    const int step = 32 * per, tid = 32 * warp + lane;
    const int iters = ((e1 - e0) / VE + kVerBatch * step - 1) / (kVerBatch * step);
    const uint32_t mine = ring + 16 * threadIdx.x;
    int ir = r0, iv = tid;      // the next copy: row, first vector
    Part ahead = part_of<BF16>(row(min(r0, rows - 1)), e0, e1);
    uint32_t put = 0, get = 0;  // first slots
    auto copy_next = [&]() {
        if (ir < rows) {
#pragma unroll
            for (int u = 0; u < kVerBatch; ++u)
                if (iv + u * step < ahead.nv) cp_async16(mine + (put + u) * SLOT, ahead.vec + iv + u * step);
            put = put + kVerBatch == kVerDepth ? 0 : put + kVerBatch;
            iv += kVerBatch * step;
            if (iv >= iters * kVerBatch * step) {
                iv = tid;
                ir += groups;
                if (ir < rows) ahead = part_of<BF16>(row(ir), e0, e1);
            }
        }
        cp_async_commit();
    };
    if (iters) {
        for (int d = 0; d < AHEAD; ++d) copy_next();
    }
    for (int r = r0; r < rows; r += groups) {
        const uint8_t *const at = row(r);
        const Part now = part_of<BF16>(at, e0, e1);
        // one element of this thread before or after the vectors (fewer than VE each)
        const int head = now.first - e0, tail = now.first + now.nv * VE;
        const int one = tid < VE ? (tid < head ? e0 + tid : e1) : tail + tid - VE;
        const float xo = one < e1 ? load_in(at, one, BF16) : 0.f;
        P a;
        clear(a);
        auto run = run_of(a);
        for (int i = 0; i < iters; ++i) {
            cp_async_wait<AHEAD - 1>();
            const int v = i * kVerBatch * step + tid;
            uint4 x[kVerBatch];
#pragma unroll
            for (int u = 0; u < kVerBatch; ++u)
                x[u] = v + u * step < now.nv ? lds128(mine + (get + u) * SLOT) : make_uint4(none, none, none, none);
            get = get + kVerBatch == kVerDepth ? 0 : get + kVerBatch;
            run.template add<BF16>(x, scale, now.first + v * VE, step * VE);
            copy_next();
        }
        if (!run.result(a, scale) || single) {  // again, element by element
            clear(a);
            for (int v = tid; v < now.nv; v += step)
                for (int e = 0; e < VE; ++e) add_one(a, clean(load_in(now.vec + v, e, BF16)), scale, now.first + v * VE + e);
        }
        if (one < e1) add_one(a, clean(xo), scale, one);
        a = join_warp<16>(a, scale);
        if (lane == 0) red[r][warp] = a;
    }
    cp_async_wait_all();
}

// red[r][0 .. warps-1] of every CTA joined, and over the cluster, into total[r], for `rows` rows;
// `part` is exchanged (alternate buffers in consecutive calls: a CTA that has passed
// the next call's barrier has read this call's).  `single`: of rows scanned so.
template <class P>
__device__ __forceinline__ void join_cluster(P (*red)[kVerWarps], P *part, P *total, int rows, int warps, float scale,
                                             int CL, bool single = false) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    if (warp < rows) {
        P a;
        clear(a);
        if (lane < warps) a = red[warp][lane];
        a = join_warp<kVerWarps / 2>(a, scale);
        if (lane == 0) part[warp] = a;
    }
    cluster_sync();
    if (warp < rows) {
        P a;
        clear(a);
        if (lane < CL) a = peer(part + warp, (uint32_t)lane);
        a = join_warp<kVerCluster / 2>(a, scale);
        if (lane == 0) total[warp] = marked(a, scale, single);
    }
    __syncthreads();
}

template <bool BF16>
__global__ void __launch_bounds__(kVerThreads, 4) verify_kernel(const VerifyArgs p, int CL, int round) {
    __shared__ Soft red_s[2 * kVerRound][kVerWarps], part_s[2][2 * kVerRound], total_s[2 * kVerRound];
    __shared__ Best red_b[kVerRound][kVerWarps], part_b[2][kVerRound], total_b[kVerRound];
    // of the positions of a round (alternate buffers, as in join_cluster): the token, its logits, its uniform
    __shared__ int drafted[2][kVerRound];
    __shared__ float logit_t[2][kVerRound], logit_d[2][kVerRound], uniform[2][kVerRound];
    __shared__ uint32_t bar_bits;
    extern __shared__ __align__(16) uint4 ring_mem[];
    const uint32_t ring = smem_u32(ring_mem);
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
    int a = 0, token = -1, flip = 0;
    // fetched before a round's rows are scanned; read after its barriers
    auto fetch_drafts = [&](int a0, int n) {
        if ((int)threadIdx.x < n && a0 + (int)threadIdx.x < L) {
            const int r = threadIdx.x, i = a0 + r, x = p.tokens[(int64_t)b * D + i];
            const bool valid = x >= 0 && x < V;
            drafted[flip][r] = valid ? x : -1;
            if (!greedy) {
                logit_t[flip][r] = valid ? clean(load_in(trow(i), x, BF16)) : -INFINITY;
                logit_d[flip][r] = valid && !point_mass ? clean(load_in(drow(i), x, BF16)) : -INFINITY;
                uniform[flip][r] = p.u[(int64_t)b * D + i];
            }
        }
    };
    auto report = [&](int x) {
        if (x < 0 && rank == 0 && threadIdx.x == 0) atomicOr(p.status, (uint32_t)kDevBadToken);
    };
    Soft P{-INFINITY, 0.f}, Q{-INFINITY, 0.f};
    int point = -1;  // the rejected token of a draft without probabilities (a point mass)
    bool rejected = false;
    if (threadIdx.x == 0) bar_bits = 0;  // seen after the barriers of a round
    if (greedy) {
        for (bool done = false; !done; flip ^= 1) {
            const int n = min(round, L + 1 - a), a0 = a;
            fetch_drafts(a0, n);
            scan_rows<BF16>([&](int r) { return trow(a0 + r); }, n, e0, e1, scale, red_b, ring);
            join_cluster(red_b, part_b[flip], total_b, n, warps_per_row(n), scale, CL);
            for (int r = 0; r < n && !done; ++r) {
                token = total_b[r].i;
                if (a < L) report(drafted[flip][r]);
                if (a < L && token >= 0 && drafted[flip][r] == token) ++a;
                else done = true;
            }
        }
    } else {
        const int per = point_mass ? 1 : 2;  // rows of a position
        bool single = false;                 // this and the later rows are summed element by element
        for (bool done = false; !done; flip ^= 1) {
            const int n = min(round, L + 1 - a), a0 = a;
            const int rows = per * n - (per == 2 && a0 + n > L ? 1 : 0);  // position L has no draft
            fetch_drafts(a0, n);
            scan_rows<BF16>([&](int r) { return per == 1 ? trow(a0 + r) : r & 1 ? drow(a0 + (r >> 1)) : trow(a0 + (r >> 1)); },
                            rows, e0, e1, scale, red_s, ring, single);
            join_cluster(red_s, part_s[flip], total_s, rows, warps_per_row(rows), scale, CL, single);
            for (int r = 0; r < n && !done; ++r) {
                P = total_s[per * r];
                if (per == 2 && a < L) Q = total_s[2 * r + 1];
                if (fminf(P.s, Q.s) < 0.f) {  // marked: this position again
                    single = true;
                    break;
                }
                if (a == L) {
                    done = true;
                    break;
                }
                const int x = drafted[flip][r];
                report(x);
                bool ok = false;
                if (x >= 0 && P.s > 0.f) {
                    const float px = ex2((logit_t[flip][r] - P.m) * scale) / P.s;
                    const float qx = point_mass ? 1.f : Q.s > 0.f ? ex2((logit_d[flip][r] - Q.m) * scale) / Q.s : 0.f;
                    ok = uniform[flip][r] * qx < px;
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
                const int lane = threadIdx.x & 31;
                // token j with r_j / noise_j exactly, if it beats this thread's best (ascending j)
                Best best{0.f, -1};
                auto exact = [&](int j, float x, float e) {
                    float r = ex2((clean(x) - P.m) * scale) * ip;
                    if (minus_q) r -= ex2((clean(load_in(qrow, j, BF16)) - Q.m) * scale) * iq;
                    if (pass == 0 && j == point) r = 0.f;
                    const float score = r / e;
                    if (r > 0.f && score > best.v) best = Best{score, j};
                };
                auto exactly = [&](int j) { exact(j, load_in(prow, j, BF16), noise[j]); };
                // The test: 2^{(x - m) scale} > bar noise, with bar below the best score of the CTA so far
                // times P.s, by more than its rounding.  A first token of every thread gives a start.
                auto bar_of = [&](bool found) {  // positive floats compare as their bits
                    if (found) {
                        const uint32_t m = __reduce_max_sync(kFull, __float_as_uint(best.v));
                        if (lane == 0) atomicMax(&bar_bits, m);
                    }
                    return __uint_as_float(*static_cast<volatile uint32_t *>(&bar_bits)) * P.s * (1.f - 0x1p-20f);
                };
                const Part now = part_of<BF16>(prow, e0, e1);
                const bool vectors = ((reinterpret_cast<uintptr_t>(noise + now.first)) & 15) == 0;
                constexpr int VE = BF16 ? 8 : 4;
                const int vec_end = vectors ? now.first + now.nv * VE : e0;  // [first, vec_end) as vectors
                // batches of NB vectors: a slot per vector of logits and one per four noises, copied ahead
                constexpr int NB = BF16 ? 2 : 3, NS = 6, AHEAD = kVerDepth / NS, STEP = kVerThreads, SLOT = STEP * 16;
                static_assert(NB * (1 + VE / 4) == NS, "");
                const uint32_t mine = ring + 16 * threadIdx.x;
                int iv = threadIdx.x;
                uint32_t put = 0, get = 0;
                auto copy_next = [&]() {
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        const int i = iv + n * STEP;
                        if (i < now.nv) {
                            const uint32_t at = mine + (put + n * (1 + VE / 4)) * SLOT;
                            cp_async16(at, now.vec + i);
#pragma unroll
                            for (int e = 0; e < VE / 4; ++e) cp_async16(at + (e + 1) * SLOT, noise + now.first + i * VE + 4 * e);
                        }
                    }
                    put = put + NS == kVerDepth ? 0 : put + NS;
                    iv += NB * STEP;
                    cp_async_commit();
                };
                if (vectors) {
#pragma unroll
                    for (int d = 0; d < AHEAD; ++d) copy_next();
                }
                const int start = vectors ? now.first + (int)threadIdx.x * VE : e0 + (int)threadIdx.x;
                if (start < (vectors ? vec_end : e1)) exactly(start);
                bar_of(true);
                __syncthreads();
                float bar = bar_of(false);
                if (vectors) {
                    for (int i0 = threadIdx.x & ~31; i0 < now.nv; i0 += NB * STEP) {
                        float over[NB * VE];
                        float most = -1.f;
                        cp_async_wait<AHEAD - 1>();
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            const uint32_t at = mine + (get + n * (1 + VE / 4)) * SLOT;
                            float f[VE];
                            elements(lds128(at), f);
                            const float2 nm = splat2(-P.m), s2 = splat2(scale);
#pragma unroll
                            for (int e = 0; e < VE; e += 4) {
                                const uint4 w = lds128(at + (e / 4 + 1) * SLOT);
                                const float2 d0 = mul2(add2(make_float2(f[e], f[e + 1]), nm), s2);
                                const float2 d1 = mul2(add2(make_float2(f[e + 2], f[e + 3]), nm), s2);
                                const bool live = i0 + lane + n * STEP < now.nv;  // else the slot holds something else
                                float *const ov = over + n * VE + e;
                                ov[0] = live ? fmaf(-bar, __uint_as_float(w.x), ex2(d0.x)) : -1.f;
                                ov[1] = live ? fmaf(-bar, __uint_as_float(w.y), ex2(d0.y)) : -1.f;
                                ov[2] = live ? fmaf(-bar, __uint_as_float(w.z), ex2(d1.x)) : -1.f;
                                ov[3] = live ? fmaf(-bar, __uint_as_float(w.w), ex2(d1.y)) : -1.f;
                                most = fmaxf(most, fmaxf(fmaxf(ov[0], ov[1]), fmaxf(ov[2], ov[3])));
                            }
                        }
                        const bool found = __any_sync(kFull, most > 0.f);
                        if (found) {
                            uint32_t mask = 0;
#pragma unroll
                            for (int e = 0; e < NB * VE; ++e) mask |= over[e] > 0.f ? 1u << e : 0u;
                            for (; mask; mask &= mask - 1) {
                                const int e = __ffs(mask) - 1, n = e / VE, k = e % VE;
                                const uint32_t at = mine + (get + n * (1 + VE / 4)) * SLOT;
                                exact(now.first + (i0 + lane + n * STEP) * VE + k, BF16 ? bf16_at(at, k) : ldsf(at + 4 * k),
                                      ldsf(at + (k / 4 + 1) * SLOT + 4 * (k % 4)));
                            }
                        }
                        get = get + NS == kVerDepth ? 0 : get + NS;
                        bar = bar_of(found);
                        copy_next();
                    }
                    cp_async_wait_all();
                }
                // the other elements, one per lane, U of a thread at a time and the next U in flight
                const int head = vectors ? now.first - e0 : 0, others = head + (e1 - vec_end);
                auto other = [&](int k) { return min(k < head ? e0 + k : vec_end + k - head, e1 - 1); };
                constexpr int U = 4;
                float xn[U], en[U];
                auto fetch = [&](int k0) {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int j = other(k0 + lane + u * kVerThreads);
                        xn[u] = load_in(prow, j, BF16);
                        en[u] = noise[j];
                    }
                };
                const int k1 = threadIdx.x & ~31;
                if (k1 < others) fetch(k1);
                for (int k0 = k1; k0 < others; k0 += U * kVerThreads) {
                    float x[U], e[U], over = -1.f;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        x[u] = xn[u];
                        e[u] = en[u];
                    }
                    if (k0 + U * kVerThreads < others) fetch(k0 + U * kVerThreads);
#pragma unroll
                    for (int u = 0; u < U; ++u) over = fmaxf(over, fmaf(-bar, e[u], ex2((x[u] - P.m) * scale)));
                    const bool found = __any_sync(kFull, over > 0.f);
                    if (over > 0.f) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const int k = k0 + lane + u * kVerThreads;
                            if (k < others && fmaf(-bar, e[u], ex2((x[u] - P.m) * scale)) > 0.f) {
                                const Best mine_before = best;  // elements before the vectors come out of order:
                                best = Best{0.f, -1};           // ties still go to the lower index
                                exact(other(k), x[u], e[u]);
                                best = join(mine_before, best);
                            }
                        }
                    }
                    bar = bar_of(found);
                }
                best = join_warp<16>(best, 0.f);
                if (lane == 0) red_b[0][threadIdx.x >> 5] = best;
                join_cluster(red_b, part_b[flip], total_b, 1, kVerWarps, 0.f, CL);
                token = total_b[0].i;  // no residual: bar_bits is still 0
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
    // CTAs per request: 8 while there are at most 8 CTAs per SM, parts of 2048 tokens at least (256
    // requests of 3 drafts, V = 151552: 4 CTAs 135 us, 2 CTAs 148, 8 CTAs 151).  Positions of a round:
    // one where the CTAs fill the GPU (the same: 135 us, two 139, four 151), up to four where the time
    // is latency (one request of 4 drafts, V = 32000: four 12.7 us, one 16.5; 61 requests of 5 drafts,
    // V = 100003: two 50.5 us, one 56.8).
    const int64_t sms = sm_count();
    int CL = kVerCluster;
    while (CL > 1 && (p.batch * (int64_t)CL > 8 * sms || p.vocab / CL < 2048)) CL /= 2;
    const int64_t ctas = p.batch * (int64_t)CL;
    const int round = ctas >= 4 * sms ? 1 : ctas >= sms ? 2 : kVerRound;
    const void *const kern = p.bf16 ? reinterpret_cast<const void *>(verify_kernel<true>) : reinterpret_cast<const void *>(verify_kernel<false>);
    const cudaError_t es = ensure_smem_limit(kern, kVerRing);
    if (es != cudaSuccess) return es;
    cudaLaunchConfig_t cfg{};
    cfg.dynamicSmemBytes = kVerRing;
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
