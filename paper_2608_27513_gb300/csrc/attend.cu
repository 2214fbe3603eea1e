// attend.cu -- attention over the 8-bit cache: o_r = sum_j softmax_j(scale q_r.k_j) v_j.
//
// The rows of an item are the (query token, query head) pairs that share a (batch row, KV head), 16 of
// them; its keys are the pages from the first that its first query sees to the last that
// its last query sees.  All pages of all items form one sequence, which is cut into equal ranges,
// one per warp: the work is even whatever the lengths are, and the host need not know them.  A warp
// keeps one item's running maximum m, sum l and output o in registers and passes over each page
// once.  An item that lies inside a warp's range is written at once; parts of an item are left in
// the workspace as (o, m, l) and joined by a second, dependent launch.
//
// A warp's pages come by one bulk copy each (keys, values, scales) into a ring of its own; no warp
// waits for another.  Products run on m16n8k16 with FP16 operands and FP32 sums.  Codes minus 128
// are exact in FP16.  A query row is scaled by a power of two to below 2^15 and rounded to FP16:
// BF16 values lose nothing above 2^-39 of the row's largest (FP32: two FP16 parts, 22 bits).
// Weights p s_v / 2^e, where 2^e is the running power of two above the value scales that a row has seen, lie in
// 0 .. 1 and enter as FP16 times 2^10 (2^-11 relative down to 2^-24 of the largest; an output in
// BF16 is rounded by 2^-8 anyway), as two parts for FP32.  Sums, maxima and outputs are FP32.
//
// The contraction index of Q K^T is permuted so that a lane's operands are 16 consecutive codes,
// and the columns of P V so that a lane reads 16 consecutive codes of 4 tokens: 16-byte loads
// without bank conflicts, one byte permute and one subtraction per two codes.
//
// Few rows of short contexts run a CTA per item and one launch (attend_items_kernel).  Where all warps of a
// CTA lie inside one item, of a long context, the CTA joins their parts before it leaves one.
//
// Bound by the cache's bytes: 256 rows of up to 4096 tokens, 32 heads, 8 KV heads, d = 128 take 215 us (6.3 TB/s
// of codes, the join 8 of them); a row of 131071 tokens 54 us, of which 4 are the start (lengths, tables and first
// copies, one after the other) and 5 the join.  A page costs a warp 1.2 us from copy to copy with 3 to 4
// in flight, 8 warps to an SM: rows of 1000 tokens, a page or four to a warp, are bound by that (9 us).
#include "attend.cuh"

#include <algorithm>

namespace damp {

static __device__ uint32_t g_status_attend;

namespace {

constexpr int kJoinThreads = 256;
constexpr int kNoScale = -1000;  // below every exponent field
template <int D, bool F32>
struct AttCfg {
    static constexpr int R = 16;
    static constexpr int parts = F32 ? 2 : 1;
    static constexpr int warps = D == 256 ? 4 : 8;
    static constexpr int threads = warps * 32;
    static constexpr int rec = cache_record_bytes(D);
    static constexpr bool q_smem = D / 2 + parts * D / 4 > 128;  // registers of o and q
    static constexpr int qbytes = q_smem ? parts * (D / 16) * 512 : 0;
    static constexpr int stages = std::min(4, (215000 / warps - qbytes) / (rec + 48));
    static constexpr int ring = stages * rec;
    static constexpr int warp_bytes = ring + qbytes + stages * 48;  // 32 bytes about the page, the barrier
    static_assert(stages >= 2, "ring");
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d += (sum of a's parts) b.  The tensor cores cut their sums off where FP32 additions round: errors of one sign, which
// add up over the pages.  For FP32 inputs 16 products at a time, the small part's first, are summed there and added
// here.  Error norm against 64 bits, all sums there and as it is: a row of 1000 tokens, d = 64,
// 7.3e-7 and 3.1e-7 (FP32 matrix products: 3.1e-7), 2 rows of up to 300 queries in up to 3000 tokens, d = 128, 2.4e-6
// and 4.0e-7 (1.2e-6), 4 rows of 640 queries in 8000 tokens, d = 64, 7.1e-6 before.  It costs 16 rows of 4000 tokens, 8 KV heads, d = 128, 53 us instead of 45, 64 rows with 2 KV heads,
// d = 256, 113 instead of 73.  (BF16 outputs are rounded by 2^-8 anyway.)
template <int PARTS>
__device__ __forceinline__ void mma_add(float (&d)[4], const uint32_t (&a)[PARTS][4], uint32_t b0, uint32_t b1) {
    if constexpr (PARTS == 2) {
        float z[4] = {0.f, 0.f, 0.f, 0.f};
        mma16816(z, a[1], b0, b1);
        mma16816(z, a[0], b0, b1);
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] += z[i];
    } else {
        mma16816(d, a[0], b0, b1);
    }
}
// a and b as FP16 parts
__device__ __forceinline__ void split_pair(float a, float b, uint32_t &hi, uint32_t &lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 f = __half22float2(h);
    hi = *reinterpret_cast<const uint32_t *>(&h);
    lo = half_pair(a - f.x, b - f.y);
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor_sync(kFull, x, 1));
    return fmaxf(x, __shfl_xor_sync(kFull, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(kFull, x, 1);
    return x + __shfl_xor_sync(kFull, x, 2);
}
// 16 values of a query row
template <bool BF>
__device__ __forceinline__ void load16(const void *p, int64_t at, bool live, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    if (!live) return;
    if (BF) {
        const uint4 *g = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p) + at);
        const uint4 w[2] = {g[0], g[1]};
        const uint32_t *u = reinterpret_cast<const uint32_t *>(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    } else {
        const float4 *g = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 w = g[i];
            x[4 * i] = w.x, x[4 * i + 1] = w.y, x[4 * i + 2] = w.z, x[4 * i + 3] = w.w;
        }
    }
}
// 16 rows of queries and what a warp has of their outputs.
template <int D, bool F32>
struct AttRows {
    using C = AttCfg<D, F32>;
    static constexpr int R = C::R, kSteps = D / 16, kCols = D / 8;  // K steps of Q K^T, column tiles of P V
    static constexpr bool BF = !F32;
    float o[kCols][4], m[2], l[2], factor[2];
    int limit[2];  // the last token that a row sees
    uint32_t q[C::q_smem ? 1 : C::parts][C::q_smem ? 1 : kSteps][4];
    int ve[2];  // exponent field of a row's unit: above the value scales of the pages that it has seen

    // tile rt of a batch row's queries; qs: where in shared memory the operands go that registers do not hold
    __device__ __forceinline__ void start(const AttendArgs &p, AttRow w, int b, int rt, int h, uint32_t qs, int lane) {
        const int G = p.group, g = lane >> 2, c = lane & 3;
        __syncwarp();
        int64_t from[2];
        bool live[2];
        float up[2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int row = rt * R + hh * 8 + g, t = att_div(p, row);
            live[hh] = t < w.n;
            limit[hh] = live[hh] ? w.len - w.n + t : kNoRow;
            from[hh] = ((int64_t)b * p.T + t) * p.q_stride + (int64_t)(h * G + (row - t * G)) * D;
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                float x[16];
                load16<BF>(p.q, from[hh] + 16 * (c + 4 * j), live[hh], x);
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
            }
            top = quad_max(top);
            const int e = min(max((int)(__float_as_uint(top) >> 23), 15), 254);  // up to below 2^15
            up[hh] = __uint_as_float((uint32_t)(268 - e) << 23);
            factor[hh] = p.scale * (kLog2e * __uint_as_float((uint32_t)(e - 14) << 23));  // over up: the scale meets its inverse first
            m[hh] = -INFINITY;
            l[hh] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            float x[2][16];
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                load16<BF>(p.q, from[hh] + 16 * (c + 4 * j), live[hh], x[hh]);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[hh][i] *= up[hh];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        if (F32)
                            split_pair(x[hh][4 * i + 2 * k], x[hh][4 * i + 2 * k + 1], hi[2 * k + hh], lo[2 * k + hh]);
                        else
                            hi[2 * k + hh] = half_pair(x[hh][4 * i + 2 * k], x[hh][4 * i + 2 * k + 1]);
                    }
                }
                const int step = 4 * j + i;
                if constexpr (C::q_smem) {
                    const uint32_t at = qs + step * 512 + lane * 16;
                    sts128(at, make_uint4(hi[0], hi[1], hi[2], hi[3]));
                    if (F32) sts128(at + kSteps * 512, make_uint4(lo[0], lo[1], lo[2], lo[3]));
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        q[0][step][k] = hi[k];
                        if constexpr (F32) q[1][step][k] = lo[k];
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kCols; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        ve[0] = ve[1] = 0;
        __syncwarp();
    }
    // one page, whose record lies at kb in shared memory
    __device__ __forceinline__ void page(const AttendArgs &p, uint32_t kb, int page, uint32_t qs, int lane) {
        const int g = lane >> 2, c = lane & 3;
        const int kswz = cache_swizzle(g, D), vswz[2] = {cache_swizzle(2 * c, D), cache_swizzle(2 * c + 1, D)};
        const uint32_t vb = kb + cache_rows_bytes(D);
        const float ks = __uint_as_float(lds32(vb + cache_rows_bytes(D))), vs = __uint_as_float(lds32(vb + cache_rows_bytes(D) + 4));
        float s[4][4];
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            uint4 kk[4];
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) kk[nt] = lds128(kb + (8 * nt + g) * D + 16 * ((c + 4 * j) ^ kswz));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int step = 4 * j + i;
                uint32_t a[C::parts][4];
#pragma unroll
                for (int pt = 0; pt < C::parts; ++pt) {
                    if constexpr (C::q_smem) {
                        const uint4 w = lds128(qs + (pt * kSteps + step) * 512 + lane * 16);
                        a[pt][0] = w.x, a[pt][1] = w.y, a[pt][2] = w.z, a[pt][3] = w.w;
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) a[pt][k] = q[pt][step][k];
                    }
                }
#pragma unroll
                for (int nt = 0; nt < 4; ++nt) {
                    const uint32_t w = i == 0 ? kk[nt].x : i == 1 ? kk[nt].y : i == 2 ? kk[nt].z : kk[nt].w;
                    const uint32_t b0 = half_codes(w, 0x4140u), b1 = half_codes(w, 0x4342u);
                    mma_add<C::parts>(s[nt], a, b0, b1);
                }
            }
        }
        const int at = page * kCachePage;
        bool edge = false;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int k = limit[hh];
            edge = edge || (k != kNoRow && (k < at + kCachePage - 1 || (p.window && k - (p.window - 1) > at)));
        }
        const bool masked = __any_sync(kFull, edge);
        // vs = 2^(e - 127) mantissa / 2^10
        const int e = vs > 0.f ? min((int)(__float_as_uint(vs) >> 23) + 1, 253) : kNoScale;
        const float mantissa = vs > 0.f ? vs * __uint_as_float((uint32_t)(254 - e) << 23) * 1024.f : 0.f;
        bool moved = false;
        int fall[2];
        uint32_t pa[C::parts][4][2];  // [column tile][row half]
        float corr[2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const float fac = factor[hh] * ks;
            const int last = limit[hh], from = p.window ? last - (p.window - 1) : 0;
            // a row's unit: a power of two above the value scales of all pages so far of which it sees a token
            const int mine = !masked || (last >= at && from < at + kCachePage) ? e : kNoScale, up = max(ve[hh], mine);
            const float wscale = mantissa * __uint_as_float((uint32_t)max(127 + mine - up, 0) << 23);
            fall[hh] = ve[hh] - up;
            ve[hh] = up;
            float x[8], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = s[i >> 1][2 * hh + (i & 1)] * fac;
            if (masked) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int token = at + 8 * (i >> 1) + 2 * c + (i & 1);
                    if (token > last || token < from) x[i] = -INFINITY;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i]);
            const float mn = fmaxf(m[hh], quad_max(top)), mu = mn == -INFINITY ? 0.f : mn;
            corr[hh] = ex2(m[hh] - mu);
            moved = moved || mn != m[hh] || fall[hh] != 0;
            m[hh] = mn;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = ex2(x[i] - mu);
                sum += x[i];
                x[i] *= wscale;
            }
            l[hh] = fmaf(l[hh], corr[hh], sum);
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
                if constexpr (F32)
                    split_pair(x[2 * nt], x[2 * nt + 1], pa[0][nt][hh], pa[1][nt][hh]);
                else
                    pa[0][nt][hh] = half_pair(x[2 * nt], x[2 * nt + 1]);
            }
        }
        if (__any_sync(kFull, moved)) {
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) corr[hh] *= __uint_as_float((uint32_t)max(127 + fall[hh], 0) << 23);
#pragma unroll
            for (int i = 0; i < kCols; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i][k] *= corr[k >> 1];
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
            uint32_t a[C::parts][4];
#pragma unroll
            for (int pt = 0; pt < C::parts; ++pt)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[pt][k] = pa[pt][2 * s2 + (k >> 1)][k & 1];
#pragma unroll
            for (int grp = 0; grp < (D + 127) / 128; ++grp) {
                constexpr int W = D == 64 ? 2 : 4;  // words of codes per token
                uint32_t w[4][W];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t row = vb + (16 * s2 + 8 * (k >> 1) + 2 * c + (k & 1)) * D;
                    if constexpr (D == 64) {
                        const uint2 y = lds64(row + 16 * ((g >> 1) ^ vswz[k & 1]) + 8 * (g & 1));
                        w[k][0] = y.x, w[k][1] = y.y;
                    } else {
                        const uint4 y = lds128(row + 16 * ((g + 8 * grp) ^ vswz[k & 1]));
                        w[k][0] = y.x, w[k][1] = y.y, w[k][W - 2] = y.z, w[k][W - 1] = y.w;
                    }
                }
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const uint32_t t0 = prmt(w[0][i], w[1][i], 0x5140u), t1 = prmt(w[0][i], w[1][i], 0x7362u);
                    const uint32_t u0 = prmt(w[2][i], w[3][i], 0x5140u), u1 = prmt(w[2][i], w[3][i], 0x7362u);
                    const uint32_t b0[4] = {half_codes(t0, 0x4140u), half_codes(t0, 0x4342u), half_codes(t1, 0x4140u), half_codes(t1, 0x4342u)};
                    const uint32_t b1[4] = {half_codes(u0, 0x4140u), half_codes(u0, 0x4342u), half_codes(u1, 0x4140u), half_codes(u1, 0x4342u)};
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_add<C::parts>(o[grp * 16 + 4 * i + k], a, b0[k], b1[k]);
                }
            }
        }
    }
    // the outputs, where all pages were this warp's; else a part of them: rows of D values, and their (m, l)
    __device__ __forceinline__ void leave(const AttendArgs &p, int b, int rt, int h, bool whole, float *parts, float2 *mls, int lane) {
        const int G = p.group, g = lane >> 2, c = lane & 3;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const float unit = __uint_as_float((uint32_t)ve[hh] << 23) * (1.f / 1024.f);
            const int r = hh * 8 + g;  // in the item
            const int row = rt * R + r, t = att_div(p, row);
            const float sum = quad_sum(l[hh]);
            const bool live = limit[hh] != kNoRow;
            const float y = whole ? (sum == 0.f ? 0.f : unit / sum) : unit;
            const int64_t to = ((int64_t)(b * (int64_t)p.T + t) * p.H + h * G + (row - t * G)) * D;
            float *const part = parts + r * D;
            if (live) {
                if (!whole && c == 0) mls[r] = make_float2(m[hh], sum);
                constexpr int N = D == 64 ? 8 : 16;
#pragma unroll
                for (int k = 0; k < 2 * kCols / N; ++k) {  // runs of N columns
                    const int col = (k >> 1) * 128 + 2 * N * c + N * (k & 1);
                    float x[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] = o[(k >> 1) * 16 + i][2 * hh + (k & 1)] * y;
                    if (whole)
                        store_out<BF, N>(p.o, to + col, x);
                    else
                        store_out<false, N>(part, col, x);
                }
            }
        }
    }
};

struct AttPage {  // a page of the sequence, 32 bytes
    int b, rt, h, page;    // page: in the row's table
    int begin, count;      // of its item, in the sequence
    int bad, unused;
};

template <int D, bool F32, bool TEST>
__global__ void __launch_bounds__(AttCfg<D, F32>::threads, 1) attend_kernel(const AttendArgs p) {
    using C = AttCfg<D, F32>;
    constexpr int R = C::R;
    extern __shared__ __align__(128) uint8_t sm[];
    int32_t *const before = reinterpret_cast<int32_t *>(sm + C::warps * C::warp_bytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.group;
    uint8_t *const mine = sm + warp * C::warp_bytes;
    uint8_t *const about = mine + C::ring + C::qbytes;  // [stages] AttPage, then the barriers
    const uint32_t ring = smem_u32(mine), qs = ring + C::ring, bars = smem_u32(about) + C::stages * 32;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the join waits for the end of this grid itself
    if (lane == 0) {
        for (int i = 0; i < C::stages; ++i) mbar_init(bars + 8 * i, 1);
        fence_mbar_init();
    }
    att_count(p, R, 1, before);
    const int warps = gridDim.x * C::warps;
    const AttWork work = att_work(p.workspace, warps, R);
    const int total = before[p.batch] * p.Hk, per = att_per(total, warps);
    const int range = blockIdx.x * C::warps + warp;
    const int end = min(total, (int)min((int64_t)total, ((int64_t)range + 1) * per));
    const int begin = (int)min((int64_t)end, (int64_t)range * per);

    // ---- the ring: lane l knows page base + l of the sequence ----
    int base = begin - 32;
    AttPage my{};
    int my_tile = 0;  // where the tile of rows of `my` begins in the sequence
    const uint8_t *my_record = nullptr;
    bool failed = false;
    auto fetch = [&](int f, int stage) {  // all lanes
        if (f - base >= 32) {
            base = f;
            const int x = f + lane;
            if (x < end) {
                int lo = 0, hi = p.batch;  // before[lo] Hk <= x < before[hi] Hk
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (before[mid] * p.Hk <= x) lo = mid;
                    else hi = mid;
                }
                const AttRow w = att_row(p, lo);
                int rt = 0, tile = before[lo] * p.Hk;
                if (my_record && lo == my.b) rt = my.rt, tile = my_tile;  // pages come in order
                AttItem it = att_item(p, w, rt, R);
                while (x - tile >= it.pages * p.Hk) {
                    tile += it.pages * p.Hk;
                    it = att_item(p, w, ++rt, R);
                }
                my_tile = tile;
                const int at = x - tile;
                my.b = lo;
                my.rt = rt;
                my.h = at / it.pages;
                const int i = at - my.h * it.pages;
                my.page = it.first + i;
                my.begin = x - i;
                my.count = it.pages;
                const int64_t slot = cache_page(p.pages[(int64_t)lo * p.table + my.page], p.num_pages);
                my.bad = slot < 0;
                my_record = p.pool + (slot * p.Hk + my.h) * C::rec;
            }
        }
        if (lane == f - base) {
            AttPage *const to = reinterpret_cast<AttPage *>(about) + stage;
            *to = my;
            const uint32_t bar = bars + 8 * stage;
            fence_proxy_async_smem();
            if (my.bad) {
                atomicOr(p.status, kDevBadSlot);
                mbar_arrive_expect_tx(bar, 0);
            } else {
                mbar_arrive_expect_tx(bar, C::rec + att_extra<TEST>(p, range, 1));
                bulk_g2s(ring + stage * C::rec, my_record, C::rec, bar);
            }
        }
    };
    __syncwarp();
    for (int i = 0; i < C::stages - 1; ++i)
        if (begin + i < end) fetch(begin + i, i);

    // ---- the item at hand ----
    int item = -1;  // its first page in the sequence
    AttPage now{};
    AttRows<D, F32> rows;

    // the item at hand: written if it lies in the range, else a part of it, in the workspace or (own: for the CTA to
    // join) in this warp's ring
    auto finish = [&](bool own) {
        const bool whole = now.begin >= begin && now.begin + now.count <= end;
        const int64_t slot = 2 * range + (now.begin >= begin ? 1 : 0);
        float *const parts = own ? reinterpret_cast<float *>(mine) : work.o + slot * R * D;
        rows.leave(p, now.b, now.rt, now.h, whole, parts, own ? reinterpret_cast<float2 *>(parts + R * D) : work.ml + slot * R, lane);
    };

    int stage = 0;
    uint32_t parity = 0;
    for (int f = begin; f < end && !failed; ++f) {
        {
            const int ahead = f + C::stages - 1;
            __syncwarp();  // the stage that is filled next has been read by all lanes
            if (ahead < end) fetch(ahead, stage == 0 ? C::stages - 1 : stage - 1);
        }
        if (!mbar_wait_bounded(bars + 8 * stage, parity, kAttWait<TEST>)) failed = true;
        if (__any_sync(kFull, failed)) {
            failed = true;
            for (int x = f + 1; x < min(end, f + C::stages); ++x) {  // the other copies in flight
                if (++stage == C::stages) stage = 0, parity ^= 1u;
                mbar_wait_bounded(bars + 8 * stage, parity, kAttWait<TEST>);
            }
            break;
        }
        const AttPage *const info = reinterpret_cast<const AttPage *>(about) + stage;
        if (info->begin != item) {
            if (item >= 0) finish(false);
            now = *info;
            item = now.begin;
            rows.start(p, att_row(p, now.b), now.b, now.rt, now.h, qs, lane);
        }
        if (!info->bad) rows.page(p, ring + stage * C::rec, info->page, qs, lane);
        if (++stage == C::stages) {
            stage = 0;
            parity ^= 1u;
        }
    }
    if (failed) {  // the join finds no part of an item that this range should have left, and makes NaN of it
        if (lane == 0) atomicOr(p.status, kDevWaitTimeout);
        work.ml[(int64_t)2 * range * R + lane] = make_float2(NAN, NAN);
        static_assert(2 * R == 32, "both parts");
    }
    // All warps of a CTA inside one item (a long context): their parts become one.
    __shared__ int tails[C::warps];
    const bool open = !failed && item >= 0 && !(now.begin >= begin && now.begin + now.count <= end);
    if (lane == 0) tails[warp] = open ? item : -1;
    __syncthreads();
    bool one = true;
#pragma unroll
    for (int i = 0; i < C::warps; ++i) one = one && tails[i] >= 0 && tails[i] == tails[0];
    if (!failed && item >= 0) finish(one);
    if (one) {
        static_assert(R * (D + 2) * 4 <= C::ring, "parts");
        __syncthreads();
        const int n = min(R, p.T * G - now.rt * R);  // rows (those of no query hold what they will)
        const int first = blockIdx.x * C::warps, slot = 2 * first + (item >= first * (int64_t)per ? 1 : 0);
        auto part = [&](int w) { return reinterpret_cast<const float *>(sm + w * C::warp_bytes); };
        for (int i = threadIdx.x; i < n * (D / 4); i += C::threads) {
            const int r = i / (D / 4), col = 4 * (i - r * (D / 4));
            float M = -INFINITY, f[C::warps];
#pragma unroll
            for (int w = 0; w < C::warps; ++w) M = fmaxf(M, reinterpret_cast<const float2 *>(part(w) + R * D)[r].x);
            const float mu = M == -INFINITY ? 0.f : M;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            float L = 0.f;
#pragma unroll
            for (int w = 0; w < C::warps; ++w) {
                const float2 ml = reinterpret_cast<const float2 *>(part(w) + R * D)[r];
                f[w] = ex2(ml.x - mu);
                L = fmaf(ml.y, f[w], L);
                const float4 z = *reinterpret_cast<const float4 *>(part(w) + r * D + col);
                y.x = fmaf(z.x, f[w], y.x), y.y = fmaf(z.y, f[w], y.y), y.z = fmaf(z.z, f[w], y.z), y.w = fmaf(z.w, f[w], y.w);
            }
            *reinterpret_cast<float4 *>(work.o + ((int64_t)slot * R + r) * D + col) = y;
            if (col == 0) {
                work.ml[(int64_t)slot * R + r] = make_float2(M, L);
                for (int w = 1; w < C::warps; ++w) work.ml[(int64_t)2 * (first + w) * R + r] = make_float2(-INFINITY, 0.f);  // nothing there
            }
        }
    }
    if (lane == 0) {
        const bool split = open && now.begin >= begin;
        work.split[range] = split ? AttSplit{now.b, now.rt, now.h, (now.begin + now.count - 1) / per, min(R, att_row(p, now.b).n * G - now.rt * R)} : AttSplit{0, 0, 0, -1};
    }
}

// A CTA per item, for contexts so short that its warps alone read them in the time that a second launch takes:
// warp w has every C::warps-th page from w on, and the CTA joins the warps' parts and writes all of the item's rows.
template <int D, bool F32, bool TEST>
__global__ void __launch_bounds__(AttCfg<D, F32>::threads, 1) attend_items_kernel(const AttendArgs p, int tiles, int items) {
    using C = AttCfg<D, F32>;
    constexpr int R = C::R;
    extern __shared__ __align__(128) uint8_t sm[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *const mine = sm + warp * C::warp_bytes;
    const uint32_t ring = smem_u32(mine), qs = ring + C::ring, bars = qs + C::qbytes;
    if (lane == 0) {
        for (int i = 0; i < C::stages; ++i) mbar_init(bars + 8 * i, 1);
        fence_mbar_init();
    }
    __syncwarp();
    uint32_t seq = 0;  // copies so far: stage seq % stages, its parity (seq / stages) % 2
    bool failed = false;
    for (int x = blockIdx.x; x < items; x += gridDim.x) {
        const int h = x % p.Hk, bt = x / p.Hk, rt = bt % tiles, b = bt / tiles;
        const AttRow w = att_row(p, b);
        const AttItem it = att_item(p, w, rt, R);
        const int n = failed || it.pages <= warp ? 0 : (it.pages - warp + C::warps - 1) / C::warps;  // pages of this warp, 32 at most
        int64_t slot = -1;  // lane = one of them
        if (lane < n) slot = cache_page(p.pages[(int64_t)b * p.table + it.first + warp + C::warps * lane], p.num_pages);
        const unsigned bad = __ballot_sync(kFull, lane < n && slot < 0);
        auto fetch = [&](int k) {
            if (lane == k) {
                const uint32_t s = (seq + k) % C::stages, bar = bars + 8 * s;
                fence_proxy_async_smem();
                if (slot < 0) {
                    atomicOr(p.status, kDevBadSlot);
                    mbar_arrive_expect_tx(bar, 0);
                } else {
                    mbar_arrive_expect_tx(bar, C::rec + att_extra<TEST>(p, blockIdx.x, 1));
                    bulk_g2s(ring + s * C::rec, p.pool + (slot * p.Hk + h) * C::rec, C::rec, bar);
                }
            }
        };
        for (int k = 0; k < min(n, C::stages); ++k) fetch(k);
        AttRows<D, F32> rows;
        if (n) rows.start(p, w, b, rt, h, qs, lane);
        for (int k = 0; k < n; ++k) {
            const uint32_t s = (seq + k) % C::stages;
            if (!mbar_wait_bounded(bars + 8 * s, ((seq + k) / C::stages) & 1, kAttWait<TEST>)) failed = true;
            if (__any_sync(kFull, failed)) {
                failed = true;
                for (int y = k + 1; y < min(n, k + C::stages); ++y)  // the other copies in flight
                    mbar_wait_bounded(bars + 8 * ((seq + y) % C::stages), ((seq + y) / C::stages) & 1, kAttWait<TEST>);
                break;
            }
            if (!((bad >> k) & 1)) rows.page(p, ring + s * C::rec, it.first + warp + C::warps * k, qs, lane);
            __syncwarp();
            if (k + C::stages < n) fetch(k + C::stages);
        }
        seq += n;
        static_assert(R * (D + 2) * 4 <= C::ring, "parts");
        if (n) rows.leave(p, b, rt, h, false, reinterpret_cast<float *>(mine), reinterpret_cast<float2 *>(mine + R * D * 4), lane);
        const bool lost = __syncthreads_or(failed);  // rows without all of their pages are not written
        const int parts = min(C::warps, it.pages);
        for (int i = threadIdx.x; i < R * (D / 4) && !lost; i += C::threads) {
            const int r = i / (D / 4), col = 4 * (i - r * (D / 4)), row = rt * R + r, t = att_div(p, row);
            if (t >= p.T) break;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (t < w.n) {
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int k = 0; k < C::warps; ++k)
                    if (k < parts) M = fmaxf(M, reinterpret_cast<const float2 *>(sm + k * C::warp_bytes + R * D * 4)[r].x);
                const float mu = M == -INFINITY ? 0.f : M;
#pragma unroll
                for (int k = 0; k < C::warps; ++k) {
                    if (k < parts) {
                        const float2 ml = reinterpret_cast<const float2 *>(sm + k * C::warp_bytes + R * D * 4)[r];
                        const float f = ex2(ml.x - mu);
                        L = fmaf(ml.y, f, L);
                        const float4 z = *reinterpret_cast<const float4 *>(sm + k * C::warp_bytes + (r * D + col) * 4);
                        y.x = fmaf(z.x, f, y.x), y.y = fmaf(z.y, f, y.y), y.z = fmaf(z.z, f, y.z), y.w = fmaf(z.w, f, y.w);
                    }
                }
                const float u = L == 0.f ? 0.f : 1.f / L;
                y.x *= u, y.y *= u, y.z *= u, y.w *= u;
            }
            const int64_t to = (((int64_t)b * p.T + t) * p.H + h * p.group + (row - t * p.group)) * D + col;
            if (F32) {
                *reinterpret_cast<float4 *>(static_cast<float *>(p.o) + to) = y;
            } else {
                uint2 z;
                const __nv_bfloat162 lo = __floats2bfloat162_rn(y.x, y.y), hi = __floats2bfloat162_rn(y.z, y.w);
                memcpy(&z.x, &lo, 4);
                memcpy(&z.y, &hi, 4);
                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.o) + to) = z;
            }
        }
        __syncthreads();  // the parts are read before the rings take copies again
    }
    if (failed && lane == 0) atomicOr(p.status, kDevWaitTimeout);
}

// Joins the parts of items that several ranges hold, blockIdx.x: the range that the item starts in; the blocks
// after those clear.  Items of many rows have few parts each: a thread per row and 4 columns.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attend_join_rows_kernel(const AttendArgs p, int R, int ranges, int slice) {
    if ((int)blockIdx.x >= ranges) {
        if (blockIdx.y == 0) att_clear<D, true>(p, blockIdx.x - ranges, slice);
        return;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const AttWork work = att_work(p.workspace, ranges, R);
    const int first = blockIdx.x;
    const AttSplit it = work.split[first];
    const int r = (blockIdx.y * kJoinThreads + threadIdx.x) / (D / 4), col = 4 * (threadIdx.x % (D / 4));
    if (it.last < 0 || r >= it.rows) return;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float M = -INFINITY, L = 0.f;
    constexpr int U = 4;
    for (int x0 = first; x0 <= it.last; x0 += U) {
        float2 ml[U];
        float4 y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t slot = (2 * (int64_t)min(x0 + u, it.last) + (x0 + u == first ? 1 : 0)) * R + r;
            ml[u] = work.ml[slot];
            y[u] = *reinterpret_cast<const float4 *>(work.o + slot * D + col);
            if (x0 + u > it.last) ml[u] = make_float2(-INFINITY, 0.f);
        }
        float Mn = M;
#pragma unroll
        for (int u = 0; u < U; ++u) Mn = fmaxf(Mn, ml[u].x);
        const float mu = Mn == -INFINITY ? 0.f : Mn, old = ex2(M - mu);
        M = Mn;
        L *= old;
        o.x *= old, o.y *= old, o.z *= old, o.w *= old;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = ex2(ml[u].x - mu);
            L = fmaf(ml[u].y, f, L);
            if (x0 + u <= it.last) o.x = fmaf(y[u].x, f, o.x), o.y = fmaf(y[u].y, f, o.y), o.z = fmaf(y[u].z, f, o.z), o.w = fmaf(y[u].w, f, o.w);
        }
    }
    const int G = p.group, row = it.rt * R + r, t = att_div(p, row);
    const float y = L == 0.f ? 0.f : 1.f / L;
    uint2 w;
    const __nv_bfloat162 a = __floats2bfloat162_rn(o.x * y, o.y * y), b = __floats2bfloat162_rn(o.z * y, o.w * y);
    memcpy(&w.x, &a, 4);
    memcpy(&w.y, &b, 4);
    *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.o) + (((int64_t)it.b * p.T + t) * p.H + it.h * G + (row - t * G)) * D + col) = w;
}

// Items of 16 rows may have many parts: `wpr` warps of a CTA per row.
template <int D, bool BF>
__global__ void __launch_bounds__(kJoinThreads) attend_join_kernel(const AttendArgs p, int ranges, int wpr, int slice) {
    constexpr int R = 16;
    constexpr int V = D / 32;  // columns of a lane
    __shared__ float part[kJoinThreads / 32][D + 2];
    const int G = p.group;
    if ((int)blockIdx.x >= ranges) {
        if (blockIdx.y == 0) att_clear<D, BF>(p, blockIdx.x - ranges, slice);
        return;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const AttWork work = att_work(p.workspace, ranges, R);
    const int first = blockIdx.x;
    const AttSplit it = work.split[first];
    if (it.last < 0) return;
    const int rows = it.rows;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int team = warp / wpr, mate = warp % wpr, teams = kJoinThreads / 32 / wpr;
    for (int r0 = blockIdx.y * teams; r0 < rows; r0 += gridDim.y * teams) {
        const int r = r0 + team;
        const int row = it.rt * R + r, t = att_div(p, row);
        const bool live = r < rows;
        if (!live && wpr == 1) continue;
        float o[V], M = -INFINITY, L = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = 0.f;
        if (live) {
            // 32 ranges at a time: lane = range reads its (m, l); then the parts that hold something, U at once
            constexpr int U = D == 256 ? 4 : 8;
            for (int x0 = first + 32 * mate; x0 <= it.last; x0 += 32 * wpr) {
                const int x = x0 + lane;
                auto at = [&](int y) { return (2 * (int64_t)y + (y == first ? 1 : 0)) * R + r; };
                const float2 ml = x <= it.last ? work.ml[at(x)] : make_float2(-INFINITY, 0.f);
                float Mn = ml.x;
#pragma unroll
                for (int i = 16; i; i >>= 1) Mn = fmaxf(Mn, __shfl_xor_sync(kFull, Mn, i));
                Mn = fmaxf(M, Mn);
                const float mu = Mn == -INFINITY ? 0.f : Mn, old = ex2(M - mu), f = ex2(ml.x - mu);
                M = Mn;
                float l = ml.y * f;
#pragma unroll
                for (int i = 16; i; i >>= 1) l += __shfl_xor_sync(kFull, l, i);
                L = fmaf(L, old, l);
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] *= old;
                unsigned some = __ballot_sync(kFull, x <= it.last && ml.x != -INFINITY);
                while (some) {
                    float g[U], y[U][V];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int src = __ffs(some) - 1;  // -1: none left
                        g[u] = __shfl_sync(kFull, f, max(src, 0));
                        if (src < 0) g[u] = 0.f;
#pragma unroll
                        for (int i = 0; i < V; i += 2) {
                            const float2 z = src < 0 ? make_float2(0.f, 0.f) : *reinterpret_cast<const float2 *>(work.o + at(x0 + src) * D + lane * V + i);
                            y[u][i] = z.x;
                            y[u][i + 1] = z.y;
                        }
                        some &= some - 1;
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < V; ++i) o[i] = fmaf(y[u][i], g[u], o[i]);
                }
            }
        }
        if (wpr > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) part[warp][lane * V + i] = o[i];
            if (lane == 0) part[warp][D] = M, part[warp][D + 1] = L;
            __syncthreads();
            if (live && mate == 0) {
                float Mn = -INFINITY;
                for (int x = 0; x < wpr; ++x) Mn = fmaxf(Mn, part[warp + x][D]);
                const float mu = Mn == -INFINITY ? 0.f : Mn;
                L = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = 0.f;
                for (int x = 0; x < wpr; ++x) {
                    const float f = ex2(part[warp + x][D] - mu);
                    L = fmaf(part[warp + x][D + 1], f, L);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] = fmaf(part[warp + x][lane * V + i], f, o[i]);
                }
            }
        }
        if (live && mate == 0) {
            const float y = L == 0.f ? 0.f : 1.f / L;
            const int64_t to = (((int64_t)it.b * p.T + t) * p.H + it.h * G + (row - t * G)) * D + lane * V;
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                if (BF)
                    *reinterpret_cast<__nv_bfloat162 *>(static_cast<__nv_bfloat16 *>(p.o) + to + i) = __floats2bfloat162_rn(o[i] * y, o[i + 1] * y);
                else
                    *reinterpret_cast<float2 *>(static_cast<float *>(p.o) + to + i) = make_float2(o[i] * y, o[i + 1] * y);
            }
        }
    }
}

int64_t att_items(const AttendArgs &a, int R) { return (int64_t)a.batch * (((int64_t)a.T * (a.H / a.Hk) + R - 1) / R) * a.Hk; }

// The second launch of a call, enqueued while the first runs.
template <int D, bool BF>
cudaError_t launch_join(const AttendArgs &a, int R, int ranges, cudaStream_t s) {
    constexpr int kWarps = kJoinThreads / 32;
    const int64_t rows = std::min<int64_t>(R, (int64_t)a.T * (a.H / a.Hk));
    const int slice = att_clear_slice(a.H, D, BF ? 2 : 4);
    const int64_t clear = (int64_t)a.batch * ((a.T + slice - 1) / slice);
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if constexpr (BF)
        if (R > 16) {
            cfg.gridDim = dim3((unsigned)(ranges + clear), (unsigned)((rows * (D / 4) + kJoinThreads - 1) / kJoinThreads));
            return cudaLaunchKernelEx(&cfg, attend_join_rows_kernel<D>, a, R, ranges, slice);
        }
    // few items may have many parts: a CTA per row (a context of 131071 tokens, 8 items of 4 rows: 10.2 us against 12.3
    // with a CTA per item; 2048 items: 25 against 9.6)
    const int64_t items = att_items(a, R);
    int wpr = kWarps;
    if (items * rows > 4 * (int64_t)sm_count())
        while (wpr > 1 && wpr * rows > kWarps) wpr /= 2;
    cfg.gridDim = dim3((unsigned)(ranges + clear), (unsigned)((rows * wpr + kWarps - 1) / kWarps));
    return cudaLaunchKernelEx(&cfg, attend_join_kernel<D, BF>, a, ranges, wpr, slice);
}
// Whether an item is a CTA's: two items per SM at most, of 8 pages per warp at most.  On the GPU alone (8 KV heads,
// d = 128): 16 rows of 1000 tokens 10.9 us against 17.5 by ranges, of 2000 16.0 against 23.1; one row of 500 7.6 against
// 11.3, of 1000 10.2 against 11.8, of 2000 15.5 against 12.8, of 4000 25.5 against 12.9; 60 rows of 1000 (480 items) 42
// against 33.  2 KV heads, d = 256 (4 warps): 8 rows of 2000 28.7 against 21.1.  It saves the host a launch too.
constexpr int kItemWarpPages = 8;
bool att_by_items(const AttendArgs &a) {
    return a.table <= kItemWarpPages * (a.d == 256 ? 4 : 8) && att_items(a, 16) <= 2 * (int64_t)sm_count();
}

template <int D, bool F32, bool TEST>
cudaError_t launch_as(const AttendArgs &a, cudaStream_t s) {
    using C = AttCfg<D, F32>;
    static_assert(kItemWarpPages <= 32 && (C::warps == 4) == (D == 256), "a page per lane");
    if (att_by_items(a)) {
        const int smem = C::warps * C::warp_bytes;
        const cudaError_t e = ensure_smem_limit(reinterpret_cast<const void *>(attend_items_kernel<D, F32, TEST>), smem);
        if (e != cudaSuccess) return e;
        const int items = (int)att_items(a, C::R);
        attend_items_kernel<D, F32, TEST><<<std::min(items, sm_count()), C::threads, smem, s>>>(a, (int)(items / a.Hk / a.batch), items);
        return cudaGetLastError();
    }
    const int smem = C::warps * C::warp_bytes + (a.batch + 1) * 4;
    cudaError_t e = ensure_smem_limit(reinterpret_cast<const void *>(attend_kernel<D, F32, TEST>), smem);
    if (e != cudaSuccess) return e;
    const int grid = sm_count();
    attend_kernel<D, F32, TEST><<<grid, C::threads, smem, s>>>(a);
    e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_join<D, !F32>(a, C::R, grid * C::warps, s);
}
template <int D>
cudaError_t launch_d(const AttendArgs &a, cudaStream_t s) {
    if (attend_tc_takes(a)) {
        const cudaError_t e = launch_attend_tc(a, sm_count(), s);
        return e != cudaSuccess || attend_tc_whole(a) ? e : launch_join<D, true>(a, attend_tc_rows(a), sm_count(), s);
    }
    if (a.test) {
        if constexpr (D == 128) return a.in_bf16 ? launch_as<D, false, true>(a, s) : cudaErrorNotSupported;
        return cudaErrorNotSupported;
    }
    return a.in_bf16 ? launch_as<D, false, false>(a, s) : launch_as<D, true, false>(a, s);
}

}  // namespace

int64_t attend_workspace(const AttendArgs &a) {
    const bool tc = attend_tc_takes(a);
    if (tc ? attend_tc_whole(a) : att_by_items(a)) return 0;
    return att_work_bytes(sm_count() * (tc ? 1 : a.d == 256 ? 4 : 8), tc ? attend_tc_rows(a) : 16, a.d);
}

cudaError_t launch_attend(AttendArgs a, cudaStream_t s) {
    static std::atomic<uint32_t *> cache[64];
    const cudaError_t e = symbol_address_cached(&g_status_attend, cache, &a.status);
    if (e != cudaSuccess) return e;
    a.group = a.H / a.Hk;
    a.by_group = fast_div_by(a.group);
    return a.d == 64 ? launch_d<64>(a, s) : a.d == 128 ? launch_d<128>(a, s) : launch_d<256>(a, s);
}

cudaError_t take_status_attend(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_attend, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_attend, &zero, sizeof(uint32_t));
}

}  // namespace damp
