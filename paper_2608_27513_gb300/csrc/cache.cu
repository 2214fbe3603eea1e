// cache.cu -- writing and reading the 8-bit cache of softmax-attention layers.
//
// Append.  With s the scale of a (page, KV head, keys or values), r = 1/s, a value x is stored as
// code rne(x r) + 128, held to 1 .. 255; s = amax/127 over the values that the call writes into the
// page, or the scale that the page's earlier tokens have, if that is larger.  Where an open page's
// scale grows from s to s', its earlier codes become rne(c (s r')): off by another half step of s'.
// Every operation is one FP32 rounding, so that the codes are defined to the bit.  Scales below
// 2^-126 are 0 (the block then holds zeros).  A NaN is stored as 0; an infinity takes no part in
// the maximum and is held to 127 s; both set a status bit.
//
// An item is one (row, page, head, keys or values): 128 threads, or a warp where a page receives 8
// tokens at most.  A thread keeps the values of its chunks of 16 in registers between the maximum
// and the codes, so each value is read once; codes are stored 16 bytes at a time.
//
// Measured: 8 rows of 1000 to 2000 tokens, 8 KV heads, d = 128, BF16, are written in 13.4 to 14.6 us (72 % of the issue
// slots, 14 instructions a value with all that an item costs; the floor of the bytes is 11) and read back in 14; 256 rows
// of one token each, written (earlier codes requantised where a scale grows) and their open pages read back, in 9.9;
// one token of one row 4.2, two launches.  64 threads an item take 17.1 us for those prompts and 23.9 for 16 heads,
// d = 64 (128: 16.1), a warp 15.2 and 13.2 to 14.5 (but d = 256 10.1 where 128 threads take 7.2, and d = 64 in FP32
// 22 where they take 20; calls of 9 to 64 tokens 0.1 to 0.4 us longer).  Below 9 tokens 128 threads would find no work.
//
// Read.  A thread turns whole 16 bytes of values, several on their way at once.  Bound by the bytes.
#include "cache.cuh"

#include <algorithm>
#include <cfloat>

namespace damp {

static __device__ uint32_t g_status_cache;

namespace {

constexpr int kAppThreads = 128;
constexpr int kReadThreads = 256;

// 16 values of a row
template <bool BF>
struct Sixteen {
    uint4 w[BF ? 2 : 4];
    __device__ __forceinline__ void load(const void *p, int64_t at) {
        const uint4 *g = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p) + at * (BF ? 2 : 4));
#pragma unroll
        for (int i = 0; i < (BF ? 2 : 4); ++i) w[i] = g[i];
    }
    __device__ __forceinline__ float2 pair(int i) const {  // values 2 i and 2 i + 1
        const uint32_t *u = reinterpret_cast<const uint32_t *>(w);
        if (BF) return make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
        return make_float2(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
    }
};

__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a <= FLT_MAX ? a : 0.f;
}
// rne(x) + 128 in the low byte, |x| <= 127
__device__ __forceinline__ uint32_t code_of(float x) { return __float_as_uint(__fadd_rn(x, 12582912.f + 128.f)); }
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
    return prmt(prmt(code_of(a), code_of(b), 0x0040u), prmt(code_of(c), code_of(d), 0x0040u), 0x5410u);
}
__device__ __forceinline__ float scaled(float x, float r) {  // held to the codes' range; NaN: 0
    const float y = __fmul_rn(x, r);
    return y == y ? fminf(fmaxf(y, -127.f), 127.f) : 0.f;
}

// TPI threads per item (32: warps on their own, 128: the CTA)
template <int D, int TPI, bool BF>
__global__ void __launch_bounds__(kAppThreads) cache_append_kernel(const CacheArgs p, int touched) {
    constexpr int kChunks = D / 16;
    constexpr int kUnits = TPI == 32 ? 8 * kChunks / 32 : kCachePage * kChunks / kAppThreads;  // of a thread
    static_assert(kUnits >= 1, "units");
    __shared__ float part[4];
    const int lane = threadIdx.x & 31;
    const int tid = TPI == 32 ? lane : threadIdx.x;
    // of row blockIdx.y, from the fastest: keys and values, heads, pages
    const int item = TPI == 32 ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    const int which = item & 1, b = blockIdx.y;
    const int ahead = fast_div(item >> 1, p.Hk, p.by_heads), h = (item >> 1) - ahead * p.Hk;
    if (ahead >= touched) return;  // (a whole warp; with 128 threads an item, never)
    const int start = p.start[b];
    const int fresh = p.lengths ? max(0, min(p.lengths[b], p.T)) : p.T;
    const int first_page = max(start, 0) / kCachePage;
    const int64_t page = first_page + ahead;  // of the row
    const int64_t lo = max((int64_t)start, page * kCachePage), hi = min((int64_t)start + fresh, (page + 1) * kCachePage);
    if (start < 0 || lo >= hi) {
        if (start < 0 && fresh > 0 && tid == 0) atomicOr(p.status, kDevBadSlot);
        return;
    }
    const int t0 = (int)(lo - page * kCachePage);  // in the page
    const int n = (int)(hi - lo) * kChunks;
    const void *const x = which ? p.v : p.k;
    const int64_t stride = which ? p.v_stride : p.k_stride;
    const int64_t from = ((int64_t)b * p.T + (lo - start)) * stride + (int64_t)h * D;

    Sixteen<BF> val[kUnits];  // on their way while the page is looked up
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int u = tid + i * TPI;
        if (u < n) val[i].load(x, from + (u / kChunks) * stride + (u % kChunks) * 16);
    }
    const int64_t slot = page < p.table ? cache_page(p.pages[(int64_t)b * p.table + page], p.num_pages) : -1;
    if (slot < 0) {
        if (tid == 0) atomicOr(p.status, kDevBadSlot);
        return;
    }
    uint8_t *const record = p.pool + (slot * p.Hk + h) * cache_record_bytes(D);
    uint8_t *const rows = record + which * cache_rows_bytes(D);
    float *const scale_at = reinterpret_cast<float *>(record + 2 * cache_rows_bytes(D)) + which;
    const float before = t0 ? *scale_at : 0.f;
    // magnitudes as integers, which order them and show what is not finite
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        if (tid + i * TPI < n) {
            const uint32_t *const w = reinterpret_cast<const uint32_t *>(val[i].w);
#pragma unroll
            for (int e = 0; e < (BF ? 8 : 16); ++e) most = BF ? __vmaxu2(most, w[e] & 0x7fff7fffu) : max(most, w[e] & 0x7fffffffu);
        }
    }
    if (BF) most = max(most & 0xffff0000u, most << 16);
    float top = __uint_as_float(most);
    const bool bad = most >= 0x7f800000u;
    if (bad) {
        atomicOr(p.status, kDevNotFinite);
        top = 0.f;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if (tid + i * TPI < n) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 y = val[i].pair(e);
                    top = fmaxf(top, fmaxf(finite_abs(y.x), finite_abs(y.y)));
                }
            }
        }
    }
    top = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(top)));  // not negative: ordered as integers
    if (TPI == 128) {
        if (lane == 0) part[threadIdx.x >> 5] = top;
        __syncthreads();
        top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    }
    float s = __fdiv_rn(top, 127.f);
    if (s < FLT_MIN) s = 0.f;
    s = fmaxf(s, before);  // before is read by all threads above, written below, after the barrier or in step
    const float r = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
    if (TPI == 32) __syncwarp();
    if (tid == 0 && (s != before || t0 == 0)) *scale_at = s;
    if (t0 && s != before) {  // the earlier tokens of an open page
        const float f = __fmul_rn(before, r);
        for (int u = tid; u < t0 * kChunks; u += TPI) {
            uint4 *const at = reinterpret_cast<uint4 *>(rows + 16 * u);  // each chunk where it lies
            uint4 c = *at;
            uint32_t *const w = reinterpret_cast<uint32_t *>(&c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = __fmul_rn((float)((int)((w[i] >> (8 * e)) & 255u) - 128), f);
                w[i] = code4(y[0], y[1], y[2], y[3]);
            }
            *at = c;
        }
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int u = tid + i * TPI;
        if (u < n) {
            uint32_t w[4];
            if (bad) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 y = val[i].pair(2 * e), z = val[i].pair(2 * e + 1);
                    w[e] = code4(scaled(y.x, r), scaled(y.y, r), scaled(z.x, r), scaled(z.y, r));
                }
            } else {  // |x| <= 127 s, s and r rounded once each: x r rounds to 127 at most where all is finite
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 y = val[i].pair(2 * e), z = val[i].pair(2 * e + 1);
                    w[e] = code4(__fmul_rn(y.x, r), __fmul_rn(y.y, r), __fmul_rn(z.x, r), __fmul_rn(z.y, r));
                }
            }
            *reinterpret_cast<uint4 *>(rows + cache_chunk(t0 + u / kChunks, u % kChunks, D)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// A thread turns N keys and N values, 16 bytes each once they are turned (so that a warp's stores are whole
// lines), of kReadPairs (token, head) pairs, all on their way at once.  Indices are divided in 32 bits by a
// multiplication: with 64-bit divisions the instructions, not the bytes, took the time.
constexpr int kReadPairs = 4;
template <int D, bool BF>
__global__ void __launch_bounds__(kReadThreads) cache_read_kernel(const CacheArgs p) {
    constexpr int N = BF ? 8 : 4, kParts = D / N, kStep = kReadThreads / kParts;  // threads of a pair; pairs at a time
    uint32_t code[kReadPairs][2][N / 4];
    float2 scale[kReadPairs];
    const int b = blockIdx.y, m = threadIdx.x % kParts, pairs = p.T * p.Hk;
    const int pair0 = blockIdx.x * (kReadPairs * kStep) + threadIdx.x / kParts;
    const int64_t first = p.start ? (int64_t)p.start[b] : 0;
    const int held = cache_clamp(p.lengths[b], p.table);
#pragma unroll
    for (int i = 0; i < kReadPairs; ++i) {
        const int pair = pair0 + i * kStep;
        scale[i] = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < N / 4; ++k) code[i][0][k] = code[i][1][k] = 0x80808080u;  // zeros
        if (pair < pairs) {
            const int t = fast_div(pair, p.Hk, p.by_heads), h = pair - t * p.Hk;
            const int64_t token = first + t;
            if (token >= 0 && token < held) {
                const int64_t slot = cache_page(p.pages[(int64_t)b * p.table + (int)token / kCachePage], p.num_pages);
                if (slot < 0) {
                    if (m == 0) atomicOr(p.status, kDevBadSlot);
                } else {
                    const uint8_t *const record = p.pool + (slot * p.Hk + h) * cache_record_bytes(D);
                    const uint8_t *const at = record + cache_chunk((int)(token % kCachePage), m * N / 16, D) + m * N % 16;
#pragma unroll
                    for (int which = 0; which < 2; ++which) {
                        const uint8_t *const from = at + which * cache_rows_bytes(D);
                        if constexpr (N == 8) {
                            const uint2 w = __ldg(reinterpret_cast<const uint2 *>(from));
                            code[i][which][0] = w.x, code[i][which][N / 4 - 1] = w.y;
                        } else {
                            code[i][which][0] = __ldg(reinterpret_cast<const uint32_t *>(from));
                        }
                    }
                    scale[i] = __ldg(reinterpret_cast<const float2 *>(record + 2 * cache_rows_bytes(D)));
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kReadPairs; ++i) {
        const int pair = pair0 + i * kStep;
        if (pair >= pairs) continue;
        const int64_t unit = ((int64_t)b * pairs + pair) * kParts + m;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const float s = which ? scale[i].y : scale[i].x;
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = (u8_biased(code[i][which][e / 4], e % 4) - (8388608.f + 128.f)) * s;
            uint32_t y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (BF) {
                    const __nv_bfloat162 z = __floats2bfloat162_rn(x[2 * e % N], x[(2 * e + 1) % N]);
                    memcpy(&y[e], &z, 4);
                } else {
                    y[e] = __float_as_uint(x[e]);
                }
            }
            stg128(static_cast<uint4 *>(which ? p.v : p.k) + unit, make_uint4(y[0], y[1], y[2], y[3]));
        }
    }
}

template <int D, bool BF>
void append_as(const CacheArgs &a, cudaStream_t s) {
    const int touched = (a.T + kCachePage - 2) / kCachePage + 1;  // pages that T tokens may lie in
    const unsigned items = 2u * a.Hk * touched;
    if (a.T <= 8)
        cache_append_kernel<D, 32, BF><<<dim3((items + 3) / 4, a.batch), kAppThreads, 0, s>>>(a, touched);
    else
        cache_append_kernel<D, 128, BF><<<dim3(items, a.batch), kAppThreads, 0, s>>>(a, touched);
}
template <int D, bool BF>
void read_as(const CacheArgs &a, cudaStream_t s) {
    const int per = kReadPairs * kReadThreads / (D / (BF ? 8 : 4)), pairs = a.T * a.Hk;
    cache_read_kernel<D, BF><<<dim3((unsigned)((pairs - 1) / per + 1), a.batch), kReadThreads, 0, s>>>(a);
}
#define DAMP_BY_D(f, a, s)                                                                      \
    do {                                                                                        \
        if (a.d == 64)                                                                          \
            a.in_bf16 ? f<64, true>(a, s) : f<64, false>(a, s);                                 \
        else if (a.d == 128)                                                                    \
            a.in_bf16 ? f<128, true>(a, s) : f<128, false>(a, s);                               \
        else                                                                                    \
            a.in_bf16 ? f<256, true>(a, s) : f<256, false>(a, s);                               \
    } while (0)

cudaError_t status_word(uint32_t **out) {
    static std::atomic<uint32_t *> cache[64];
    return symbol_address_cached(&g_status_cache, cache, out);
}

}  // namespace

cudaError_t launch_cache_append(CacheArgs a, cudaStream_t s) {
    const cudaError_t e = status_word(&a.status);
    if (e != cudaSuccess) return e;
    a.by_heads = fast_div_by(a.Hk);
    DAMP_BY_D(append_as, a, s);
    return cudaGetLastError();
}

cudaError_t launch_cache_read(CacheArgs a, cudaStream_t s) {
    const cudaError_t e = status_word(&a.status);
    if (e != cudaSuccess) return e;
    a.by_heads = fast_div_by(a.Hk);
    DAMP_BY_D(read_as, a, s);
    return cudaGetLastError();
}

cudaError_t take_status_cache(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_cache, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_cache, &zero, sizeof(uint32_t));
}

}  // namespace damp
