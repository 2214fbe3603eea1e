// rotary.cu -- rotary positions of queries and keys.
//
// Pair i of a head turns by position * f_i: (a, b) -> m (a cos - b sin, b cos + a sin).  The pair is
// (x_i, x_{i + r/2}) or, interleaved, (x_2i, x_2i+1) of the first r values of a head; the others are
// copied.  cos and sin are the same for all heads, so a CTA computes them once for its tokens and
// its threads then walk over the heads of q and k with 16-byte loads and stores.
//
// Angles.  position * f in 32 bits loses 2^-24 of the whole angle, 0.06 radians at position 2^20.
// Here f / 2 pi becomes a fixed-point fraction of a turn in 64 bits, by integers from the double's own bits and 128 bits
// of 1 / 2 pi (in doubles the product is off by up to 2^-56 of a turn, 2^-25 at position 2^31), and its product
// with the position modulo 2^64 keeps the fraction exactly: 2^-64 of a turn per position, whatever
// the position.  What is left of it after quarter turns, half a quarter at most, goes to sincospif: rounding it
// to FP32 costs 2^-24 of that rest (of a whole turn's range it cost up to 2^-25 half turns).
//
// Bound by the bytes (each value read and written once): 4 rows of 2048 tokens, 32 and 8 heads, d = 128, BF16, take
// 29 us, 5.8 TB/s; a single token 1.9 us, a launch.
#include "damp_common.cuh"
#include "damp_internal.h"

#include <algorithm>

namespace damp {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotPairs = 512;   // cosines and sines of a CTA

// The fraction of a turn per position, f / 2 pi, in units of 2^-64.  f = m 2^(e - 1086) with a mantissa m of 64 bits,
// 1 / 2 pi = c 2^-130 with c of 128 bits, of whose product the upper 128 bits are taken.
__device__ __forceinline__ uint64_t turns_of(double f) {
    constexpr uint64_t c_hi = 0xa2f9836e4e441529ull, c_lo = 0xfc2757d1f534ddc0ull;
    const uint64_t bits = (uint64_t)__double_as_longlong(f);
    const int e = (int)(bits >> 52) & 0x7ff;
    const uint64_t m = (bits << 11) | (1ull << 63);
    const uint64_t low = __umul64hi(m, c_lo), mid = m * c_hi;
    const uint64_t lo = mid + low, hi = __umul64hi(m, c_hi) + (lo < low ? 1 : 0);  // f / 2 pi = (hi, lo) 2^(e - 1152)
    const int right = 1088 - e;  // places to units of 2^-64; 65 for f = 1
    uint64_t t = 0;
    if (e == 0x7ff || right >= 129) t = 0;  // not finite; below 2^-65 turns
    else if (right > 64) t = ((hi >> (right - 65)) + 1) >> 1;  // to the nearest
    else if (right == 64) t = hi;
    else if (right > 0) t = (hi << (64 - right)) | (lo >> right);
    else if (right > -64) t = lo << -right;  // (frequencies from 2^65 on: the bits of 1 / 2 pi run out)
    return bits >> 63 ? 0 - t : t;
}
// cosine and sine of an angle in units of 2^-64 turns
__device__ __forceinline__ void sincos_of(uint64_t turn, float &s, float &c) {
    const uint32_t quarter = (uint32_t)((turn + (1ull << 61)) >> 62);  // (4 is 0)
    const int32_t rest = (int32_t)((int64_t)(turn - ((uint64_t)quarter << 62)) >> 30);  // of 2^-34 turns, an eighth at most
    float a, b;
    sincospif((float)rest * 1.1641532182693481e-10f, &a, &b);  // half turns: 2^-33
    s = quarter & 1 ? b : a;
    c = quarter & 1 ? a : b;
    if (quarter & 2) s = -s;
    if ((quarter + 1) & 2) c = -c;
}

template <int V>
struct alignas(V * 4 < 16 ? V * 4 : 16) F32 {
    float x[V];
};
template <int V>
struct alignas(V * 2) B16 {
    __nv_bfloat16 x[V];
};

// V values: a vector load or store of 16 bytes where V says so, single values for V = 1
template <int V, bool BF>
__device__ __forceinline__ void rot_load(const void *p, int64_t at, float (&x)[V]) {
    if (BF) {
        const B16<V> w = *reinterpret_cast<const B16<V> *>(static_cast<const __nv_bfloat16 *>(p) + at);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = __bfloat162float(w.x[i]);
    } else {
        const F32<V> w = *reinterpret_cast<const F32<V> *>(static_cast<const float *>(p) + at);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = w.x[i];
    }
}
template <int V, bool BF>
__device__ __forceinline__ void rot_store(void *p, int64_t at, const float (&x)[V]) {
    if (BF) {
        B16<V> w;
#pragma unroll
        for (int i = 0; i < V; ++i) w.x[i] = __float2bfloat16_rn(x[i]);
        *reinterpret_cast<B16<V> *>(static_cast<__nv_bfloat16 *>(p) + at) = w;
    } else {
        F32<V> w;
#pragma unroll
        for (int i = 0; i < V; ++i) w.x[i] = x[i];
        *reinterpret_cast<F32<V> *>(static_cast<float *>(p) + at) = w;
    }
}

// A unit of work: V pairs of a head (half layout: two vectors; interleaved: 2 V neighbouring values)
// or 2 V values to copy.  V = 1 takes any r, d, stride and alignment.
template <int V, bool BF, bool INTER>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const RotaryArgs p, int tb) {
    __shared__ __align__(16) float cs[kRotPairs], sn[kRotPairs];
    const int half = p.r / 2;
    const int64_t t0 = (int64_t)blockIdx.x * tb;
    const int n = (int)min((int64_t)tb, p.tokens - t0);
    for (int i = threadIdx.x; i < n * half; i += kRotThreads) {
        const int t = i / half, j = i - t * half;
        const int64_t token = t0 + t;
        const int64_t row = p.per_row ? token / p.T : token;
        const int64_t pos = (int64_t)p.positions[row] + (p.per_row ? token - row * p.T : 0);
        float s, c;
        sincos_of(turns_of(p.freq[j]) * (uint64_t)pos, s, c);
        cs[i] = p.scale * c;
        sn[i] = p.scale * s;
    }
    __syncthreads();
    const int turned = half / V, units = p.units, heads = p.heads[0] + p.heads[1];
    const int all = n * heads * units;
    for (int i = threadIdx.x; i < all; i += kRotThreads) {
        const int th = fast_div(i, units, p.by_units), u = i - th * units;
        const int t = fast_div(th, heads, p.by_heads);
        int h = th - t * heads;
        const bool second = h >= p.heads[0];
        const void *x = second ? p.x[1] : p.x[0];
        void *out = second ? p.out[1] : p.out[0];
        const int nh = second ? p.heads[1] : p.heads[0];
        if (second) h -= p.heads[0];
        const int64_t from = (t0 + t) * (second ? p.stride[1] : p.stride[0]) + (int64_t)h * p.d;
        const int64_t to = ((t0 + t) * nh + h) * p.d;
        float a[V], b[V];
        if (u < turned) {
            const int j = u * V;
            if (INTER) {
                if constexpr (V == 1) {
                    rot_load<1, BF>(x, from + 2 * j, a);
                    rot_load<1, BF>(x, from + 2 * j + 1, b);
                } else {
                    float w[V], z[V];
                    rot_load<V, BF>(x, from + 2 * j, w);
                    rot_load<V, BF>(x, from + 2 * j + V, z);
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) {
                        a[e] = w[2 * e];
                        b[e] = w[2 * e + 1];
                        a[V / 2 + e] = z[2 * e];
                        b[V / 2 + e] = z[2 * e + 1];
                    }
                }
            } else {
                rot_load<V, BF>(x, from + j, a);
                rot_load<V, BF>(x, from + half + j, b);
            }
            float y[V], z[V], cv[V], sv[V];
            rot_load<V, false>(cs, t * half + j, cv);
            rot_load<V, false>(sn, t * half + j, sv);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                y[e] = a[e] * cv[e] - b[e] * sv[e];
                z[e] = b[e] * cv[e] + a[e] * sv[e];
            }
            if (INTER) {
                if constexpr (V == 1) {
                    rot_store<1, BF>(out, to + 2 * j, y);
                    rot_store<1, BF>(out, to + 2 * j + 1, z);
                } else {
                    float w[V];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
#pragma unroll
                        for (int e = 0; e < V / 2; ++e) {
                            w[2 * e] = y[k * (V / 2) + e];
                            w[2 * e + 1] = z[k * (V / 2) + e];
                        }
                        rot_store<V, BF>(out, to + 2 * j + k * V, w);
                    }
                }
            } else {
                rot_store<V, BF>(out, to + j, y);
                rot_store<V, BF>(out, to + half + j, z);
            }
        } else {
            const int j = p.r + (u - turned) * 2 * V;
            rot_load<V, BF>(x, from + j, a);
            const bool more = j + V < p.d;  // the rest of a head may be an odd number of vectors
            if (more) rot_load<V, BF>(x, from + j + V, b);
            rot_store<V, BF>(out, to + j, a);
            if (more) rot_store<V, BF>(out, to + j + V, b);
        }
    }
}

template <int V, bool BF>
void launch_layout(const RotaryArgs &a, unsigned grid, int tb, cudaStream_t s) {
    if (a.interleaved)
        rotary_kernel<V, BF, true><<<grid, kRotThreads, 0, s>>>(a, tb);
    else
        rotary_kernel<V, BF, false><<<grid, kRotThreads, 0, s>>>(a, tb);
}

}  // namespace

cudaError_t launch_rotary(RotaryArgs a, cudaStream_t s) {
    // Vectors of 16 bytes where both halves of a pair, the rest of a head and every row start on one.
    const int V = a.in_bf16 ? 8 : 4;
    bool wide = (a.r / 2) % V == 0 && a.d % V == 0;
    for (int i = 0; i < 2; ++i)
        if (a.heads[i])
            wide = wide && reinterpret_cast<uintptr_t>(a.x[i]) % 16 == 0 && reinterpret_cast<uintptr_t>(a.out[i]) % 16 == 0 &&
                   a.stride[i] % V == 0;
    const int unit = wide ? V : 1;
    a.units = a.r / 2 / unit + (a.d - a.r + 2 * unit - 1) / (2 * unit);
    a.by_units = fast_div_by(a.units);
    a.by_heads = fast_div_by(a.heads[0] + a.heads[1]);
    // Tokens of a CTA: one while there are few (the time is latency), then enough to fill its threads
    // with cosines.
    const int most = std::max(1, std::min(kRotPairs, kRotThreads) / (a.r / 2));
    const int64_t fill = a.tokens / (4 * (int64_t)sm_count());
    const int tb = (int)std::max<int64_t>(1, std::min<int64_t>(most, fill));
    const unsigned grid = (unsigned)((a.tokens + tb - 1) / tb);
    if (a.in_bf16)
        wide ? launch_layout<8, true>(a, grid, tb, s) : launch_layout<1, true>(a, grid, tb, s);
    else
        wide ? launch_layout<4, false>(a, grid, tb, s) : launch_layout<1, false>(a, grid, tb, s);
    return cudaGetLastError();
}

}  // namespace damp
