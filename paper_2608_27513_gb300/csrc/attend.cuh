// attend.cuh -- what the kernels of attention over the 8-bit cache share: the items and their pages, the
// sequence of all items' pages, the workspace of parts.
//
// The rows of an item are R (query token, query head) pairs that share a (batch row, KV head); its keys
// are the pages from the first that its first query sees to the last that its last query sees.
// The items' pages, `unit` at a time, form one sequence, in the order of batch rows, tiles of R rows and
// KV heads, which is cut into equal ranges.
#pragma once

#include "cache.cuh"

#include <cfloat>
#include <climits>

namespace damp {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kNoRow = INT_MIN / 2;  // below every token, with a window too (2^30 at most)

// the pages of an item in its row's table
struct AttItem {
    int first, pages;
};
// the rows' tokens: held tokens, queries
struct AttRow {
    int len, n;
};
__device__ __forceinline__ AttRow att_row(const AttendArgs &p, int b) {
    AttRow r;
    r.len = cache_clamp(p.lengths[b], p.table);
    r.n = p.q_lengths ? max(0, min(p.q_lengths[b], p.T)) : p.T;
    return r;
}
__device__ __forceinline__ int att_div(const AttendArgs &p, int x) { return fast_div(x, p.group, p.by_group); }
__device__ __forceinline__ AttItem att_item(const AttendArgs &p, AttRow w, int rt, int R) {
    const int t0 = att_div(p, rt * R), t1 = min(w.n - 1, att_div(p, rt * R + R - 1));
    const int hi = w.len - w.n + t1;  // the last token that its last query sees
    if (t0 > t1 || hi < 0) return AttItem{0, 0};
    const int lo = p.window ? max(0, w.len - w.n + t0 - (p.window - 1)) : 0;
    return AttItem{lo / kCachePage, hi / kCachePage - lo / kCachePage + 1};
}
__device__ __forceinline__ int att_tiles(int n, int R, int G) { return (n * G + R - 1) / R; }
__device__ __forceinline__ int att_units(int pages, int unit) { return (pages + unit - 1) / unit; }

// limit of a wait; in the variant that tests the waits
template <bool TEST>
constexpr uint64_t kAttWait = TEST ? 10000000ull : 2000000000ull;
// bytes that a barrier of range (or CTA) i expects beyond what is copied: none but in that variant
template <bool TEST>
__device__ __forceinline__ uint32_t att_extra(const AttendArgs &p, int i, int test) {
    return TEST && p.test == test && (i & 1) ? 16u : 0u;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// bytes 0 and 2 (or as `sel` says) of w as FP16 codes minus 128: 0x64 above a byte is 1024 + byte
__device__ __forceinline__ uint32_t half_codes(uint32_t w, uint32_t sel) {
    const uint32_t h = prmt(w, 0x64646464u, sel);
    const __half2 y = __hadd2(*reinterpret_cast<const __half2 *>(&h), __half2(__ushort_as_half(0xE480), __ushort_as_half(0xE480)));  // -1152
    return *reinterpret_cast<const uint32_t *>(&y);
}
// a in the low half
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// N (8 or 16) consecutive outputs
template <bool BF, int N>
__device__ __forceinline__ void store_out(void *o, int64_t at, const float (&x)[N]) {
    if (BF) {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const __nv_bfloat162 z = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            memcpy(&w[i], &z, 4);
        }
#pragma unroll
        for (int i = 0; i < N / 8; ++i)
            stg128(static_cast<__nv_bfloat16 *>(o) + at + 8 * i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
    } else {
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            *reinterpret_cast<float4 *>(static_cast<float *>(o) + at + 4 * i) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
}

// Workspace: for each range the item that starts in it and does not end in it, the parts' (m, l) [range][2][R]
// and o [range][2][R][D].  A range leaves part 1 of an item that starts in it, else part 0.
struct AttSplit {
    int b, rt, h;
    int last;  // the range that it ends in; -1: there is no such item
    int rows;  // of queries
    int unused[3];
};
struct AttWork {
    AttSplit *split;
    float2 *ml;
    float *o;
};
__host__ __device__ inline int64_t att_work_bytes(int ranges, int R, int D) {
    return (int64_t)ranges * (32 + 2 * (int64_t)R * (8 + 4 * D));
}
__host__ __device__ inline AttWork att_work(uint8_t *w, int ranges, int R) {
    AttWork a;
    a.split = reinterpret_cast<AttSplit *>(w);
    a.ml = reinterpret_cast<float2 *>(a.split + ranges);
    a.o = reinterpret_cast<float *>(a.ml + (int64_t)ranges * 2 * R);
    return a;
}
__device__ __forceinline__ int att_per(int total, int ranges) { return max(1, (total + ranges - 1) / ranges); }

// before[b]: the units of batch rows before b, for one KV head (all threads)
__device__ inline void att_count(const AttendArgs &p, int R, int unit, int32_t *before) {
    const int tiles = att_tiles(p.T, R, p.group);
    for (int b = threadIdx.x; b <= p.batch; b += blockDim.x) before[b] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < p.batch * tiles; i += blockDim.x) {
        const int b = i / tiles;
        const int n = att_units(att_item(p, att_row(p, b), i - b * tiles, R).pages, unit);
        if (tiles == 1) before[b + 1] = n;
        else if (n) atomicAdd(before + b + 1, n);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int sum = 0;
        for (int at = 0; at < p.batch; at += 32) {
            const int b = at + threadIdx.x;
            int n = b < p.batch ? before[b + 1] : 0;
#pragma unroll
            for (int i = 1; i < 32; i <<= 1) {
                const int y = __shfl_up_sync(kFull, n, i);
                if ((int)threadIdx.x >= i) n += y;
            }
            if (b < p.batch) before[b + 1] = sum + n;
            sum += __shfl_sync(kFull, n, 31);
        }
    }
    __syncthreads();
}

// Clears the outputs of queries that see no token or are none: block i, `slice` queries of a row.
template <int D, bool BF>
__device__ __forceinline__ void att_clear(const AttendArgs &p, int i, int slice) {
    const int slices = (p.T + slice - 1) / slice, b = i / slices;
    const AttRow w = att_row(p, b);
    const int t0 = (i - b * slices) * slice, t1 = min(p.T, t0 + slice);
    const int64_t token = (int64_t)p.H * D / (BF ? 8 : 4);  // 16 bytes at a time
    for (int side = 0; side < 2; ++side) {  // before the first token, after the last query
        const int lo = side ? max(t0, w.n) : t0, hi = side ? t1 : min(t1, w.n - w.len);
        uint4 *const o = static_cast<uint4 *>(p.o) + ((int64_t)b * p.T + lo) * token;
        for (int64_t k = threadIdx.x; k < (hi - lo) * token; k += blockDim.x) o[k] = make_uint4(0, 0, 0, 0);
    }
}
// queries of a block that clears: 256 KB of outputs
__host__ __device__ inline int att_clear_slice(int H, int D, int es) {
    const int n = (256 << 10) / (H * D * es);
    return n < 1 ? 1 : n;
}

// the products of prompts and drafts on the tensor cores (attend_tc.cu)
bool attend_tc_takes(const AttendArgs &a);
int attend_tc_rows(const AttendArgs &a);  // of an item
bool attend_tc_whole(const AttendArgs &a);  // no item is split, one launch
cudaError_t launch_attend_tc(AttendArgs a, int grid, cudaStream_t s);

}  // namespace damp
