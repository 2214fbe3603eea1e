// slots.cu -- whole slots of state pools: copy (save, fork, reorder), compact and free.
//
// A model keeps one pool per layer with the same slot numbers, so a call takes every
// layer's pool (blockIdx.y) and one list of slot numbers.
//
// Copy.  dst[i] receives what src[i] held before the call, for any overlap of the two
// lists (a reorder, a rotation): a CTA owns a slice of W bytes of every slot named, reads
// the slice of all sources into shared memory and only then writes the destinations, so
// no slice is read after it was written.  Slices of different CTAs are disjoint.
// Bound by the bytes moved.
#include "damp_common.cuh"
#include "damp_internal.h"

#include <algorithm>

namespace damp {

static __device__ uint32_t g_status_slots;

// the slot of an entry: -1 for an entry to skip (negative, or out of range: flagged)
__device__ __forceinline__ int64_t slot_of(int32_t i, int64_t num_slots, bool &bad) {
    if (i >= num_slots) bad = true;
    return i < 0 || i >= num_slots ? -1 : (int64_t)i;
}

__global__ void __launch_bounds__(kSlotThreads) copy_slots_kernel(const SlotArgs p) {
    extern __shared__ __align__(16) uint4 stage[];
    const SlotPool pool = p.pools[blockIdx.y];
    const int64_t off = (int64_t)blockIdx.x * p.slice;
    if (off >= pool.slot_bytes) return;
    const int units = (int)(min((int64_t)p.slice, pool.slot_bytes - off) / 16);
    bool bad = false;
    const int64_t total = (int64_t)p.n * units;
    for (int64_t i = threadIdx.x; i < total; i += kSlotThreads) {
        const int e = (int)(i / units), u = (int)(i % units);
        const int64_t s = slot_of(p.src[e], p.num_slots, bad), d = slot_of(p.dst[e], p.num_slots, bad);
        if (s < 0 || d < 0 || s == d) continue;
        stage[i] = *reinterpret_cast<const uint4 *>(pool.base + s * pool.slot_bytes + off + 16 * u);
    }
    __syncthreads();
    for (int64_t i = threadIdx.x; i < total; i += kSlotThreads) {
        const int e = (int)(i / units), u = (int)(i % units);
        const int64_t s = slot_of(p.src[e], p.num_slots, bad), d = slot_of(p.dst[e], p.num_slots, bad);
        if (s < 0 || d < 0 || s == d) continue;
        *reinterpret_cast<uint4 *>(pool.base + d * pool.slot_bytes + off + 16 * u) = stage[i];
    }
    if (bad) atomicOr(p.status, (uint32_t)kDevBadSlot);
}

__global__ void __launch_bounds__(kSlotThreads) zero_slots_kernel(const SlotArgs p) {
    const SlotPool pool = p.pools[blockIdx.y];
    bool bad = false;
    const int64_t s = slot_of(p.dst[blockIdx.z], p.num_slots, bad);
    if (bad && threadIdx.x == 0) atomicOr(p.status, (uint32_t)kDevBadSlot);
    if (s < 0) return;
    const int64_t off = (int64_t)blockIdx.x * p.slice, end = min(off + (int64_t)p.slice, pool.slot_bytes);
    for (int64_t i = off + 16 * threadIdx.x; i < end; i += 16 * kSlotThreads)
        *reinterpret_cast<uint4 *>(pool.base + s * pool.slot_bytes + i) = make_uint4(0, 0, 0, 0);
}

// The new slot numbers of a compaction.  With n distinct live slots, the live slots below
// n stay and those at or above it move, in ascending order, into the free slots below n
// in ascending order: no slot is both a source and a destination.  One CTA; a bit per
// slot and the running count of set bits per word in shared memory.
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(const SlotArgs p, int32_t *out, int words) {
    extern __shared__ __align__(16) uint32_t sm[];
    uint32_t *const live = sm, *const before = sm + words;  // bits; set bits in the words before
    __shared__ uint32_t warp_sum[kPlanThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int w = tid; w < words; w += kPlanThreads) live[w] = 0;
    __syncthreads();
    bool bad = false;
    for (int i = tid; i < p.n; i += kPlanThreads) {
        const int64_t s = slot_of(p.src[i], p.num_slots, bad);
        if (s >= 0) atomicOr(&live[s >> 5], 1u << (s & 31));
    }
    if (bad) atomicOr(p.status, (uint32_t)kDevBadSlot);
    __syncthreads();
    uint32_t n = 0;  // live slots counted so far
    for (int w0 = 0; w0 < words; w0 += kPlanThreads) {
        const int w = w0 + tid;
        const uint32_t own = w < words ? __popc(live[w]) : 0;
        uint32_t x = own;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const uint32_t y = __shfl_up_sync(kFull, x, m);
            if (lane >= m) x += y;
        }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        uint32_t base = n, all = 0;
        for (int i = 0; i < kPlanThreads / 32; ++i) {
            if (i < warp) base += warp_sum[i];
            all += warp_sum[i];
        }
        if (w < words) before[w] = base + x - own;
        n += all;
        __syncthreads();
    }
    const uint32_t below = before[n >> 5 < (uint32_t)words ? n >> 5 : words - 1];
    // live slots below n
    const uint32_t kept = (n >> 5) < (uint32_t)words ? below + __popc(live[n >> 5] & ((1u << (n & 31)) - 1)) : n;
    for (int i = tid; i < p.n; i += kPlanThreads) {
        bool b2 = false;
        const int64_t s = slot_of(p.src[i], p.num_slots, b2);
        if (s < (int64_t)n) {
            out[i] = (int32_t)s;  // stays, or -1
            continue;
        }
        // rank among the movers, then the free slot of that rank: the last word with at most
        // `rank` free slots before it
        uint32_t rank = before[s >> 5] + __popc(live[s >> 5] & ((1u << (s & 31)) - 1)) - kept;
        int lo = 0, hi = words - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (32u * mid - before[mid] <= rank) lo = mid;
            else hi = mid - 1;
        }
        rank -= 32u * lo - before[lo];
        uint32_t free_bits = ~live[lo];
        for (uint32_t r = 0; r < rank; ++r) free_bits &= free_bits - 1;
        out[i] = 32 * lo + __ffs(free_bits) - 1;
    }
}

static cudaError_t slots_status_word(SlotArgs &p) {
    static std::atomic<uint32_t *> cache[64];
    return symbol_address_cached(&g_status_slots, cache, &p.status);
}

static int64_t largest_slot(const SlotArgs &p) {
    int64_t m = 0;
    for (int i = 0; i < p.n_pools; ++i) m = std::max(m, p.pools[i].slot_bytes);
    return m;
}

cudaError_t launch_copy_slots(SlotArgs p, cudaStream_t s) {
    cudaError_t e = slots_status_word(p);
    if (e != cudaSuccess) return e;
    // slices of all entries within 64 KB of shared memory (three CTAs per SM), 16 bytes at
    // least: kMaxSlotEntries of them take 192 KB
    int slice = 16;
    while (slice < 16384 && (int64_t)p.n * slice * 2 <= 65536) slice *= 2;
    p.slice = slice;
    const int smem = p.n * slice;
    if ((e = ensure_smem_limit(reinterpret_cast<const void *>(copy_slots_kernel), smem)) != cudaSuccess) return e;
    const int64_t slices = (largest_slot(p) + slice - 1) / slice;
    copy_slots_kernel<<<dim3((unsigned)slices, (unsigned)p.n_pools), kSlotThreads, smem, s>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_zero_slots(SlotArgs p, cudaStream_t s) {
    const cudaError_t e = slots_status_word(p);
    if (e != cudaSuccess) return e;
    p.slice = 65536;
    const int64_t slices = (largest_slot(p) + p.slice - 1) / p.slice;
    for (int z0 = 0; z0 < p.n; z0 += 65535) {
        SlotArgs q = p;
        q.dst = p.dst + z0;
        zero_slots_kernel<<<dim3((unsigned)slices, (unsigned)p.n_pools, (unsigned)std::min(65535, p.n - z0)), kSlotThreads, 0,
                            s>>>(q);
    }
    return cudaGetLastError();
}

cudaError_t launch_compact_plan(SlotArgs p, int32_t *out, cudaStream_t s) {
    cudaError_t e = slots_status_word(p);
    if (e != cudaSuccess) return e;
    const int words = (int)((p.num_slots + 31) / 32);
    const int smem = words * 8;
    if ((e = ensure_smem_limit(reinterpret_cast<const void *>(compact_plan_kernel), smem)) != cudaSuccess) return e;
    compact_plan_kernel<<<1, kPlanThreads, smem, s>>>(p, out, words);
    return cudaGetLastError();
}

cudaError_t take_status_slots(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_status_slots, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_status_slots, &zero, sizeof(uint32_t));
}

}  // namespace damp
