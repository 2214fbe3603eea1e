// slots.cu -- whole slots of state pools: copy (save, fork, reorder), compact and free.
//
// A model keeps one pool per layer with the same slot numbers, so a call takes every
// layer's pool (blockIdx.y) and one list of slot numbers.
//
// Copy.  dst[i] receives what src[i] held before the call, for any overlap of the two
// lists (a reorder, a rotation): the bytes of a slot are cut into slices, and a CTA reads
// a slice of every source into shared memory before it writes one of the destinations.
// Slices are disjoint, so no byte is read after it was written.  Bulk copies (the TMA
// engine) move whole slices both ways; while a slice's destinations are written, the next
// slice's sources are read into the other buffer.  A source named in consecutive entries
// (a fork) is read once.  Bound by the bytes moved: of 10 layers of 627 KB slots, one slot
// forked to 64 in 67 us (6.1 TB/s), a pool of 256 slots compacted to 131 in 132 us (6.1 TB/s,
// the plan included).
//
// Free.  Plain 16-byte stores; 37 of those slots in 34 us (6.8 TB/s).
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

// shared memory -> global memory, 16-byte aligned, in the thread's bulk group
__device__ __forceinline__ void bulk_s2g(void *dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// this thread's bulk stores have read their shared memory / are done
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// Shared memory: [2 buffers][from n][to n][buffer row n][source n].  stage: bytes of a buffer;
// least: the slice below which CTAs would run out of work.
__global__ void __launch_bounds__(kSlotThreads) copy_slots_kernel(const SlotArgs p, int stage, int least) {
    extern __shared__ __align__(128) uint8_t copy_sm[];
    __shared__ __align__(8) uint64_t bars[2];
    __shared__ int counts[2];  // entries to copy, distinct sources
    const int tid = threadIdx.x, lane = tid & 31;
    int32_t *const from = reinterpret_cast<int32_t *>(copy_sm + 2 * stage), *const to = from + p.n, *const row = to + p.n,
                   *const source = row + p.n;
    const uint32_t bar = smem_u32(bars), buffer = smem_u32(copy_sm);
    if (tid == 0) {
        mbar_init(bar, 1);
        mbar_init(bar + 8, 1);
        fence_mbar_init();
    }
    bool bad = false;
    for (int i = tid; i < p.n; i += kSlotThreads) {
        const int64_t s = slot_of(p.src[i], p.num_slots, bad), d = slot_of(p.dst[i], p.num_slots, bad);
        from[i] = s < 0 || d < 0 || s == d ? -1 : (int32_t)s;
        to[i] = (int32_t)d;
    }
    if (bad && blockIdx.x == 0) atomicOr(p.status, (uint32_t)kDevBadSlot);
    __syncthreads();
    if (tid < 32) {  // the entries to copy, in order; a run of one source has one buffer row
        int m = 0, rows = 0, last = -1;
        for (int i0 = 0; i0 < p.n; i0 += 32) {
            const int s = i0 + lane < p.n ? from[i0 + lane] : -1, d = s >= 0 ? to[i0 + lane] : 0;
            const uint32_t live = __ballot_sync(kFull, s >= 0), before = live & ((1u << lane) - 1);
            const int prev = __shfl_sync(kFull, s, before ? 31 - __clz(before) : 0);
            const bool head = s >= 0 && s != (before ? prev : last);
            const uint32_t heads = __ballot_sync(kFull, head);
            const int r = rows + __popc(heads & ((2u << lane) - 1)) - 1;
            __syncwarp();
            if (s >= 0) {
                to[m + __popc(before)] = d;
                row[m + __popc(before)] = r;
            }
            if (head) source[r] = s;
            __syncwarp();
            if (live) last = __shfl_sync(kFull, s, 31 - __clz(live));
            m += __popc(live);
            rows += __popc(heads);
        }
        if (lane == 0) {
            counts[0] = m;
            counts[1] = rows;
        }
    }
    __syncthreads();
    const int m = counts[0], rows = counts[1];
    if (m == 0) return;
    const int slice = min(stage / rows, least) & ~15;
    // slices of the pools in order
    struct At {
        int pool;
        int64_t off;
        uint32_t bytes;
    };
    int pool = 0;
    int64_t first = 0;  // number of pool's first slice
    auto at = [&](int64_t k) -> At {  // k ascends; bytes 0: no slice left
        while (pool < p.n_pools) {
            const int64_t here = (p.pools[pool].slot_bytes + slice - 1) / slice;
            if (k < first + here) break;
            first += here;
            ++pool;
        }
        if (pool == p.n_pools) return At{pool, 0, 0};
        const int64_t off = (k - first) * slice;
        return At{pool, off, (uint32_t)min((int64_t)slice, p.pools[pool].slot_bytes - off)};
    };
    auto load = [&](const At &a, int b) {
        if (tid == 0) mbar_arrive_expect_tx(bar + 8 * b, a.bytes * (uint32_t)rows);
        const uint8_t *const base = p.pools[a.pool].base + a.off;
        for (int r = tid; r < rows; r += kSlotThreads)
            bulk_g2s(buffer + (uint32_t)(b * stage + r * slice), base + source[r] * p.pools[a.pool].slot_bytes, a.bytes, bar + 8 * b);
    };
    At now = at(blockIdx.x);
    if (now.bytes) load(now, 0);
    bool ok = true;
    for (int64_t k = blockIdx.x, i = 0; now.bytes; k += gridDim.x, ++i) {
        const int b = (int)(i & 1);
        const At next = at(k + gridDim.x);
        bulk_wait_read();  // the stores out of the other buffer
        __syncthreads();
        if (next.bytes) load(next, b ^ 1);
        ok = mbar_wait_bounded(bar + 8 * b, (uint32_t)(i >> 1) & 1u);
        if (!__syncthreads_and(ok)) {
            if (next.bytes) mbar_wait_bounded(bar + 8 * (b ^ 1), (uint32_t)((i + 1) >> 1) & 1u);
            mbar_wait_bounded(bar + 8 * b, (uint32_t)(i >> 1) & 1u);
            if (tid == 0) atomicOr(p.status, (uint32_t)kDevWaitTimeout);
            break;
        }
        uint8_t *const base = p.pools[now.pool].base + now.off;
        for (int e = tid; e < m; e += kSlotThreads)
            bulk_s2g(base + to[e] * p.pools[now.pool].slot_bytes, buffer + (uint32_t)(b * stage + row[e] * slice), now.bytes);
        bulk_commit();
        now = next;
    }
    bulk_wait();
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
    extern __shared__ __align__(16) uint32_t plan_sm[];
    uint32_t *const live = plan_sm, *const before = plan_sm + words;  // bits; set bits in the words before
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

cudaError_t launch_copy_slots(SlotArgs p, cudaStream_t s) {
    cudaError_t e = slots_status_word(p);
    if (e != cudaSuccess) return e;
    // One CTA per SM with two buffers of all its shared memory: the longest slices for the number of
    // sources (short bulk copies are slow), but four slices per CTA where there are few sources.
    const int64_t ctas = sm_count();
    int64_t bytes = 0;
    for (int i = 0; i < p.n_pools; ++i) bytes += p.pools[i].slot_bytes;
    const int lists = 16 * p.n;
    const int stage = ((max_smem_per_block() - 2048 - lists) / 2) & ~127;
    const int least = (int)std::min<int64_t>(std::max<int64_t>(bytes / (4 * ctas), 1024) & ~127, 1 << 20);
    const int smem = 2 * stage + lists;
    if ((e = ensure_smem_limit(reinterpret_cast<const void *>(copy_slots_kernel), smem)) != cudaSuccess) return e;
    const int shortest = std::max(std::min(stage / p.n, least) & ~15, 16);  // every entry with its own source
    const int64_t grid = std::min(ctas, bytes / shortest + p.n_pools);
    copy_slots_kernel<<<(unsigned)grid, kSlotThreads, smem, s>>>(p, stage, least);
    return cudaGetLastError();
}

static int64_t largest_slot(const SlotArgs &p) {
    int64_t m = 0;
    for (int i = 0; i < p.n_pools; ++i) m = std::max(m, p.pools[i].slot_bytes);
    return m;
}

cudaError_t launch_zero_slots(SlotArgs p, cudaStream_t s) {
    const cudaError_t e = slots_status_word(p);
    if (e != cudaSuccess) return e;
    p.slice = 65536;
    const int64_t slices = (largest_slot(p) + p.slice - 1) / p.slice;
    for (int64_t z0 = 0; z0 < p.n; z0 += 65535) {  // (the last step may pass 2^31)
        SlotArgs q = p;
        q.dst = p.dst + z0;
        zero_slots_kernel<<<dim3((unsigned)slices, (unsigned)p.n_pools, (unsigned)std::min<int64_t>(65535, p.n - z0)),
                            kSlotThreads, 0, s>>>(q);
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
