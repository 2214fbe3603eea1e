// damp_abi.cu -- the extern "C" entry points of libdamp (include/damp.h):
// host-side argument checks, then one launch on the caller's stream.
#include <atomic>
#include <climits>

#include "damp.h"
#include "damp_common.cuh"
#include "damp_internal.h"

namespace damp {

namespace {

constexpr int kMaxDevices = 64;
std::atomic<int> g_sm_count[kMaxDevices];
std::atomic<int> g_smem_optin[kMaxDevices];
std::atomic<int> g_smem_sm[kMaxDevices];

int device_attr(std::atomic<int> *cache, cudaDeviceAttr attr, int fallback) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return fallback;
    int v = cache[dev].load(std::memory_order_relaxed);
    if (v > 0) return v;
    if (cudaDeviceGetAttribute(&v, attr, dev) != cudaSuccess || v <= 0) return fallback;
    cache[dev].store(v, std::memory_order_relaxed);
    return v;
}

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct Range {
    uintptr_t lo, hi;  // [lo, hi)
};
Range range_of(const void *p, int64_t bytes) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Range{lo, lo + (uintptr_t)(bytes > 0 ? bytes : 0)};
}
bool overlap(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi && a.hi > a.lo && b.hi > b.lo; }

// value heads of the operand tensors (H_m)
int64_t model_heads_of(const damp_layout *L) { return L->model_heads > 0 ? L->model_heads : L->num_heads; }

damp_status check_layout(const damp_layout *L) {
    if (!L) return DAMP_ERR_NULL;
    if (L->num_heads < 1 || L->num_qk_heads < 1 || L->model_heads < 0) return DAMP_ERR_SHAPE;
    const int64_t Hm = model_heads_of(L);
    if (Hm < L->num_heads || Hm % L->num_qk_heads) return DAMP_ERR_SHAPE;
    if (!L->head_map && Hm != L->num_heads) return DAMP_ERR_SHAPE;
    if (L->head_map && !aligned(L->head_map, 4)) return DAMP_ERR_ALIGN;
    if (Hm > (1 << 20)) return DAMP_ERR_SHAPE;
    if (L->d_k != 32 && L->d_k != 64 && L->d_k != 128) return DAMP_ERR_SHAPE;
    if (L->d_v < 32 || L->d_v > 1024 || L->d_v % 32) return DAMP_ERR_SHAPE;
    if (L->k_hi < 0 || L->k_hi > L->d_k) return DAMP_ERR_SHAPE;
    if (L->lo_format < DAMP_LO_U8_AFFINE_G32_H32 || L->lo_format > DAMP_LO_FP8_E4M3_G32) return DAMP_ERR_FORMAT;
    return DAMP_OK;
}

int64_t slot_bytes_of(const damp_layout *L) {
    return (int64_t)L->num_heads * (L->d_v / 32) * rec_geom(L->d_k, L->k_hi, L->lo_format).bytes;
}

// Slots, batch rows and the pool's byte range; shared by every call on a pool.
damp_status check_pool(const void *state, int64_t num_slots, const int32_t *slot_idx, int32_t batch,
                       int64_t slot_bytes, Range *pool) {
    if (batch < 0 || num_slots < 0) return DAMP_ERR_SHAPE;
    if (!state) return DAMP_ERR_NULL;
    if (!aligned(state, 16)) return DAMP_ERR_ALIGN;
    if (slot_idx && !aligned(slot_idx, 4)) return DAMP_ERR_ALIGN;
    if (!slot_idx && num_slots < batch) return DAMP_ERR_SHAPE;
    if (num_slots < 1) return DAMP_ERR_SHAPE;
    if (slot_bytes > 0 && num_slots > INT64_MAX / slot_bytes) return DAMP_ERR_SHAPE;
    *pool = range_of(state, num_slots * slot_bytes);
    return DAMP_OK;
}

// The single-token kernels take the query head of head m as (m H_qk) / H_m in 32 bits.
bool heads_fit_step(const damp_layout *L) { return (model_heads_of(L) - 1) * L->num_qk_heads <= INT32_MAX; }

cudaError_t launch_step(const StepArgs &a, bool packed, cudaStream_t s, bool waittest = false) {
    if (waittest) return launch_packed_kda_waittest(a, s);
    if (!packed) return launch_fp32_step(a, s);
    if (a.fmt == DAMP_LO_S8_ABSMAX_ROW) {
        if (a.dv > 4 * 32) return launch_rowabs_step(a, s);  // the two-sweep step for d_v > 128
        // d_k = d_v = 128: the full-row quad step (four warps share each row's maximum)
        const cudaError_t eq = a.kda ? launch_quad_rowabs_kda(a, s) : launch_quad_rowabs_gdn(a, s);
        if (eq != cudaErrorNotSupported) return eq;
        StepArgs one = a;  // otherwise a one-token chunk: four warps share each row's maximum
        one.T = 1;
        one.lengths = nullptr;
        return a.kda ? launch_prefill_kda(one, s) : launch_prefill_gdn(one, s);
    }
    if (a.fmt == DAMP_LO_U4_AFFINE_G32_H32 || a.fmt == DAMP_LO_U4_AFFINE_G32)
        return a.kda ? launch_packed_kda_u4(a, s) : launch_packed_gdn_u4(a, s);
    if (a.fmt == DAMP_LO_FP8_E4M3_G32) return a.kda ? launch_packed_kda_f8(a, s) : launch_packed_gdn_f8(a, s);
    return a.kda ? launch_packed_kda(a, s) : launch_packed_gdn(a, s);
}

damp_status step(const damp_layout *L, void *state, int64_t num_slots, const int32_t *slot_idx, int32_t batch,
                 const uint8_t *perm, const void *q, const void *k, const void *v, const float *g,
                 const float *beta, float *o, int32_t in_dtype, void *stream, bool kda, bool packed,
                 bool uniform, bool waittest = false, StepArgs *prepared = nullptr) {
    damp_status st = check_layout(L);
    if (st != DAMP_OK && packed) return st;
    if (!packed) {  // the FP32 state ignores k_hi and lo_format and holds every model head
        if (!L) return DAMP_ERR_NULL;
        damp_layout l2 = *L;
        l2.k_hi = 0;
        l2.lo_format = 0;
        if ((st = check_layout(&l2)) != DAMP_OK) return st;
        if (L->head_map) return DAMP_ERR_SHAPE;
    }
    if (uniform && L->k_hi != 0) return DAMP_ERR_SHAPE;
    // (the row-absmax step goes to a kernel with 64-bit products)
    if (!heads_fit_step(L) && !(packed && L->lo_format == DAMP_LO_S8_ABSMAX_ROW)) return DAMP_ERR_SHAPE;
    if (in_dtype != DAMP_IN_BF16 && in_dtype != DAMP_IN_FP32) return DAMP_ERR_FORMAT;
    if (waittest && (L->d_k != 128 || L->d_v != 128 || L->k_hi != 10 || L->lo_format != DAMP_LO_U8_AFFINE_G32_H32 ||
                     in_dtype != DAMP_IN_BF16 || L->head_map))
        return DAMP_ERR_SHAPE;
    if (batch < 0) return DAMP_ERR_SHAPE;
    if (batch == 0) return DAMP_OK;
    const int64_t sb = packed ? slot_bytes_of(L) : (int64_t)L->num_heads * L->d_k * L->d_v * 4;
    Range pool;
    if ((st = check_pool(state, num_slots, slot_idx, batch, sb, &pool)) != DAMP_OK) return st;
    if ((packed && !perm) || !q || !k || !v || !g || !beta || !o) return DAMP_ERR_NULL;
    if ((packed && !aligned(perm, 16)) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) ||
        !aligned(g, kda ? 16 : 4) || !aligned(beta, 4) || !aligned(o, 4))
        return DAMP_ERR_ALIGN;
    const int64_t B = batch, H = L->num_heads, Hm = model_heads_of(L), Hq = L->num_qk_heads, dk = L->d_k,
                  dv = L->d_v;
    const int64_t esz = in_dtype == DAMP_IN_BF16 ? 2 : 4;
    const Range ro = range_of(o, B * Hm * dv * 4);
    const Range inputs[] = {range_of(q, B * Hq * dk * esz), range_of(k, B * Hq * dk * esz),
                            range_of(v, B * Hm * dv * esz), range_of(g, B * Hm * (kda ? dk : 1) * 4),
                            range_of(beta, B * Hm * 4), range_of(perm, packed ? H * dk : 0),
                            range_of(slot_idx, slot_idx ? B * 4 : 0), range_of(L->head_map, L->head_map ? H * 4 : 0)};
    if (overlap(ro, pool)) return DAMP_ERR_ALIAS;
    for (const Range &r : inputs)
        if (overlap(ro, r) || overlap(pool, r)) return DAMP_ERR_ALIAS;

    StepArgs a{};
    a.H = L->num_heads;
    a.Hqk = L->num_qk_heads;
    a.Hm = (int32_t)Hm;
    a.head_map = L->head_map;
    a.dk = L->d_k;
    a.dv = L->d_v;
    a.K = packed ? L->k_hi : 0;
    a.fmt = packed ? L->lo_format : 0;
    a.state = state;
    a.num_slots = num_slots;
    a.slot_idx = slot_idx;
    a.batch = batch;
    a.perm = perm;
    a.q = q;
    a.k = k;
    a.v = v;
    a.g = g;
    a.beta = beta;
    a.o = o;
    a.in_bf16 = in_dtype == DAMP_IN_BF16;
    a.kda = kda;
    if (prepared) {  // checked, not launched (the head-group step launches)
        *prepared = a;
        return DAMP_OK;
    }
    return launch_step(a, packed, static_cast<cudaStream_t>(stream), waittest) == cudaSuccess ? DAMP_OK
                                                                                           : DAMP_ERR_CUDA;
}

// The head groups of one layer (App. E): each group checked as a one-group step, the
// groups against each other (same operand shapes and format, pools disjoint from each
// other); two groups with a compile-time pair of K_hi run in one launch, other groups
// one launch each.
damp_status step_groups(const damp_layout *layouts, int32_t n_groups, void *const *states, const int64_t *num_slots,
                        const uint8_t *const *perms, const int32_t *slot_idx, int32_t batch, const void *q,
                        const void *k, const void *v, const float *g, const float *beta, float *o, int32_t in_dtype,
                        void *stream, bool kda) {
    constexpr int kMaxGroups = 8;
    if (!layouts || !states || !num_slots || !perms) return DAMP_ERR_NULL;
    if (n_groups < 1 || n_groups > kMaxGroups) return DAMP_ERR_SHAPE;
    if (batch < 0) return DAMP_ERR_SHAPE;
    StepArgs a[kMaxGroups];
    Range pools[kMaxGroups];
    for (int i = 0; i < n_groups; ++i) {
        const damp_layout &L = layouts[i];
        damp_status st = check_layout(&L);
        if (st != DAMP_OK) return st;
        if (!L.head_map) return DAMP_ERR_SHAPE;  // a group is a head subset
        const damp_layout &L0 = layouts[0];
        if (L.model_heads != L0.model_heads || L.num_qk_heads != L0.num_qk_heads || L.d_k != L0.d_k ||
            L.d_v != L0.d_v)
            return DAMP_ERR_SHAPE;
        if (L.lo_format != L0.lo_format) return DAMP_ERR_FORMAT;
        if (batch == 0) continue;
        st = step(&L, states[i], num_slots[i], slot_idx, batch, perms[i], q, k, v, g, beta, o, in_dtype, stream, kda,
                  true, false, false, &a[i]);
        if (st != DAMP_OK) return st;
        pools[i] = range_of(states[i], num_slots[i] * slot_bytes_of(&L));
        for (int j = 0; j < i; ++j)
            if (overlap(pools[i], pools[j])) return DAMP_ERR_ALIAS;
    }
    if (batch == 0) return DAMP_OK;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (n_groups == 2) {
        const cudaError_t e = kda ? launch_packed2_kda(a[0], a[1], s) : launch_packed2_gdn(a[0], a[1], s);
        if (e != cudaErrorNotSupported) return e == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
    }
    for (int i = 0; i < n_groups; ++i)
        if (launch_step(a[i], true, s) != cudaSuccess) return DAMP_ERR_CUDA;
    return DAMP_OK;
}

damp_status prefill(const damp_layout *L, void *state, int64_t num_slots, const int32_t *slot_idx, int32_t batch,
                    int32_t chunk_len, const int32_t *lengths, const uint8_t *perm, const void *q, const void *k,
                    const void *v, const float *g, const float *beta, float *o, int32_t in_dtype, void *stream,
                    bool kda) {
    damp_status st = check_layout(L);
    if (st != DAMP_OK) return st;
    if (L->lo_format == DAMP_LO_S8_ABSMAX_ROW && L->d_v > 128) return DAMP_ERR_SHAPE;
    if (in_dtype != DAMP_IN_BF16 && in_dtype != DAMP_IN_FP32) return DAMP_ERR_FORMAT;
    if (batch < 0 || chunk_len < 0) return DAMP_ERR_SHAPE;
    if (batch == 0 || chunk_len == 0) return DAMP_OK;
    Range pool;
    if ((st = check_pool(state, num_slots, slot_idx, batch, slot_bytes_of(L), &pool)) != DAMP_OK) return st;
    if (!perm || !q || !k || !v || !g || !beta || !o) return DAMP_ERR_NULL;
    if (!aligned(perm, 16) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(g, kda ? 16 : 4) ||
        !aligned(beta, 4) || !aligned(o, 4) || (lengths && !aligned(lengths, 4)))
        return DAMP_ERR_ALIGN;
    const int64_t B = batch, T = chunk_len, H = L->num_heads, Hm = model_heads_of(L), Hq = L->num_qk_heads,
                  dk = L->d_k, dv = L->d_v;
    const int64_t esz = in_dtype == DAMP_IN_BF16 ? 2 : 4;
    const Range ro = range_of(o, B * T * Hm * dv * 4);
    const Range inputs[] = {range_of(q, B * T * Hq * dk * esz), range_of(k, B * T * Hq * dk * esz),
                            range_of(v, B * T * Hm * dv * esz), range_of(g, B * T * Hm * (kda ? dk : 1) * 4),
                            range_of(beta, B * T * Hm * 4), range_of(perm, H * dk),
                            range_of(slot_idx, slot_idx ? B * 4 : 0), range_of(lengths, lengths ? B * 4 : 0),
                            range_of(L->head_map, L->head_map ? H * 4 : 0)};
    if (overlap(ro, pool)) return DAMP_ERR_ALIAS;
    for (const Range &r : inputs)
        if (overlap(ro, r) || overlap(pool, r)) return DAMP_ERR_ALIAS;

    StepArgs a{};
    a.H = L->num_heads;
    a.Hqk = L->num_qk_heads;
    a.Hm = (int32_t)Hm;
    a.head_map = L->head_map;
    a.dk = L->d_k;
    a.dv = L->d_v;
    a.K = L->k_hi;
    a.fmt = L->lo_format;
    a.state = state;
    a.num_slots = num_slots;
    a.slot_idx = slot_idx;
    a.batch = batch;
    a.perm = perm;
    a.q = q;
    a.k = k;
    a.v = v;
    a.g = g;
    a.beta = beta;
    a.o = o;
    a.in_bf16 = in_dtype == DAMP_IN_BF16;
    a.kda = kda;
    a.T = chunk_len;
    a.lengths = lengths;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return (kda ? launch_prefill_kda(a, s) : launch_prefill_gdn(a, s)) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

// Linear attention with a decay per head on an FP32 pool: T tokens per row (the step: 1).
damp_status lin(const damp_layout *L, float *state, int64_t num_slots, const int32_t *slot_idx, int32_t batch, int32_t T,
                const int32_t *lengths, const void *q, const void *k, const void *v, const float *g, int32_t g_per_head,
                float *o, int32_t in_dtype, void *workspace, int64_t workspace_bytes, void *stream, bool step) {
    if (!L) return DAMP_ERR_NULL;
    damp_layout l2 = *L;  // the FP32 state ignores k_hi and lo_format and holds every model head
    l2.k_hi = 0;
    l2.lo_format = 0;
    damp_status st = check_layout(&l2);
    if (st != DAMP_OK) return st;
    if (L->head_map) return DAMP_ERR_SHAPE;
    if (in_dtype != DAMP_IN_BF16 && in_dtype != DAMP_IN_FP32) return DAMP_ERR_FORMAT;
    if (batch < 0 || T < 0) return DAMP_ERR_SHAPE;
    if (batch == 0 || T == 0) return DAMP_OK;
    const int64_t B = batch, N = B * T, H = L->num_heads, Hq = L->num_qk_heads, dk = L->d_k, dv = L->d_v;
    if (B * H * (dv / 32) > INT32_MAX) return DAMP_ERR_SHAPE;  // CTAs of one launch
    Range pool;
    if ((st = check_pool(state, num_slots, slot_idx, batch, H * dk * dv * 4, &pool)) != DAMP_OK) return st;
    if (!q || !k || !v || !g || !o) return DAMP_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(g, 4) || !aligned(o, 4) ||
        (lengths && !aligned(lengths, 4)))
        return DAMP_ERR_ALIGN;
    const int64_t esz = in_dtype == DAMP_IN_BF16 ? 2 : 4;
    const Range ro = range_of(o, N * H * dv * 4);
    const Range inputs[] = {range_of(q, N * Hq * dk * esz), range_of(k, N * Hq * dk * esz),
                            range_of(v, N * H * dv * esz), range_of(g, (g_per_head ? H : N * H) * 4),
                            range_of(slot_idx, slot_idx ? B * 4 : 0), range_of(lengths, lengths ? B * 4 : 0)};
    if (overlap(ro, pool)) return DAMP_ERR_ALIAS;
    for (const Range &r : inputs)
        if (overlap(ro, r) || overlap(pool, r)) return DAMP_ERR_ALIAS;
    LinArgs a{};
    a.H = L->num_heads;
    a.Hqk = L->num_qk_heads;
    a.dk = L->d_k;
    a.dv = L->d_v;
    a.state = state;
    a.num_slots = num_slots;
    a.slot_idx = slot_idx;
    a.batch = batch;
    a.T = T;
    a.lengths = lengths;
    a.q = q;
    a.k = k;
    a.v = v;
    a.g = g;
    a.g_per_head = g_per_head != 0;
    a.o = o;
    a.in_bf16 = in_dtype == DAMP_IN_BF16;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (step) return launch_lin_step(a, s) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
    const bool tc = lin_tc_takes(a);
    const int64_t need = (int64_t)(tc ? lin_tc_workspace(a) : lin_chunk_workspace(a));
    if (need) {
        if (!workspace) return DAMP_ERR_NULL;
        if (workspace_bytes < need) return DAMP_ERR_SHAPE;
        if (!aligned(workspace, 16)) return DAMP_ERR_ALIGN;
        const Range rw = range_of(workspace, need);
        if (overlap(rw, ro) || overlap(rw, pool)) return DAMP_ERR_ALIAS;
        for (const Range &r : inputs)
            if (overlap(rw, r)) return DAMP_ERR_ALIAS;
    }
    return (tc ? launch_lin_tc(a, workspace, s) : launch_lin_chunk(a, workspace, s)) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

// Whole slots of several pools.  Entries src (live slots of a compaction) and dst; launches
// take kSlotPools pools each.
enum SlotOp { kCopySlots, kZeroSlots, kCompactSlots };

damp_status slots(void *const *pools, const int64_t *slot_bytes, int32_t n_pools, int64_t num_slots, const int32_t *src,
                  int32_t *dst, int32_t n, void *stream, SlotOp op) {
    constexpr int kMaxPools = 1024;
    if (n_pools < 0 || n_pools > kMaxPools || num_slots < 0 || n < 0) return DAMP_ERR_SHAPE;
    if (n == 0 || (n_pools == 0 && op != kCompactSlots)) return DAMP_OK;
    if (num_slots < 1 || num_slots > INT32_MAX) return DAMP_ERR_SHAPE;
    if (op != kZeroSlots && n > kMaxSlotEntries) return DAMP_ERR_SHAPE;
    if (op == kCompactSlots && num_slots > kMaxPlanSlots) return DAMP_ERR_SHAPE;
    if ((n_pools && (!pools || !slot_bytes)) || !dst || (op != kZeroSlots && !src)) return DAMP_ERR_NULL;
    if (!aligned(dst, 4) || (src && !aligned(src, 4))) return DAMP_ERR_ALIGN;
    const Range rd = range_of(dst, (int64_t)n * 4), rs = range_of(src, src ? (int64_t)n * 4 : 0);
    if (op == kCompactSlots && overlap(rd, rs)) return DAMP_ERR_ALIAS;
    for (int i = 0; i < n_pools; ++i) {
        if (!pools[i]) return DAMP_ERR_NULL;
        if (!aligned(pools[i], 16)) return DAMP_ERR_ALIGN;
        if (slot_bytes[i] < 16 || slot_bytes[i] % 16 || slot_bytes[i] / 16 > INT32_MAX ||
            slot_bytes[i] > INT64_MAX / num_slots)
            return DAMP_ERR_SHAPE;
        const Range r = range_of(pools[i], num_slots * slot_bytes[i]);
        if (overlap(r, rd) || overlap(r, rs)) return DAMP_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(r, range_of(pools[j], num_slots * slot_bytes[j]))) return DAMP_ERR_ALIAS;
    }
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    SlotArgs a{};
    a.n = n;
    a.num_slots = num_slots;
    a.src = src;
    a.dst = dst;
    if (op == kCompactSlots && launch_compact_plan(a, dst, s) != cudaSuccess) return DAMP_ERR_CUDA;
    for (int i0 = 0; i0 < n_pools; i0 += kSlotPools) {
        a.n_pools = n_pools - i0 < kSlotPools ? n_pools - i0 : kSlotPools;
        for (int i = 0; i < a.n_pools; ++i)
            a.pools[i] = SlotPool{static_cast<uint8_t *>(pools[i0 + i]), slot_bytes[i0 + i]};
        if ((op == kZeroSlots ? launch_zero_slots(a, s) : launch_copy_slots(a, s)) != cudaSuccess) return DAMP_ERR_CUDA;
    }
    return DAMP_OK;
}

enum ConvKind { kQ, kDQ, kPack, kUnpack };

damp_status convert(const damp_layout *L, void *state, int64_t num_slots, const int32_t *slot_idx, int32_t batch,
                    const uint8_t *perm, float *S, uint16_t *hi, uint8_t *codes, uint16_t *meta, void *stream,
                    ConvKind kind) {
    damp_status st = check_layout(L);
    if (st != DAMP_OK) return st;
    if (batch < 0) return DAMP_ERR_SHAPE;
    if (batch == 0) return DAMP_OK;
    Range pool;
    if ((st = check_pool(state, num_slots, slot_idx, batch, slot_bytes_of(L), &pool)) != DAMP_OK) return st;
    const int64_t B = batch, H = L->num_heads, Hm = model_heads_of(L), dk = L->d_k, dv = L->d_v, K = L->k_hi;
    if (kind == kQ || kind == kDQ) {
        if (!perm || !S) return DAMP_ERR_NULL;
        if (!aligned(perm, 16) || !aligned(S, 16)) return DAMP_ERR_ALIGN;
        const Range rs = range_of(S, B * Hm * dk * dv * 4);
        if (overlap(rs, pool) || overlap(rs, range_of(perm, H * dk)) ||
            overlap(rs, range_of(slot_idx, slot_idx ? B * 4 : 0)) || overlap(pool, range_of(perm, H * dk)))
            return DAMP_ERR_ALIAS;
    } else {
        const int64_t nh = B * H * K * dv * 2, nc = B * H * (dk - K) * dv * fmt_code_bits(L->lo_format) / 8;
        const int64_t nm = B * H * (dk - K) * (L->lo_format == DAMP_LO_S8_ABSMAX_ROW ? 1 : dv / 32) * 4;
        if ((nh && !hi) || (nc && !codes) || (nm && !meta)) return DAMP_ERR_NULL;
        if ((hi && !aligned(hi, 4)) || (codes && !aligned(codes, 4)) || (meta && !aligned(meta, 4)))
            return DAMP_ERR_ALIGN;
        const Range t[] = {range_of(hi, nh), range_of(codes, nc), range_of(meta, nm)};
        for (const Range &r : t) {
            if (overlap(r, pool) || overlap(r, range_of(slot_idx, slot_idx ? B * 4 : 0))) return DAMP_ERR_ALIAS;
        }
        if (overlap(t[0], t[1]) || overlap(t[0], t[2]) || overlap(t[1], t[2])) return DAMP_ERR_ALIAS;
    }
    ConvArgs a{};
    a.H = L->num_heads;
    a.Hm = (int32_t)Hm;
    a.head_map = kind == kQ || kind == kDQ ? L->head_map : nullptr;  // tiers are pool-indexed
    a.dk = L->d_k;
    a.dv = L->d_v;
    a.K = L->k_hi;
    a.fmt = L->lo_format;
    a.state = state;
    a.num_slots = num_slots;
    a.slot_idx = slot_idx;
    a.batch = batch;
    a.perm = perm;
    a.S = S;
    a.hi = hi;
    a.codes = codes;
    a.meta = meta;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.fmt == DAMP_LO_S8_ABSMAX_ROW)
        return launch_rowabs_convert(a, (int)kind, s) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
    cudaError_t e = kind == kQ ? launch_quantize(a, s)
                    : kind == kDQ ? launch_dequantize(a, s)
                    : kind == kPack ? launch_pack_tiers(a, s)
                                    : launch_unpack_tiers(a, s);
    return e == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

damp_status check_cache(const damp_cache_layout *L) {
    if (!L) return DAMP_ERR_NULL;
    if (L->num_kv_heads < 1 || L->num_heads < 1 || L->num_heads > 65536 || L->num_heads % L->num_kv_heads)
        return DAMP_ERR_SHAPE;
    return L->d == 64 || L->d == 128 || L->d == 256 ? DAMP_OK : DAMP_ERR_SHAPE;
}

// what the calls on a cache have in common; es: bytes of an element
damp_status cache_args(const damp_cache_layout *L, void *cache, int64_t num_pages, const int32_t *pages, int32_t table,
                       int32_t batch, int32_t T, int32_t dtype, CacheArgs *a, Range *pool, Range *lists, int64_t *es) {
    const damp_status st = check_cache(L);
    if (st != DAMP_OK) return st;
    if (dtype != DAMP_IN_BF16 && dtype != DAMP_IN_FP32) return DAMP_ERR_FORMAT;
    if (num_pages < 1 || num_pages > INT32_MAX || table < 1 || table > (1 << 25) || batch < 0 || batch > kCacheMaxBatch || T < 0)
        return DAMP_ERR_SHAPE;
    a->H = L->num_heads;
    a->Hk = L->num_kv_heads;
    a->d = L->d;
    a->pool = static_cast<uint8_t *>(cache);
    a->num_pages = num_pages;
    a->pages = pages;
    a->table = table;
    a->batch = batch;
    a->T = T;
    a->in_bf16 = dtype == DAMP_IN_BF16;
    *es = a->in_bf16 ? 2 : 4;
    *pool = range_of(cache, num_pages * a->Hk * (64 * L->d + 16));
    *lists = range_of(pages, (int64_t)batch * table * 4);
    return DAMP_OK;
}

}  // namespace

int sm_count() { return device_attr(g_sm_count, cudaDevAttrMultiProcessorCount, 1); }

namespace {
struct SmemEntry {
    std::atomic<const void *> kernel{nullptr};
    std::atomic<int> bytes{0};
};
constexpr int kSmemEntries = 256;
SmemEntry g_smem_set[kMaxDevices][kSmemEntries];
}  // namespace

cudaError_t ensure_smem_limit(const void *kernel, int bytes) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    SmemEntry *slot = nullptr;
    if (dev >= 0 && dev < kMaxDevices) {
        const size_t h = (reinterpret_cast<uintptr_t>(kernel) >> 4) % kSmemEntries;
        for (size_t i = 0; i < kSmemEntries; ++i) {
            SmemEntry &en = g_smem_set[dev][(h + i) % kSmemEntries];
            const void *k = en.kernel.load(std::memory_order_acquire);
            if (k == kernel) {
                if (en.bytes.load(std::memory_order_acquire) >= bytes) return cudaSuccess;
                slot = &en;
                break;
            }
            if (k == nullptr) {
                const void *expected = nullptr;
                if (en.kernel.compare_exchange_strong(expected, kernel) || expected == kernel) {
                    slot = &en;
                    break;
                }
            }
        }
    }
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && slot) {
        int cur = slot->bytes.load(std::memory_order_relaxed);
        while (cur < bytes && !slot->bytes.compare_exchange_weak(cur, bytes)) {
        }
    }
    return e;
}

cudaError_t symbol_address_cached(const void *symbol, std::atomic<uint32_t *> *cache, uint32_t **out) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < kMaxDevices) {
        uint32_t *known = cache[dev].load(std::memory_order_acquire);
        if (known) {
            *out = known;
            return cudaSuccess;
        }
    }
    e = cudaGetSymbolAddress(reinterpret_cast<void **>(out), symbol);
    if (e == cudaSuccess && dev >= 0 && dev < kMaxDevices) cache[dev].store(*out, std::memory_order_release);
    return e;
}
int max_smem_per_block() { return device_attr(g_smem_optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, 48 * 1024); }
int max_smem_per_sm() { return device_attr(g_smem_sm, cudaDevAttrMaxSharedMemoryPerMultiprocessor, 0); }

}  // namespace damp

using namespace damp;

extern "C" {

damp_status damp_validate_layout(const damp_layout *layout) { return check_layout(layout); }

size_t damp_record_bytes(const damp_layout *layout) {
    if (check_layout(layout) != DAMP_OK) return 0;
    return (size_t)rec_geom(layout->d_k, layout->k_hi, layout->lo_format).bytes;
}

size_t damp_slot_bytes(const damp_layout *layout) {
    if (check_layout(layout) != DAMP_OK) return 0;
    return (size_t)slot_bytes_of(layout);
}

double damp_bits_per_value(const damp_layout *L) {
    if (check_layout(L) != DAMP_OK) return -1.0;
    const double hi = 16.0 * L->k_hi * L->d_v;
    const double lo = L->lo_format == DAMP_LO_S8_ABSMAX_ROW
                          ? (8.0 * L->d_v + 32.0) * (double)(L->d_k - L->k_hi)  // int8 + one FP32 scale
                          : (fmt_code_bits(L->lo_format) + 32.0 / 32.0) * (double)(L->d_k - L->k_hi) *
                                L->d_v;  // codes + 32 bits of metadata per 32 values
    return (hi + lo) / ((double)L->d_k * L->d_v);
}

damp_status damp_gdn_decode_step(const damp_layout *layout, void *state, int64_t num_slots, const int32_t *slot_idx,
                                 int32_t batch, const uint8_t *perm, const void *q, const void *k, const void *v,
                                 const float *g, const float *beta, float *o, int32_t in_dtype, void *stream) {
    return step(layout, state, num_slots, slot_idx, batch, perm, q, k, v, g, beta, o, in_dtype, stream, false, true,
                false);
}

damp_status damp_kda_decode_step(const damp_layout *layout, void *state, int64_t num_slots, const int32_t *slot_idx,
                                 int32_t batch, const uint8_t *perm, const void *q, const void *k, const void *v,
                                 const float *g, const float *beta, float *o, int32_t in_dtype, void *stream) {
    return step(layout, state, num_slots, slot_idx, batch, perm, q, k, v, g, beta, o, in_dtype, stream, true, true,
                false);
}

damp_status damp_gdn_decode_step_groups(const damp_layout *layouts, int32_t n_groups, void *const *states,
                                        const int64_t *num_slots, const uint8_t *const *perms,
                                        const int32_t *slot_idx, int32_t batch, const void *q, const void *k,
                                        const void *v, const float *g, const float *beta, float *o,
                                        int32_t in_dtype, void *stream) {
    return step_groups(layouts, n_groups, states, num_slots, perms, slot_idx, batch, q, k, v, g, beta, o, in_dtype,
                       stream, false);
}

damp_status damp_kda_decode_step_groups(const damp_layout *layouts, int32_t n_groups, void *const *states,
                                        const int64_t *num_slots, const uint8_t *const *perms,
                                        const int32_t *slot_idx, int32_t batch, const void *q, const void *k,
                                        const void *v, const float *g, const float *beta, float *o,
                                        int32_t in_dtype, void *stream) {
    return step_groups(layouts, n_groups, states, num_slots, perms, slot_idx, batch, q, k, v, g, beta, o, in_dtype,
                       stream, true);
}

damp_status damp_test_kda_wait_timeout(const damp_layout *layout, void *state, int64_t num_slots,
                                       const int32_t *slot_idx, int32_t batch, const uint8_t *perm, const void *q,
                                       const void *k, const void *v, const float *g, const float *beta, float *o,
                                       int32_t in_dtype, void *stream) {
    return step(layout, state, num_slots, slot_idx, batch, perm, q, k, v, g, beta, o, in_dtype, stream, true, true,
                false, true);
}

damp_status damp_u8_gdn_decode_step(const damp_layout *layout, void *state, int64_t num_slots,
                                    const int32_t *slot_idx, int32_t batch, const uint8_t *perm, const void *q,
                                    const void *k, const void *v, const float *g, const float *beta, float *o,
                                    int32_t in_dtype, void *stream) {
    return step(layout, state, num_slots, slot_idx, batch, perm, q, k, v, g, beta, o, in_dtype, stream, false, true,
                true);
}

damp_status damp_u8_kda_decode_step(const damp_layout *layout, void *state, int64_t num_slots,
                                    const int32_t *slot_idx, int32_t batch, const uint8_t *perm, const void *q,
                                    const void *k, const void *v, const float *g, const float *beta, float *o,
                                    int32_t in_dtype, void *stream) {
    return step(layout, state, num_slots, slot_idx, batch, perm, q, k, v, g, beta, o, in_dtype, stream, true, true,
                true);
}

damp_status damp_fp32_gdn_decode_step(const damp_layout *layout, float *state, int64_t num_slots,
                                      const int32_t *slot_idx, int32_t batch, const void *q, const void *k,
                                      const void *v, const float *g, const float *beta, float *o, int32_t in_dtype,
                                      void *stream) {
    return step(layout, state, num_slots, slot_idx, batch, nullptr, q, k, v, g, beta, o, in_dtype, stream, false,
                false, false);
}

damp_status damp_fp32_kda_decode_step(const damp_layout *layout, float *state, int64_t num_slots,
                                      const int32_t *slot_idx, int32_t batch, const void *q, const void *k,
                                      const void *v, const float *g, const float *beta, float *o, int32_t in_dtype,
                                      void *stream) {
    return step(layout, state, num_slots, slot_idx, batch, nullptr, q, k, v, g, beta, o, in_dtype, stream, true,
                false, false);
}

damp_status damp_gdn_prefill_chunk(const damp_layout *layout, void *state, int64_t num_slots, const int32_t *slot_idx,
                                   int32_t batch, int32_t chunk_len, const int32_t *lengths, const uint8_t *perm,
                                   const void *q, const void *k, const void *v, const float *g, const float *beta,
                                   float *o, int32_t in_dtype, void *stream) {
    return prefill(layout, state, num_slots, slot_idx, batch, chunk_len, lengths, perm, q, k, v, g, beta, o, in_dtype,
                   stream, false);
}

damp_status damp_kda_prefill_chunk(const damp_layout *layout, void *state, int64_t num_slots, const int32_t *slot_idx,
                                   int32_t batch, int32_t chunk_len, const int32_t *lengths, const uint8_t *perm,
                                   const void *q, const void *k, const void *v, const float *g, const float *beta,
                                   float *o, int32_t in_dtype, void *stream) {
    return prefill(layout, state, num_slots, slot_idx, batch, chunk_len, lengths, perm, q, k, v, g, beta, o, in_dtype,
                   stream, true);
}

damp_status damp_lin_decode_step(const damp_layout *layout, float *state, int64_t num_slots, const int32_t *slot_idx,
                                 int32_t batch, const void *q, const void *k, const void *v, const float *g,
                                 int32_t g_per_head, float *o, int32_t in_dtype, void *stream) {
    return lin(layout, state, num_slots, slot_idx, batch, 1, nullptr, q, k, v, g, g_per_head, o, in_dtype, nullptr, 0,
               stream, true);
}

damp_status damp_lin_prefill_chunk(const damp_layout *layout, float *state, int64_t num_slots, const int32_t *slot_idx,
                                   int32_t batch, int32_t chunk_len, const int32_t *lengths, const void *q,
                                   const void *k, const void *v, const float *g, int32_t g_per_head, float *o,
                                   int32_t in_dtype, void *workspace, int64_t workspace_bytes, void *stream) {
    return lin(layout, state, num_slots, slot_idx, batch, chunk_len, lengths, q, k, v, g, g_per_head, o, in_dtype,
               workspace, workspace_bytes, stream, false);
}

int64_t damp_lin_prefill_workspace(const damp_layout *layout, int32_t batch, int32_t chunk_len, int32_t in_dtype) {
    if (!layout || batch <= 0 || chunk_len <= 0) return 0;
    damp_layout l2 = *layout;
    l2.k_hi = 0;
    l2.lo_format = 0;
    if (check_layout(&l2) != DAMP_OK) return 0;
    LinArgs a{};
    a.H = layout->num_heads;
    a.dk = layout->d_k;
    a.dv = layout->d_v;
    a.batch = batch;
    a.T = chunk_len;
    a.in_bf16 = in_dtype == DAMP_IN_BF16;
    return (int64_t)(lin_tc_takes(a) ? lin_tc_workspace(a) : lin_chunk_workspace(a));
}

damp_status damp_copy_slots(void *const *pools, const int64_t *slot_bytes, int32_t n_pools, int64_t num_slots,
                            const int32_t *src, const int32_t *dst, int32_t n, void *stream) {
    return slots(pools, slot_bytes, n_pools, num_slots, src, const_cast<int32_t *>(dst), n, stream, kCopySlots);
}

damp_status damp_zero_slots(void *const *pools, const int64_t *slot_bytes, int32_t n_pools, int64_t num_slots,
                            const int32_t *idx, int32_t n, void *stream) {
    return slots(pools, slot_bytes, n_pools, num_slots, nullptr, const_cast<int32_t *>(idx), n, stream, kZeroSlots);
}

damp_status damp_compact_slots(void *const *pools, const int64_t *slot_bytes, int32_t n_pools, int64_t num_slots,
                               const int32_t *slot_idx, int32_t n, int32_t *slot_idx_out, void *stream) {
    return slots(pools, slot_bytes, n_pools, num_slots, slot_idx, slot_idx_out, n, stream, kCompactSlots);
}

damp_status damp_verify_drafts(const void *target_logits, const void *draft_logits, int32_t logits_dtype,
                               int64_t row_stride, int32_t vocab, const int32_t *draft_tokens, const int32_t *draft_len,
                               int32_t n_draft, const float *u, const float *noise, const float *temperature,
                               int32_t batch, int32_t *tokens_out, int32_t *count_out, void *stream) {
    if (logits_dtype != DAMP_IN_BF16 && logits_dtype != DAMP_IN_FP32) return DAMP_ERR_FORMAT;
    if (batch < 0 || n_draft < 0 || vocab < 1 || vocab > (1 << 30) || row_stride < vocab) return DAMP_ERR_SHAPE;
    if (batch == 0) return DAMP_OK;
    const int64_t B = batch, D = n_draft, esz = logits_dtype == DAMP_IN_BF16 ? 2 : 4;
    if (row_stride > INT64_MAX / 8 / (B * (D + 1))) return DAMP_ERR_SHAPE;
    if (!target_logits || !noise || !tokens_out || !count_out || (D && (!draft_tokens || !u))) return DAMP_ERR_NULL;
    if (!aligned(target_logits, 16) || (draft_logits && !aligned(draft_logits, 16)) || !aligned(noise, 16) ||
        !aligned(draft_tokens, 4) || !aligned(draft_len, 4) || !aligned(u, 4) || !aligned(temperature, 4) ||
        !aligned(tokens_out, 4) || !aligned(count_out, 4))
        return DAMP_ERR_ALIGN;
    const Range rt = range_of(tokens_out, B * (D + 1) * 4), rc = range_of(count_out, B * 4);
    const Range inputs[] = {range_of(target_logits, ((B * (D + 1) - 1) * row_stride + vocab) * esz),
                            range_of(draft_logits, draft_logits && D ? ((B * D - 1) * row_stride + vocab) * esz : 0),
                            range_of(draft_tokens, draft_tokens ? B * D * 4 : 0),
                            range_of(draft_len, draft_len ? B * 4 : 0), range_of(u, u ? B * D * 4 : 0),
                            range_of(noise, B * vocab * 4), range_of(temperature, temperature ? B * 4 : 0)};
    if (overlap(rt, rc)) return DAMP_ERR_ALIAS;
    for (const Range &r : inputs)
        if (overlap(rt, r) || overlap(rc, r)) return DAMP_ERR_ALIAS;
    VerifyArgs a{};
    a.target = target_logits;
    a.draft = draft_logits;
    a.tokens = draft_tokens;
    a.draft_len = draft_len;
    a.u = u;
    a.noise = noise;
    a.temperature = temperature;
    a.batch = batch;
    a.n_draft = n_draft;
    a.vocab = vocab;
    a.bf16 = logits_dtype == DAMP_IN_BF16;
    a.row_stride = row_stride;
    a.tokens_out = tokens_out;
    a.count_out = count_out;
    return launch_verify(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

damp_status damp_rotary(const void *q, int64_t q_stride, int32_t heads, const void *k, int64_t k_stride,
                        int32_t kv_heads, int32_t d, int32_t dtype, const int32_t *positions, int32_t positions_per_row,
                        int32_t batch, int32_t T, const double *freq, int32_t rotary_dim, int32_t interleaved,
                        float scale, void *q_out, void *k_out, void *stream) {
    if (dtype != DAMP_IN_BF16 && dtype != DAMP_IN_FP32) return DAMP_ERR_FORMAT;
    if (d < 1 || d > 1024 || rotary_dim < 2 || rotary_dim > d || rotary_dim % 2 || heads < 1 || heads > 1024 ||
        kv_heads < 0 || kv_heads > 1024 || batch < 0 || T < 0)
        return DAMP_ERR_SHAPE;
    const int64_t n = (int64_t)batch * T, es = dtype == DAMP_IN_BF16 ? 2 : 4;
    if (n > INT32_MAX) return DAMP_ERR_SHAPE;
    if (n == 0) return DAMP_OK;
    RotaryArgs a{};
    a.x[0] = q, a.x[1] = k;
    a.out[0] = q_out, a.out[1] = k_out;
    a.stride[0] = q_stride, a.stride[1] = k_stride;
    a.heads[0] = heads, a.heads[1] = kv_heads;
    Range in[2] = {}, out[2] = {};
    if (!positions || !freq) return DAMP_ERR_NULL;
    for (int i = 0; i < 2; ++i) {
        if (a.heads[i] == 0) continue;
        const int64_t row = (int64_t)a.heads[i] * d;
        if (!a.x[i] || !a.out[i]) return DAMP_ERR_NULL;
        if (a.stride[i] < row || a.stride[i] > INT64_MAX / 16 / n) return DAMP_ERR_SHAPE;
        if (!aligned(a.x[i], es) || !aligned(a.out[i], es)) return DAMP_ERR_ALIGN;
        in[i] = range_of(a.x[i], ((n - 1) * a.stride[i] + row) * es);
        out[i] = range_of(a.out[i], n * row * es);
    }
    if (!aligned(positions, 4) || !aligned(freq, 8)) return DAMP_ERR_ALIGN;
    const Range rp = range_of(positions, (positions_per_row ? (int64_t)batch : n) * 4), rf = range_of(freq, (int64_t)rotary_dim * 4);
    if (overlap(out[0], out[1])) return DAMP_ERR_ALIAS;
    for (int i = 0; i < 2; ++i) {
        if (overlap(out[i], rp) || overlap(out[i], rf) || overlap(out[i], in[1 - i])) return DAMP_ERR_ALIAS;
        const bool in_place = a.out[i] == a.x[i] && a.stride[i] == (int64_t)a.heads[i] * d;
        if (!in_place && overlap(out[i], in[i])) return DAMP_ERR_ALIAS;
    }
    a.d = d;
    a.r = rotary_dim;
    a.positions = positions;
    a.per_row = positions_per_row != 0;
    a.T = T;
    a.tokens = n;
    a.freq = freq;
    a.scale = scale;
    a.interleaved = interleaved != 0;
    a.in_bf16 = dtype == DAMP_IN_BF16;
    return launch_rotary(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

int64_t damp_cache_page_bytes(const damp_cache_layout *layout) {
    return check_cache(layout) == DAMP_OK ? (int64_t)layout->num_kv_heads * (64 * layout->d + 16) : 0;
}

damp_status damp_cache_append(const damp_cache_layout *layout, void *cache, int64_t num_pages, const int32_t *pages,
                              int32_t table, int32_t batch, int32_t T, const int32_t *start, const int32_t *lengths,
                              const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t dtype,
                              void *stream) {
    CacheArgs a{};
    Range pool, lists;
    int64_t es = 0;
    damp_status st = cache_args(layout, cache, num_pages, pages, table, batch, T, dtype, &a, &pool, &lists, &es);
    if (st != DAMP_OK) return st;
    const int64_t n = (int64_t)batch * T, row = (int64_t)a.Hk * a.d;
    if (k_stride < row || v_stride < row || k_stride * es % 16 || v_stride * es % 16) return DAMP_ERR_SHAPE;
    if (n == 0) return DAMP_OK;
    if (k_stride > INT64_MAX / 16 / n || v_stride > INT64_MAX / 16 / n) return DAMP_ERR_SHAPE;
    if (T > (1 << 30) || 2 * row / a.d * batch > INT32_MAX / ((T + 30) / 32 + 1)) return DAMP_ERR_SHAPE;  // a table's tokens; CTAs
    if (!cache || !pages || !start || !k || !v) return DAMP_ERR_NULL;
    if (!aligned(cache, 16) || !aligned(pages, 4) || !aligned(start, 4) || !aligned(lengths, 4) || !aligned(k, 16) ||
        !aligned(v, 16))
        return DAMP_ERR_ALIGN;
    const Range inputs[] = {lists, range_of(start, (int64_t)batch * 4), range_of(lengths, lengths ? (int64_t)batch * 4 : 0),
                            range_of(k, ((n - 1) * k_stride + row) * es), range_of(v, ((n - 1) * v_stride + row) * es)};
    for (const Range &r : inputs)
        if (overlap(pool, r)) return DAMP_ERR_ALIAS;
    a.start = start;
    a.lengths = lengths;
    a.k = const_cast<void *>(k);
    a.v = const_cast<void *>(v);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    return launch_cache_append(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

damp_status damp_cache_read(const damp_cache_layout *layout, const void *cache, int64_t num_pages, const int32_t *pages,
                            int32_t table, int32_t batch, int32_t T, const int32_t *start, const int32_t *lengths,
                            void *k, void *v, int32_t dtype, void *stream) {
    CacheArgs a{};
    Range pool, lists;
    int64_t es = 0;
    damp_status st = cache_args(layout, const_cast<void *>(cache), num_pages, pages, table, batch, T, dtype, &a, &pool,
                                &lists, &es);
    if (st != DAMP_OK) return st;
    const int64_t n = (int64_t)batch * T, row = (int64_t)a.Hk * a.d;
    if (n == 0) return DAMP_OK;
    if (T > INT32_MAX / 2 / a.Hk) return DAMP_ERR_SHAPE;  // (token, head) pairs of a row
    if (!cache || !pages || !lengths || !k || !v) return DAMP_ERR_NULL;
    if (!aligned(cache, 16) || !aligned(pages, 4) || !aligned(start, 4) || !aligned(lengths, 4) || !aligned(k, 16) ||
        !aligned(v, 16))
        return DAMP_ERR_ALIGN;
    const Range rk = range_of(k, n * row * es), rv = range_of(v, n * row * es);
    const Range inputs[] = {pool, lists, range_of(start, start ? (int64_t)batch * 4 : 0), range_of(lengths, (int64_t)batch * 4)};
    if (overlap(rk, rv)) return DAMP_ERR_ALIAS;
    for (const Range &r : inputs)
        if (overlap(rk, r) || overlap(rv, r)) return DAMP_ERR_ALIAS;
    a.start = start;
    a.lengths = lengths;
    a.k = k;
    a.v = v;
    return launch_cache_read(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

int64_t damp_cache_attend_workspace(const damp_cache_layout *layout, int32_t batch, int32_t T, int32_t table,
                                    int32_t dtype) {
    if (check_cache(layout) != DAMP_OK || batch < 1 || batch > kCacheMaxBatch || T < 1 || table < 1) return 0;
    AttendArgs a{};
    a.H = layout->num_heads;
    a.Hk = layout->num_kv_heads;
    a.d = layout->d;
    a.batch = batch;
    a.T = T;
    a.table = table;
    a.in_bf16 = dtype == DAMP_IN_BF16;
    return attend_workspace(a);
}

static damp_status cache_attend(const damp_cache_layout *layout, const void *cache, int64_t num_pages,
                                const int32_t *pages, int32_t table, int32_t batch, int32_t T, const int32_t *lengths,
                                const int32_t *q_lengths, const void *q, int64_t q_stride, float scale, int32_t window,
                                void *o, int32_t dtype, void *workspace, int64_t workspace_bytes, void *stream,
                                int32_t test) {
    CacheArgs c{};
    Range pool, lists;
    int64_t es = 0;
    damp_status st = cache_args(layout, const_cast<void *>(cache), num_pages, pages, table, batch, T, dtype, &c, &pool,
                                &lists, &es);
    if (st != DAMP_OK) return st;
    const int64_t n = (int64_t)batch * T, row = (int64_t)c.H * c.d, G = c.H / c.Hk;
    if (window < 0 || !(scale > 0.f) || !(scale <= 3.4e38f) || q_stride < row || q_stride * es % 16) return DAMP_ERR_SHAPE;
    if (n == 0) return DAMP_OK;
    if (q_stride > INT64_MAX / 16 / n || T * G > (1 << 26)) return DAMP_ERR_SHAPE;
    // pages of all items of 16 rows: 32-bit indices in the kernels, with room for what is added to them
    if (((T * G + 15) / 16) * batch * c.Hk > (1 << 30) / table) return DAMP_ERR_SHAPE;
    AttendArgs a{};
    a.H = c.H;
    a.Hk = c.Hk;
    a.d = c.d;
    a.batch = batch;
    a.T = T;
    a.table = table;
    a.in_bf16 = c.in_bf16;
    const int64_t need = attend_workspace(a);
    if (workspace_bytes < need) return DAMP_ERR_SHAPE;
    if (!cache || !pages || !lengths || !q || !o || (need && !workspace)) return DAMP_ERR_NULL;
    if (!aligned(cache, 16) || !aligned(pages, 4) || !aligned(lengths, 4) || !aligned(q_lengths, 4) || !aligned(q, 16) ||
        !aligned(o, 16) || !aligned(workspace, 16))
        return DAMP_ERR_ALIGN;
    const Range ro = range_of(o, n * row * es), rw = range_of(workspace, workspace ? workspace_bytes : 0);
    const Range inputs[] = {pool, lists, range_of(lengths, (int64_t)batch * 4), range_of(q_lengths, q_lengths ? (int64_t)batch * 4 : 0),
                            range_of(q, ((n - 1) * q_stride + row) * es)};
    if (overlap(ro, rw)) return DAMP_ERR_ALIAS;
    for (const Range &r : inputs)
        if (overlap(ro, r) || overlap(rw, r)) return DAMP_ERR_ALIAS;
    a.pool = c.pool;
    a.num_pages = num_pages;
    a.pages = pages;
    a.lengths = lengths;
    a.q_lengths = q_lengths;
    a.q = q;
    a.q_stride = q_stride;
    a.scale = scale;
    a.window = window >= (1 << 30) ? 0 : window;  // a table holds 2^30 tokens at most
    a.o = o;
    a.workspace = static_cast<uint8_t *>(workspace);
    a.test = test;
    return launch_attend(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? DAMP_OK : DAMP_ERR_CUDA;
}

damp_status damp_cache_attend(const damp_cache_layout *layout, const void *cache, int64_t num_pages,
                              const int32_t *pages, int32_t table, int32_t batch, int32_t T, const int32_t *lengths,
                              const int32_t *q_lengths, const void *q, int64_t q_stride, float scale, int32_t window,
                              void *o, int32_t dtype, void *workspace, int64_t workspace_bytes, void *stream) {
    return cache_attend(layout, cache, num_pages, pages, table, batch, T, lengths, q_lengths, q, q_stride, scale, window, o,
                        dtype, workspace, workspace_bytes, stream, 0);
}

damp_status damp_test_cache_attend_wait_timeout(const damp_cache_layout *layout, const void *cache, int64_t num_pages,
                                                const int32_t *pages, int32_t table, int32_t batch, int32_t T,
                                                const int32_t *lengths, const int32_t *q_lengths, const void *q,
                                                int64_t q_stride, float scale, int32_t window, void *o, int32_t dtype,
                                                void *workspace, int64_t workspace_bytes, int32_t queries, void *stream) {
    if (check_cache(layout) == DAMP_OK && (layout->d != 128 || dtype != DAMP_IN_BF16)) return DAMP_ERR_SHAPE;
    return cache_attend(layout, cache, num_pages, pages, table, batch, T, lengths, q_lengths, q, q_stride, scale, window, o,
                        dtype, workspace, workspace_bytes, stream, queries ? 2 : 1);
}

damp_status damp_quantize_state(const damp_layout *layout, const float *S, const uint8_t *perm, void *state,
                                int64_t num_slots, const int32_t *slot_idx, int32_t batch, void *stream) {
    return convert(layout, state, num_slots, slot_idx, batch, perm, const_cast<float *>(S), nullptr, nullptr,
                   nullptr, stream, kQ);
}

damp_status damp_dequantize_state(const damp_layout *layout, const void *state, int64_t num_slots,
                                  const int32_t *slot_idx, int32_t batch, const uint8_t *perm, float *S,
                                  void *stream) {
    return convert(layout, const_cast<void *>(state), num_slots, slot_idx, batch, perm, S, nullptr, nullptr, nullptr,
                   stream, kDQ);
}

damp_status damp_pack_tiers(const damp_layout *layout, const uint16_t *hi, const uint8_t *codes, const uint16_t *meta,
                            void *state, int64_t num_slots, const int32_t *slot_idx, int32_t batch, void *stream) {
    return convert(layout, state, num_slots, slot_idx, batch, nullptr, nullptr, const_cast<uint16_t *>(hi),
                   const_cast<uint8_t *>(codes), const_cast<uint16_t *>(meta), stream, kPack);
}

damp_status damp_unpack_tiers(const damp_layout *layout, const void *state, int64_t num_slots,
                              const int32_t *slot_idx, int32_t batch, uint16_t *hi, uint8_t *codes, uint16_t *meta,
                              void *stream) {
    return convert(layout, const_cast<void *>(state), num_slots, slot_idx, batch, nullptr, nullptr, hi, codes, meta,
                   stream, kUnpack);
}

damp_status damp_calib_error_energy(const damp_layout *layout, const float *S, int32_t batch, float *E_acc,
                                    void *stream) {
    damp_status st = check_layout(layout);
    if (st != DAMP_OK) return st;
    if (batch < 0) return DAMP_ERR_SHAPE;
    if (!E_acc) return DAMP_ERR_NULL;
    if (batch == 0) return DAMP_OK;
    if (!S) return DAMP_ERR_NULL;
    if (!aligned(S, 16) || !aligned(E_acc, 4)) return DAMP_ERR_ALIGN;
    const int64_t H = layout->num_heads, Hm = model_heads_of(layout), dk = layout->d_k, dv = layout->d_v;
    if (overlap(range_of(S, (int64_t)batch * Hm * dk * dv * 4), range_of(E_acc, Hm * dk * 4))) return DAMP_ERR_ALIAS;
    return launch_calib_error_energy(S, batch, (int32_t)H, (int32_t)Hm, layout->head_map, (int32_t)dk, (int32_t)dv,
                                     layout->lo_format, E_acc, static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? DAMP_OK
               : DAMP_ERR_CUDA;
}

damp_status damp_calib_log_decay(const damp_layout *layout, const float *g, int32_t batch, int32_t kda, float *G_acc,
                                 void *stream) {
    damp_status st = check_layout(layout);
    if (st != DAMP_OK) return st;
    if (batch < 0) return DAMP_ERR_SHAPE;
    if (!G_acc) return DAMP_ERR_NULL;
    if (batch == 0) return DAMP_OK;
    if (!g) return DAMP_ERR_NULL;
    if (!aligned(g, 4) || !aligned(G_acc, 4)) return DAMP_ERR_ALIGN;
    const int64_t H = layout->num_heads, Hm = model_heads_of(layout), dk = layout->d_k;
    if (overlap(range_of(g, (int64_t)batch * Hm * (kda ? dk : 1) * 4), range_of(G_acc, Hm * dk * 4)))
        return DAMP_ERR_ALIAS;
    return launch_calib_log_decay(g, batch, (int32_t)H, (int32_t)Hm, layout->head_map, (int32_t)dk, kda ? 1 : 0,
                                  G_acc, static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? DAMP_OK
               : DAMP_ERR_CUDA;
}

damp_status damp_calib_accumulate(const damp_layout *layout, float *S, int32_t n_docs, int32_t n_tokens,
                                  const void *q, const void *k, const void *v, const float *g, const float *beta,
                                  int32_t in_dtype, int32_t kda, int32_t every, float *E_acc, float *G_acc,
                                  void *stream) {
    damp_status st = check_layout(layout);
    if (st != DAMP_OK) return st;
    if (layout->head_map) return DAMP_ERR_SHAPE;  // the trajectories hold every head of the layer
    if (!heads_fit_step(layout)) return DAMP_ERR_SHAPE;
    if (in_dtype != DAMP_IN_BF16 && in_dtype != DAMP_IN_FP32) return DAMP_ERR_FORMAT;
    if (n_docs < 0 || n_tokens < 0 || every < 1) return DAMP_ERR_SHAPE;
    if (!E_acc || !G_acc) return DAMP_ERR_NULL;
    if (n_docs == 0 || n_tokens == 0) return DAMP_OK;
    if (!S || !q || !k || !v || !g || !beta) return DAMP_ERR_NULL;
    if (!aligned(S, 16) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(g, kda ? 16 : 4) ||
        !aligned(beta, 4) || !aligned(E_acc, 4) || !aligned(G_acc, 4))
        return DAMP_ERR_ALIGN;
    const int64_t B = n_docs, T = n_tokens, H = layout->num_heads, Hq = layout->num_qk_heads, dk = layout->d_k,
                  dv = layout->d_v;
    if (B * T > INT32_MAX) return DAMP_ERR_SHAPE;  // the log-decay call takes the (token, document) rows
    const int64_t esz = in_dtype == DAMP_IN_BF16 ? 2 : 4;
    const int64_t sq = B * Hq * dk * esz, sv = B * H * dv * esz, sg = B * H * (kda ? dk : 1) * 4, sb = B * H * 4;
    const Range rs = range_of(S, B * H * dk * dv * 4), re = range_of(E_acc, H * dk * 4), rg = range_of(G_acc, H * dk * 4);
    const Range inputs[] = {range_of(q, T * sq), range_of(k, T * sq), range_of(v, T * sv), range_of(g, T * sg),
                            range_of(beta, T * sb)};
    if (overlap(rs, re) || overlap(rs, rg) || overlap(re, rg)) return DAMP_ERR_ALIAS;
    for (const Range &r : inputs)
        if (overlap(rs, r) || overlap(re, r) || overlap(rg, r)) return DAMP_ERR_ALIAS;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    StepArgs a{};
    a.H = (int32_t)H;
    a.Hqk = (int32_t)Hq;
    a.Hm = (int32_t)H;
    a.dk = (int32_t)dk;
    a.dv = (int32_t)dv;
    a.state = S;
    a.num_slots = B;
    a.batch = n_docs;
    a.o = nullptr;  // the trajectories' outputs are not needed
    a.in_bf16 = in_dtype == DAMP_IN_BF16;
    a.kda = kda ? 1 : 0;
    for (int64_t t = 0; t < T; ++t) {
        a.q = static_cast<const uint8_t *>(q) + t * sq;
        a.k = static_cast<const uint8_t *>(k) + t * sq;
        a.v = static_cast<const uint8_t *>(v) + t * sv;
        a.g = reinterpret_cast<const float *>(reinterpret_cast<const uint8_t *>(g) + t * sg);
        a.beta = reinterpret_cast<const float *>(reinterpret_cast<const uint8_t *>(beta) + t * sb);
        if (launch_fp32_step(a, s) != cudaSuccess) return DAMP_ERR_CUDA;
        if ((t + 1) % every == 0 &&
            launch_calib_error_energy(S, n_docs, (int32_t)H, (int32_t)H, nullptr, (int32_t)dk, (int32_t)dv,
                                      layout->lo_format, E_acc, s) != cudaSuccess)
            return DAMP_ERR_CUDA;
    }
    // the log-decay sums of every (token, document) row: the stacked gates as one batch
    return launch_calib_log_decay(g, (int32_t)(B * T), (int32_t)H, (int32_t)H, nullptr, (int32_t)dk, kda ? 1 : 0,
                                  G_acc, s) == cudaSuccess
               ? DAMP_OK
               : DAMP_ERR_CUDA;
}

damp_status damp_calib_select(const damp_layout *layout, const float *E_acc, int64_t n_samples, const float *G_acc,
                              int64_t n_tokens, float tau, float *C_out, uint8_t *perm_out, void *stream) {
    damp_status st = check_layout(layout);
    if (st != DAMP_OK) return st;
    if (!E_acc || !G_acc || !C_out || !perm_out) return DAMP_ERR_NULL;
    if (n_samples < 1 || n_tokens < 1 || !(tau > 0.0f) || !(tau <= 1.0f)) return DAMP_ERR_SHAPE;
    if (!aligned(E_acc, 4) || !aligned(G_acc, 4) || !aligned(C_out, 4)) return DAMP_ERR_ALIGN;
    const int64_t H = layout->num_heads, Hm = model_heads_of(layout), dk = layout->d_k;
    const Range rc = range_of(C_out, H * dk * 4), rp = range_of(perm_out, H * dk);
    const Range ins[] = {range_of(E_acc, Hm * dk * 4), range_of(G_acc, Hm * dk * 4)};
    if (overlap(rc, rp)) return DAMP_ERR_ALIAS;
    for (const Range &r : ins)
        if (overlap(r, rc) || overlap(r, rp)) return DAMP_ERR_ALIAS;
    return launch_calib_select(E_acc, n_samples, G_acc, n_tokens, tau, (int32_t)H, (int32_t)Hm, layout->head_map,
                               (int32_t)dk, layout->k_hi, C_out, perm_out,
                               static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? DAMP_OK
               : DAMP_ERR_CUDA;
}

damp_status damp_device_status(uint32_t *status) {
    if (!status) return DAMP_ERR_NULL;
    // Kernels on non-blocking streams do not order with the copies below: wait for
    // all of them first, so a bit set by a kernel in flight is not cleared unread.
    if (cudaDeviceSynchronize() != cudaSuccess) return DAMP_ERR_CUDA;
    uint32_t all = 0, bits = 0;
    if (take_status_packed_gdn(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_packed_kda(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_packed_gdn_u4(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_packed_kda_u4(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_packed_gdn_f8(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_packed_kda_f8(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_groups_gdn(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_groups_kda(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_quad_gdn(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_quad_kda(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_fp32(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_lin(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_lin_tc(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_slots(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_verify(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_cache(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_attend(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_attend_tc(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_convert(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_rowabs(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_prefill_gdn(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_prefill_kda(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_prefill_gdn_x(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_prefill_kda_x(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    if (take_status_calib(&bits) != cudaSuccess) return DAMP_ERR_CUDA;
    all |= bits;
    *status = all;
    return DAMP_OK;
}

const char *damp_status_string(damp_status s) {
    switch (s) {
        case DAMP_OK: return "DAMP_OK";
        case DAMP_ERR_NULL: return "DAMP_ERR_NULL: a required pointer is NULL";
        case DAMP_ERR_SHAPE: return "DAMP_ERR_SHAPE: a size is outside what the kernels support";
        case DAMP_ERR_ALIGN: return "DAMP_ERR_ALIGN: a pointer is not aligned as documented";
        case DAMP_ERR_ALIAS: return "DAMP_ERR_ALIAS: an output overlaps the state pool or another argument";
        case DAMP_ERR_FORMAT: return "DAMP_ERR_FORMAT: unknown or unsupported lo_format / in_dtype";
        case DAMP_ERR_CUDA: return "DAMP_ERR_CUDA: the CUDA runtime reported an error while enqueueing";
    }
    return "unknown damp_status";
}

int32_t damp_version(void) { return 100; }

}  // extern "C"
