"""libdamp: the DAMP decode-step recurrent-state update on GB300 (sm_103a).

Python binding over the C ABI of include/damp.h.  The functions carry the
ABI's names and only marshal arguments: every step of the path runs in the
library's CUDA kernels.  PyTorch provides device memory and streams.  There is
no CPU fallback: without the built library every call raises
DampLibraryError.

    layout = Layout(num_heads=32, num_qk_heads=32, d_k=128, d_v=128, k_hi=10)
    state = new_state(layout, num_slots=256, device="cuda")
    quantize_state(layout, S_fp32, perm, state)            # prefill hand-off
    o = kda_decode_step(layout, state, perm, q, k, v, g, beta)

Linear attention with a decay per head and no delta rule runs on an FP32 pool
(new_fp32_state) with lin_prefill_chunk and lin_decode_step.  copy_slots, zero_slots and
compact_slots move whole slots of all layers' pools, packed or FP32; verify_drafts accepts
drafted tokens, and its counts are the lengths with which a chunk replays them.

The softmax-attention layers of hybrid models keep their keys and values in 8 bits, in pages of
32 tokens (CacheLayout, new_cache): rotary turns q and k, cache_append writes new tokens,
cache_attend attends over the cache (one token a row, drafted tokens, prompts), cache_read
reads values back.  Pages are slots of copy_slots and zero_slots.

A layer whose heads keep different numbers of FP16 key channels (the decay-tiered
allocation of App. E) is a list of head groups (`head_groups`), one uniform layout,
pool and permutation table per K_hi, each with a head map into the layer's heads.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, field

from ._lib import DampCacheLayout, DampLayout, DampLibraryError, lib

__all__ = [
    "Layout", "DampError", "DampLibraryError", "LO_U8_AFFINE_G32_H32", "LO_U8_AFFINE_G32", "LO_S8_ABSMAX_ROW", "LO_U4_AFFINE_G32_H32",
    "LO_U4_AFFINE_G32", "LO_FP8_E4M3_G32",
    "record_bytes", "slot_bytes", "bits_per_value", "new_state", "new_fp32_state",
    "gdn_decode_step", "kda_decode_step", "gdn_prefill_chunk", "kda_prefill_chunk", "calib_error_energy", "calib_log_decay", "calib_select", "u8_gdn_decode_step", "u8_kda_decode_step",
    "fp32_gdn_decode_step", "fp32_kda_decode_step", "quantize_state", "dequantize_state",
    "pack_tiers", "unpack_tiers", "device_status", "version", "DEV_WAIT_TIMEOUT", "DEV_BAD_SLOT", "DEV_BAD_HEAD",
    "head_groups", "test_kda_wait_timeout", "gdn_decode_step_groups", "kda_decode_step_groups",
    "calib_accumulate", "lin_decode_step", "lin_prefill_chunk", "copy_slots", "zero_slots", "compact_slots",
    "verify_drafts", "DEV_BAD_TOKEN", "CacheLayout", "CACHE_PAGE", "new_cache", "cache_page_bytes", "cache_append",
    "cache_read", "cache_attend", "test_cache_attend_wait_timeout", "rotary", "rotary_frequencies", "DEV_NOT_FINITE",
]

LO_U8_AFFINE_G32_H32 = 0
LO_U8_AFFINE_G32 = 1
LO_S8_ABSMAX_ROW = 2  # per-row symmetric absmax INT8, FP32 row scale
LO_U4_AFFINE_G32_H32 = 3  # UINT4 affine G32 + H32
LO_U4_AFFINE_G32 = 4  # UINT4 affine G32
LO_FP8_E4M3_G32 = 5  # FP8 E4M3, FP32 scale per 32
IN_BF16 = 0
IN_FP32 = 1
DEV_WAIT_TIMEOUT = 1
DEV_BAD_SLOT = 2
DEV_BAD_HEAD = 4
DEV_BAD_TOKEN = 8
DEV_NOT_FINITE = 16
CACHE_PAGE = 32  # tokens of a page of the 8-bit cache


class DampError(RuntimeError):
    def __init__(self, status: int, what: str):
        msg = lib().damp_status_string(status).decode()
        super().__init__(f"{what}: {msg}")
        self.status = status


@dataclass(frozen=True)
class Layout:
    """damp_layout: num_heads held heads (one state per slot and head), q/k heads of the
    operands, d_k x d_v states, K_hi FP16 key channels, the low-tier format; for a head
    group of a layer, model_heads (value heads of the operand tensors) and head_map
    (int32 CUDA tensor [num_heads]: the model head of each held head)."""
    num_heads: int
    num_qk_heads: int
    d_k: int
    d_v: int
    k_hi: int
    lo_format: int = LO_U8_AFFINE_G32_H32
    model_heads: int = 0
    head_map: object = field(default=None, compare=False, repr=False)

    def __post_init__(self):
        if self.head_map is not None:
            import torch
            m = self.head_map
            if (not isinstance(m, torch.Tensor) or m.dtype != torch.int32 or not m.is_cuda or not m.is_contiguous()
                    or m.shape != (self.num_heads,)):
                raise ValueError(f"head_map must be a contiguous int32 CUDA tensor of shape [{self.num_heads}]")

    @property
    def heads_of_operands(self) -> int:
        """H_m: value heads of v, g, beta, o and S."""
        return self.model_heads or self.num_heads

    def c(self) -> DampLayout:
        return DampLayout(self.num_heads, self.num_qk_heads, self.d_k, self.d_v, self.k_hi, self.lo_format,
                          self.model_heads, None if self.head_map is None else self.head_map.data_ptr())


def head_groups(k_hi_of_head, num_qk_heads: int, d_k: int, d_v: int, lo_format: int = LO_U8_AFFINE_G32_H32,
                device="cuda"):
    """Layouts of a layer whose heads keep different numbers of FP16 key channels
    (App. E, decay-tiered allocation): one layout per distinct K_hi, held heads in
    ascending model-head order, each with its head map.  Returns [(layout, heads)],
    heads the list of model heads of the group."""
    import torch
    ks = [int(k) for k in k_hi_of_head]
    H = len(ks)
    out = []
    for K in sorted(set(ks)):
        heads = [h for h in range(H) if ks[h] == K]
        m = torch.tensor(heads, dtype=torch.int32, device=device)
        out.append((Layout(len(heads), num_qk_heads, d_k, d_v, K, lo_format, model_heads=H, head_map=m), heads))
    return out


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # a Stream object costs microseconds
    if raw is None:
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    return ctypes.c_void_p(raw(torch.cuda.current_device()))


def _check(status: int, what: str):
    if status != 0:
        raise DampError(status, what)


def _in_dtype(*ts) -> int:
    import torch
    dts = {t.dtype for t in ts}
    if dts == {torch.bfloat16}:
        return IN_BF16
    if dts == {torch.float32}:
        return IN_FP32
    raise TypeError("q, k, v must all be bfloat16 or all float32")


def _cuda_contig(name, t):
    if t is None:
        return
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")


def _want(name, t, shape, *, dtype=None, esize=None):
    """Raise ValueError unless tensor t (if given) has exactly `shape` (and dtype or
    element size).  The C ABI sees only pointers, so a mis-sized tensor would make a
    kernel read or write outside it: every size is checked here, before any call."""
    if t is None:
        return
    if tuple(t.shape) != tuple(int(x) for x in shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(int(x) for x in shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if esize is not None and t.element_size() not in ((esize,) if isinstance(esize, int) else esize):
        raise ValueError(f"{name} has {t.element_size()}-byte elements, expected {esize}")


def _want_pool(layout, state, num_slots, fp32=False):
    """The packed pool (uint8 [slots, slot_bytes]) or FP32 state (float32 [slots, H, d_k,
    d_v]) must hold num_slots slots; returns num_slots (default: all of them)."""
    import torch
    if state is None:
        raise ValueError("state is required")
    if fp32:
        _want("state", state, (state.shape[0], layout.num_heads, layout.d_k, layout.d_v), dtype=torch.float32)
    else:
        if state.dim() != 2:
            raise ValueError(f"state has shape {tuple(state.shape)}, expected [slots, {slot_bytes(layout)}]")
        _want("state", state, (state.shape[0], slot_bytes(layout)), dtype=torch.uint8)
    n = state.shape[0] if num_slots is None else int(num_slots)
    if n < 0 or n > state.shape[0]:
        raise ValueError(f"num_slots {n} exceeds the {state.shape[0]} slots of state")
    return n


def _want_batch(slot_idx, B, num_slots):
    import torch
    _want("slot_idx", slot_idx, (B,), dtype=torch.int32)
    if slot_idx is None and B > num_slots:
        raise ValueError(f"batch {B} exceeds num_slots {num_slots} without slot_idx")


def _want_operands(layout, kind, q, k, v, g, beta, o, lead):
    """q, k [*lead, H_qk, d_k]; v [*lead, H_m, d_v]; g [*lead, H_m] (GDN) or [*lead, H_m,
    d_k] (KDA); beta [*lead, H_m]; o float32 [*lead, H_m, d_v]."""
    import torch
    Hm = layout.heads_of_operands
    for n, t in (("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta)):
        if t is None:
            raise ValueError(f"{n} is required")
    lead = tuple(lead)
    _want("q", q, lead + (layout.num_qk_heads, layout.d_k))
    _want("k", k, lead + (layout.num_qk_heads, layout.d_k))
    _want("v", v, lead + (Hm, layout.d_v))
    _want("g", g, lead + ((Hm, layout.d_k) if kind == "kda" else (Hm,)), dtype=torch.float32)
    _want("beta", beta, lead + (Hm,), dtype=torch.float32)
    _want("o", o, lead + (Hm, layout.d_v), dtype=torch.float32)


def version() -> int:
    return int(lib().damp_version())


def record_bytes(layout: Layout) -> int:
    c = layout.c()
    return int(lib().damp_record_bytes(ctypes.byref(c)))


def slot_bytes(layout: Layout) -> int:
    c = layout.c()
    n = int(lib().damp_slot_bytes(ctypes.byref(c)))
    if n == 0:
        _check(lib().damp_validate_layout(ctypes.byref(c)), "layout")
    return n


def bits_per_value(layout: Layout) -> float:
    c = layout.c()
    return float(lib().damp_bits_per_value(ctypes.byref(c)))


def new_state(layout: Layout, num_slots: int, device="cuda"):
    """A zero-filled packed pool of num_slots slots (uint8, 16-B aligned by the allocator)."""
    import torch
    return torch.zeros((num_slots, slot_bytes(layout)), dtype=torch.uint8, device=device)


def new_fp32_state(layout: Layout, num_slots: int, device="cuda"):
    import torch
    return torch.zeros((num_slots, layout.num_heads, layout.d_k, layout.d_v), dtype=torch.float32, device=device)


def _step(fn_name, layout, state, perm, q, k, v, g, beta, o, slot_idx, num_slots, stream):
    import torch
    fp32 = fn_name.startswith("damp_fp32")
    if v is None or v.dim() < 1:
        raise ValueError("v must be a [B, H, d_v] tensor")
    B = v.shape[0]
    num_slots = _want_pool(layout, state, num_slots, fp32=fp32)
    _want_batch(slot_idx, B, num_slots)
    if not fp32:
        _want("perm", perm, (layout.num_heads, layout.d_k), dtype=torch.uint8)
    _want_operands(layout, "kda" if "_kda_" in fn_name else "gdn", q, k, v, g, beta, o, (B,))
    for n, t in (("state", state), ("perm", perm), ("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta),
                 ("o", o), ("slot_idx", slot_idx)):
        _cuda_contig(n, t)
    if o is None:
        # a head group writes only its heads' rows: the others start at zero
        alloc = torch.empty if layout.head_map is None else torch.zeros
        o = alloc((B, layout.heads_of_operands, layout.d_v), dtype=torch.float32, device=v.device)
    c = layout.c()
    args = [ctypes.byref(c), _ptr(state), num_slots, _ptr(slot_idx), B]
    if perm is not None or not fn_name.startswith("damp_fp32"):
        args.append(_ptr(perm))
    args += [_ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(o), _in_dtype(q, k, v), _stream(stream)]
    _check(getattr(lib(), fn_name)(*args), fn_name)
    return o


def gdn_decode_step(layout, state, perm, q, k, v, g, beta, o=None, slot_idx=None, num_slots=None, stream=None):
    """One GDN decode step on the packed state (in place); returns o [B, H, d_v] float32."""
    return _step("damp_gdn_decode_step", layout, state, perm, q, k, v, g, beta, o, slot_idx, num_slots, stream)


def kda_decode_step(layout, state, perm, q, k, v, g, beta, o=None, slot_idx=None, num_slots=None, stream=None):
    """One KDA decode step on the packed state (in place); returns o [B, H, d_v] float32."""
    return _step("damp_kda_decode_step", layout, state, perm, q, k, v, g, beta, o, slot_idx, num_slots, stream)


def _step_groups(fn_name, groups, q, k, v, g, beta, o, slot_idx, stream):
    """groups: [(layout, state, perm)] of one layer (head_groups layouts)."""
    import torch
    n = len(groups)
    if n < 1:
        raise ValueError("at least one head group is required")
    if v is None or v.dim() < 1:
        raise ValueError("v must be a [B, H_m, d_v] tensor")
    B = v.shape[0]
    kind = "kda" if "_kda_" in fn_name else "gdn"
    layouts = (DampLayout * n)()
    states = (ctypes.c_void_p * n)()
    perms = (ctypes.c_void_p * n)()
    slots = (ctypes.c_int64 * n)()
    for i, (layout, state, perm) in enumerate(groups):
        if layout.head_map is None:
            raise ValueError(f"group {i} has no head map (build the groups with head_groups)")
        ns = _want_pool(layout, state, None)
        _want_batch(slot_idx, B, ns)
        _want("perm", perm, (layout.num_heads, layout.d_k), dtype=torch.uint8)
        _want_operands(layout, kind, q, k, v, g, beta, o, (B,))
        _cuda_contig("state", state)
        _cuda_contig("perm", perm)
        layouts[i] = layout.c()
        states[i] = state.data_ptr()
        perms[i] = perm.data_ptr()
        slots[i] = ns
    for nm, t in (("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta), ("o", o), ("slot_idx", slot_idx)):
        _cuda_contig(nm, t)
    if o is None:
        o = torch.empty((B, groups[0][0].heads_of_operands, groups[0][0].d_v), dtype=torch.float32, device=v.device)
    _check(getattr(lib(), fn_name)(layouts, n, states, slots, perms, _ptr(slot_idx), B, _ptr(q), _ptr(k), _ptr(v),
                                   _ptr(g), _ptr(beta), _ptr(o), _in_dtype(q, k, v), _stream(stream)), fn_name)
    return o


def gdn_decode_step_groups(groups, q, k, v, g, beta, o=None, slot_idx=None, stream=None):
    """One GDN decode step of a layer stored as head groups, groups = [(layout, state, perm)]
    (one launch for two groups with a compile-time K_hi pair); returns o [B, H_m, d_v]."""
    return _step_groups("damp_gdn_decode_step_groups", groups, q, k, v, g, beta, o, slot_idx, stream)


def kda_decode_step_groups(groups, q, k, v, g, beta, o=None, slot_idx=None, stream=None):
    """One KDA decode step of a layer stored as head groups (see gdn_decode_step_groups)."""
    return _step_groups("damp_kda_decode_step_groups", groups, q, k, v, g, beta, o, slot_idx, stream)


def test_kda_wait_timeout(layout, state, perm, q, k, v, g, beta, o=None, slot_idx=None, num_slots=None,
                          stream=None):
    """The bounded-wait test hook (damp_test_kda_wait_timeout): every wait of the KDA step's
    kernel runs out after ~1 ms; nothing is written and the status word reports
    DEV_WAIT_TIMEOUT.  For tests of the timeout path only."""
    return _step("damp_test_kda_wait_timeout", layout, state, perm, q, k, v, g, beta, o, slot_idx, num_slots,
                 stream)


def u8_gdn_decode_step(layout, state, perm, q, k, v, g, beta, o=None, slot_idx=None, num_slots=None, stream=None):
    return _step("damp_u8_gdn_decode_step", layout, state, perm, q, k, v, g, beta, o, slot_idx, num_slots, stream)


def u8_kda_decode_step(layout, state, perm, q, k, v, g, beta, o=None, slot_idx=None, num_slots=None, stream=None):
    return _step("damp_u8_kda_decode_step", layout, state, perm, q, k, v, g, beta, o, slot_idx, num_slots, stream)


def fp32_gdn_decode_step(layout, state, q, k, v, g, beta, o=None, slot_idx=None, num_slots=None, stream=None):
    """One GDN decode step on an FP32 state [slots, H, d_k, d_v] (in place)."""
    return _step("damp_fp32_gdn_decode_step", layout, state, None, q, k, v, g, beta, o, slot_idx, num_slots, stream)


def fp32_kda_decode_step(layout, state, q, k, v, g, beta, o=None, slot_idx=None, num_slots=None, stream=None):
    return _step("damp_fp32_kda_decode_step", layout, state, None, q, k, v, g, beta, o, slot_idx, num_slots, stream)


def _prefill(fn_name, layout, state, perm, q, k, v, g, beta, o, lengths, slot_idx, num_slots, stream):
    import torch
    if v is None or v.dim() < 2:
        raise ValueError("v must be a [B, T, H, d_v] tensor")
    B, T = v.shape[0], v.shape[1]
    num_slots = _want_pool(layout, state, num_slots)
    _want_batch(slot_idx, B, num_slots)
    _want("lengths", lengths, (B,), dtype=torch.int32)
    _want("perm", perm, (layout.num_heads, layout.d_k), dtype=torch.uint8)
    _want_operands(layout, "kda" if "_kda_" in fn_name else "gdn", q, k, v, g, beta, o, (B, T))
    for n, t in (("state", state), ("perm", perm), ("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta),
                 ("o", o), ("lengths", lengths), ("slot_idx", slot_idx)):
        _cuda_contig(n, t)
    if o is None:
        o = torch.zeros((B, T, layout.heads_of_operands, layout.d_v), dtype=torch.float32, device=v.device)
    c = layout.c()
    _check(getattr(lib(), fn_name)(ctypes.byref(c), _ptr(state), num_slots, _ptr(slot_idx), B, T, _ptr(lengths),
                                   _ptr(perm), _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(o),
                                   _in_dtype(q, k, v), _stream(stream)), fn_name)
    return o


def gdn_prefill_chunk(layout, state, perm, q, k, v, g, beta, o=None, lengths=None, slot_idx=None, num_slots=None,
                      stream=None):
    """One GDN prefill chunk on the packed state (in place): q, k [B, T, H_qk, d_k], v [B, T, H, d_v],
    g, beta [B, T, H]; returns o [B, T, H, d_v] float32."""
    return _prefill("damp_gdn_prefill_chunk", layout, state, perm, q, k, v, g, beta, o, lengths, slot_idx,
                    num_slots, stream)


def kda_prefill_chunk(layout, state, perm, q, k, v, g, beta, o=None, lengths=None, slot_idx=None, num_slots=None,
                      stream=None):
    """One KDA prefill chunk on the packed state (in place): as gdn_prefill_chunk with g [B, T, H, d_k]."""
    return _prefill("damp_kda_prefill_chunk", layout, state, perm, q, k, v, g, beta, o, lengths, slot_idx,
                    num_slots, stream)


def calib_error_energy(layout, S, E_acc, stream=None):
    """E_acc [H, d_k] += per-channel squared low-tier round-trip error of S [B, H, d_k, d_v]."""
    import torch
    Hm = layout.heads_of_operands
    if S is None or S.dim() != 4:
        raise ValueError("S must be a [B, H, d_k, d_v] tensor")
    _want("S", S, (S.shape[0], Hm, layout.d_k, layout.d_v), dtype=torch.float32)
    _want("E_acc", E_acc, (Hm, layout.d_k), dtype=torch.float32)
    _cuda_contig("S", S)
    _cuda_contig("E_acc", E_acc)
    _check(lib().damp_calib_error_energy(ctypes.byref(layout.c()), _ptr(S), S.shape[0], _ptr(E_acc), _stream(stream)),
           "damp_calib_error_energy")
    return E_acc


def calib_log_decay(layout, g, G_acc, stream=None):
    """G_acc [H, d_k] += log-decay g summed over the batch (g [B, H] GDN or [B, H, d_k] KDA)."""
    import torch
    Hm = layout.heads_of_operands
    if g is None or g.dim() not in (2, 3):
        raise ValueError("g must be a [B, H] or [B, H, d_k] tensor")
    _want("g", g, (g.shape[0], Hm) + ((layout.d_k,) if g.dim() == 3 else ()), dtype=torch.float32)
    _want("G_acc", G_acc, (Hm, layout.d_k), dtype=torch.float32)
    _cuda_contig("g", g)
    _cuda_contig("G_acc", G_acc)
    _check(lib().damp_calib_log_decay(ctypes.byref(layout.c()), _ptr(g), g.shape[0], 1 if g.dim() == 3 else 0,
                                      _ptr(G_acc), _stream(stream)), "damp_calib_log_decay")
    return G_acc


def calib_accumulate(layout, kind, S, q, k, v, g, beta, E_acc, G_acc, every=8, stream=None):
    """One calibration run's statistics in one call (damp_calib_accumulate): q, k [T, B, H_qk,
    d_k]; v [T, B, H, d_v]; g [T, B, H, d_k] (KDA) or [T, B, H] (GDN); beta [T, B, H]; S the
    FP32 states [B, H, d_k, d_v] (updated); E_acc, G_acc [H, d_k] accumulated.  Returns
    (n_samples, n_token_rows) for calib_select."""
    import torch
    if layout.head_map is not None:
        raise ValueError("the calibration trajectories hold every head: use a layout without a head map")
    if v is None or v.dim() != 4:
        raise ValueError("v must be a [T, B, H, d_v] tensor")
    T, B = v.shape[0], v.shape[1]
    H = layout.num_heads
    _want("S", S, (B, H, layout.d_k, layout.d_v), dtype=torch.float32)
    _want_operands(layout, kind, q, k, v, g, beta, None, (T, B))
    _want("E_acc", E_acc, (H, layout.d_k), dtype=torch.float32)
    _want("G_acc", G_acc, (H, layout.d_k), dtype=torch.float32)
    for n, t in (("S", S), ("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta), ("E_acc", E_acc),
                 ("G_acc", G_acc)):
        _cuda_contig(n, t)
    _check(lib().damp_calib_accumulate(ctypes.byref(layout.c()), _ptr(S), B, T, _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                                       _ptr(beta), _in_dtype(q, k, v), 1 if kind == "kda" else 0, int(every),
                                       _ptr(E_acc), _ptr(G_acc), _stream(stream)), "damp_calib_accumulate")
    return max(B * (T // int(every)), 1), B * T


def calib_select(layout, E_acc, n_samples, G_acc, n_tokens, tau=1e-4, stream=None):
    """Scores C [H, d_k] float32 and permutations pi [H, d_k] uint8 (Algorithm 1)."""
    import torch
    Hm = layout.heads_of_operands
    _want("E_acc", E_acc, (Hm, layout.d_k), dtype=torch.float32)
    _want("G_acc", G_acc, (Hm, layout.d_k), dtype=torch.float32)
    _cuda_contig("E_acc", E_acc)
    _cuda_contig("G_acc", G_acc)
    C = torch.empty((layout.num_heads, layout.d_k), dtype=torch.float32, device=E_acc.device)
    perm = torch.empty((layout.num_heads, layout.d_k), dtype=torch.uint8, device=E_acc.device)
    _check(lib().damp_calib_select(ctypes.byref(layout.c()), _ptr(E_acc), int(n_samples), _ptr(G_acc), int(n_tokens),
                                   float(tau), _ptr(C), _ptr(perm), _stream(stream)), "damp_calib_select")
    return C, perm


def quantize_state(layout, S, perm, state, slot_idx=None, num_slots=None, stream=None):
    """Write natural-order FP32 states S [B, H, d_k, d_v] into packed slots."""
    import torch
    if S is None or S.dim() != 4:
        raise ValueError("S must be a [B, H, d_k, d_v] tensor")
    n_slots = _want_pool(layout, state, num_slots)
    _want_batch(slot_idx, S.shape[0], n_slots)
    _want("S", S, (S.shape[0], layout.heads_of_operands, layout.d_k, layout.d_v), dtype=torch.float32)
    _want("perm", perm, (layout.num_heads, layout.d_k), dtype=torch.uint8)
    for n, t in (("S", S), ("perm", perm), ("state", state), ("slot_idx", slot_idx)):
        _cuda_contig(n, t)
    c = layout.c()
    _check(lib().damp_quantize_state(ctypes.byref(c), _ptr(S), _ptr(perm), _ptr(state), n_slots, _ptr(slot_idx),
                                     S.shape[0], _stream(stream)), "damp_quantize_state")


def dequantize_state(layout, state, perm, batch=None, S=None, slot_idx=None, num_slots=None, stream=None):
    """Reconstruct natural-order FP32 states [B, H, d_k, d_v] from packed slots."""
    import torch
    n_slots = _want_pool(layout, state, num_slots)
    B = (slot_idx.shape[0] if slot_idx is not None else n_slots) if batch is None else int(batch)
    _want_batch(slot_idx, B, n_slots)
    _want("S", S, (B, layout.heads_of_operands, layout.d_k, layout.d_v), dtype=torch.float32)
    _want("perm", perm, (layout.num_heads, layout.d_k), dtype=torch.uint8)
    for n, t in (("S", S), ("perm", perm), ("state", state), ("slot_idx", slot_idx)):
        _cuda_contig(n, t)
    if S is None:
        S = torch.zeros((B, layout.heads_of_operands, layout.d_k, layout.d_v), dtype=torch.float32, device=state.device)
    c = layout.c()
    _check(lib().damp_dequantize_state(ctypes.byref(c), _ptr(state), n_slots, _ptr(slot_idx), B,
                                       _ptr(perm), _ptr(S), _stream(stream)), "damp_dequantize_state")
    return S


def _tier_shapes(layout, B, hi, codes, meta):
    """(name, tensor, shape, element bytes) of the logical tiers of B slots (damp_pack_tiers)."""
    H, dk, dv, K, f = layout.num_heads, layout.d_k, layout.d_v, layout.k_hi, layout.lo_format
    lo = dk - K
    codes_cols = dv // 2 if f in (LO_U4_AFFINE_G32_H32, LO_U4_AFFINE_G32) else dv
    if f == LO_S8_ABSMAX_ROW:
        meta_shape, meta_es = (B, H, lo), 4
    elif f == LO_FP8_E4M3_G32:
        meta_shape, meta_es = (B, H, lo, dv // 32), 4
    else:
        meta_shape, meta_es = (B, H, lo, dv // 32, 2), 2
    return [("hi", hi, (B, H, K, dv), 2), ("codes", codes, (B, H, lo, codes_cols), 1),
            ("meta", meta, meta_shape, meta_es)]


def pack_tiers(layout, hi, codes, meta, state, slot_idx=None, num_slots=None, stream=None):
    """Copy logical tiers (hi uint16/fp16 [B,H,K,d_v], codes uint8 [B,H,d_k-K,d_v],
    meta uint16/fp16 [B,H,d_k-K,d_v/32,2]; row-absmax format: codes int8, meta float32
    [B,H,d_k-K]) into packed slots, bit for bit."""
    B = codes.shape[0] if codes is not None else (hi.shape[0] if hi is not None else 0)
    n_slots = _want_pool(layout, state, num_slots)
    _want_batch(slot_idx, B, n_slots)
    for n, t, shape, es in _tier_shapes(layout, B, hi, codes, meta):
        _want(n, t, shape, esize=es)
    for n, t in (("hi", hi), ("codes", codes), ("meta", meta), ("state", state), ("slot_idx", slot_idx)):
        _cuda_contig(n, t)
    c = layout.c()
    _check(lib().damp_pack_tiers(ctypes.byref(c), _ptr(hi if hi is not None and hi.numel() else None),
                                 _ptr(codes if codes is not None and codes.numel() else None),
                                 _ptr(meta if meta is not None and meta.numel() else None), _ptr(state),
                                 n_slots, _ptr(slot_idx), B,
                                 _stream(stream)), "damp_pack_tiers")


def unpack_tiers(layout, state, batch=None, slot_idx=None, num_slots=None, stream=None):
    """Logical tiers (hi int16 bits, codes uint8, meta int16 bits; row-absmax format: codes
    int8, meta float32 [B,H,d_k-K]) of `batch` packed slots."""
    import torch
    n_slots = _want_pool(layout, state, num_slots)
    B = (slot_idx.shape[0] if slot_idx is not None else n_slots) if batch is None else int(batch)
    _want_batch(slot_idx, B, n_slots)
    _cuda_contig("state", state)
    _cuda_contig("slot_idx", slot_idx)
    H, dk, dv, K = layout.num_heads, layout.d_k, layout.d_v, layout.k_hi
    dev = state.device
    hi = torch.empty((B, H, K, dv), dtype=torch.int16, device=dev)
    if layout.lo_format == LO_S8_ABSMAX_ROW:
        codes = torch.empty((B, H, dk - K, dv), dtype=torch.int8, device=dev)
        meta = torch.empty((B, H, dk - K), dtype=torch.float32, device=dev)
    elif layout.lo_format in (LO_U4_AFFINE_G32_H32, LO_U4_AFFINE_G32):
        codes = torch.empty((B, H, dk - K, dv // 2), dtype=torch.uint8, device=dev)
        meta = torch.empty((B, H, dk - K, dv // 32, 2), dtype=torch.int16, device=dev)
    elif layout.lo_format == LO_FP8_E4M3_G32:
        codes = torch.empty((B, H, dk - K, dv), dtype=torch.uint8, device=dev)
        meta = torch.empty((B, H, dk - K, dv // 32), dtype=torch.float32, device=dev)
    else:
        codes = torch.empty((B, H, dk - K, dv), dtype=torch.uint8, device=dev)
        meta = torch.empty((B, H, dk - K, dv // 32, 2), dtype=torch.int16, device=dev)
    c = layout.c()
    _check(lib().damp_unpack_tiers(ctypes.byref(c), _ptr(state), n_slots,
                                   _ptr(slot_idx), B, _ptr(hi if hi.numel() else None),
                                   _ptr(codes if codes.numel() else None), _ptr(meta if meta.numel() else None),
                                   _stream(stream)), "damp_unpack_tiers")
    return hi, codes, meta


def _new(shape, dtype, like, stream):
    """An uninitialized output, allocated for the stream that the call runs on."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _given(name, t, shape, dtype):
    """The address of t; ValueError unless it is a contiguous CUDA tensor of the shape and type."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.shape != shape or t.dtype != dtype:
        _want(name, t, shape, dtype=dtype)
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    return t.data_ptr()


def _lin(layout, state, q, k, v, g, o, lengths, slot_idx, num_slots, stream, lead_dims):
    import torch
    f32, i32 = torch.float32, torch.int32
    if v is None or v.dim() != lead_dims + 2:
        raise ValueError(f"v must have {lead_dims + 2} dimensions")
    if layout.head_map is not None:
        raise ValueError("the FP32 state holds every head: use a layout without a head map")
    dtype = v.dtype
    bf16 = dtype == torch.bfloat16
    if not bf16 and dtype != f32 or q is not None and q.dtype != dtype or k is not None and k.dtype != dtype:
        raise TypeError("q, k, v must all be bfloat16 or all float32")
    if state is None or state.dim() != 4:
        raise ValueError("state must be a [slots, H, d_k, d_v] tensor")
    lead = v.shape[:lead_dims]
    B, H, dk, dv = lead[0], layout.num_heads, layout.d_k, layout.d_v
    slots = state.shape[0]
    pool = _given("state", state, (slots, H, dk, dv), f32)
    if num_slots is not None:
        if not 0 <= num_slots <= slots:
            raise ValueError(f"num_slots {num_slots} exceeds the {slots} slots of state")
        slots = int(num_slots)
    idx = None
    if slot_idx is not None:
        idx = _given("slot_idx", slot_idx, (B,), i32)
    elif B > slots:
        raise ValueError(f"batch {B} exceeds num_slots {slots} without slot_idx")
    qk_shape, o_shape = lead + (layout.num_qk_heads, dk), lead + (H, dv)
    per_head = g is not None and g.dim() == 1
    qp, kp, vp = _given("q", q, qk_shape, dtype), _given("k", k, qk_shape, dtype), _given("v", v, o_shape, dtype)
    gp = _given("g", g, (H,) if per_head else lead + (H,), f32)
    n = None if lengths is None else _given("lengths", lengths, (B,), i32)
    if o is None:
        o = _new(o_shape, f32, v, stream)
    op = _given("o", o, o_shape, f32)
    c = ctypes.byref(layout.c())
    in_dtype = IN_BF16 if bf16 else IN_FP32
    L = lib()
    if lead_dims == 1:
        _check(L.damp_lin_decode_step(c, pool, slots, idx, B, qp, kp, vp, gp, per_head, op, in_dtype, _stream(stream)),
               "damp_lin_decode_step")
    else:
        T = lead[1]
        need = L.damp_lin_prefill_workspace(c, B, T, in_dtype)
        ws = _new((need,), torch.uint8, v, stream) if need else None
        _check(L.damp_lin_prefill_chunk(c, pool, slots, idx, B, T, n, qp, kp, vp, gp, per_head, op, in_dtype,
                                        ws.data_ptr() if need else None, need, _stream(stream)), "damp_lin_prefill_chunk")
    return o


def lin_decode_step(layout, state, q, k, v, g, o=None, slot_idx=None, num_slots=None, stream=None):
    """One token of linear attention with a decay per head on an FP32 state [slots, H, d_k, d_v]
    (in place): S = e^g S + k v^T, o = S^T q.  q, k [B, H_qk, d_k], v [B, H, d_v], g [B, H] or
    [H]; returns o [B, H, d_v] float32."""
    return _lin(layout, state, q, k, v, g, o, None, slot_idx, num_slots, stream, 1)


def lin_prefill_chunk(layout, state, q, k, v, g, o=None, lengths=None, slot_idx=None, num_slots=None, stream=None):
    """A chunk of T tokens of linear attention with a decay per head on an FP32 state (in place):
    q, k [B, T, H_qk, d_k], v [B, T, H, d_v], g [B, T, H] or [H]; row b runs its first lengths[b]
    tokens.  Returns o [B, T, H, d_v] float32, zero past a row's length."""
    return _lin(layout, state, q, k, v, g, o, lengths, slot_idx, num_slots, stream, 2)


def _pools(pools):
    """(pointers, bytes per slot, number of pools, slots) of one pool or a list of pools: CUDA
    tensors [slots, ...], contiguous, of any type, all with the same number of slots."""
    import torch
    if isinstance(pools, torch.Tensor):
        pools = (pools,)
    n = len(pools)
    if n == 0:
        raise ValueError("at least one pool is required")
    slots = pools[0].shape[0] if pools[0].dim() else 0
    ptrs, sizes = (ctypes.c_void_p * n)(), (ctypes.c_int64 * n)()
    for i, t in enumerate(pools):
        if t.dim() < 2 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"pool {i} must be a contiguous CUDA tensor [slots, ...]")
        if t.shape[0] != slots or slots == 0:
            raise ValueError(f"pool {i} has {t.shape[0]} slots, expected {slots} (one at least)")
        ptrs[i] = t.data_ptr()
        sizes[i] = t.nbytes // slots
    return ptrs, sizes, n, slots


def _slot_list(name, t):
    import torch
    if t is None or t.dim() != 1:
        raise ValueError(f"{name} must be a one-dimensional int32 CUDA tensor")
    return _given(name, t, t.shape, torch.int32)


def copy_slots(pools, src, dst, stream=None):
    """Slot dst[i] of every pool receives what slot src[i] held before the call (int32 [n], dst
    distinct; the lists may overlap).  A source named n times is forked n ways.  An entry with a
    negative slot is skipped.  pools: one pool or the list of a model's layers, packed or FP32."""
    if src is not None and dst is not None and src.shape != dst.shape:
        raise ValueError(f"src has shape {tuple(src.shape)}, dst {tuple(dst.shape)}")
    ptrs, sizes, n, slots = _pools(pools)
    _check(lib().damp_copy_slots(ptrs, sizes, n, slots, _slot_list("src", src), _slot_list("dst", dst), src.shape[0],
                                 _stream(stream)), "damp_copy_slots")


def zero_slots(pools, idx, stream=None):
    """Free slots idx (int32 [n]) of every pool: an all-zero slot is the zero state, the start of
    a sequence.  Negative entries are skipped."""
    ptrs, sizes, n, slots = _pools(pools)
    _check(lib().damp_zero_slots(ptrs, sizes, n, slots, _slot_list("idx", idx), idx.shape[0], _stream(stream)),
           "damp_zero_slots")


def compact_slots(pools, slot_idx, out=None, stream=None):
    """Move the live slots slot_idx (int32 [B], negative for a finished request) of every pool
    into the lowest slot numbers; returns the new slot_idx.  With n distinct live slots, those
    below n stay, the others move in ascending order into the free slots below n in ascending
    order.  The slots left behind keep their bytes (zero_slots frees them)."""
    import torch
    idx = _slot_list("slot_idx", slot_idx)
    ptrs, sizes, n, slots = _pools(pools)
    if out is None:
        out = _new(slot_idx.shape, torch.int32, slot_idx, stream)
    _check(lib().damp_compact_slots(ptrs, sizes, n, slots, idx, slot_idx.shape[0],
                                    _given("out", out, slot_idx.shape, torch.int32), _stream(stream)),
           "damp_compact_slots")
    return out


def verify_drafts(target_logits, draft_tokens, u, noise, draft_logits=None, temperature=None, draft_len=None,
                  vocab=None, tokens=None, count=None, stream=None):
    """Speculative sampling: accept a prefix of the drafted tokens and draw the next one.

    target_logits [B, D + 1, ld], draft_logits [B, D, ld] (None: each draft is certain) bfloat16 or
    float32, of which the first vocab (default ld) entries of a row are tokens; draft_tokens int32
    [B, D], row b of which the first draft_len[b] (default D) count; u float32 [B, D] uniform in
    [0, 1); noise float32 [B, vocab] exponential; temperature float32 [B] (default 1, 0: greedy).
    Returns tokens int32 [B, D + 1] (the accepted drafts, the drawn token, then -1) and count int32
    [B], the number of tokens of each row: the lengths to replay a chunk with."""
    import torch
    if target_logits is None or target_logits.dim() != 3 or target_logits.shape[1] < 1:
        raise ValueError("target_logits must be a [B, D + 1, vocab] tensor")
    B, D1, ld = target_logits.shape
    D = D1 - 1
    dtype = target_logits.dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("logits must be bfloat16 or float32")
    V = ld if vocab is None else int(vocab)
    if not 1 <= V <= ld:
        raise ValueError(f"vocab {V} is outside 1 .. {ld}")
    i32, f32 = torch.int32, torch.float32
    opt = lambda name, t, shape, dt: None if t is None else _given(name, t, shape, dt)
    target = _given("target_logits", target_logits, target_logits.shape, dtype)
    draft = opt("draft_logits", draft_logits, (B, D, ld), dtype)
    drafted = _given("draft_tokens", draft_tokens, (B, D), i32) if D else None
    uniform = _given("u", u, (B, D), f32) if D else None
    args = [target, draft if D else None, IN_BF16 if dtype == torch.bfloat16 else IN_FP32, ld, V, drafted,
            opt("draft_len", draft_len, (B,), i32), D, uniform, _given("noise", noise, (B, V), f32),
            opt("temperature", temperature, (B,), f32), B]
    if tokens is None:
        tokens = _new((B, D1), i32, target_logits, stream)
    if count is None:
        count = _new((B,), i32, target_logits, stream)
    _check(lib().damp_verify_drafts(*args, _given("tokens", tokens, (B, D1), i32), _given("count", count, (B,), i32),
                                    _stream(stream)), "damp_verify_drafts")
    return tokens, count


_cache_layouts = {}


@dataclass(frozen=True)
class CacheLayout:
    """damp_cache_layout: query heads, KV heads (a divisor of them) and the head dimension (64, 128 or
    256) of a softmax-attention layer."""
    num_heads: int
    num_kv_heads: int
    d: int

    def __post_init__(self):
        # what every call needs of the layout, made once for equal ones: the struct, a reference to it, and the
        # sizes of the workspaces by device, batch, tokens, table and type
        key = (self.num_heads, self.num_kv_heads, self.d)
        shared = _cache_layouts.get(key)
        if shared is None:
            c = DampCacheLayout(*key)
            shared = _cache_layouts[key] = (c, ctypes.byref(c), {})
        object.__setattr__(self, "_shared", shared)

    def __reduce__(self):  # copies and pickles: the reference to the struct is not for them
        return CacheLayout, (self.num_heads, self.num_kv_heads, self.d)

    def c(self) -> DampCacheLayout:
        return self._shared[0]

    @property
    def record_bytes(self) -> int:
        """Bytes of a page of one KV head."""
        return 2 * CACHE_PAGE * self.d + 16


def cache_page_bytes(layout: CacheLayout) -> int:
    """Bytes of a page, all KV heads; 0 if the layout is invalid."""
    return int(lib().damp_cache_page_bytes(layout._shared[1]))


def new_cache(layout: CacheLayout, num_pages: int, device="cuda"):
    """A zeroed pool uint8 [num_pages, num_kv_heads, record_bytes] of pages of CACHE_PAGE tokens."""
    import torch
    return torch.zeros((num_pages, layout.num_kv_heads, layout.record_bytes), dtype=torch.uint8, device=device)


def _token_rows(name, t, shape, dtype, device):
    """(address, elements from token to token) of t [B, T, H, d] on the device: a tensor whose tokens are evenly
    spaced (contiguous, or a slice of the heads of a larger projection)."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.shape != shape or t.dtype != dtype:
        _want(name, t, shape, dtype=dtype)
    if t.get_device() != device:
        _wrong_device(name, t, device)
    B, T, H, d = shape
    if B * T > 0x7fffffff:
        raise ValueError(f"{name} holds more than 2^31 - 1 tokens")
    if t.is_contiguous():
        return t.data_ptr(), H * d
    sb, st, sh, sd = t.stride()
    step = st if T > 1 else sb
    if (sd != 1 and d > 1) or (sh != d and H > 1) or (T > 1 and B > 1 and sb != T * st) or step < H * d:
        raise ValueError(f"{name} must hold whole contiguous tokens [heads, d] at an even distance")
    return t.data_ptr(), step


def _wrong_device(name, t, device):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    raise ValueError(f"{name} lies on device {t.get_device()}, the current device is {device}")


def _here(name, t, shape, dtype, device):
    """As _given, for a tensor of the current device."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.shape != shape or t.dtype != dtype:
        _want(name, t, shape, dtype=dtype)
    if t.get_device() != device:
        _wrong_device(name, t, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _call_device(torch, first):
    """The current device (no call on it where there is none: the first tensor is then refused)."""
    if not first.is_cuda:
        return 0
    get = getattr(torch._C, "_cuda_getDevice", None)  # current_device() costs a microsecond
    return torch.cuda.current_device() if get is None else get()


def _raw_stream(torch, stream, device):
    if stream is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(device)
    return _stream(stream)


def _output(torch, like, contiguous, stream):
    """An uninitialized contiguous tensor of like's shape and type (empty_like costs half of what empty does)."""
    if stream is not None:
        return _new(like.shape, like.dtype, like, stream)
    return torch.empty_like(like) if contiguous else torch.empty_like(like, memory_format=torch.contiguous_format)


def rotary_frequencies(dim, base=10000.0, scaling="none", factor=1.0, trained=4096, turns=(32.0, 1.0), device="cuda"):
    """(freq, scale) for rotary: float64 [dim / 2] radians per position, base^(-2 i / dim), and the factor
    of the rotated part.  For contexts `factor` times the `trained` length: "linear" divides every
    frequency by factor; "ntk" raises the base to base factor^(dim / (dim - 2)), which divides the lowest
    by factor and leaves the highest; "yarn" divides those that make fewer than turns[1] turns within the
    trained length, keeps those that make more than turns[0], mixes linearly in i between the two, and
    gives the scale 0.1 ln(factor) + 1."""
    import math

    import torch
    if dim < 2 or dim % 2:
        raise ValueError("dim must be even, 2 at least")
    if not base > 1 or not factor >= 1:
        raise ValueError("base must be above 1, factor 1 at least")
    i = torch.arange(dim // 2, dtype=torch.float64)
    if scaling == "ntk":
        if dim == 2:
            raise ValueError("ntk scaling needs a dim above 2")
        base = base * factor ** (dim / (dim - 2))
    freq, scale = base ** (-2.0 * i / dim), 1.0
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "yarn":
        at = [dim * math.log(trained / (2 * math.pi * n)) / (2 * math.log(base)) for n in turns]
        low, high = max(math.floor(at[0]), 0), min(math.ceil(at[1]), dim - 1)
        stretched = ((i - low) / max(high - low, 0.001)).clamp(0, 1)
        freq = freq * (1 - stretched) + freq / factor * stretched
        scale = 0.1 * math.log(factor) + 1.0
    elif scaling not in ("none", "ntk"):
        raise ValueError("scaling must be none, linear, ntk or yarn")
    return freq.to(device), scale


def rotary(q, k, positions, freq, interleaved=False, scale=1.0, q_out=None, k_out=None, stream=None):
    """Rotary positions: q [B, T, H, d] and k [B, T, H_kv, d] (or None) bfloat16 or float32, of each head the
    first 2 len(freq) values turned by position * freq (float64, rotary_frequencies) and multiplied by scale,
    the others copied.  positions int32 [B, T], or [B]: of the first token of each row.  q and k may be
    slices of the heads of one projection.  Returns (q, k) rotated, contiguous; q_out and k_out may be
    q and k themselves where those are contiguous."""
    import torch
    if q is None or q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("q and k must be [B, T, heads, d] tensors")
    if freq is None or freq.dim() != 1:
        raise ValueError("freq must be a float64 tensor [rotary_dim / 2]")
    if positions is None or positions.dim() not in (1, 2):
        raise ValueError("positions must be an int32 tensor [B, T] or [B]")
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    dtype, dev = q.dtype, _call_device(torch, q)
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError("q must be bfloat16 or float32")
    shape = q.shape
    B, T, H, d = shape
    per_row = positions.dim() == 1
    qp, qs = _token_rows("q", q, shape, dtype, dev)
    if q_out is None:
        q_out = _output(torch, q, qs == H * d, stream)
        qo = q_out.data_ptr()
    else:
        qo = _here("q_out", q_out, shape, dtype, dev)
    kp = ko = None
    Hk = ks = 0
    if k is not None:
        Hk = k.shape[2]
        k_shape = (B, T, Hk, d)
        kp, ks = _token_rows("k", k, k_shape, dtype, dev)
        if k_out is None:
            k_out = _output(torch, k, ks == Hk * d, stream)
            ko = k_out.data_ptr()
        else:
            ko = _here("k_out", k_out, k_shape, dtype, dev)
    r = freq.shape[0]
    status = lib().damp_rotary(qp, qs, H, kp, ks, Hk, d, IN_BF16 if dtype == torch.bfloat16 else IN_FP32,
                               _here("positions", positions, (B,) if per_row else (B, T), torch.int32, dev), per_row, B, T,
                               _here("freq", freq, (r,), torch.float64, dev), 2 * r, bool(interleaved), scale, qo, ko,
                               _raw_stream(torch, stream, dev))
    if status:
        raise DampError(status, "damp_rotary")
    return q_out, k_out


def _cache(layout, cache, pages, B, dev, i32, u8):
    """(pool address, pages, table address, entries of a row) of a cache and its page table."""
    if cache is None or cache.dim() != 3:
        raise ValueError("cache must be a [num_pages, num_kv_heads, record_bytes] tensor")
    if pages is None or pages.dim() != 2:
        raise ValueError("pages must be an int32 tensor [B, pages of a row]")
    n, W = cache.shape[0], pages.shape[1]
    if W > 1 << 25:
        raise ValueError("pages holds more than 2^25 pages of a row")
    return (_here("cache", cache, (n, layout.num_kv_heads, 2 * CACHE_PAGE * layout.d + 16), u8, dev), n,
            _here("pages", pages, (B, W), i32, dev), W)


def cache_append(layout, cache, k, v, pages, start, lengths=None, stream=None):
    """Write new tokens into the 8-bit cache (in place): k, v [B, T, H_kv, d] bfloat16 or float32; token t of
    row b becomes token start[b] + t of the row (start int32 [B]: the tokens it holds), whose page is
    pages[b, (start[b] + t) // CACHE_PAGE] (int32 [B, W]).  Row b has lengths[b] new tokens (default T).
    k and v may be slices of the heads of one projection.  The pages written must be distinct.

    Tokens are taken back by a smaller start; the page that then is open keeps the scale that they gave it, and its
    codes the rounding.  To leave no trace of them (a rejected draft), copy that page before (copy_slots) and
    put it back."""
    import torch
    if k is None or k.dim() != 4:
        raise ValueError("k must be a [B, T, num_kv_heads, d] tensor")
    dtype, dev, i32 = k.dtype, _call_device(torch, k), torch.int32
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError("k must be bfloat16 or float32")
    B, T = k.shape[0], k.shape[1]
    shape = (B, T, layout.num_kv_heads, layout.d)
    kp, ks = _token_rows("k", k, shape, dtype, dev)
    vp, vs = _token_rows("v", v, shape, dtype, dev)
    pool, n, table, W = _cache(layout, cache, pages, B, dev, i32, torch.uint8)
    status = lib().damp_cache_append(layout._shared[1], pool, n, table, W, B, T, _here("start", start, (B,), i32, dev),
                                     None if lengths is None else _here("lengths", lengths, (B,), i32, dev), kp, ks, vp, vs,
                                     IN_BF16 if dtype == torch.bfloat16 else IN_FP32, _raw_stream(torch, stream, dev))
    if status:
        raise DampError(status, "damp_cache_append")


def cache_read(layout, cache, pages, lengths, tokens, start=None, dtype=None, k=None, v=None, stream=None):
    """Read values back: k, v [B, tokens, H_kv, d] of dtype (default bfloat16) hold tokens start[b] ..
    start[b] + tokens - 1 of each row (start int32 [B], default 0), zeros from lengths[b] on (the tokens
    that row b holds)."""
    import torch
    if cache is None:
        raise ValueError("cache is required")
    if pages is None or pages.dim() != 2:
        raise ValueError("pages must be an int32 tensor [B, pages of a row]")
    B, T, dev, i32 = pages.shape[0], int(tokens), _call_device(torch, cache), torch.int32
    if T < 0:
        raise ValueError("tokens must not be negative")
    if dtype is None:
        dtype = torch.bfloat16 if k is None else k.dtype
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError("dtype must be bfloat16 or float32")
    pool, n, table, W = _cache(layout, cache, pages, B, dev, i32, torch.uint8)
    held = _here("lengths", lengths, (B,), i32, dev)
    shape = (B, T, layout.num_kv_heads, layout.d)
    if k is None:
        k = _new(shape, dtype, cache, stream)
    kp = _here("k", k, shape, dtype, dev)
    if v is None:
        v = _output(torch, k, True, stream)
    vp = _here("v", v, shape, dtype, dev)
    status = lib().damp_cache_read(layout._shared[1], pool, n, table, W, B, T, None if start is None else _here("start", start, (B,), i32, dev),
                                   held, kp, vp, IN_BF16 if dtype == torch.bfloat16 else IN_FP32, _raw_stream(torch, stream, dev))
    if status:
        raise DampError(status, "damp_cache_read")
    return k, v


def _attend_workspace(layout, key):
    """Bytes of cache_attend's workspace for key (device, B, T, W, type), kept for the next call: 1024 of them at most."""
    sizes = layout._shared[2]
    if len(sizes) >= 1024:
        sizes.clear()
    need = sizes[key] = int(lib().damp_cache_attend_workspace(layout._shared[1], *key[1:]))
    return need


def cache_attend(layout, cache, q, pages, lengths, q_lengths=None, scale=None, window=None, o=None, stream=None):
    """Attention over the 8-bit cache: q [B, T, H, d] bfloat16 or float32; row b holds lengths[b] tokens
    (int32 [B]), the last q_lengths[b] (default T) of which are its queries' own: query t is token
    j = lengths[b] - q_lengths[b] + t and sees tokens up to j, the last `window` of them if given.
    scale: of q.k (default d^-1/2).  Returns o [B, T, H, d] of q's type, zeros past q_lengths[b].  T = 1 is a
    decode step, a few tokens a draft, many a prompt (append their keys and values first)."""
    import torch
    if q is None or q.dim() != 4:
        raise ValueError("q must be a [B, T, num_heads, d] tensor")
    if window is not None and window < 1:
        raise ValueError("window must be 1 at least")
    dtype, dev, i32 = q.dtype, _call_device(torch, q), torch.int32
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError("q must be bfloat16 or float32")
    B, T, d = q.shape[0], q.shape[1], layout.d
    shape, dt = (B, T, layout.num_heads, d), IN_BF16 if dtype == torch.bfloat16 else IN_FP32
    qp, qs = _token_rows("q", q, shape, dtype, dev)
    pool, n, table, W = _cache(layout, cache, pages, B, dev, i32, torch.uint8)
    held = _here("lengths", lengths, (B,), i32, dev)
    if o is None:
        o = _output(torch, q, qs == layout.num_heads * d, stream)
        op = o.data_ptr()
    else:
        op = _here("o", o, shape, dtype, dev)
    L = lib()
    need = layout._shared[2].get((dev, B, T, W, dt))
    if need is None:
        need = _attend_workspace(layout, (dev, B, T, W, dt))
    ws = None
    if need:
        ws = q.new_empty(need // (4 if dt else 2)) if stream is None else _new((need,), torch.uint8, q, stream)
    status = L.damp_cache_attend(layout._shared[1], pool, n, table, W, B, T, held,
                                 None if q_lengths is None else _here("q_lengths", q_lengths, (B,), i32, dev), qp, qs,
                                 d ** -0.5 if scale is None else scale, 0 if window is None else min(window, 0x7fffffff), op, dt,
                                 None if ws is None else ws.data_ptr(), need, _raw_stream(torch, stream, dev))
    if status:
        raise DampError(status, "damp_cache_attend")
    return o


def test_cache_attend_wait_timeout(layout, cache, q, pages, lengths, o, queries=False):
    """The bounded-wait test hook of cache_attend (damp_test_cache_attend_wait_timeout): in every second range of the work
    the waits for pages (or for queries) run out after 10 ms.  For tests of the timeout path only."""
    import torch
    B, T, dt = q.shape[0], q.shape[1], IN_BF16 if q.dtype == torch.bfloat16 else IN_FP32
    dev = _call_device(torch, q)
    shape = (B, T, layout.num_heads, layout.d)
    pool, n, table, W = _cache(layout, cache, pages, B, dev, torch.int32, torch.uint8)
    need = lib().damp_cache_attend_workspace(layout._shared[1], B, T, W, dt)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    status = lib().damp_test_cache_attend_wait_timeout(
        layout._shared[1], pool, n, table, W, B, T, _here("lengths", lengths, (B,), torch.int32, dev), None,
        _here("q", q, shape, q.dtype, dev), layout.num_heads * layout.d, layout.d ** -0.5, 0, _here("o", o, shape, q.dtype, dev), dt,
        ws.data_ptr(), need, bool(queries), _raw_stream(torch, None, dev))
    if status:
        raise DampError(status, "damp_test_cache_attend_wait_timeout")


def device_status() -> int:
    """Read and clear the device status word (DEV_* bits)."""
    v = ctypes.c_uint32(0)
    _check(lib().damp_device_status(ctypes.byref(v)), "damp_device_status")
    return int(v.value)
