"""Thin ctypes binding over libmoa.so (the C ABI declared in include/moa.h).

Argument marshalling only: torch provides device memory and streams, every step
of the drafter forward runs in the library's CUDA kernels. There is no CPU or
PyTorch fallback: if the library is missing or no sm_100 GPU is present, the
calls fail loudly.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import build as _build

MOA_MAX_BATCH = 64
STATUS_NAMES = ["OK", "ERR_NULL", "ERR_SHAPE", "ERR_DTYPE", "ERR_ALIGN", "ERR_WORKSPACE", "ERR_CAPACITY",
                "ERR_STATE", "ERR_ARCH", "ERR_CUDA", "ERR_TIMEOUT"]
MOA_OK = 0

EXPORTS = ["moa_create", "moa_destroy", "moa_tli_configure", "moa_state_bytes", "moa_status_str", "moa_last_cuda_error",
           "moa_state_set_len", "moa_lsa_forward", "moa_sa_append", "moa_sa_append_static", "moa_drafter_prefill", "moa_tree_begin", "moa_draft_step",
           "moa_tree_expand", "moa_tree_attn_mask", "moa_verify_greedy", "moa_pack_tree", "moa_unpack_tree", "moa_quantize_rows", "moa_dequantize_rows",
           "moa_paged_workspace_bytes", "moa_paged_append", "moa_paged_attention", "moa_paged_commit", "moa_paged_evict_workspace_bytes",
           "moa_paged_evict", "moa_token_record", "moa_logit_rules", "moa_verify_greedy_rules", "moa_state_status", "moa_profile_begin", "moa_profile_end", "moa_profile_phases",
           "moa_launch_count", "moa_trace_begin", "moa_trace_end"]


class MoaConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "d_model", "n_stack", "d_stack", "vocab", "head_dim", "lsa_hq", "lsa_hkv", "lsa_mlp",
        "sa_hq", "sa_hkv", "sa_mlp", "ca_hq", "ca_hkv", "ca_mlp", "max_batch", "max_ctx",
        "tree_topk", "tree_depth", "tree_keep")] + [("rms_eps", C.c_float), ("sa_rope_theta", C.c_float),
                                                    ("dtype", C.c_int32)]


WEIGHT_FIELDS = ["embed", "lm_head", "final_norm",
                 "lsa_norm1", "lsa_wq", "lsa_wk", "lsa_wv", "lsa_wo", "lsa_norm2", "lsa_wgate", "lsa_wup", "lsa_wdown",
                 "sa_norm1", "sa_wq", "sa_wk", "sa_wv", "sa_wo", "sa_norm2", "sa_wgate", "sa_wup", "sa_wdown",
                 "ca_normq", "ca_normkv", "ca_wq", "ca_wk", "ca_wv", "ca_wo", "ca_norm2", "ca_wgate", "ca_wup",
                 "ca_wdown"]


class MoaWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_FIELDS]


MOA_MAX_TLI = 4
TLI_LAYER_FIELDS = ["norm1", "wq", "wk", "wv", "wo", "norm2", "wgate", "wup", "wdown"]


class MoaTliConfig(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hq", C.c_int32), ("hkv", C.c_int32), ("mlp", C.c_int32),
                ("rope_theta", C.c_float)]


class MoaTliLayer(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in TLI_LAYER_FIELDS]


class MoaTliCaches(C.Structure):
    _fields_ = [("k", C.c_void_p * MOA_MAX_TLI), ("v", C.c_void_p * MOA_MAX_TLI)]


class MoaState(C.Structure):
    _fields_ = [("ca_k", C.c_void_p), ("ca_v", C.c_void_p), ("sa_k", C.c_void_p), ("sa_v", C.c_void_p),
                ("ca_len", C.c_void_p), ("sa_len", C.c_void_p), ("tree", C.c_void_p),
                ("ca_len_host", C.c_void_p), ("sa_len_host", C.c_void_p), ("step", C.c_int32)]


class MoaPagedCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64)] + [
        (n, C.c_void_p) for n in ("page_table", "len", "weight", "pos", "seen")] + [
        (n, C.c_int32) for n in ("batch", "max_pages", "n_pages", "page_size", "hkv", "head_dim", "dtype")]


class MoaLogitRuleSet(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("counts", "seen", "repetition", "frequency", "presence", "bias_id", "bias_value",
                                          "allow")] + [("n_bias", C.c_int32)]


class MoaError(RuntimeError):
    def __init__(self, status: int, what: str, detail: str = ""):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{what}: MOA_{name}" + (f" ({detail})" if detail else ""))


_lib = None


def lib_path() -> str:
    return _build.LIB


def load_library(rebuild_if_stale: bool = True) -> C.CDLL:
    """Loads libmoa.so, building it first if it is missing or older than its sources and nvcc is around."""
    global _lib
    if _lib is not None:
        return _lib
    trace = os.environ.get("MOA_TRACE_BUILD", "") == "1"          # the variant whose kernels stamp the stage trace
    checks = os.environ.get("MOA_CHECKS_BUILD", "") == "1"        # the debug variant with device-side index checks
    path = _build.LIB_TRACE if trace else _build.LIB_CHECKS if checks else _build.LIB
    if rebuild_if_stale and (os.path.exists("/usr/local/cuda/bin/nvcc") or os.environ.get("NVCC")):
        path = _build.build(trace=trace, checks=checks)
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found: build it with `python -m paper_2410_03804_b200.build`")
    lib = C.CDLL(path)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    lib.moa_create.argtypes = [C.POINTER(MoaConfig), C.POINTER(MoaWeights), C.POINTER(vp)]
    lib.moa_destroy.argtypes = [vp]
    lib.moa_destroy.restype = None
    lib.moa_state_bytes.argtypes = [vp, i32, C.POINTER(sz), C.POINTER(sz)]
    lib.moa_status_str.argtypes = [i32]
    lib.moa_status_str.restype = C.c_char_p
    lib.moa_last_cuda_error.argtypes = []
    lib.moa_last_cuda_error.restype = C.c_char_p
    lib.moa_tli_configure.argtypes = [vp, C.POINTER(MoaTliConfig), vp, C.POINTER(MoaTliCaches)]
    lib.moa_state_set_len.argtypes = [vp, C.POINTER(MoaState), i32, vp, i32, vp]
    lib.moa_lsa_forward.argtypes = [vp, C.POINTER(MoaState), vp, vp, i32, vp, vp, sz, vp]
    lib.moa_sa_append.argtypes = [vp, C.POINTER(MoaState), vp, vp, i32, vp, sz, vp]
    lib.moa_drafter_prefill.argtypes = [vp, C.POINTER(MoaState), vp, vp, i32, vp, vp, vp, sz, vp]
    lib.moa_sa_append_static.argtypes = [vp, C.POINTER(MoaState), vp, vp, i32, vp]
    lib.moa_tree_begin.argtypes = [vp, C.POINTER(MoaState), vp, i32, vp]
    lib.moa_draft_step.argtypes = [vp, C.POINTER(MoaState), i32, vp, vp, vp, vp, sz, vp]
    lib.moa_tree_expand.argtypes = [vp, C.POINTER(MoaState), i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.moa_tree_attn_mask.argtypes = [vp, i32, i32, vp, i32, vp]
    lib.moa_verify_greedy.argtypes = [vp, vp, i32, i32, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.moa_pack_tree.argtypes = [vp, vp, C.c_int64, vp, vp]
    lib.moa_unpack_tree.argtypes = [vp, C.c_int64, vp, vp, vp]
    lib.moa_quantize_rows.argtypes = [vp, i32, C.c_int64, i32, vp, vp, vp]
    lib.moa_dequantize_rows.argtypes = [vp, vp, C.c_int64, i32, vp, i32, vp]
    lib.moa_paged_workspace_bytes.argtypes = [vp, i32, i32, i32, C.POINTER(sz)]
    lib.moa_paged_append.argtypes = [vp, vp, vp, C.c_int64, i32, vp, vp]
    lib.moa_paged_attention.argtypes = [vp, vp, C.c_int64, vp, vp, C.c_int64, i32, i32, i32, vp, C.c_float, vp, vp, vp, sz, vp]
    lib.moa_paged_commit.argtypes = [vp, i32, vp, vp, i32, i32, vp]
    lib.moa_paged_evict_workspace_bytes.argtypes = [vp, i32, C.POINTER(sz)]
    lib.moa_paged_evict.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.moa_token_record.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp]
    lib.moa_logit_rules.argtypes = [vp, vp, vp, i32, i32, vp, i32, i32, vp, vp, vp]
    lib.moa_verify_greedy_rules.argtypes = [vp, vp, vp, i32, i32, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.moa_state_status.argtypes = [vp, C.POINTER(MoaState), vp]
    lib.moa_profile_begin.argtypes = [vp]
    lib.moa_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i32)]
    lib.moa_profile_phases.argtypes = [vp, vp, sz, i32, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(i32),
                                       C.POINTER(i32), vp]
    lib.moa_launch_count.argtypes = []
    lib.moa_trace_begin.argtypes = [vp, i32]
    lib.moa_trace_end.argtypes = [C.POINTER(i32)]
    for n in EXPORTS:
        if n not in ("moa_destroy", "moa_status_str", "moa_last_cuda_error", "moa_launch_count"):
            getattr(lib, n).restype = i32
    lib.moa_launch_count.restype = C.c_int64
    _lib = lib
    return lib


def _check(status: int, what: str):
    if status != MOA_OK:
        detail = load_library().moa_last_cuda_error().decode() if status in (5, 9) else ""
        raise MoaError(status, what, detail)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _host_i32(vals):
    arr = (C.c_int32 * len(vals))(*[int(v) for v in vals])
    return arr


def moa_tree_attn_mask(parent: torch.Tensor, packed: bool = False, stream=None) -> torch.Tensor:
    """Ancestor-or-self mask of a batch of trees. parent: int32 cuda [batch, n]."""
    assert parent.is_cuda and parent.dtype == torch.int32 and parent.dim() == 2 and parent.is_contiguous()
    batch, n = parent.shape
    if packed:
        out = torch.empty((batch, n, (n + 63) // 64), dtype=torch.int64, device=parent.device)
    else:
        out = torch.empty((batch, n, n), dtype=torch.uint8, device=parent.device)
    st = load_library().moa_tree_attn_mask(_ptr(parent), batch, n, _ptr(out) if out.numel() else C.c_void_p(16),
                                           1 if packed else 0, _stream(stream))
    _check(st, "moa_tree_attn_mask")
    return out


def moa_verify_greedy(tok: torch.Tensor, parent: torch.Tensor, target_logits: torch.Tensor, cap: int, out=None,
                      stream=None):
    """tok, parent: cuda int32 [batch, n] (the kept tree); target_logits: cuda float32 / bfloat16 [batch, n, V].
    Returns (choice [batch, n], acc_slot [batch, cap], acc_tok [batch, cap], acc_len [batch], next_tok [batch]);
    out: the same five int32 tensors preallocated by the caller."""
    assert tok.is_cuda and tok.dtype == torch.int32 and tok.is_contiguous() and tok.dim() == 2
    assert parent.is_cuda and parent.dtype == torch.int32 and parent.is_contiguous() and parent.shape == tok.shape
    assert target_logits.is_cuda and target_logits.is_contiguous() and target_logits.shape[:2] == tok.shape
    assert target_logits.dtype in (torch.float32, torch.bfloat16)
    b, n = tok.shape
    dev = tok.device
    if out is not None:
        choice, acc_slot, acc_tok, acc_len, next_tok = out
    else:
        choice = torch.empty((b, n), dtype=torch.int32, device=dev)
        acc_slot = torch.empty((b, cap), dtype=torch.int32, device=dev)
        acc_tok = torch.empty((b, cap), dtype=torch.int32, device=dev)
        acc_len = torch.empty((b,), dtype=torch.int32, device=dev)
        next_tok = torch.empty((b,), dtype=torch.int32, device=dev)
    _check(load_library().moa_verify_greedy(_ptr(tok), _ptr(parent), b, n, _ptr(target_logits),
                                            0 if target_logits.dtype == torch.float32 else 1, target_logits.shape[2],
                                            int(cap), _ptr(choice), _ptr(acc_slot), _ptr(acc_tok), _ptr(acc_len),
                                            _ptr(next_tok), _stream(stream)), "moa_verify_greedy")
    return choice, acc_slot, acc_tok, acc_len, next_tok


def moa_pack_tree(tok: torch.Tensor, parent: torch.Tensor, stream=None) -> torch.Tensor:
    """cuda int32 [..., n] token ids and parent slots -> cuda uint8 [..., n, 4] (the client's 4-bytes-per-node message)."""
    assert tok.is_cuda and tok.dtype == torch.int32 and tok.is_contiguous() and parent.shape == tok.shape
    assert parent.is_cuda and parent.dtype == torch.int32 and parent.is_contiguous()
    msg = torch.empty(tuple(tok.shape) + (4,), dtype=torch.uint8, device=tok.device)
    _check(load_library().moa_pack_tree(_ptr(tok), _ptr(parent), tok.numel(), _ptr(msg), _stream(stream)), "moa_pack_tree")
    return msg


def moa_unpack_tree(msg: torch.Tensor, stream=None):
    assert msg.is_cuda and msg.dtype == torch.uint8 and msg.is_contiguous() and msg.shape[-1] == 4
    tok = torch.empty(tuple(msg.shape[:-1]), dtype=torch.int32, device=msg.device)
    parent = torch.empty_like(tok)
    _check(load_library().moa_unpack_tree(_ptr(msg), tok.numel(), _ptr(tok), _ptr(parent), _stream(stream)), "moa_unpack_tree")
    return tok, parent


def moa_quantize_rows(x: torch.Tensor, out=None, stream=None):
    """x cuda float32 / bfloat16 [rows, width] -> (int8 codes [rows, width], float32 scales [rows])."""
    assert x.is_cuda and x.is_contiguous() and x.dim() == 2 and x.dtype in (torch.float32, torch.bfloat16)
    codes, scales = out if out is not None else (torch.empty(x.shape, dtype=torch.int8, device=x.device),
                                                 torch.empty((x.shape[0],), dtype=torch.float32, device=x.device))
    _check(load_library().moa_quantize_rows(_ptr(x), 0 if x.dtype == torch.float32 else 1, x.shape[0], x.shape[1],
                                            _ptr(codes), _ptr(scales), _stream(stream)), "moa_quantize_rows")
    return codes, scales


def moa_dequantize_rows(codes: torch.Tensor, scales: torch.Tensor, dtype=torch.float32, out=None, stream=None):
    assert codes.is_cuda and codes.dtype == torch.int8 and codes.is_contiguous() and codes.dim() == 2
    assert scales.is_cuda and scales.dtype == torch.float32 and scales.numel() == codes.shape[0]
    if out is None:
        out = torch.empty(codes.shape, dtype=dtype, device=codes.device)
    _check(load_library().moa_dequantize_rows(_ptr(codes), _ptr(scales), codes.shape[0], codes.shape[1], _ptr(out),
                                              0 if out.dtype == torch.float32 else 1, _stream(stream)), "moa_dequantize_rows")
    return out


# The serving operators are called once per layer and token, so their checks read each attribute of a tensor once.
_raw_stream = torch._C._cuda_getCurrentRawStream


def _serving_call(index: int, stream, call, what: str, *args):
    """Makes a call of the serving operators with its tensors' device current, on the given or that device's current stream."""
    assert stream is None or stream.device_index == index, "the stream is of another device"
    if torch._C._cuda_getDevice() == index:
        status = call(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(index):
            status = call(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    if status != MOA_OK:
        _check(status, what)


def _made(make, stream):
    """A tensor that a call makes for itself: of the call's stream, so that its memory's earlier uses and its fill come before."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        t = make()
    t.record_stream(torch.cuda.current_stream(t.device))       # where a result is read afterwards
    return t


def _is(t: torch.Tensor, dtype, index: int) -> bool:
    """A contiguous tensor of a type on a device."""
    return t.dtype is dtype and t.get_device() == index and t.is_contiguous()


def _rows(t: torch.Tensor, batch: int, heads: int, head_dim: int, dtype, index: int, what: str):
    """Checks rows [batch, n, heads, head_dim] whose heads are contiguous; returns (n, elements between two rows)."""
    assert t.dim() == 4 and t.dtype is dtype and t.get_device() == index, what
    b, n, h, d = t.shape
    s0, s1, s2, s3 = t.stride()
    assert b == batch and h == heads and d == head_dim and n >= 1, what
    assert s3 == 1 and (s2 == head_dim or heads == 1), what + ": heads must be contiguous"
    if n == 1:
        return 1, s0 if batch > 1 else heads * head_dim
    assert batch == 1 or s0 == n * s1, what + ": rows must be evenly spaced"
    return n, s1


class PagedCache:
    """The key / value cache of one attention layer in pages (moa_paged_cache of include/moa.h). k, v: cuda float32 /
    bfloat16 [n_pages, page_size, hkv, head_dim], contiguous within a page (views of one block are fine); page_table: int32
    [batch, max_pages]; length: int32 [batch], committed slots, < 0 for a sequence not in use; weight, pos: float32 / int32
    [batch, hkv, max_pages * page_size] and seen: int32 [batch] for accumulated weights and eviction. The tensors are held,
    not copied; the caller fills the table."""

    def __init__(self, k, v, page_table, length, weight=None, pos=None, seen=None):
        assert k.is_cuda and k.dim() == 4 and k.dtype in (torch.float32, torch.bfloat16), "k: cuda [n_pages, page_size, hkv, head_dim]"
        dev, (n_pages, ps, hkv, dh) = k.device, k.shape
        at = k.get_device()
        assert v.get_device() == at and v.shape == k.shape and v.dtype == k.dtype and v.stride() == k.stride(), "v must be laid out as k"
        assert k.stride(3) == 1 and (hkv == 1 or k.stride(2) == dh) and (ps == 1 or k.stride(1) == hkv * dh), "a page must be contiguous"
        assert _is(page_table, torch.int32, at) and page_table.dim() == 2 and page_table.shape[1] >= 1, "page_table: int32 [batch, max_pages]"
        batch, per = page_table.shape
        assert _is(length, torch.int32, at) and length.shape == (batch,), "length: int32 [batch]"
        full = (batch, hkv, per * ps)
        assert weight is None or (_is(weight, torch.float32, at) and weight.shape == full), "weight: float32 [batch, hkv, slots]"
        assert pos is None or (_is(pos, torch.int32, at) and pos.shape == full), "pos: int32 [batch, hkv, slots]"
        assert seen is None or (_is(seen, torch.int32, at) and seen.shape == (batch,)), "seen: int32 [batch]"
        self.k, self.v, self.page_table, self.len, self.weight, self.pos, self.seen = k, v, page_table, length, weight, pos, seen
        self.device, self.dtype, self.batch, self.hkv, self.head_dim, self.slots = dev, k.dtype, batch, hkv, dh, per * ps
        self.index, self._full = at, torch.Size(full)
        self.c = MoaPagedCache(k.data_ptr(), v.data_ptr(), k.stride(0) if n_pages > 1 else ps * hkv * dh, page_table.data_ptr(),
                               length.data_ptr(), weight.data_ptr() if weight is not None else None,
                               pos.data_ptr() if pos is not None else None, seen.data_ptr() if seen is not None else None, batch,
                               per, n_pages, ps, hkv, dh, 0 if k.dtype == torch.float32 else 1)
        self._ref = C.addressof(self.c)

    def _scratch(self, status_of, what: str) -> int:
        n = C.c_size_t()
        with torch.cuda.device(self.device):
            _check(status_of(C.byref(n)), what)
        return n.value

    def workspace(self, n: int, hq: int, weights: bool = False) -> torch.Tensor:
        """Scratch for moa_paged_attention with n rows per sequence and hq query heads (zeroed, as its first call needs it)."""
        lib = load_library()
        return torch.zeros(self._scratch(lambda b: lib.moa_paged_workspace_bytes(self._ref, n, hq, 1 if weights else 0, b),
                                         "moa_paged_workspace_bytes"), dtype=torch.uint8, device=self.device)

    def evict_workspace(self, budget: int) -> torch.Tensor:
        """Scratch for moa_paged_evict."""
        lib = load_library()
        return torch.empty(self._scratch(lambda b: lib.moa_paged_evict_workspace_bytes(self._ref, budget, b),
                                         "moa_paged_evict_workspace_bytes"), dtype=torch.uint8, device=self.device)

    def _own_scratch(self, ws, make, stream):
        if ws is None:
            ws = _made(make, stream)
        assert _is(ws, torch.uint8, self.index), "ws: cuda uint8, contiguous"
        return ws


def moa_paged_append(cache: PagedCache, k_new: torch.Tensor, v_new: torch.Tensor, n_new=None, stream=None):
    """Writes rows [batch, n, hkv, head_dim] behind the committed slots (the first n_new[b] of each sequence), without
    committing them."""
    at, b, hkv, dh, dt = cache.index, cache.batch, cache.hkv, cache.head_dim, cache.dtype
    n, step = _rows(k_new, b, hkv, dh, dt, at, "k_new")
    assert _rows(v_new, b, hkv, dh, dt, at, "v_new") == (n, step), "v_new must be laid out as k_new"
    assert n_new is None or (_is(n_new, torch.int32, at) and n_new.shape == (b,)), "n_new: int32 [batch]"
    _serving_call(at, stream, load_library().moa_paged_append, "moa_paged_append", cache._ref, k_new.data_ptr(), v_new.data_ptr(), step, n,
                  None if n_new is None else n_new.data_ptr())


def moa_paged_attention(cache: PagedCache, q: torch.Tensor, k_new=None, v_new=None, mask=None, scale: float = 0.0,
                        new_rows: bool = True, out=None, weight_out=None, ws=None, stream=None) -> torch.Tensor:
    """Attention of q [batch, n, hq, head_dim] over the cache and the n new rows (k_new, v_new [batch, n, hkv, head_dim] are
    appended by the call; without them the rows are in the pages already; new_rows=False: there are none). mask: int64
    [batch, n] or [batch, n, 1], one packed word per row as moa_tree_attn_mask(packed=True) gives it; None: causal.
    weight_out (n = 1): float32 [batch, hkv, slots], may be cache.weight. Returns out [batch, n, hq, head_dim]."""
    at, b, hkv, dh, dt = cache.index, cache.batch, cache.hkv, cache.head_dim, cache.dtype
    assert q.dim() == 4, "q: [batch, n, hq, head_dim]"
    hq = q.shape[2]
    n, q_step = _rows(q, b, hq, dh, dt, at, "q")
    kp = vp = mp = wp = None
    new_step = 0
    assert (k_new is None) == (v_new is None), "k_new and v_new come together"
    if k_new is not None:
        assert new_rows, "k_new and v_new are new rows"
        m, new_step = _rows(k_new, b, hkv, dh, dt, at, "k_new")
        assert m == n and _rows(v_new, b, hkv, dh, dt, at, "v_new") == (n, new_step), "v_new must be laid out as k_new, with q's rows"
        kp, vp = k_new.data_ptr(), v_new.data_ptr()
    if mask is not None:
        assert (_is(mask, torch.int64, at) or _is(mask, torch.uint64, at)) and mask.numel() == b * n, "mask: int64 [batch, n]"
        mp = mask.data_ptr()
    if out is None:
        out = _made(lambda: torch.empty((b, n, hq, dh), dtype=dt, device=cache.device), stream)
    else:
        assert _is(out, dt, at) and out.shape == q.shape, "out: [batch, n, hq, head_dim]"
    if weight_out is not None:
        assert _is(weight_out, torch.float32, at) and weight_out.shape == cache._full, "weight_out: float32 [batch, hkv, slots]"
        wp = weight_out.data_ptr()
    ws = cache._own_scratch(ws, lambda: cache.workspace(n, hq, wp is not None), stream)
    _serving_call(at, stream, load_library().moa_paged_attention, "moa_paged_attention", cache._ref, q.data_ptr(), q_step, kp, vp, new_step, n,
                  n if new_rows else 0, hq, mp, scale, out.data_ptr(), wp, ws.data_ptr(), ws.numel())
    return out


def moa_paged_commit(cache: PagedCache, n: int, acc_slot=None, acc_len=None, advance: bool = True, stream=None):
    """Keeps the accepted path (acc_slot [batch, cap], acc_len [batch] of moa_verify_greedy) of n uncommitted rows, or all of
    them, and advances cache.len (and cache.seen) when asked to."""
    at, cap = cache.index, 0
    assert acc_len is None or (_is(acc_len, torch.int32, at) and acc_len.shape == (cache.batch,)), "acc_len: int32 [batch]"
    if acc_slot is not None:
        assert acc_len is not None and _is(acc_slot, torch.int32, at) and acc_slot.dim() == 2, "acc_slot: int32 [batch, cap]"
        b, cap = acc_slot.shape
        assert b == cache.batch, "acc_slot: int32 [batch, cap]"
    _serving_call(at, stream, load_library().moa_paged_commit, "moa_paged_commit", cache._ref, n, None if acc_slot is None else acc_slot.data_ptr(),
                  None if acc_len is None else acc_len.data_ptr(), cap, 1 if advance else 0)


def moa_paged_evict(cache: PagedCache, budget: int, sink: int = 4, recent: int = 64, weight_out=None, pos_out=None, len_out=None,
                    update_len: bool = True, ws=None, stream=None):
    """Cuts every sequence's heads to `budget` slots (see include/moa.h). weight_out and pos_out default to the cache's own;
    len_out to cache.len, or to nothing with update_len=False (layers that share len)."""
    assert cache.weight is not None and cache.pos is not None and cache.seen is not None, "the cache needs weight, pos and seen"
    at = cache.index
    w, p = cache.weight if weight_out is None else weight_out, cache.pos if pos_out is None else pos_out
    assert _is(w, torch.float32, at) and w.shape == cache._full, "weight_out: float32 [batch, hkv, slots]"
    assert _is(p, torch.int32, at) and p.shape == cache._full, "pos_out: int32 [batch, hkv, slots]"
    n = len_out if len_out is not None else cache.len if update_len else None
    assert n is None or (_is(n, torch.int32, at) and n.shape == (cache.batch,)), "len_out: int32 [batch]"
    ws = cache._own_scratch(ws, lambda: cache.evict_workspace(budget), stream)
    _serving_call(at, stream, load_library().moa_paged_evict, "moa_paged_evict", cache._ref, budget, sink, recent, w.data_ptr(), p.data_ptr(),
                  None if n is None else n.data_ptr(), ws.data_ptr(), ws.numel())


class LogitRules:
    """The rules of a batch of sequences (moa_logit_rule_set of include/moa.h); every tensor may be None. vocab: V; counts:
    int32 [batch, V]; seen: int32 [batch, ceil(V / 32)] bits; repetition, frequency, presence: float32 [batch]; bias_id,
    bias_value: int32 / float32 [batch, n_bias]; allow: int32 [batch, n, ceil(V / 32)] bits. The tensors are held, not
    copied: counts and seen may grow (moa_token_record) and penalties change between calls."""

    def __init__(self, vocab: int, counts=None, seen=None, repetition=None, frequency=None, presence=None, bias_id=None,
                 bias_value=None, allow=None):
        words = (vocab + 31) // 32
        given = [t for t in (counts, seen, repetition, frequency, presence, bias_id, bias_value, allow) if t is not None]
        assert (bias_id is None) == (bias_value is None), "bias_id and bias_value come together"
        self.index = given[0].get_device() if given else None
        self.batch = given[0].shape[0] if given else None
        self.rows = None if allow is None else allow.shape[1]
        n_bias = 0 if bias_id is None else bias_id.shape[1]
        for t, dt, shape, what in ((counts, torch.int32, (self.batch, vocab), "counts"), (seen, torch.int32, (self.batch, words), "seen"),
                                   (repetition, torch.float32, (self.batch,), "repetition"), (frequency, torch.float32, (self.batch,), "frequency"),
                                   (presence, torch.float32, (self.batch,), "presence"), (bias_id, torch.int32, (self.batch, n_bias), "bias_id"),
                                   (bias_value, torch.float32, (self.batch, n_bias), "bias_value"),
                                   (allow, torch.int32, (self.batch, self.rows, words), "allow")):
            assert t is None or (t.is_cuda and _is(t, dt, self.index) and t.shape == shape), what
        self.vocab, self.counts, self.seen, self.held = vocab, counts, seen, given
        p = lambda t: None if t is None or t.numel() == 0 else t.data_ptr()  # noqa: E731
        self.c = MoaLogitRuleSet(p(counts), p(seen), p(repetition), p(frequency), p(presence), p(bias_id), p(bias_value), p(allow), n_bias)
        self._ref = C.addressof(self.c)


def moa_token_record(tok: torch.Tensor, vocab: int, counts=None, seen=None, n_tok=None, stream=None):
    """Adds tokens tok int32 [batch, cap] (the first n_tok[b] of each sequence; ids outside 0..vocab-1 are left out) to the
    record: bits in seen, and numbers in counts (None for a prompt)."""
    assert tok.is_cuda and tok.dtype == torch.int32 and tok.dim() == 2 and tok.is_contiguous(), "tok: cuda int32 [batch, cap]"
    b, cap = tok.shape
    at = tok.get_device()
    assert counts is None or (_is(counts, torch.int32, at) and counts.shape == (b, vocab)), "counts: int32 [batch, vocab]"
    assert seen is None or (_is(seen, torch.int32, at) and seen.shape == (b, (vocab + 31) // 32)), "seen: int32 [batch, ceil(vocab / 32)]"
    assert n_tok is None or (_is(n_tok, torch.int32, at) and n_tok.shape == (b,)), "n_tok: int32 [batch]"
    _serving_call(at, stream, load_library().moa_token_record, "moa_token_record", *(None if t is None else t.data_ptr() for t in (counts, seen)),
                  b, vocab, tok.data_ptr(), None if n_tok is None else n_tok.data_ptr(), cap)


def _rule_rows(rules: LogitRules, logits: torch.Tensor, tok, parent):
    at, dt = logits.get_device(), logits.dtype
    assert at >= 0 and logits.is_contiguous() and logits.dim() == 3 and dt in (torch.float32, torch.bfloat16), "logits: cuda [batch, n, V]"
    b, n, v = logits.shape
    assert v == rules.vocab and rules.batch in (None, b) and rules.rows in (None, n), "the rules are of another batch"
    assert rules.index in (None, at), "the rules are on another device"
    assert (tok is None) == (parent is None), "tok and parent come together"
    if tok is not None:
        assert _is(tok, torch.int32, at) and tok.shape == (b, n), "tok: int32 [batch, n]"
        assert _is(parent, torch.int32, at) and parent.shape == (b, n), "parent: int32 [batch, n]"
    return at, b, n, v, 0 if dt is torch.float32 else 1


def moa_logit_rules(rules: LogitRules, logits: torch.Tensor, tok=None, parent=None, out=None, choice=None, stream=None):
    """Applies the rules to logits [batch, n, V]; tok, parent int32 [batch, n]: the kept tree whose slots the rows are.
    Returns (adjusted logits, arg-max int32 [batch, n]); out may be the logits themselves."""
    at, b, n, v, dt = _rule_rows(rules, logits, tok, parent)
    if out is None:
        out = _made(lambda: torch.empty_like(logits), stream)
    else:
        assert _is(out, logits.dtype, at) and out.shape == logits.shape, "out: as the logits"
    if choice is None:
        choice = _made(lambda: torch.empty((b, n), dtype=torch.int32, device=logits.device), stream)
    else:
        assert _is(choice, torch.int32, at) and choice.shape == (b, n), "choice: int32 [batch, n]"
    _serving_call(at, stream, load_library().moa_logit_rules, "moa_logit_rules", rules._ref, None if tok is None else tok.data_ptr(),
                  None if parent is None else parent.data_ptr(), b, n, logits.data_ptr(), dt, v, out.data_ptr(), choice.data_ptr())
    return out, choice


def moa_verify_greedy_rules(rules: LogitRules, tok: torch.Tensor, parent: torch.Tensor, target_logits: torch.Tensor, cap: int, out=None,
                            stream=None):
    """moa_verify_greedy with the arg-max of the adjusted logits; none are written. Returns the same five tensors."""
    assert tok is not None, "a verification needs the tree"
    at, b, n, v, dt = _rule_rows(rules, target_logits, tok, parent)
    if out is None:
        out = tuple(_made(lambda: torch.empty(s, dtype=torch.int32, device=target_logits.device), stream)
                    for s in ((b, n), (b, cap), (b, cap), (b,), (b,)))
    else:
        for t, s in zip(out, ((b, n), (b, cap), (b, cap), (b,), (b,))):
            assert _is(t, torch.int32, at) and t.shape == s, "out: int32 [batch, n], [batch, cap] twice, [batch] twice"
    c, slot, acc, length, following = out
    _serving_call(at, stream, load_library().moa_verify_greedy_rules, "moa_verify_greedy_rules", rules._ref, tok.data_ptr(), parent.data_ptr(), b, n,
                  target_logits.data_ptr(), dt, v, cap, c.data_ptr(), slot.data_ptr(), acc.data_ptr(), length.data_ptr(), following.data_ptr())
    return c, slot, acc, length, following


class MoA:
    """A drafter context plus one decoding state on the current CUDA device.

    weights: dict name -> CUDA tensor (dtype float32 or bfloat16, as cfg['dtype'] says).
    cfg keys: the fields of moa_config except dtype/max_* (given separately). Target Layer Inference: with
    cfg['n_tli'] = N > 0 (plus 'tli_hq', 'tli_hkv', 'tli_mlp') the weights also hold 'tli{l}_{norm1,wq,...}' for
    l < N, and the LLM's caches of those layers are the tensors tli_k[l], tli_v[l] (fill_tli_cache)."""

    def __init__(self, cfg: dict, weights: dict, max_batch: int, max_ctx: int, lsa_chunk_tokens: int = 8):
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2410_03804_b200 needs a CUDA device (B200, sm_100a); there is no CPU path")
        self.dtype = torch.float32 if cfg["dtype"] == "f32" else torch.bfloat16
        c = MoaConfig()
        for n in ("d_model", "n_stack", "d_stack", "vocab", "head_dim", "lsa_hq", "lsa_hkv", "lsa_mlp", "sa_hq",
                  "sa_hkv", "sa_mlp", "ca_hq", "ca_hkv", "ca_mlp", "tree_topk", "tree_depth", "tree_keep"):
            setattr(c, n, int(cfg[n]))
        c.max_batch, c.max_ctx = int(max_batch), int(max_ctx)
        c.rms_eps = float(cfg.get("rms_eps", 1e-5))
        c.sa_rope_theta = float(cfg.get("rope_theta", 500000.0))
        c.dtype = 0 if cfg["dtype"] == "f32" else 1
        self.cfg = c
        self.weights = {}
        w = MoaWeights()
        for n in WEIGHT_FIELDS:
            t = weights[n]
            assert t.is_cuda and t.dtype == self.dtype and t.is_contiguous(), n
            self.weights[n] = t          # keep alive
            setattr(w, n, t.data_ptr())
        self._w = w
        h = C.c_void_p()
        _check(self.lib.moa_create(C.byref(c), C.byref(w), C.byref(h)), "moa_create")
        self.h = h
        self.device = weights["embed"].device
        self.n_tli = int(cfg.get("n_tli", 0))
        self.tli_k, self.tli_v = [], []
        if self.n_tli > 0:
            self.moa_tli_configure(cfg, weights, max_batch, max_ctx)
        tb, wb = C.c_size_t(), C.c_size_t()
        _check(self.lib.moa_state_bytes(self.h, int(lsa_chunk_tokens), C.byref(tb), C.byref(wb)), "moa_state_bytes")
        self.tree_bytes, self.ws_bytes = tb.value, wb.value
        dev, dh = self.device, c.head_dim
        self.ca_k = torch.zeros((max_batch, max_ctx, c.ca_hkv, dh), dtype=self.dtype, device=dev)
        self.ca_v = torch.zeros_like(self.ca_k)
        self.sa_k = torch.zeros((max_batch, max_ctx, c.sa_hkv, dh), dtype=self.dtype, device=dev)
        self.sa_v = torch.zeros_like(self.sa_k)
        self.ca_len = torch.zeros(MOA_MAX_BATCH, dtype=torch.int32, device=dev)
        self.sa_len = torch.zeros(MOA_MAX_BATCH, dtype=torch.int32, device=dev)
        self.tree = torch.zeros(self.tree_bytes, dtype=torch.uint8, device=dev)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self._ca_len_host = (C.c_int32 * MOA_MAX_BATCH)()
        self._sa_len_host = (C.c_int32 * MOA_MAX_BATCH)()
        st = MoaState()
        st.ca_k, st.ca_v, st.sa_k, st.sa_v = (t.data_ptr() for t in (self.ca_k, self.ca_v, self.sa_k, self.sa_v))
        st.ca_len, st.sa_len, st.tree = self.ca_len.data_ptr(), self.sa_len.data_ptr(), self.tree.data_ptr()
        st.ca_len_host = C.addressof(self._ca_len_host)
        st.sa_len_host = C.addressof(self._sa_len_host)
        st.step = -1
        self.st = st

    def close(self):
        if getattr(self, "h", None):
            self.lib.moa_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the C-ABI calls, same names -------------------------------------------------------
    def moa_tli_configure(self, cfg: dict, weights: dict, max_batch: int, max_ctx: int):
        """Turns Target Layer Inference on: binds the N decoder layers' weights and allocates their caches."""
        n = int(cfg["n_tli"])
        tc = MoaTliConfig(n, int(cfg["tli_hq"]), int(cfg["tli_hkv"]), int(cfg["tli_mlp"]),
                          float(cfg.get("rope_theta", 500000.0)))
        layers = (MoaTliLayer * n)()
        for l in range(n):
            for f in TLI_LAYER_FIELDS:
                t = weights[f"tli{l}_{f}"]
                assert t.is_cuda and t.dtype == self.dtype and t.is_contiguous(), (l, f)
                self.weights[f"tli{l}_{f}"] = t
                setattr(layers[l], f, t.data_ptr())
        caches = MoaTliCaches()
        shape = (max_batch, max_ctx, tc.hkv, self.cfg.head_dim)
        self.tli_k = [torch.zeros(shape, dtype=self.dtype, device=self.device) for _ in range(n)]
        self.tli_v = [torch.zeros(shape, dtype=self.dtype, device=self.device) for _ in range(n)]
        for l in range(n):
            caches.k[l], caches.v[l] = self.tli_k[l].data_ptr(), self.tli_v[l].data_ptr()
        _check(self.lib.moa_tli_configure(self.h, C.byref(tc), C.cast(layers, C.c_void_p), C.byref(caches)),
               "moa_tli_configure")

    def moa_state_set_len(self, which: str, lens, stream=None):
        lens = [int(v) for v in lens]
        _check(self.lib.moa_state_set_len(self.h, C.byref(self.st), 0 if which == "ca" else 1, _host_i32(lens),
                                          len(lens), _stream(stream)), "moa_state_set_len")

    def moa_lsa_forward(self, h_stack: torch.Tensor, n_tok, want_kv: bool = True, stream=None):
        """h_stack: T cuda [sum n_tok, S, D_in]; n_tok: list of per-sequence token counts."""
        assert h_stack.is_cuda and h_stack.dtype == self.dtype and h_stack.is_contiguous()
        n_tok = [int(v) for v in n_tok]
        assert h_stack.shape[0] == sum(n_tok)
        kv = torch.empty((sum(n_tok), self.cfg.d_stack), dtype=self.dtype, device=self.device) if want_kv else None
        _check(self.lib.moa_lsa_forward(self.h, C.byref(self.st), _ptr(h_stack), _host_i32(n_tok), len(n_tok),
                                        _ptr(kv), _ptr(self.ws), self.ws_bytes, _stream(stream)), "moa_lsa_forward")
        return kv

    def moa_sa_append(self, tok: torch.Tensor, n, stream=None):
        assert tok.is_cuda and tok.dtype == torch.int32 and tok.is_contiguous()
        n = [int(v) for v in n]
        assert tok.numel() == sum(n)
        _check(self.lib.moa_sa_append(self.h, C.byref(self.st), _ptr(tok), _host_i32(n), len(n), _ptr(self.ws),
                                      self.ws_bytes, _stream(stream)), "moa_sa_append")

    def moa_drafter_prefill(self, tok: torch.Tensor, n, ca_limit=None, out=None, stream=None):
        """The drafter over whole sequences in one pass: tok cuda int32 [sum n]; ca_limit cuda int32 [sum n] or
        None. Returns hidden [sum n, E] and appends the tokens to the self-attention prefix."""
        assert tok.is_cuda and tok.dtype == torch.int32 and tok.is_contiguous()
        n = [int(v) for v in n]
        assert tok.numel() == sum(n)
        if ca_limit is not None:
            assert ca_limit.is_cuda and ca_limit.dtype == torch.int32 and ca_limit.numel() == sum(n)
        hid = out if out is not None else torch.empty((sum(n), self.cfg.d_model), dtype=self.dtype, device=self.device)
        _check(self.lib.moa_drafter_prefill(self.h, C.byref(self.st), _ptr(tok), _host_i32(n), len(n), _ptr(ca_limit),
                                            _ptr(hid), _ptr(self.ws), self.ws_bytes, _stream(stream)), "moa_drafter_prefill")
        return hid

    def moa_sa_append_static(self, tok: torch.Tensor, n, stream=None):
        """moa_sa_append without a workspace: the library's fixed scratch array is used, nothing is allocated.
        For callers that cannot allocate device memory; at most 32 tokens per call (see include/moa.h)."""
        assert tok.is_cuda and tok.dtype == torch.int32 and tok.is_contiguous()
        n = [int(v) for v in n]
        assert tok.numel() == sum(n)
        _check(self.lib.moa_sa_append_static(self.h, C.byref(self.st), _ptr(tok), _host_i32(n), len(n),
                                             _stream(stream)), "moa_sa_append_static")

    def moa_tree_begin(self, root_tok: torch.Tensor, stream=None):
        assert root_tok.is_cuda and root_tok.dtype == torch.int32 and root_tok.is_contiguous()
        self.batch = root_tok.numel()
        _check(self.lib.moa_tree_begin(self.h, C.byref(self.st), _ptr(root_tok), self.batch, _stream(stream)),
               "moa_tree_begin")

    def rows(self) -> int:
        return self.batch if self.st.step == 0 else self.batch * self.cfg.tree_topk

    def moa_draft_step(self, want_hidden: bool = False, out=None, stream=None):
        """Returns (topk_id [R,B] int32, topk_logp [R,B] float32, hidden [R,E] or None)."""
        R, B = self.rows(), self.cfg.tree_topk
        if out is None:
            ids = torch.empty((R, B), dtype=torch.int32, device=self.device)
            lp = torch.empty((R, B), dtype=torch.float32, device=self.device)
            hid = torch.empty((R, self.cfg.d_model), dtype=self.dtype, device=self.device) if want_hidden else None
        else:
            ids, lp, hid = out
        _check(self.lib.moa_draft_step(self.h, C.byref(self.st), self.batch, _ptr(ids), _ptr(lp), _ptr(hid),
                                       _ptr(self.ws), self.ws_bytes, _stream(stream)), "moa_draft_step")
        return ids, lp, hid

    def moa_tree_expand(self, ids: torch.Tensor, lp: torch.Tensor, out=None, stream=None):
        """Expands with the given top-B lists. After the last step returns the kept tree as
        (tok, parent, depth, score, n) tensors of shape [batch, m+1] / [batch]; otherwise None."""
        assert ids.is_cuda and ids.dtype == torch.int32 and lp.dtype == torch.float32
        last = self.st.step + 1 == self.cfg.tree_depth
        outs = out
        if last and outs is None:
            W = self.cfg.tree_keep + 1
            outs = (torch.empty((self.batch, W), dtype=torch.int32, device=self.device),
                    torch.empty((self.batch, W), dtype=torch.int32, device=self.device),
                    torch.empty((self.batch, W), dtype=torch.int32, device=self.device),
                    torch.empty((self.batch, W), dtype=torch.float32, device=self.device),
                    torch.empty((self.batch,), dtype=torch.int32, device=self.device))
        p = [_ptr(t) for t in outs] if outs is not None else [None] * 5
        _check(self.lib.moa_tree_expand(self.h, C.byref(self.st), self.batch, _ptr(ids), _ptr(lp), *p, _stream(stream)),
               "moa_tree_expand")
        return outs if last else None

    def moa_state_status(self, stream=None) -> int:
        return int(self.lib.moa_state_status(self.h, C.byref(self.st), _stream(stream)))

    def moa_profile_begin(self):
        _check(self.lib.moa_profile_begin(self.h), "moa_profile_begin")

    def moa_profile_end(self):
        """Returns (summed LM-head kernel milliseconds, launches timed)."""
        ms, n = C.c_double(), C.c_int32()
        _check(self.lib.moa_profile_end(self.h, C.byref(ms), C.byref(n)), "moa_profile_end")
        return ms.value, n.value

    PHASE_KINDS = ["gemm", "rows_norm", "res_norm", "mean_norm", "cache_append", "lsa_attention"]

    def moa_profile_phases(self, stream=None):
        """[(kind name, microseconds, of which in the closing barrier)] of the last dense LSA pass launched while
        profiling was on."""
        cap = 32
        us, wait, kinds, n = (C.c_double * cap)(), (C.c_double * cap)(), (C.c_int32 * cap)(), C.c_int32()
        _check(self.lib.moa_profile_phases(self.h, _ptr(self.ws), self.ws_bytes, cap, us, wait, kinds, C.byref(n),
                                           _stream(stream)), "moa_profile_phases")
        return [(self.PHASE_KINDS[kinds[i]], us[i], wait[i]) for i in range(n.value)]

    def moa_launch_count(self) -> int:
        return int(self.lib.moa_launch_count())

    TRACE_KINDS = ["other", "embed", "gemm", "attention", "attn_merge", "lm_merge", "tree_expand", "row_norm", "res_norm",
                   "swiglu", "sum_cast", "rope", "cache_append", "layer_mean"]

    def moa_trace_begin(self, cap: int = 4096):
        """Starts the stage trace (library built with MOA_TRACE_BUILD=1 only)."""
        self._trace = torch.zeros(2 * cap, dtype=torch.int64, device=self.device)
        _check(self.lib.moa_trace_begin(_ptr(self._trace), cap), "moa_trace_begin")

    def moa_trace_end(self):
        """[(kernel kind, gridDim.x, nanosecond stamp)] in launch order."""
        n = C.c_int32()
        _check(self.lib.moa_trace_end(C.byref(n)), "moa_trace_end")
        t = self._trace.cpu().tolist()
        return [(self.TRACE_KINDS[(t[2 * i + 1] >> 32) & 0xff], t[2 * i + 1] & 0xffffffff, t[2 * i]) for i in range(min(n.value, len(t) // 2))]

    # ---- convenience for tests / bench: raw views of the tree blob ---------------------------
    def fill_cache(self, which: str, k: torch.Tensor, v: torch.Tensor):
        """Copies caller-made cache content [batch, n, hkv, dh] in and sets the lengths."""
        ck, cv = (self.ca_k, self.ca_v) if which == "ca" else (self.sa_k, self.sa_v)
        b, n = k.shape[0], k.shape[1]
        ck[:b, :n].copy_(k)
        cv[:b, :n].copy_(v)
        self.moa_state_set_len(which, [n] * b)

    def fill_tli_cache(self, layer: int, k: torch.Tensor, v: torch.Tensor):
        """Copies the LLM's cache of one Target-Layer-Inference layer [batch, n, hkv, dh] in (positions 0..n-1;
        the valid length is the self-attention prefix length)."""
        b, n = k.shape[0], k.shape[1]
        self.tli_k[layer][:b, :n].copy_(k)
        self.tli_v[layer][:b, :n].copy_(v)
