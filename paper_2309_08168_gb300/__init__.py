"""Python binding of libssd, batch-1 self-speculative decoding on GB300.

Argument marshalling only: every step of the decode path runs in the CUDA
library (csrc/, built for sm_103a by build.py).  The functions keep the C
ABI's names (include/ssd.h, include/ssd_ops.h, include/ssd_step.h).  Importing this module fails
loudly when the library has not been built; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libssd.so")

SSD_OK = 0
SSD_ERR_INVALID_ARG = -1
SSD_ERR_OOM = -2
SSD_ERR_CUDA = -3
SSD_ERR_CAPACITY = -4
SSD_ERR_TIMEOUT = -5
SSD_ERR_STATE = -6
SSD_GREEDY = 0
SSD_SAMPLE = 1

# every symbol include/ssd.h declares
EXPORTS = ("ssd_create", "ssd_set_skip", "ssd_set_sampling", "ssd_set_draft_exit", "ssd_prefill", "ssd_generate",
           "ssd_debug_forward", "ssd_debug_spec_accept", "ssd_debug_time_forward", "ssd_destroy",
           "ssd_last_error", "ssd_linear_noalloc", "ssd_debug_trace_forward", "ssd_debug_stall_barrier")

# the operators that include/ssd_ops.h declares (and ssd_debug_tree_stall)
OPERATOR_EXPORTS = ("ssd_tree_plan", "ssd_rope_init", "ssd_rope_kv", "ssd_tree_attention",
                    "ssd_tree_attention_workspace", "ssd_tree_commit")
# and those of include/ssd_step.h
STEP_EXPORTS = ("ssd_rope_axes_init", "ssd_norm_rope_kv", "ssd_logits_adjust", "ssd_logits_choose", "ssd_moe_route", "ssd_moe_mlp",
                "ssd_moe_workspace")
SSD_AXES_SECTIONS, SSD_AXES_IN_TURNS = 0, 1
SSD_MOE_SOFTMAX, SSD_MOE_SIGMOID = 0, 1
SSD_F32, SSD_F16, SSD_BF16 = 0, 1, 2
SSD_STATUS_PAGES, SSD_STATUS_TABLE, SSD_STATUS_PARENT, SSD_STATUS_TIMEOUT = 1, 2, 4, 8
SSD_ROPE_PLAIN, SSD_ROPE_LINEAR, SSD_ROPE_BY_PARTS = 0, 1, 2


class ssd_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in
                ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "ffn", "vocab", "max_seq")] + \
               [("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float)]


_VP = ctypes.c_void_p
_VPP = ctypes.POINTER(ctypes.c_void_p)
LAYER_TENSORS = ("wq", "wk", "wv", "wo", "attn_norm", "w_gate", "w_up", "w_down", "mlp_norm")


class ssd_weights(ctypes.Structure):
    _fields_ = [("embed", _VP), ("final_norm", _VP), ("lm_head", _VP)] + \
               [(n, _VPP) for n in LAYER_TENSORS] + [("on_device", ctypes.c_int)]


class ssd_stats(ctypes.Structure):
    _fields_ = [("rounds", ctypes.c_int), ("drafted", ctypes.c_int), ("accepted", ctypes.c_int),
                ("emitted", ctypes.c_int), ("accept_rate", ctypes.c_double), ("hist", ctypes.c_int * 33),
                ("draft_ms", ctypes.c_float), ("verify_ms", ctypes.c_float), ("total_ms", ctypes.c_float),
                ("kernel_launches", ctypes.c_longlong), ("gamma", ctypes.c_float)]

    def as_dict(self) -> dict:
        return {"rounds": self.rounds, "drafted": self.drafted, "accepted": self.accepted,
                "emitted": self.emitted, "accept_rate": self.accept_rate, "hist": list(self.hist),
                "draft_ms": self.draft_ms, "verify_ms": self.verify_ms, "total_ms": self.total_ms,
                "kernel_launches": self.kernel_launches, "gamma": self.gamma}


class ssd_pages(ctypes.Structure):
    _fields_ = [("k", _VP), ("v", _VP)] + \
               [(n, ctypes.c_int) for n in ("dtype", "n_layers", "n_pages", "n_kv_heads", "page_size", "head_dim")] + \
               [(n, ctypes.c_int64) for n in ("layer_stride", "page_stride", "head_stride", "pos_stride")]


class ssd_batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_requests", "n_rows", "max_rows", "max_blocks")] + \
               [("row_start", _VP), ("lens", _VP), ("block_table", _VP)]


class ssd_rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int), ("amplitude", ctypes.c_float),
                ("turns", ctypes.c_uint64 * 64)]


class ssd_rope_axes(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int), ("axis", ctypes.c_uint8 * 64)]


class ssd_head_norm(ctypes.Structure):
    _fields_ = [("q_gain", _VP), ("k_gain", _VP), ("eps", ctypes.c_float)]


class ssd_logit_rules(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("vocab", "n_requests", "n_rows", "max_rows")] + \
               [(n, _VP) for n in ("row_start", "history", "history_len", "prompt_len")] + \
               [("history_stride", ctypes.c_int64), ("max_history", ctypes.c_int), ("mask_words", ctypes.c_int)] + \
               [(n, _VP) for n in ("tokens", "masks", "repetition", "presence", "frequency", "bias", "bias_of", "allowed", "allowed_of")] + \
               [("bias_stride", ctypes.c_int64), ("allowed_stride", ctypes.c_int64), ("n_bias", ctypes.c_int), ("n_allowed", ctypes.c_int)]


class ssd_moe(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("gate", "up", "down")] + [(n, ctypes.c_int64) for n in ("gate_stride", "up_stride", "down_stride")] + \
               [(n, ctypes.c_int) for n in ("dtype", "n_experts", "d", "f")]


class SSDError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{msg} (code {code})")
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libssd is not built ({LIB_PATH} missing); run "
                          "`python -c 'import __graft_entry__ as g; g.build()'` first")
    lib = ctypes.CDLL(LIB_PATH)
    H = ctypes.c_void_p
    lib.ssd_create.argtypes = [ctypes.POINTER(ssd_config), ctypes.POINTER(ssd_weights), _VP, ctypes.POINTER(H)]
    lib.ssd_set_skip.argtypes = [H, _VP, ctypes.c_int]
    lib.ssd_set_sampling.argtypes = [H, ctypes.c_float, ctypes.c_float]
    lib.ssd_set_draft_exit.argtypes = [H, ctypes.c_int] + [ctypes.c_float] * 5
    lib.ssd_prefill.argtypes = [H, _VP, ctypes.c_int]
    lib.ssd_generate.argtypes = [H, _VP, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                 ctypes.c_uint64, _VP, ctypes.POINTER(ssd_stats)]
    lib.ssd_debug_forward.argtypes = [H, ctypes.c_int, _VP, ctypes.c_int, ctypes.c_int, _VP]
    lib.ssd_debug_spec_accept.argtypes = [H, _VP, _VP, ctypes.c_int, _VP, _VP, ctypes.c_int, ctypes.c_int, _VP]
    lib.ssd_debug_time_forward.argtypes = [H, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                           _VP, _VP, _VP]
    lib.ssd_debug_trace_forward.argtypes = [H, ctypes.c_int, ctypes.c_int, _VP, _VP, ctypes.c_int, _VP,
                                            ctypes.c_int, _VP, _VP, ctypes.c_int, _VP]
    lib.ssd_debug_trace_forward.restype = ctypes.c_int
    lib.ssd_debug_stall_barrier.argtypes = [H, ctypes.c_int, ctypes.c_double]
    lib.ssd_debug_stall_barrier.restype = ctypes.c_int
    lib.ssd_linear_noalloc.argtypes = [_VP, _VP, _VP, ctypes.c_int, ctypes.c_int, ctypes.c_int, _VP]
    lib.ssd_linear_noalloc.restype = ctypes.c_int
    I, L, BP, PP, RP = ctypes.c_int, ctypes.c_int64, ctypes.POINTER(ssd_batch), ctypes.POINTER(ssd_pages), ctypes.POINTER(ssd_rope)
    lib.ssd_tree_plan.argtypes = [BP, I, I] + [_VP] * 9 + [I, _VP, _VP]
    lib.ssd_rope_init.argtypes = [I, I, I] + [ctypes.c_double] * 6 + [RP]
    lib.ssd_rope_kv.argtypes = [PP, I, RP, I, I, I, _VP, L, _VP, L, _VP, L, _VP, _VP, _VP, L, _VP]
    lib.ssd_tree_attention.argtypes = [BP, PP, I, I, I, _VP, L, _VP, I, ctypes.c_float, _VP, L, _VP, ctypes.c_size_t, _VP, _VP]
    lib.ssd_tree_attention_workspace.argtypes = [I, ctypes.POINTER(ctypes.c_size_t)]
    lib.ssd_tree_commit.argtypes = [BP, PP] + [_VP] * 9
    lib.ssd_debug_tree_stall.argtypes, lib.ssd_debug_tree_stall.restype = [I, ctypes.c_double], None
    AP, NP, LP, MP = (ctypes.POINTER(x) for x in (ssd_rope_axes, ssd_head_norm, ssd_logit_rules, ssd_moe))
    lib.ssd_rope_axes_init.argtypes = [RP, I, I, ctypes.POINTER(I), AP]
    lib.ssd_norm_rope_kv.argtypes = [PP, I, RP, AP, NP, I, I, I, _VP, L, _VP, L, _VP, L, _VP, _VP, _VP, L, _VP]
    lib.ssd_logits_adjust.argtypes = [LP, I, _VP, L, _VP, L, _VP]
    lib.ssd_logits_choose.argtypes = [LP, I, _VP, L, I, _VP, _VP, _VP, _VP]
    lib.ssd_moe_route.argtypes = [I, I, I, I, I, _VP, L, _VP, _VP, I, I, ctypes.c_float, _VP, _VP, _VP]
    lib.ssd_moe_mlp.argtypes = [MP, I, I, _VP, L, _VP, _VP, _VP, L, _VP, L, _VP, ctypes.c_size_t, _VP, _VP]
    lib.ssd_debug_moe_stall.argtypes, lib.ssd_debug_moe_stall.restype = [I, ctypes.c_double], None
    lib.ssd_moe_workspace.argtypes = [MP, I, I, ctypes.POINTER(ctypes.c_size_t)]
    for n in OPERATOR_EXPORTS + STEP_EXPORTS:
        getattr(lib, n).restype = ctypes.c_int
    lib.ssd_destroy.argtypes = [H]
    lib.ssd_destroy.restype = None
    lib.ssd_last_error.argtypes = []
    lib.ssd_last_error.restype = ctypes.c_char_p
    for n in ("ssd_create", "ssd_set_skip", "ssd_set_sampling", "ssd_set_draft_exit", "ssd_prefill",
              "ssd_generate", "ssd_debug_forward", "ssd_debug_spec_accept", "ssd_debug_time_forward"):
        getattr(lib, n).restype = ctypes.c_int
    return lib


lib = _load()


def _check(rc: int):
    if rc != SSD_OK:
        raise SSDError(rc, lib.ssd_last_error().decode())


def _ptr(a) -> int:
    """Address of a numpy array or a torch tensor."""
    if hasattr(a, "data_ptr"):
        return a.data_ptr()
    return a.ctypes.data


# -- the C ABI, one function each -------------------------------------------

def ssd_create(cfg: ssd_config, weights: ssd_weights, cuda_stream: int | None = None) -> int:
    h = ctypes.c_void_p()
    _check(lib.ssd_create(ctypes.byref(cfg), ctypes.byref(weights), cuda_stream, ctypes.byref(h)))
    _configs[h.value] = cfg
    return h.value


def ssd_set_skip(h: int, mask) -> None:
    m = np.ascontiguousarray(mask, dtype=np.uint8)
    _check(lib.ssd_set_skip(h, m.ctypes.data, m.size))


def ssd_set_sampling(h: int, temperature: float, top_p: float) -> None:
    _check(lib.ssd_set_sampling(h, temperature, top_p))


def ssd_set_draft_exit(h: int, enable: bool, gamma0: float = 0.6, alpha: float = 0.9, eps: float = 0.01,
                       beta1: float = 0.5, beta2: float = 0.9) -> None:
    _check(lib.ssd_set_draft_exit(h, int(bool(enable)), gamma0, alpha, eps, beta1, beta2))


def ssd_prefill(h: int, prompt) -> None:
    p = np.ascontiguousarray(prompt, dtype=np.int32)
    _check(lib.ssd_prefill(h, p.ctypes.data, p.size))


def ssd_generate(h: int, prompt, n_new: int, K: int, mode: int = SSD_GREEDY, seed: int = 0,
                 out=None):
    """prompt: host int32 tokens or None (restart from the last prefill).
    Returns (tokens np.int32[n_new], stats dict)."""
    if prompt is None:
        pp, pn = None, 0
    else:
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        pp, pn = p.ctypes.data, p.size
    toks = out if out is not None else np.zeros(n_new, dtype=np.int32)
    st = ssd_stats()
    _check(lib.ssd_generate(h, pp, pn, n_new, K, mode, seed, _ptr(toks) if n_new else None, ctypes.byref(st)))
    return toks, st.as_dict()


def ssd_debug_forward(h: int, draft: bool, tokens, pos0: int) -> np.ndarray:
    t = np.ascontiguousarray(tokens, dtype=np.int32)
    out = np.empty((t.size, config_of(h).vocab), dtype=np.float32)
    _check(lib.ssd_debug_forward(h, int(draft), t.ctypes.data, t.size, pos0, out.ctypes.data))
    return out


def ssd_debug_stall_barrier(h: int, barrier: int, wait_limit_s: float) -> None:
    _check(lib.ssd_debug_stall_barrier(h, int(barrier), float(wait_limit_s)))


def ssd_debug_spec_accept(h: int, p, q, drafts, seeds, pos0: int):
    p = np.ascontiguousarray(p, dtype=np.float32)
    q = np.ascontiguousarray(q, dtype=np.float32)
    d = np.ascontiguousarray(drafts, dtype=np.int32)
    s = np.ascontiguousarray(seeds, dtype=np.uint64)
    T, Kd = d.shape
    out = np.empty((T, 2), dtype=np.int32)
    _check(lib.ssd_debug_spec_accept(h, p.ctypes.data, q.ctypes.data, Kd, d.ctypes.data, s.ctypes.data,
                                     T, pos0, out.ctypes.data))
    return out[:, 0], out[:, 1]


def ssd_debug_time_forward(h: int, draft: bool, rows: int, gemm_only: bool, reps: int):
    """Returns (ms per forward replay, kernels per replay, weight bytes per replay)."""
    ms = ctypes.c_float()
    n = ctypes.c_int()
    b = ctypes.c_double()
    _check(lib.ssd_debug_time_forward(h, int(draft), rows, int(gemm_only), reps, ctypes.addressof(ms),
                                      ctypes.addressof(n), ctypes.addressof(b)))
    return ms.value, n.value, b.value


def ssd_linear_noalloc(w, x, y, N: int, K: int, M: int, cuda_stream: int | None = None) -> None:
    """y[M][N] = x[M][K] @ w[N][K]^T on device tensors, without allocating."""
    _check(lib.ssd_linear_noalloc(_ptr(w), _ptr(x), _ptr(y), N, K, M, cuda_stream))


OP_NAMES = ("embed", "qkv", "attention", "o/down", "gate/up", "lm_head")


def ssd_debug_trace_forward(h: int, draft: bool, rows: int, detail_op: int = -1):
    """Returns [(op name, microseconds)] for one forward of the forward kernel.
    With detail_op >= 0 (op index + 65536 x a CTA index) it returns (ops,
    units, ctas): units = [64][4] stamps (ns) of that CTA's first work units
    of that op (producer issue, MMAs issued, 0, segment flush done; for
    attention 8 stamps per item), ctas = [grid][8] stamps per CTA in the
    order ssd.h lists."""
    cfg = config_of(h)
    cap = 2 + 5 * cfg.n_layers
    us = np.zeros(cap, dtype=np.float32)
    ty = np.zeros(cap, dtype=np.int32)
    ut = np.zeros((64, 4), dtype=np.uint64)
    max_ctas = 1024
    ct = np.zeros((max_ctas, 8), dtype=np.uint64)
    n = ctypes.c_int()
    n_ctas = ctypes.c_int()
    detail = detail_op >= 0
    _check(lib.ssd_debug_trace_forward(h, int(draft), rows, us.ctypes.data, ty.ctypes.data, cap,
                                       ctypes.addressof(n), int(detail_op), ut.ctypes.data if detail else None,
                                       ct.ctypes.data if detail else None, max_ctas, ctypes.addressof(n_ctas)))
    ops = [(OP_NAMES[ty[i]], float(us[i])) for i in range(n.value)]
    return (ops, ut, ct[:n_ctas.value]) if detail else ops


# -- operators on the caller's device tensors (include/ssd_ops.h) -------------

_TYPES: dict = {}  # name -> type, those met so far
_ROW_TYPES = {"torch.float32": SSD_F32, "torch.float16": SSD_F16, "torch.bfloat16": SSD_BF16}


def _refuse(what: str):
    raise SSDError(SSD_ERR_INVALID_ARG, what)


def _dev(t, what: str, dtype, device: int, n: int):
    """Address of a contiguous tensor of n values of this type on CUDA device `device`, or None for None."""
    if t is None:
        return None
    if t.get_device() != device or t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        _refuse(f"{what}: a contiguous {dtype} tensor of {n} values on CUDA device {device} is wanted, got {t.dtype}, shape {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(t, what: str, device: int, dtype, n_rows: int, heads: int, hd: int):
    """(address, row stride) of rows [row][head][dim] whose heads lie behind one another."""
    shape, stride = t.shape, t.stride()
    if shape != (n_rows, heads, hd) or t.dtype is not dtype or t.get_device() != device:
        _refuse(f"{what}: {dtype} of shape ({n_rows}, {heads}, {hd}) on CUDA device {device} is wanted, got {t.dtype}, {tuple(shape)} on {t.device}")
    if n_rows == 0:  # (strides of no rows mean nothing)
        return None, heads * hd
    if stride[2] != 1 or (stride[1] != hd and heads > 1):
        _refuse(f"{what}: the heads of a row must lie behind one another")
    return t.data_ptr(), stride[0] if n_rows > 1 else heads * hd


def _row_type(t, what: str) -> int:
    k = _ROW_TYPES.get(t.dtype)
    if k is None:
        k = _ROW_TYPES.get(str(t.dtype))
        if k is None or t.dim() != 3:
            _refuse(f"{what}: fp32, fp16 or bf16 rows [row][head][dim] are wanted")
        _ROW_TYPES[t.dtype] = k
    if t.dim() != 3:
        _refuse(f"{what}: rows [row][head][dim] are wanted")
    return k


def _of_type(t, what: str, name: str):
    """t's type, which has to be this one."""
    if t is None:
        return None
    k = t.dtype
    if _TYPES.get(name) is not k:
        if str(k) != name:
            _refuse(f"{what}: {name} is wanted, got {k}")
        _TYPES[name] = k
    return k


class PagedKV:
    """A paged cache: k and v are fp16 or bf16 CUDA tensors indexed [layer][page][kv_head][position in page][dim],
    of equal shape and strides (any memory order in which dims are adjacent).  Keeps the tensors."""

    def __init__(self, k, v):
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device or not k.is_cuda:
            _refuse("k and v: CUDA tensors [layer][page][kv_head][position][dim] of one shape, type and memory order are wanted")
        if str(k.dtype) not in ("torch.float16", "torch.bfloat16") or k.stride(4) != 1:
            _refuse("k and v: fp16 or bf16 with adjacent dims are wanted")
        self.k, self.v, self.device = k, v, k.get_device()
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        self.struct = ssd_pages(k.data_ptr(), v.data_ptr(), _ROW_TYPES[str(k.dtype)], *(k.shape[i] for i in (0, 1, 2, 3, 4)), *k.stride()[:4])


class TreeBatch:
    """A round's rows: row_start int32 [n + 1], lens int32 [n] and block_table int32 [n][max_blocks] on one device.
    Keeps the tensors; their contents may change between calls."""

    def __init__(self, row_start, lens, block_table, n_rows: int, max_rows: int):
        n, self.i32 = lens.numel(), _of_type(lens, "lens", "torch.int32")
        if not lens.is_cuda or block_table.dim() != 2 or block_table.shape[0] != n:
            _refuse("lens [request] and block_table [request][block] on a CUDA device are wanted")
        self.device = lens.get_device()
        self.keep = (row_start, lens, block_table)
        self.n_requests, self.n_rows, self.max_rows, self.max_blocks = n, n_rows, max_rows, block_table.shape[1]
        self.struct = ssd_batch(n, n_rows, max_rows, self.max_blocks, _dev(row_start, "row_start", self.i32, self.device, n + 1),
                                _dev(lens, "lens", self.i32, self.device, n),
                                _dev(block_table, "block_table", self.i32, self.device, n * self.max_blocks))


def ssd_tree_plan(batch: TreeBatch, page_size: int, n_pages: int, parents, held, held_out, ring, ends, ends_out, slots,
                  positions, masks=None, status=None, cuda_stream: int | None = None) -> None:
    """Pages, slots, positions and ancestor masks of a round.  parents int32 [n_rows] or None (chains); held, held_out
    int32 [n]; ring int32 [n_pages]; ends, ends_out int64 [2]; slots, positions int32 [n_rows]; masks int64 [n_rows][words]
    (bit patterns) with parents; status int32 [1] or None."""
    d, n, r, i32, i64 = batch.device, batch.n_requests, batch.n_rows, batch.i32, _of_type(ends, "ends", "torch.int64")
    if r == 0:  # (pages only)
        parents = masks = None
    words = _words(masks)
    _check(lib.ssd_tree_plan(batch.struct, page_size, n_pages, _dev(parents, "parents", i32, d, r), _dev(held, "held", i32, d, n),
                             _dev(held_out, "held_out", i32, d, n), _dev(ring, "ring", i32, d, n_pages), _dev(ends, "ends", i64, d, 2),
                             _dev(ends_out, "ends_out", i64, d, 2), _dev(slots, "slots", i32, d, r),
                             _dev(positions, "positions", i32, d, r), _dev(masks, "masks", i64, d, r * words), words,
                             _dev(status, "status", i32, d, 1), cuda_stream))


def _words(masks) -> int:
    if masks is None:
        return 0
    if masks.dim() != 2 or masks.shape[1] == 0:
        _refuse("masks: [row][word] is wanted")
    return masks.shape[1]


def ssd_rope_init(rot_dim: int, theta: float = 1e4, interleaved: bool = False, scaling: int = SSD_ROPE_PLAIN, factor: float = 1.0,
                  original_len: float = 0.0, slow: float = 1.0, fast: float = 32.0, amplitude: float = 1.0) -> ssd_rope:
    out = ssd_rope()
    _check(lib.ssd_rope_init(rot_dim, int(bool(interleaved)), scaling, theta, factor, original_len, slow, fast, amplitude, out))
    return out


def ssd_rope_kv(cache: PagedKV, layer: int, rope: ssd_rope, q, k, v, positions, slots, q_out,
                cuda_stream: int | None = None) -> None:
    """Turns q [n][heads][hd] and k [n][kv_heads][hd] to positions int32 [n]; q to q_out, k and v [n][kv_heads][hd] to
    rows slots int32 [n] of the cache's layer."""
    kind, d, t, n, h, g, hd = _row_type(q, "q"), cache.device, q.dtype, q.shape[0], q.shape[1], cache.n_kv_heads, cache.head_dim
    i32 = _of_type(slots, "slots", "torch.int32")
    _check(lib.ssd_rope_kv(cache.struct, layer, rope, kind, n, h, *_rows(q, "q", d, t, n, h, hd), *_rows(k, "k", d, t, n, g, hd),
                           *_rows(v, "v", d, t, n, g, hd), _dev(positions, "positions", i32, d, n), _dev(slots, "slots", i32, d, n),
                           *_rows(q_out, "q_out", d, t, n, h, hd), cuda_stream))


def ssd_tree_attention_workspace(cache: PagedKV) -> int:
    """Bytes of workspace that ssd_tree_attention wants for this cache."""
    n = ctypes.c_size_t()
    _check(lib.ssd_tree_attention_workspace(cache.head_dim, n))
    return n.value


def ssd_tree_attention(batch: TreeBatch, cache: PagedKV, layer: int, q, masks, scale: float, out, workspace, status=None,
                       cuda_stream: int | None = None) -> None:
    """out [n_rows][heads][hd] = attention of q over the requests' cached positions and the nodes that masks
    int64 [n_rows][words] show (None: chains).  workspace: a contiguous uint8 tensor.  What only the device can see (a table that is
    too narrow, a wait that gave up and left an output that is not valid) is told by status int32 [1] alone, set to 0 before."""
    kind, d, t, n, h, hd = _row_type(q, "q"), cache.device, q.dtype, batch.n_rows, q.shape[1], cache.head_dim
    if batch.device != d:
        _refuse("the batch and the cache are on different devices")
    if n == 0:
        masks = None
    words = _words(masks)
    _check(lib.ssd_tree_attention(batch.struct, cache.struct, layer, kind, h, *_rows(q, "q", d, t, n, h, hd),
                                  _dev(masks, "masks", _of_type(masks, "masks", "torch.int64"), d, n * words), words, scale,
                                  *_rows(out, "out", d, t, n, h, hd),
                                  _dev(workspace, "workspace", _of_type(workspace, "workspace", "torch.uint8"), d, workspace.numel()),
                                  workspace.numel(), _dev(status, "status", batch.i32, d, 1), cuda_stream))


def ssd_debug_tree_stall(cta: int, wait_limit_s: float = 0.01) -> None:
    """Test hook: a CTA of the next ssd_tree_attention call (tiles of more than two rows) never asks for its keys, so its waits
    give up after wait_limit_s."""
    if cta >= 0 and not 0.0 < wait_limit_s <= 10.0:
        _refuse("ssd_debug_tree_stall: 0 < wait_limit_s <= 10 is wanted")
    lib.ssd_debug_tree_stall(cta, wait_limit_s)


def ssd_tree_commit(batch: TreeBatch, cache: PagedKV | None, parents, tokens, target, accepted, next_token, lens_out, path,
                    emitted, cuda_stream: int | None = None) -> None:
    """Walks every tree along target int32 [n_rows]: accepted, next_token, lens_out int32 [n]; path, emitted int32
    [n_rows]; moves the accepted rows of every layer of the cache (None: tokens only).  parents None: chains."""
    d, n, r, i32 = batch.device, batch.n_requests, batch.n_rows, batch.i32
    if cache is not None and cache.device != d:
        _refuse("the batch and the cache are on different devices")
    _check(lib.ssd_tree_commit(batch.struct, cache.struct if cache is not None else None, _dev(parents, "parents", i32, d, r),
                               _dev(tokens, "tokens", i32, d, r), _dev(target, "target", i32, d, r),
                               _dev(accepted, "accepted", i32, d, n), _dev(next_token, "next_token", i32, d, n),
                               _dev(lens_out, "lens_out", i32, d, n), _dev(path, "path", i32, d, r),
                               _dev(emitted, "emitted", i32, d, r), cuda_stream))


# -- operators of a decoding step around those (include/ssd_step.h) -----------

def ssd_rope_axes_init(rope: ssd_rope, layout: int, pairs) -> ssd_rope_axes:
    """Which axis turns each pair: pairs has the number of pairs of every axis."""
    out, pairs = ssd_rope_axes(), [int(x) for x in pairs]
    _check(lib.ssd_rope_axes_init(rope, layout, len(pairs), (ctypes.c_int * max(1, len(pairs)))(*pairs), out))
    return out


class HeadNorm:
    """Gains fp32 [head_dim] of the queries' and the keys' heads (None: not normalised) on one CUDA device, and eps.  Keeps the tensors."""

    def __init__(self, q_gain, k_gain, eps: float):
        self.keep, self.sizes, self.device = (q_gain, k_gain), set(), None
        for t in self.keep:
            if t is not None:
                if not t.is_cuda or self.device not in (None, t.get_device()):
                    _refuse("gains on one CUDA device are wanted")
                self.device = t.get_device()
                self.sizes.add(t.numel())
        ptr = [_dev(t, "gain", _of_type(t, "gain", "torch.float32"), self.device, t.numel()) if t is not None else None for t in self.keep]
        self.struct = ssd_head_norm(*ptr, eps)


def ssd_norm_rope_kv(cache: PagedKV, layer: int, rope: ssd_rope, q, k, v, positions, slots, q_out, axes: ssd_rope_axes | None = None,
                     norm: HeadNorm | None = None, cuda_stream: int | None = None) -> None:
    """ssd_rope_kv with norms of q's and k's heads before the rotation; positions int32 [axes][n] (without axes [n])."""
    kind, d, t, n, h, g, hd = _row_type(q, "q"), cache.device, q.dtype, q.shape[0], q.shape[1], cache.n_kv_heads, cache.head_dim
    i32 = _of_type(slots, "slots", "torch.int32")
    if norm is not None and norm.device is not None and (norm.device != d or norm.sizes != {hd}):
        _refuse(f"gains of {hd} values on CUDA device {d} are wanted")
    _check(lib.ssd_norm_rope_kv(cache.struct, layer, rope, axes, norm.struct if norm is not None else None, kind, n, h, *_rows(q, "q", d, t, n, h, hd),
                                *_rows(k, "k", d, t, n, g, hd), *_rows(v, "v", d, t, n, g, hd),
                                _dev(positions, "positions", i32, d, n * (axes.n_axes if axes is not None else 1)), _dev(slots, "slots", i32, d, n),
                                *_rows(q_out, "q_out", d, t, n, h, hd), cuda_stream))


def _matrix(t, what: str, device: int, dtype, rows: int, width: int):
    """(address, row stride) of rows of `width` adjacent values."""
    if t.shape != (rows, width) or t.dtype is not dtype or t.get_device() != device:
        _refuse(f"{what}: {dtype} of shape ({rows}, {width}) on CUDA device {device} is wanted, got {t.dtype}, {tuple(t.shape)} on {t.device}")
    if rows == 0:  # (strides of no rows mean nothing)
        return None, width
    stride = t.stride()
    if stride[1] != 1 and width > 1:
        _refuse(f"{what}: the values of a row must be adjacent")
    return t.data_ptr(), stride[0] if rows > 1 else width


def _half_type(t, what: str) -> int:
    """Whether rows are fp16 or bf16."""
    k = _ROW_TYPES.get(t.dtype)
    if k is None:
        k = _ROW_TYPES.get(str(t.dtype))
        if k is not None:
            _ROW_TYPES[t.dtype] = k
    if k is None or k == SSD_F32:
        _refuse(f"{what}: fp16 or bf16 rows are wanted")
    return k


class LogitRules:
    """What is done to the logits of a round's rows (ssd_logit_rules), all tensors on one CUDA device.  Keeps the tensors; their
    contents may change between calls.  row_start int32 [requests + 1] with n_rows and max_rows, or None: a row a request.
    history int32 [requests][max_history] with history_len and prompt_len int32 [requests]; tokens int32 [n_rows] and masks
    int64 [n_rows][words] (bit patterns; None: chains) of the round's nodes; repetition, presence, frequency fp32 [requests];
    bias fp32 [sets][vocab] with bias_of int32 [requests]; allowed int32 [sets][ceil(vocab / 32)] (bit patterns) with
    allowed_of int32 [n_rows]."""

    def __init__(self, vocab: int, n_rows: int, row_start=None, max_rows: int = 1, history=None, history_len=None, prompt_len=None, tokens=None,
                 masks=None, repetition=None, presence=None, frequency=None, bias=None, bias_of=None, allowed=None, allowed_of=None):
        all_ = (row_start, history, history_len, prompt_len, tokens, masks, repetition, presence, frequency, bias, bias_of, allowed, allowed_of)
        self.keep, self.vocab, self.n_rows = all_, vocab, n_rows
        devices = {t.get_device() for t in all_ if t is not None}
        if len(devices) > 1 or -1 in devices:
            _refuse("rules: tensors on one CUDA device are wanted")
        self.device = d = devices.pop() if devices else None
        if row_start is not None and row_start.numel() < 2:
            _refuse("row_start: [requests + 1] is wanted")
        if (history is None) != (history_len is None) or (prompt_len is not None and history is None):
            _refuse("history needs history_len, prompt_len needs history")
        if (bias_of is not None and bias is None) or (allowed_of is not None and allowed is None):
            _refuse("bias_of needs bias, allowed_of needs allowed")
        n = self.n_requests = row_start.numel() - 1 if row_start is not None else n_rows

        def dev(t, what, name, size):
            return _dev(t, what, _of_type(t, what, name), d, size) if t is not None else None

        def table(t, what, name, width, rows=None):
            if t is None:
                return None, 0, 0
            if t.dim() != 2 or t.shape[1] != width or (rows is not None and t.shape[0] != rows):
                _refuse(f"{what}: [{rows or 'sets'}][{width}] is wanted, got {tuple(t.shape)}")
            return (*_matrix(t, what, d, _of_type(t, what, name), t.shape[0], width), t.shape[0])
        if history is not None and history.dim() != 2:
            _refuse("history: [request][token] is wanted")
        hist = table(history, "history", "torch.int32", history.shape[1] if history is not None else 0, n)
        bia, allo = table(bias, "bias", "torch.float32", vocab), table(allowed, "allowed", "torch.int32", -(-vocab // 32))
        words = _words(masks)
        self.struct = ssd_logit_rules(
            vocab, n, n_rows, max_rows, dev(row_start, "row_start", "torch.int32", n + 1), hist[0], dev(history_len, "history_len", "torch.int32", n),
            dev(prompt_len, "prompt_len", "torch.int32", n), hist[1], history.shape[1] if history is not None else 0, words,
            dev(tokens, "tokens", "torch.int32", n_rows), dev(masks, "masks", "torch.int64", n_rows * words),
            *(dev(t, x, "torch.float32", n) for t, x in ((repetition, "repetition"), (presence, "presence"), (frequency, "frequency"))),
            bia[0], dev(bias_of, "bias_of", "torch.int32", n), allo[0], dev(allowed_of, "allowed_of", "torch.int32", n_rows), bia[1], allo[1], bia[2], allo[2])


def _logits(rules: LogitRules, t, what: str):
    """(type, device, address, row stride) of rows of logits."""
    kind = _ROW_TYPES.get(t.dtype)
    if kind is None:
        kind = _ROW_TYPES.get(str(t.dtype))
        if kind is None:
            _refuse(f"{what}: fp32, fp16 or bf16 rows are wanted")
        _ROW_TYPES[t.dtype] = kind
    d = t.get_device()
    if d < 0 or rules.device not in (None, d):
        _refuse(f"{what}: rows on the rules' CUDA device are wanted")
    return (kind, d, *_matrix(t, what, d, t.dtype, rules.n_rows, rules.vocab))


def ssd_logits_adjust(rules: LogitRules, logits, out, cuda_stream: int | None = None) -> None:
    """out [n_rows][vocab] = the logits after the rules, of their type (out may be logits)."""
    kind, d, ptr, stride = _logits(rules, logits, "logits")
    _check(lib.ssd_logits_adjust(rules.struct, kind, ptr, stride, *_matrix(out, "out", d, logits.dtype, rules.n_rows, rules.vocab), cuda_stream))


def ssd_logits_choose(rules: LogitRules, logits, tokens, logprob, total=None, cuda_stream: int | None = None) -> None:
    """The k best tokens int32 [n_rows][k] of every row after the rules, their log probabilities fp32 [n_rows][k] and the
    logsumexp fp32 [n_rows] (or None)."""
    kind, d, ptr, stride = _logits(rules, logits, "logits")
    if tokens.dim() != 2 or tokens.shape[0] != rules.n_rows:
        _refuse("tokens: [row][k] is wanted")
    n, f32 = tokens.numel(), _of_type(logprob, "logprob", "torch.float32")
    _check(lib.ssd_logits_choose(rules.struct, kind, ptr, stride, tokens.shape[1], _dev(tokens, "tokens", _of_type(tokens, "tokens", "torch.int32"), d, n),
                                 _dev(logprob, "logprob", f32, d, n), _dev(total, "total", f32, d, rules.n_rows), cuda_stream))


class MoeWeights:
    """Experts' matrices: gate and up [expert][f][d], down [expert][d][f], fp16 or bf16, each expert's contiguous.  Keeps the tensors."""

    def __init__(self, gate, up, down):
        if gate.dim() != 3 or up.shape != gate.shape or tuple(down.shape) != (gate.shape[0], gate.shape[2], gate.shape[1]):
            _refuse("gate and up [expert][f][d] and down [expert][d][f] are wanted")
        for t in (gate, up, down):
            if str(t.dtype) not in ("torch.float16", "torch.bfloat16") or t.dtype != gate.dtype or not t.is_cuda or t.get_device() != gate.get_device():
                _refuse("gate, up and down: fp16 or bf16 of one type on one CUDA device are wanted")
            if t.numel() and (t.stride(2) != 1 or t.stride(1) != t.shape[2]):
                _refuse("an expert's matrix must be contiguous")
        self.keep, self.device, self.dtype = (gate, up, down), gate.get_device(), gate.dtype
        self.n_experts, self.f, self.d = gate.shape
        strides = [t.stride(0) if self.n_experts > 1 else self.f * self.d for t in self.keep]
        self.struct = ssd_moe(*(t.data_ptr() for t in self.keep), *strides, _ROW_TYPES[str(gate.dtype)], self.n_experts, self.d, self.f)


def ssd_moe_route(x, w_router, ids, weights, score: int = SSD_MOE_SOFTMAX, favour=None, renorm: bool = True, scale: float = 1.0,
                  cuda_stream: int | None = None) -> None:
    """The experts ids int32 [n][k] of rows x [n][d] and their weights fp32 [n][k]; w_router [experts][d] of x's type,
    favour fp32 [experts] (added to the scores that choose) or None."""
    if x.dim() != 2 or w_router.dim() != 2 or ids.dim() != 2 or not x.is_cuda:
        _refuse("x [row][d], w_router [expert][d] and ids [row][k] on a CUDA device are wanted")
    kind = _half_type(x, "x")
    (n, d), e, k, dev = x.shape, w_router.shape[0], ids.shape[1], x.get_device()
    f32 = _of_type(weights, "weights", "torch.float32")
    _check(lib.ssd_moe_route(kind, n, d, e, k, *_matrix(x, "x", dev, x.dtype, n, d), _dev(w_router, "w_router", x.dtype, dev, e * d),
                             _dev(favour, "favour", f32, dev, e), score, int(bool(renorm)), scale,
                             _dev(ids, "ids", _of_type(ids, "ids", "torch.int32"), dev, n * k), _dev(weights, "weights", f32, dev, n * k), cuda_stream))


def ssd_moe_workspace(experts: MoeWeights, n_rows: int, k: int) -> int:
    """Bytes of workspace that ssd_moe_mlp wants for this many rows and slots (never fewer than for fewer of them)."""
    n = ctypes.c_size_t()
    _check(lib.ssd_moe_workspace(experts.struct, n_rows, k, n))
    return n.value


def ssd_moe_mlp(experts: MoeWeights, x, ids, weights, out, workspace, residual=None, status=None, cuda_stream: int | None = None) -> None:
    """out [n][d] = residual + the rows x [n][d] through their experts ids int32 [n][k], by weights fp32 [n][k].
    workspace: a contiguous uint8 tensor.  A wait that gave up leaves NaN in out; status int32 [1], set to 0 before, tells the reason."""
    if x.dim() != 2 or ids.dim() != 2:
        _refuse("x [row][d] and ids [row][k] are wanted")
    n, k, d, t = x.shape[0], ids.shape[1], experts.device, experts.dtype
    _check(lib.ssd_moe_mlp(experts.struct, n, k, *_matrix(x, "x", d, t, n, experts.d), _dev(ids, "ids", _of_type(ids, "ids", "torch.int32"), d, n * k),
                           _dev(weights, "weights", _of_type(weights, "weights", "torch.float32"), d, n * k),
                           *(_matrix(residual, "residual", d, t, n, experts.d) if residual is not None else (None, 0)),
                           *_matrix(out, "out", d, t, n, experts.d),
                           _dev(workspace, "workspace", _of_type(workspace, "workspace", "torch.uint8"), d, workspace.numel()), workspace.numel(),
                           _dev(status, "status", _of_type(status, "status", "torch.int32"), d, 1), cuda_stream))


def ssd_debug_moe_stall(cta: int, wait_limit_s: float = 0.01) -> None:
    """Test hook: a CTA of the next ssd_moe_mlp call never asks for its weights, so its waits give up after wait_limit_s."""
    if cta >= 0 and not 0.0 < wait_limit_s <= 10.0:
        _refuse("ssd_debug_moe_stall: 0 < wait_limit_s <= 10 is wanted")
    lib.ssd_debug_moe_stall(cta, wait_limit_s)


def ssd_destroy(h: int) -> None:
    if h:
        _configs.pop(h, None)
        lib.ssd_destroy(h)


def ssd_last_error() -> str:
    return lib.ssd_last_error().decode()


# -- marshalling helpers -----------------------------------------------------

_configs: dict = {}


def config_of(h: int) -> ssd_config:
    return _configs[h]


def make_config(n_layers, d_model, n_heads, n_kv_heads, head_dim, ffn, vocab, max_seq,
                rms_eps=1e-5, rope_theta=1e4) -> ssd_config:
    return ssd_config(n_layers, d_model, n_heads, n_kv_heads, head_dim, ffn, vocab, max_seq,
                      rms_eps, rope_theta)


class WeightRefs:
    """ssd_weights built from a dict {embed, final_norm, lm_head, layers:[{wq..}]}
    of torch tensors (on_device=1) or numpy arrays (on_device=0).  Keeps the
    pointer arrays alive."""

    def __init__(self, weights: dict, on_device: bool):
        L = len(weights["layers"])
        self.keep = [weights]
        self.struct = ssd_weights()
        self.struct.embed = _ptr(weights["embed"])
        self.struct.final_norm = _ptr(weights["final_norm"])
        self.struct.lm_head = _ptr(weights["lm_head"])
        for name in LAYER_TENSORS:
            arr = (ctypes.c_void_p * L)(*[_ptr(layer[name]) for layer in weights["layers"]])
            self.keep.append(arr)
            setattr(self.struct, name, ctypes.cast(arr, _VPP))
        self.struct.on_device = 1 if on_device else 0


class Decoder:
    """Owns one ssd handle (thin convenience wrapper over the C ABI)."""

    def __init__(self, cfg: ssd_config, weights: dict, on_device: bool = True, stream: int | None = None):
        self.cfg = cfg
        self.refs = WeightRefs(weights, on_device)
        self.h = ssd_create(cfg, self.refs.struct, stream)

    def close(self):
        if self.h:
            ssd_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_skip(self, mask):
        ssd_set_skip(self.h, mask)

    def set_sampling(self, temperature, top_p):
        ssd_set_sampling(self.h, temperature, top_p)

    def set_draft_exit(self, enable, gamma0=0.6, alpha=0.9, eps=0.01, beta1=0.5, beta2=0.9):
        ssd_set_draft_exit(self.h, enable, gamma0, alpha, eps, beta1, beta2)

    def prefill(self, prompt):
        ssd_prefill(self.h, prompt)

    def generate(self, prompt, n_new, K, mode=SSD_GREEDY, seed=0, out=None):
        return ssd_generate(self.h, prompt, n_new, K, mode, seed, out)

    def debug_forward(self, draft, tokens, pos0):
        return ssd_debug_forward(self.h, draft, tokens, pos0)

    def debug_stall_barrier(self, barrier, wait_limit_s):
        return ssd_debug_stall_barrier(self.h, barrier, wait_limit_s)

    def debug_spec_accept(self, p, q, drafts, seeds, pos0):
        return ssd_debug_spec_accept(self.h, p, q, drafts, seeds, pos0)

    def debug_time_forward(self, draft, rows, gemm_only, reps):
        return ssd_debug_time_forward(self.h, draft, rows, gemm_only, reps)

    def debug_trace_forward(self, draft, rows, detail_op=-1):
        return ssd_debug_trace_forward(self.h, draft, rows, detail_op)
