"""Thin Python binding of the C ABI in include/*.h (argument marshalling only).

Every step of the policy forward runs in libebrl.so's HIP kernels; this
module only passes device pointers (from torch tensors), host id arrays and
the stream handle.  PyTorch supplies device memory and streams.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libebrl.so")

EBRL_OK = 0
ERRORS = {-1: "EBRL_E_INVALID", -2: "EBRL_E_OOM", -3: "EBRL_E_HIP", -4: "EBRL_E_STATE",
          -5: "EBRL_E_UNSUPPORTED"}
DTYPE_FP32, DTYPE_BF16, DTYPE_BF16_KV8 = 0, 1, 2
STATE_H_LAST_PRE, STATE_H_LAST, STATE_K, STATE_V, STATE_FLOW_V0, STATE_PREFIX_LEN, STATE_GRAPHS = range(7)
K_GEMM, K_GEMM_SKINNY, K_ATTN_PREFILL, K_ATTN_DECODE, K_OTHER = range(5)
KERNEL_CLASSES = {K_GEMM: "gemm", K_GEMM_SKINNY: "gemm_skinny", K_ATTN_PREFILL: "attn_prefill",
                  K_ATTN_DECODE: "attn_decode", K_OTHER: "other"}

_I32 = ctypes.c_int32


class Config(ctypes.Structure):
    _fields_ = [(n, _I32) for n in (
        "dtype", "n_cams", "img", "patch", "vit_layers", "vit_d", "vit_heads", "vit_mlp",
        "layers", "d", "q_heads", "kv_heads", "head_dim", "mlp", "vocab", "n_lang",
        "action_logits", "n_action_tokens", "n_bins",
        "exp_layers", "exp_d", "exp_heads", "exp_mlp", "chunk", "adim", "n_steps",
        "max_envs", "max_seq")] + [("kv_budget_bytes", ctypes.c_int64), ("init_std", ctypes.c_double),
                                   ("frame_tokens", _I32), ("frame_dim", _I32)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class ObsBatch(ctypes.Structure):
    _fields_ = [("images", ctypes.c_void_p), ("lang_ids", ctypes.c_void_p),
                ("lang_len", ctypes.c_void_p), ("lang_stride", _I32)]


_PI32, _PF64 = ctypes.POINTER(_I32), ctypes.POINTER(ctypes.c_double)


class AllocProfiles(ctypes.Structure):
    _fields_ = [("n_cenv", _I32), ("cenv", _PI32), ("n_ssim", _I32), ("ssim", _PI32), ("sim_rate", _PF64),
                ("n_sgen", _I32), ("sgen", _PI32), ("n_bgen", _I32), ("bgen", _PI32), ("gen_rate", _PF64),
                ("gen_mem", _PF64),
                ("n_strain", _I32), ("strain", _PI32), ("n_btrain", _I32), ("btrain", _PI32),
                ("train_rate", _PF64), ("train_mem", _PF64)]


class AllocLimits(ctypes.Structure):
    _fields_ = [("cores", _I32), ("mem_bytes", ctypes.c_double), ("sgen_min", _I32), ("strain_min", _I32),
                ("knee_tol", ctypes.c_double)]


class AllocResult(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("cenv", "envs", "ssim", "sgen", "strain", "bgen", "btrain", "iterations")] + \
               [(n, ctypes.c_double) for n in ("t_sim", "t_gen", "t_train", "t_rollout", "theta")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class Kv8Cache(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("block_table", ctypes.c_void_p)] + \
               [(n, _I32) for n in ("num_blocks", "table_rows", "table_stride", "kv_heads", "head_dim")]


class Kv8WriteArgs(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("dtype", "n", "rows", "max_len", "q_heads", "n_axes")] + \
               [("sections", _I32 * 3), ("tab_rows", _I32)] + \
               [(n, ctypes.c_void_p) for n in ("q", "k", "v", "q_out")] + \
               [(n, ctypes.c_int64) for n in ("ldq", "ldk", "ldv", "ldq_out")] + \
               [(n, ctypes.c_void_p) for n in ("row_start", "pos0", "seq", "axis_pos", "cos_tab", "sin_tab")]


class Kv8AttnArgs(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("dtype", "n", "rows", "max_q_len", "max_kv_len", "q_heads", "causal")] + \
               [("scale", ctypes.c_float)] + [(n, ctypes.c_void_p) for n in ("q", "out")] + \
               [(n, ctypes.c_int64) for n in ("ldq", "ldo")] + \
               [(n, ctypes.c_void_p) for n in ("row_start", "kv_len", "seq", "workspace")] + \
               [("workspace_bytes", ctypes.c_int64)]


class EbrlError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


_LIB = None

EXPORTED = [
    "ebrl_config_preset", "ebrl_policy_create", "ebrl_policy_destroy",
    "ebrl_stream_create_cu_masked", "ebrl_stream_destroy", "ebrl_policy_bind_stream",
    "ebrl_prefill", "ebrl_decode_actions", "ebrl_flow_denoise", "ebrl_wam_denoise", "ebrl_last_error",
    "ebrl_read_state", "ebrl_generate_weight_host", "ebrl_read_weight", "ebrl_write_weight",
    "ebrl_profile_enable", "ebrl_profile_read", "ebrl_op_gemm", "ebrl_op_gemm_plan",
    "ebrl_op_gemm_noalloc", "ebrl_op_stream_read",
    "ebrl_op_kv8_write", "ebrl_op_kv8_attn", "ebrl_op_kv8_attn_workspace",
    "ebrl_alloc_solve", "ebrl_alloc_objective", "ebrl_alloc_monitor_create", "ebrl_alloc_monitor_observe",
    "ebrl_alloc_monitor_destroy", "ebrl_alloc_refine",
    "ebrl_sched_create", "ebrl_sched_destroy", "ebrl_sched_dispatch", "ebrl_sched_complete",
    "ebrl_sched_next_group", "ebrl_sched_deliver", "ebrl_sched_env_state",
]


def lib():
    """Load libebrl.so; raises if it has not been built (there is no fallback)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -c 'import __graft_entry__ as g; g.build()'`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u32, u64 = ctypes.c_void_p, _I32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64
    pI32 = ctypes.POINTER(_I32)
    sig = {
        "ebrl_config_preset": (i32, [i32, ctypes.POINTER(Config)]),
        "ebrl_policy_create": (i32, [ctypes.POINTER(Config), u64, ctypes.POINTER(vp)]),
        "ebrl_policy_destroy": (None, [vp]),
        "ebrl_stream_create_cu_masked": (i32, [i32, ctypes.POINTER(u32), u32, ctypes.POINTER(vp)]),
        "ebrl_stream_destroy": (i32, [vp]),
        "ebrl_policy_bind_stream": (i32, [vp, vp]),
        "ebrl_prefill": (i32, [vp, ctypes.POINTER(ObsBatch), pI32, i32]),
        "ebrl_decode_actions": (i32, [vp, pI32, i32, vp, vp, vp]),
        "ebrl_flow_denoise": (i32, [vp, pI32, i32, vp, vp]),
        "ebrl_wam_denoise": (i32, [vp, pI32, i32, vp, vp, vp, vp]),
        "ebrl_last_error": (ctypes.c_char_p, [vp]),
        "ebrl_read_state": (i32, [vp, i32, i32, i32, vp, i64]),
        "ebrl_generate_weight_host": (i32, [u64, u32, i64, ctypes.c_double, i32, vp]),
        "ebrl_read_weight": (i32, [vp, u32, vp, i64]),
        "ebrl_write_weight": (i32, [vp, u32, vp, i64]),
        "ebrl_profile_enable": (i32, [vp, i32]),
        "ebrl_profile_read": (i32, [vp, i32, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double),
                                    ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), i32]),
        "ebrl_op_gemm": (i32, [i32, vp, vp, vp, i32, i32, i32, vp]),
        "ebrl_op_gemm_plan": (i32, [i32, i32, i32, i32, i32, i32, vp]),
        "ebrl_op_gemm_noalloc": (i32, [i32, vp, vp, vp, i32, i32, i32, vp]),
        "ebrl_op_stream_read": (i32, [vp, i64, vp, vp]),
        # structs by reference, or their bytes
        "ebrl_op_kv8_write": (i32, [vp, vp, vp]),
        "ebrl_op_kv8_attn": (i32, [vp, vp, vp]),
        "ebrl_op_kv8_attn_workspace": (i64, [vp, vp]),
        "ebrl_alloc_solve": (i32, [ctypes.POINTER(AllocProfiles), ctypes.POINTER(AllocLimits),
                                   ctypes.POINTER(AllocResult)]),
        "ebrl_alloc_objective": (i32, [ctypes.POINTER(AllocProfiles), ctypes.POINTER(AllocResult)]),
        "ebrl_alloc_monitor_create": (i32, [i32, ctypes.c_double, i32, ctypes.POINTER(vp)]),
        "ebrl_alloc_monitor_observe": (i32, [vp, ctypes.c_double, ctypes.c_double, pI32]),
        "ebrl_alloc_monitor_destroy": (None, [vp]),
        "ebrl_alloc_refine": (i32, [ctypes.POINTER(AllocProfiles), ctypes.POINTER(AllocResult), ctypes.c_double,
                                    ctypes.c_double, _PF64, _PF64]),
        "ebrl_sched_create": (i32, [i32, i32, i32, ctypes.POINTER(vp)]),
        "ebrl_sched_destroy": (None, [vp]),
        "ebrl_sched_dispatch": (i32, [vp, i32, i32, pI32]),
        "ebrl_sched_complete": (i32, [vp, i32, ctypes.c_double, pI32]),
        "ebrl_sched_next_group": (i32, [vp, pI32, pI32, i32, pI32]),
        "ebrl_sched_deliver": (i32, [vp, i32]),
        "ebrl_sched_env_state": (i32, [vp, i32, pI32, pI32, pI32, _PF64]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _LIB = L
    return L


def preset(n: int) -> Config:
    c = Config()
    rc = lib().ebrl_config_preset(n, ctypes.byref(c))
    if rc != EBRL_OK:
        raise EbrlError(rc, f"unknown preset {n}")
    return c


def _ids(env_ids) -> ctypes.Array:
    a = np.ascontiguousarray(np.asarray(env_ids, dtype=np.int32))
    return a, a.ctypes.data_as(ctypes.POINTER(_I32))


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


# ---------------------------------------------------- resource allocator --

def _alloc_profiles(P: dict):
    """Marshals a profile dict (cenv, ssim, sim[C, S], sgen, bgen, gen[G, Bg],
    gen_mem, strain, btrain, train[H, Bt], train_mem) into the C struct;
    returns the struct and the arrays it points into (kept alive by the
    caller)."""
    keep = {}

    def i32(k):
        keep[k] = np.ascontiguousarray(np.asarray(P[k], dtype=np.int32))
        return len(keep[k]), keep[k].ctypes.data_as(_PI32)

    def f64(k):
        keep[k] = np.ascontiguousarray(np.asarray(P[k], dtype=np.float64))
        return keep[k].ctypes.data_as(_PF64)

    pr = AllocProfiles()
    pr.n_cenv, pr.cenv = i32("cenv")
    pr.n_ssim, pr.ssim = i32("ssim")
    pr.sim_rate = f64("sim")
    pr.n_sgen, pr.sgen = i32("sgen")
    pr.n_bgen, pr.bgen = i32("bgen")
    pr.gen_rate, pr.gen_mem = f64("gen"), f64("gen_mem")
    pr.n_strain, pr.strain = i32("strain")
    pr.n_btrain, pr.btrain = i32("btrain")
    pr.train_rate, pr.train_mem = f64("train"), f64("train_mem")
    for k, shape in (("sim", (pr.n_cenv, pr.n_ssim)), ("gen", (pr.n_sgen, pr.n_bgen)),
                     ("train", (pr.n_strain, pr.n_btrain))):
        if keep[k].shape != shape:
            raise EbrlError(-1, f"profile table {k} has shape {keep[k].shape}, expected {shape}")
    for k, n in (("gen_mem", pr.n_bgen), ("train_mem", pr.n_btrain)):
        if keep[k].shape != (n,):
            raise EbrlError(-1, f"{k} has shape {keep[k].shape}, expected ({n},)")
    return pr, keep


def alloc_solve(P: dict, cores: int, mem_bytes: float, sgen_min: int, strain_min: int,
                knee_tol: float = 0.05) -> dict:
    """Algorithm 1 through the library (include/ebrl_alloc.h)."""
    pr, keep = _alloc_profiles(P)
    lim = AllocLimits(cores, mem_bytes, sgen_min, strain_min, knee_tol)
    out = AllocResult()
    rc = lib().ebrl_alloc_solve(ctypes.byref(pr), ctypes.byref(lim), ctypes.byref(out))
    if rc != EBRL_OK:
        raise EbrlError(rc, "ebrl_alloc_solve")
    return out.as_dict()


def alloc_objective(P: dict, cfg: dict) -> dict:
    pr, keep = _alloc_profiles(P)
    out = AllocResult(**{k: cfg[k] for k in ("sgen", "strain", "bgen", "btrain", "t_sim")})
    rc = lib().ebrl_alloc_objective(ctypes.byref(pr), ctypes.byref(out))
    if rc != EBRL_OK:
        raise EbrlError(rc, "ebrl_alloc_objective")
    return out.as_dict()


def alloc_refine(P: dict, cur: dict, observed_gen: float, observed_train: float):
    pr, keep = _alloc_profiles(P)
    res = AllocResult(**{k: cur[k] for k in ("bgen", "btrain", "t_gen", "t_train")})
    gen = np.empty_like(keep["gen"])
    train = np.empty_like(keep["train"])
    rc = lib().ebrl_alloc_refine(ctypes.byref(pr), ctypes.byref(res), observed_gen, observed_train,
                                 gen.ctypes.data_as(_PF64), train.ctypes.data_as(_PF64))
    if rc != EBRL_OK:
        raise EbrlError(rc, "ebrl_alloc_refine")
    return gen, train


class AllocMonitor:
    """The runtime adaptation trigger (ebrl_alloc_monitor_*)."""

    def __init__(self, window: int = 20, gap: float = 0.15, patience: int = 20):
        h = ctypes.c_void_p()
        rc = lib().ebrl_alloc_monitor_create(window, gap, patience, ctypes.byref(h))
        if rc != EBRL_OK:
            raise EbrlError(rc, "ebrl_alloc_monitor_create")
        self.h = h.value

    def observe(self, rollout_rate: float, train_rate: float) -> bool:
        t = _I32()
        rc = lib().ebrl_alloc_monitor_observe(self.h, rollout_rate, train_rate, ctypes.byref(t))
        if rc != EBRL_OK:
            raise EbrlError(rc, "ebrl_alloc_monitor_observe")
        return bool(t.value)

    def close(self):
        if self.h:
            lib().ebrl_alloc_monitor_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------ rollout scheduler --

class Sched:
    """The group pipeline and Algorithm 2 dispatcher (include/ebrl_sched.h)."""

    def __init__(self, n_envs: int, n_groups: int, chunk_len: int):
        h = ctypes.c_void_p()
        rc = lib().ebrl_sched_create(n_envs, n_groups, chunk_len, ctypes.byref(h))
        if rc != EBRL_OK:
            raise EbrlError(rc, "ebrl_sched_create")
        self.h = h.value
        self.n_envs = n_envs
        self._ids = np.empty(n_envs, dtype=np.int32)

    def _check(self, rc, what):
        if rc != EBRL_OK:
            raise EbrlError(rc, what)

    def dispatch(self, core: int = 0, bind_stride: int = 0) -> int:
        e = _I32()
        self._check(lib().ebrl_sched_dispatch(self.h, core, bind_stride, ctypes.byref(e)), "ebrl_sched_dispatch")
        return e.value

    def complete(self, env: int, duration: float) -> bool:
        d = _I32()
        self._check(lib().ebrl_sched_complete(self.h, env, duration, ctypes.byref(d)), "ebrl_sched_complete")
        return bool(d.value)

    def next_group(self):
        g, n = _I32(), _I32()
        self._check(lib().ebrl_sched_next_group(self.h, ctypes.byref(g), self._ids.ctypes.data_as(_PI32),
                                                self.n_envs, ctypes.byref(n)), "ebrl_sched_next_group")
        return g.value, self._ids[:n.value].copy()

    def deliver(self, group: int) -> None:
        self._check(lib().ebrl_sched_deliver(self.h, group), "ebrl_sched_deliver")

    def env_state(self, env: int):
        a, b, c, d = _I32(), _I32(), _I32(), ctypes.c_double()
        self._check(lib().ebrl_sched_env_state(self.h, env, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c),
                                               ctypes.byref(d)), "ebrl_sched_env_state")
        return a.value, bool(b.value), bool(c.value), d.value

    def close(self):
        if self.h:
            lib().ebrl_sched_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def generate_weight_host(seed: int, tensor_id: int, count: int, std: float, bf16: bool) -> np.ndarray:
    out = np.empty(count, dtype=np.uint16 if bf16 else np.float32)
    rc = lib().ebrl_generate_weight_host(seed, tensor_id, count, std, int(bf16), out.ctypes.data)
    if rc != EBRL_OK:
        raise EbrlError(rc, "generate_weight_host")
    return out


def op_gemm(A, B, C, stream=None, noalloc=False) -> None:
    """C = A B^T through the library's GEMM kernel (torch device tensors);
    noalloc: the entry point that allocates nothing (fixed device scratch)."""
    import torch
    dt = DTYPE_BF16 if A.dtype == torch.bfloat16 else DTYPE_FP32
    M, K = A.shape
    N = B.shape[0]
    s = stream if stream is not None else torch.cuda.current_stream().cuda_stream
    fn = lib().ebrl_op_gemm_noalloc if noalloc else lib().ebrl_op_gemm
    rc = fn(dt, A.data_ptr(), B.data_ptr(), C.data_ptr(), M, N, K, s)
    if rc != EBRL_OK:
        raise EbrlError(rc, "ebrl_op_gemm_noalloc" if noalloc else "ebrl_op_gemm")


def op_gemm_plan(M, N, K, dtype=DTYPE_BF16, in_order=False, cus=256) -> dict:
    """The kernel that computes an M x N x K product (no GPU needed)."""
    plan = (ctypes.c_int32 * 8)()
    rc = lib().ebrl_op_gemm_plan(dtype, M, N, K, int(in_order), cus, plan)
    if rc != EBRL_OK:
        raise EbrlError(rc, "ebrl_op_gemm_plan")
    names = ("kernel", "rows", "cols", "splits", "workgroups", "stages", "even", "cut")
    out = dict(zip(names, plan))
    out["kernel"] = ("tiles", "large", "ring", "decode", "fp32")[out["kernel"]]
    return out


def op_stream_read(buf, out, stream=None) -> None:
    """Streaming read of a device tensor's bytes (the HBM read reference)."""
    import torch
    s = stream if stream is not None else torch.cuda.current_stream().cuda_stream
    rc = lib().ebrl_op_stream_read(buf.data_ptr(), buf.numel() * buf.element_size(), out.data_ptr(), s)
    if rc != EBRL_OK:
        raise EbrlError(rc, "ebrl_op_stream_read")


# ------------------------------------------------------- 8-bit KV cache --
# include/ebrl_kv8.h.  The cache is three tensors on one GPU: codes, float8_e4m3fn
# (or their bytes, uint8 or int8), [num_blocks, 2, kv_heads, 16 * head_dim]; scales,
# float32 [num_blocks, 2, kv_heads]; block_table, int32 [sequences, pages].

KV8_PAGE = 16


def kv8_alloc(num_blocks: int, kv_heads: int, head_dim: int, device="cuda"):
    """(codes, scales) of an empty 8-bit cache, the codes as float8_e4m3fn."""
    import torch
    codes = torch.zeros((num_blocks, 2, kv_heads, KV8_PAGE * head_dim), dtype=torch.uint8, device=device)
    return codes.view(torch.float8_e4m3fn), torch.ones((num_blocks, 2, kv_heads), device=device)


def _kv8_bad(what: str, *tensors):
    raise EbrlError(-1, "kv8: " + what + "".join(
        f"; got {None if t is None else (tuple(t.shape), t.stride(), t.dtype, str(t.device))}" for t in tensors))


# The C structs, packed: these checks and this packing run before every launch
# and take longer than a small kernel, so each property of a tensor is asked for
# once and the structs are made from a format (a ctypes.Structure takes twice
# the time to fill).
_KV8_CACHE = struct.Struct("3P5i0P")
_KV8_WRITE = struct.Struct("10i4P4q6P")
_KV8_ATTN = struct.Struct("7if2P2q4Pq")


def _kv8_pack(packer, *values) -> bytes:
    try:
        return packer.pack(*values)
    except (struct.error, OverflowError) as e:
        raise EbrlError(-1, f"kv8: sizes pass 32 bits: {e}") from e


def _kv8_codes(t) -> bool:
    import torch
    dtype = t.dtype
    return dtype is torch.float8_e4m3fn or dtype is torch.uint8 or dtype is torch.int8


def _kv8_cache(codes, scales, table):
    """The packed cache, its KV heads and head dim and its GPU's index (-1: not on a GPU)."""
    import torch
    dev = codes.get_device()
    try:
        blocks, two, heads, wide = codes.shape
    except ValueError:
        two = wide = 0
    if two != 2 or not wide or wide % KV8_PAGE or not _kv8_codes(codes) or not codes.is_contiguous():
        _kv8_bad("codes are contiguous float8_e4m3fn or bytes [num_blocks, 2, kv_heads, 16 * head_dim]", codes)
    if scales.shape != (blocks, 2, heads) or scales.dtype is not torch.float32 or not scales.is_contiguous() or \
            scales.get_device() != dev:
        _kv8_bad("scales are contiguous float32 [num_blocks, 2, kv_heads] where the codes are", scales)
    pages = table.shape
    if len(pages) != 2 or table.dtype is not torch.int32 or not table.is_contiguous() or table.get_device() != dev:
        _kv8_bad("block_table is contiguous int32 [sequences, pages] where the codes are", table)
    hd = wide // KV8_PAGE
    c = _kv8_pack(_KV8_CACHE, codes.data_ptr(), scales.data_ptr(), table.data_ptr(), blocks, *pages, heads, hd)
    return c, heads, hd, dev


def _kv8_rows(name, t, dtype, dev, rows, width):
    """Pointer and row stride of a [rows, width] tensor whose rows are contiguous."""
    if t.shape != (rows, width) or t.dtype is not dtype or t.get_device() != dev:
        _kv8_bad(f"{name} is {dtype} [{rows}, {width}] where the cache is", t)
    ld, one = t.stride()
    if one != 1 and width > 1:
        _kv8_bad(f"{name} has contiguous rows", t)
    return t.data_ptr(), ld if rows > 1 else width


def _kv8_ints(dtype, dev, *named):
    """Pointers of the (name, tensor or None, elements) given; 0 for None."""
    at = []
    for name, t, n in named:
        if t is None:
            at.append(0)
            continue
        if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
            _kv8_bad(f"{name} is {n} contiguous int32 where the cache is", t)
        at.append(t.data_ptr())
    return at


def _kv8_dtype(name, t) -> int:
    import torch
    dtype = t.dtype
    if t.dim() != 2 or (dtype is not torch.bfloat16 and dtype is not torch.float32):
        _kv8_bad(f"{name} is bfloat16 or float32 [rows, heads * head_dim]", t)
    return DTYPE_BF16 if dtype is torch.bfloat16 else DTYPE_FP32


def _kv8_call(fn, name, cache, args, dev, stream):
    """The call on `stream` (None: the current one of the cache's device)."""
    import torch
    if dev < 0:
        _kv8_bad("the cache is not on a GPU")
    if dev != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            return _kv8_call(fn, name, cache, args, dev, stream)
    if stream is None:
        # the handle alone: a torch.cuda.Stream object takes 2.7 us to make,
        # as long as the launch
        stream = torch._C._cuda_getCurrentRawStream(dev)
    rc = fn(cache, args, stream)
    if rc != EBRL_OK:
        raise EbrlError(rc, name)


def op_kv8_write(codes, scales, block_table, k, v, row_start, pos0, max_len, q=None, q_out=None, sections=(),
                 axis_pos=None, cos=None, sin=None, seq=None, stream=None) -> None:
    """Rotary positions on q and k and the write of k and v into the cache
    (ebrl_op_kv8_write).  k, v, q, q_out: [rows, heads * head_dim]; row_start
    [n + 1], pos0 [n], seq [n]: int32; axis_pos: int32 [rows, axes]; sections:
    pairs of each axis (empty: no rotation); cos, sin: float32 [positions,
    head_dim / 2].  `stream`: a raw handle whose order the tensors follow."""
    import torch
    c, heads, hd, dev = _kv8_cache(codes, scales, block_table)
    n, axes, dtype = pos0.numel(), len(sections), _kv8_dtype("k", k)
    rows, torch_dtype, width = k.shape[0], k.dtype, heads * hd
    if not 0 <= max_len < 1 << 31:
        _kv8_bad(f"max_len {max_len}")
    k_at, ldk = _kv8_rows("k", k, torch_dtype, dev, rows, width)
    v_at, ldv = _kv8_rows("v", v, torch_dtype, dev, rows, width)
    if (q is None) != (q_out is None) or axes > 3 or (axes == 0 and q is not None):
        _kv8_bad("q and q_out go together, with one to three axes", q, q_out)
    q_at = ldq = qo_at = ldqo = q_heads = tab_rows = cos_at = sin_at = 0
    if q is not None:
        wide = q.shape[-1]
        if wide % hd:
            _kv8_bad(f"q has heads of {hd}", q)
        q_at, ldq = _kv8_rows("q", q, torch_dtype, dev, rows, wide)
        qo_at, ldqo = _kv8_rows("q_out", q_out, torch_dtype, dev, rows, wide)
        q_heads = wide // hd
    if axes:
        tab_rows = 0 if cos is None else cos.shape[0]
        for t in (cos, sin):
            if t is None or t.shape != (tab_rows, hd // 2) or t.dtype is not torch.float32 or not t.is_contiguous() or \
                    t.get_device() != dev:
                _kv8_bad(f"cos and sin are contiguous float32 [positions, {hd // 2}] where the cache is", cos, sin)
        cos_at, sin_at = cos.data_ptr(), sin.data_ptr()
    start_at, pos_at, seq_at, axis_at = _kv8_ints(
        torch.int32, dev, ("row_start", row_start, n + 1), ("pos0", pos0, n), ("seq", seq, n),
        ("axis_pos", axis_pos if axes else None, rows * axes))
    try:
        a = _KV8_WRITE.pack(dtype, n, rows, max_len, q_heads, axes, *sections, *(0, 0, 0)[axes:], tab_rows, q_at, k_at,
                            v_at, qo_at, ldq, ldk, ldv, ldqo, start_at, pos_at, seq_at, axis_at, cos_at, sin_at)
    except struct.error as e:
        raise EbrlError(-1, f"kv8: sections {sections}: {e}") from e
    _kv8_call(lib().ebrl_op_kv8_write, "ebrl_op_kv8_write", c, a, dev, stream)


def _kv8_bounds(max_q_len, max_kv_len):
    if not 0 <= max_q_len < 1 << 31 or not 0 <= max_kv_len <= 1 << 30:
        _kv8_bad(f"max_q_len {max_q_len}, max_kv_len {max_kv_len} (at most 2^30)")


def kv8_attn_workspace(codes, block_table, q, n, max_q_len, max_kv_len):
    """A workspace for op_kv8_attn calls with these sizes, on the cache's device."""
    import torch
    _kv8_bounds(max_q_len, max_kv_len)
    if codes.dim() != 4 or codes.shape[3] < KV8_PAGE or not _kv8_codes(codes) or block_table.dim() != 2:
        _kv8_bad("codes are [num_blocks, 2, kv_heads, 16 * head_dim], block_table [sequences, pages]", codes, block_table)
    blocks, _, heads, wide = codes.shape
    hd = wide // KV8_PAGE
    c = _kv8_pack(_KV8_CACHE, 0, 0, 0, blocks, *block_table.shape, heads, hd)
    dtype = _kv8_dtype("q", q)
    if q.shape[1] % hd:
        _kv8_bad(f"q has heads of {hd}", q)
    if not 0 <= n < 1 << 31:
        _kv8_bad(f"n {n}")
    a = _kv8_pack(_KV8_ATTN, dtype, n, q.shape[0], max_q_len, max_kv_len, q.shape[1] // hd, 1, 1.0, *(0,) * 9)
    need = lib().ebrl_op_kv8_attn_workspace(c, a)
    if need < 0:
        raise EbrlError(need, "ebrl_op_kv8_attn_workspace")
    return torch.empty(need, dtype=torch.uint8, device=codes.device)


def op_kv8_attn(codes, scales, block_table, q, out, row_start, kv_len, max_q_len, max_kv_len, causal=True, scale=None,
                workspace=None, seq=None, stream=None) -> None:
    """out = softmax(scale q K^T) V over the 8-bit cache (ebrl_op_kv8_attn).
    q, out: [rows, heads * head_dim]; row_start [n + 1], kv_len [n], seq [n]:
    int32; scale None: 1 / sqrt(head_dim).  workspace: from
    kv8_attn_workspace, one for each chain of calls that may overlap others;
    None makes one for this call (not with an explicit stream, which torch's
    allocator does not follow)."""
    import torch
    c, heads, hd, dev = _kv8_cache(codes, scales, block_table)
    n, dtype = kv_len.numel(), _kv8_dtype("q", q)
    rows, wide = q.shape
    if wide % hd:
        _kv8_bad(f"q has heads of {hd}", q)
    _kv8_bounds(max_q_len, max_kv_len)
    q_at, ldq = _kv8_rows("q", q, q.dtype, dev, rows, wide)
    out_at, ldo = _kv8_rows("out", out, q.dtype, dev, rows, wide)
    if workspace is None:
        if stream is not None:
            _kv8_bad("a call on an explicit stream needs a workspace")
        workspace = kv8_attn_workspace(codes, block_table, q, n, max_q_len, max_kv_len)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        _kv8_bad("the workspace is contiguous and where the cache is", workspace)
    start_at, len_at, seq_at = _kv8_ints(torch.int32, dev, ("row_start", row_start, n + 1), ("kv_len", kv_len, n),
                                         ("seq", seq, n))
    try:
        a = _KV8_ATTN.pack(dtype, n, rows, max_q_len, max_kv_len, wide // hd, 1 if causal else 0,
                           hd ** -0.5 if scale is None else scale, q_at, out_at, ldq, ldo, start_at, len_at, seq_at,
                           workspace.data_ptr(), workspace.nbytes)
    except (struct.error, OverflowError) as e:
        raise EbrlError(-1, f"kv8: scale {scale}: {e}") from e
    _kv8_call(lib().ebrl_op_kv8_attn, "ebrl_op_kv8_attn", c, a, dev, stream)


def create_cu_masked_stream(device: int, mask_words: Sequence[int]) -> int:
    arr = (ctypes.c_uint32 * len(mask_words))(*[int(w) & 0xFFFFFFFF for w in mask_words])
    out = ctypes.c_void_p()
    rc = lib().ebrl_stream_create_cu_masked(device, arr, len(mask_words), ctypes.byref(out))
    if rc != EBRL_OK:
        raise EbrlError(rc, lib().ebrl_last_error(None).decode())
    return out.value


def destroy_stream(s: int) -> None:
    lib().ebrl_stream_destroy(s)


class Policy:
    """One policy on the current device; calls enqueue on the bound stream."""

    def __init__(self, config, seed: int = 0, stream=None, **overrides):
        import torch
        cfg = preset(config) if isinstance(config, int) else config
        for k, v in overrides.items():
            setattr(cfg, k, v)
        self.cfg = cfg
        self.seed = seed
        h = ctypes.c_void_p()
        rc = lib().ebrl_policy_create(ctypes.byref(cfg), seed, ctypes.byref(h))
        if rc != EBRL_OK:
            raise EbrlError(rc, lib().ebrl_last_error(None).decode())
        self.h = h.value
        self.torch = torch
        self.bind_stream(stream if stream is not None else torch.cuda.current_stream().cuda_stream)

    # lifecycle -------------------------------------------------------------
    def close(self):
        if getattr(self, "h", None):
            lib().ebrl_policy_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, what):
        if rc != EBRL_OK:
            raise EbrlError(rc, f"{what}: {lib().ebrl_last_error(self.h).decode()}")

    def bind_stream(self, stream) -> None:
        self.stream = int(stream or 0)
        self._check(lib().ebrl_policy_bind_stream(self.h, self.stream or None), "bind_stream")

    @property
    def bf16(self) -> bool:
        return self.cfg.dtype != DTYPE_FP32

    # calls -----------------------------------------------------------------
    def prefill(self, env_ids, images=None, lang_ids=None, lang_len=None) -> None:
        ids, pids = _ids(env_ids)
        ob = ObsBatch()
        ob.images = _ptr(images)
        ob.lang_ids = _ptr(lang_ids)
        ob.lang_stride = int(lang_ids.shape[1]) if lang_ids is not None else 0
        ll = None
        if lang_len is not None:
            ll = np.ascontiguousarray(np.asarray(lang_len, dtype=np.int32))
            ob.lang_len = ll.ctypes.data
        self._keep = (ids, ll, images, lang_ids)
        self._check(lib().ebrl_prefill(self.h, ctypes.byref(ob), pids, len(ids)), "prefill")

    def decode_actions(self, env_ids, tokens=None, actions=None, margins=None, with_margin=True):
        torch = self.torch
        ids, pids = _ids(env_ids)
        n, nt = len(ids), self.cfg.n_action_tokens
        dev = torch.device("cuda", torch.cuda.current_device())
        if tokens is None:
            tokens = torch.empty((n, nt), dtype=torch.int32, device=dev)
        if actions is None:
            actions = torch.empty((n, nt), dtype=torch.float32, device=dev)
        if margins is None and with_margin:
            margins = torch.empty((n, nt), dtype=torch.float32, device=dev)
        self._check(lib().ebrl_decode_actions(self.h, pids, n, _ptr(tokens), _ptr(actions), _ptr(margins)),
                    "decode_actions")
        return tokens, actions, margins

    def _chunk_out(self, n, rows, cols):
        return self.torch.empty((n, rows, cols), dtype=self.torch.float32, device="cuda")

    def flow_denoise(self, env_ids, noise=None, out=None):
        """noise None: the library draws it (seeded, per-env call count)."""
        ids, pids = _ids(env_ids)
        if out is None:
            out = self._chunk_out(len(ids), self.cfg.chunk, self.cfg.adim) if noise is None else \
                self.torch.empty_like(noise)
        self._check(lib().ebrl_flow_denoise(self.h, pids, len(ids), _ptr(noise), _ptr(out)), "flow_denoise")
        return out

    def wam_denoise(self, env_ids, frame_noise=None, action_noise=None, out_frames=None, out_actions=None):
        """Joint denoising of future-frame latents and the action chunk;
        a noise of None is drawn by the library."""
        ids, pids = _ids(env_ids)
        c = self.cfg
        if out_frames is None:
            out_frames = self._chunk_out(len(ids), c.frame_tokens, c.frame_dim) if frame_noise is None else \
                self.torch.empty_like(frame_noise)
        if out_actions is None:
            out_actions = self._chunk_out(len(ids), c.chunk, c.adim) if action_noise is None else \
                self.torch.empty_like(action_noise)
        self._check(lib().ebrl_wam_denoise(self.h, pids, len(ids), _ptr(frame_noise), _ptr(action_noise),
                                           _ptr(out_frames), _ptr(out_actions)), "wam_denoise")
        return out_frames, out_actions

    # inspection ------------------------------------------------------------
    def read_state(self, what: int, env_id: int, layer: int = 0) -> np.ndarray:
        c = self.cfg
        if what in (STATE_H_LAST_PRE, STATE_H_LAST):
            out = np.empty(c.d, dtype=np.float32)
        elif what in (STATE_PREFIX_LEN, STATE_GRAPHS):
            out = np.empty(1, dtype=np.int32)
        elif what == STATE_FLOW_V0:
            out = np.empty((c.chunk, c.adim), dtype=np.float32)
        else:
            T = int(self.read_state(STATE_PREFIX_LEN, env_id)[0])
            out = np.empty((T, c.kv_heads, c.head_dim), dtype=np.uint16 if self.bf16 else np.float32)
        self._check(lib().ebrl_read_state(self.h, what, env_id, layer, out.ctypes.data, out.nbytes), "read_state")
        return out

    def read_weight(self, tensor_id: int, shape) -> np.ndarray:
        out = np.empty(shape, dtype=np.uint16 if self.bf16 else np.float32)
        self._check(lib().ebrl_read_weight(self.h, tensor_id, out.ctypes.data, out.nbytes), "read_weight")
        return out

    def write_weight(self, tensor_id: int, values: np.ndarray) -> None:
        a = np.ascontiguousarray(values, dtype=np.uint16 if self.bf16 else np.float32)
        self._check(lib().ebrl_write_weight(self.h, tensor_id, a.ctypes.data, a.nbytes), "write_weight")

    def profile_enable(self, classes=(K_GEMM, K_GEMM_SKINNY, K_ATTN_PREFILL, K_ATTN_DECODE, K_OTHER)) -> None:
        mask = 0
        for c in classes:
            mask |= 1 << c
        self._check(lib().ebrl_profile_enable(self.h, mask), "profile_enable")

    def profile_read(self, cls: int, reset: bool = False) -> dict:
        n = ctypes.c_int64()
        ms, fl, by = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
        self._check(lib().ebrl_profile_read(self.h, cls, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(fl),
                                            ctypes.byref(by), int(reset)), "profile_read")
        return {"launches": n.value, "ms": ms.value, "flop": fl.value, "bytes": by.value}
