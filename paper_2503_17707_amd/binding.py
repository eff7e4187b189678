"""Thin ctypes binding of libpipeboost.so (argument marshalling only).

Every step of the prefill runs inside the HIP library.  PyTorch is used only
to allocate the device arena and the two streams.  There is no fallback: if
the library is missing, loading fails with an error.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
# PIPEBOOST_LIB selects another build of the same library (e.g. a tuning variant)
LIB_PATH = os.environ.get("PIPEBOOST_LIB") or os.path.join(HERE, "lib", "libpipeboost.so")

PB_OK, PB_EINVAL, PB_ENOTPINNED, PB_ENOMEM, PB_EHIP, PB_ESTATE = 0, -1, -2, -3, -4, -5
PB_BF16, PB_F16 = 0, 1
LORA_BITS = {"q": 1, "k": 2, "v": 4, "o": 8}
TARGET_INDEX = {"q": 0, "k": 1, "v": 2, "o": 3}
LAYER_TENSOR_ID = {n: i for i, n in enumerate(
    ("ln1_g", "ln1_b", "wq", "bq", "wk", "bk", "wv", "bv", "wo", "bo", "ln2_g", "ln2_b",
     "w1", "b1", "w2", "b2"))}
GLOBAL_TENSOR_ID = {"embed": 0, "pos": 1, "lnf_g": 2, "lnf_b": 3}
KERNEL_KINDS = ("embed", "layernorm", "lora_shrink", "gemm_qkv", "attention", "gemm_o",
                "gemm_fc1", "gemm_fc2", "lm_head", "argmax")


class PbError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("pipeboost error %d: %s" % (code, msg))
        self.code = code


class Config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("d_ffn", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("max_pos", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("max_batch", ctypes.c_int32),
                ("max_adapters", ctypes.c_int32), ("max_rank", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("ln_eps", ctypes.c_float),
                ("max_new_tokens", ctypes.c_int32), ("merge_shadow", ctypes.c_int32)]


class KvPool(ctypes.Structure):
    """pb_kv_pool"""
    _fields_ = [("base", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("v_offset", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


_SIGS = {
    "pb_layer_bytes": (ctypes.c_size_t, [ctypes.POINTER(Config)]),
    "pb_globals_bytes": (ctypes.c_size_t, [ctypes.POINTER(Config)]),
    "pb_layer_tensor": (ctypes.c_int, [ctypes.POINTER(Config), ctypes.c_int32,
                                       ctypes.POINTER(ctypes.c_size_t),
                                       ctypes.POINTER(ctypes.c_size_t)]),
    "pb_globals_tensor": (ctypes.c_int, [ctypes.POINTER(Config), ctypes.c_int32,
                                         ctypes.POINTER(ctypes.c_size_t),
                                         ctypes.POINTER(ctypes.c_size_t)]),
    "pb_lora_layer_bytes": (ctypes.c_size_t, [ctypes.POINTER(Config), ctypes.c_int32,
                                              ctypes.c_uint32]),
    "pb_lora_tensor": (ctypes.c_int, [ctypes.POINTER(Config), ctypes.c_int32, ctypes.c_uint32,
                                      ctypes.c_int32, ctypes.c_int32,
                                      ctypes.POINTER(ctypes.c_size_t),
                                      ctypes.POINTER(ctypes.c_size_t)]),
    "pb_arena_bytes": (ctypes.c_size_t, [ctypes.POINTER(Config)]),
    "pb_host_alloc": (ctypes.c_int, [ctypes.c_size_t, ctypes.POINTER(ctypes.c_void_p)]),
    "pb_host_free": (ctypes.c_int, [ctypes.c_void_p]),
    "pb_host_numa_node": (ctypes.c_int, [ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]),
    "pb_set_host_numa_node": (ctypes.c_int, [ctypes.c_int32]),
    "pb_model_create": (ctypes.c_int, [ctypes.POINTER(Config), ctypes.c_void_p, ctypes.c_size_t,
                                       ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.POINTER(ctypes.c_void_p)]),
    "pb_stream_layers": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32),
                                        ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p),
                                        ctypes.c_void_p]),
    "pb_attach_lora": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                      ctypes.c_float, ctypes.c_uint32,
                                      ctypes.POINTER(ctypes.c_void_p)]),
    "pb_rebuild_kv": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                     ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                     ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(ctypes.c_int32),
                                     ctypes.POINTER(ctypes.c_float)]),
    "pb_invalidate_kv": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_uint8), ctypes.c_int32]),
    "pb_merge_lora": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32]),
    "pb_prefill_stage": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                        ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                        ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float)]),
    "pb_unmerge_lora": (ctypes.c_int, [ctypes.c_void_p]),
    "pb_sched_create": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p)]),
    "pb_sched_destroy": (ctypes.c_int, [ctypes.c_void_p]),
    "pb_sched_submit": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32]),
    "pb_sched_next": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64),
                                     ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32),
                                     ctypes.POINTER(ctypes.c_int32)]),
    "pb_sched_stats": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64),
                                      ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int32)]),
    "pb_plan_loading": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_uint8),
                                       ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32),
                                       ctypes.POINTER(ctypes.c_int32)]),
    "pb_decode_step": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                      ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32),
                                      ctypes.POINTER(ctypes.c_float)]),
    "pb_prefill_first_token": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32),
                                              ctypes.c_int32, ctypes.c_int32,
                                              ctypes.POINTER(ctypes.c_int32),
                                              ctypes.POINTER(ctypes.c_int32),
                                              ctypes.POINTER(ctypes.c_float)]),
    "pb_destroy": (ctypes.c_int, [ctypes.c_void_p]),
    "pb_last_error": (ctypes.c_char_p, []),
    "pb_set_chunk_bytes": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t]),
    "pb_last_load_stats": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_double),
                                          ctypes.POINTER(ctypes.c_double)]),
    "pb_set_kernel_timing": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32]),
    "pb_set_graph_replay": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32]),
    "pb_get_kernel_timing": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32,
                                            ctypes.POINTER(ctypes.c_double),
                                            ctypes.POINTER(ctypes.c_int64)]),
    "pb_reset_kernel_timing": (ctypes.c_int, [ctypes.c_void_p]),
    "pb_poison_weights": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32]),
    "pb_set_stream_delay_us": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32]),
    "pb_op_gemm": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                  ctypes.c_int32, ctypes.c_int32, ctypes.c_float, ctypes.c_int32,
                                  ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "pb_op_gemm_lora": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                       ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32,
                                       ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                       ctypes.c_uint32, ctypes.c_float, ctypes.c_int32, ctypes.c_void_p,
                                       ctypes.c_size_t, ctypes.c_void_p]),
    "pb_op_gemm_noalloc": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                          ctypes.c_int32, ctypes.c_float, ctypes.c_int32,
                                          ctypes.c_void_p]),
    "pb_op_attention": (ctypes.c_int, [ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                       ctypes.c_int32, ctypes.c_void_p]),
    "pb_op_layernorm": (ctypes.c_int, [ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                       ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                       ctypes.c_void_p]),
    "pb_op_kv_append": (ctypes.c_int, [ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                       ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]),
    "pb_op_paged_attention": (ctypes.c_int, [ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p,
                                             ctypes.c_int32, ctypes.c_int32, ctypes.c_float, ctypes.c_int32,
                                             ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t,
                                             ctypes.c_void_p]),
    "pb_op_paged_attention_workspace": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                                          ctypes.c_int32]),
    "pb_op_beam_select": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                         ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "pb_op_beam_select_workspace": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    "pb_op_page_fork": (ctypes.c_int, [ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                       ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32,
                                       ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "pb_op_page_fork_workspace": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32]),
    "pb_op_norm_q8": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32,
                                     ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                     ctypes.c_int64, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]),
    "pb_op_quant_q8": (ctypes.c_int, [ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p,
                                      ctypes.c_int64, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]),
    "pb_op_gemm_q8": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                     ctypes.c_float, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "pb_op_gemm_q8_workspace": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
}

_lib = None


def lib():
    """Load libpipeboost.so (built by ``paper_2503_17707_amd.build``); raise if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libpipeboost.so is not built (%s); run __graft_entry__.build()"
                               % LIB_PATH)
        # One HIP runtime per process: torch ships its own libamdhip64.so.7 with
        # the same soname, so it must be loaded first and the library then binds
        # to it (the streams torch creates are only valid in that runtime).
        import torch  # noqa: F401

        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def check(rc: int) -> None:
    if rc:
        raise PbError(rc, lib().pb_last_error().decode())


def make_config(w, max_tokens: Optional[int] = None, max_batch: Optional[int] = None,
                max_adapters: Optional[int] = None, max_rank: Optional[int] = None,
                max_new_tokens: int = 0, merge_shadow: bool = False) -> Config:
    """pb_config of a synth.Workload (capacities default to the workload's own sizes;
    max_new_tokens > 0 adds a KV cache for decode steps; merge_shadow keeps the
    unmerged attention weights for adapter switching)."""
    return Config(n_layers=w.n_layers, d_model=w.d_model, n_heads=w.n_heads, d_ffn=w.d_ffn,
                  vocab=w.vocab, max_pos=w.max_pos,
                  max_tokens=max_tokens or w.batch * w.seq_len,
                  max_batch=max_batch or w.batch,
                  max_adapters=w.n_adapters if max_adapters is None else max_adapters,
                  max_rank=max_rank or w.lora_rank,
                  dtype=PB_BF16 if w.dtype == "bf16" else PB_F16, ln_eps=w.ln_eps,
                  max_new_tokens=max_new_tokens, merge_shadow=1 if merge_shadow else 0)


def layer_tensor(cfg: Config, name: str):
    off, n = ctypes.c_size_t(), ctypes.c_size_t()
    check(lib().pb_layer_tensor(ctypes.byref(cfg), LAYER_TENSOR_ID[name], ctypes.byref(off),
                                ctypes.byref(n)))
    return off.value, n.value


def globals_tensor(cfg: Config, name: str):
    off, n = ctypes.c_size_t(), ctypes.c_size_t()
    check(lib().pb_globals_tensor(ctypes.byref(cfg), GLOBAL_TENSOR_ID[name], ctypes.byref(off),
                                  ctypes.byref(n)))
    return off.value, n.value


def lora_tensor(cfg: Config, rank: int, mask: int, target: str, which: str):
    off, n = ctypes.c_size_t(), ctypes.c_size_t()
    check(lib().pb_lora_tensor(ctypes.byref(cfg), rank, mask, TARGET_INDEX[target],
                               0 if which == "A" else 1, ctypes.byref(off), ctypes.byref(n)))
    return off.value, n.value


class Pinned:
    """A pinned host buffer from pb_host_alloc, freed with pb_host_free."""

    def __init__(self, nbytes: int):
        p = ctypes.c_void_p()
        check(lib().pb_host_alloc(nbytes, ctypes.byref(p)))
        self.ptr = p.value
        self.nbytes = nbytes

    def view(self, dtype=np.uint8) -> np.ndarray:
        buf = (ctypes.c_uint8 * self.nbytes).from_address(self.ptr)
        return np.frombuffer(buf, dtype=np.uint8).view(dtype)

    def free(self):
        if self.ptr:
            lib().pb_host_free(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def gpu_numa_node(device: int = 0) -> int:
    """NUMA node of the GPU (pb_host_numa_node), -1 if the system reports none."""
    n = ctypes.c_int32(-1)
    check(lib().pb_host_numa_node(device, ctypes.byref(n)))
    return n.value


def _mbind(ptr: int, nbytes: int, node: int) -> bool:
    """Prefer one NUMA node for a page-aligned, not yet touched range (mbind,
    MPOL_PREFERRED), so its pages come from that node whichever thread first
    writes them (from another node only if that one is full)."""
    if node < 0 or nbytes <= 0:
        return False
    libc = ctypes.CDLL(None, use_errno=True)
    bits = 8 * ctypes.sizeof(ctypes.c_ulong)
    mask = (ctypes.c_ulong * (1024 // bits))()
    mask[node // bits] = 1 << (node % bits)
    length = (nbytes + 4095) // 4096 * 4096
    SYS_mbind = 237  # x86_64
    return libc.syscall(SYS_mbind, ctypes.c_void_p(ptr), ctypes.c_ulong(length), 1, mask,
                        ctypes.c_ulong(1024), 0) == 0


class Pageable:
    """A page-aligned ordinary (pageable) host buffer with the interface of
    Pinned; with a NUMA node its pages are bound there before first touch."""

    def __init__(self, nbytes: int, node: int = -1):
        self._buf = np.empty(nbytes + 2 * 4096, np.uint8)
        off = (-self._buf.ctypes.data) % 4096
        self._arr = self._buf[off:off + nbytes]
        self.ptr = self._arr.ctypes.data
        self.nbytes = nbytes
        self.bound = _mbind(self.ptr, nbytes, node)

    def view(self, dtype=np.uint8) -> np.ndarray:
        return self._arr.view(dtype)

    def free(self):
        self._buf = self._arr = None
        self.ptr = None


# Host memory the layer blobs may pin (the rest stay pageable and the loader
# stages them through its own pinned ring): hosts can cap locked memory well
# below their RAM.  PIPEBOOST_PIN_BUDGET_GB overrides.
DEFAULT_PIN_BUDGET = int(float(os.environ.get("PIPEBOOST_PIN_BUDGET_GB", "48")) * (1 << 30))


class HostWeights:
    """Host blobs of a workload in the library's device layout, drawn by synth:
    the globals and LoRA blobs pinned, layer blobs pinned while they fit in
    pin_budget bytes (in layer-id order) and pageable after that.  With
    numa (default: on unless PIPEBOOST_NUMA=0) every blob sits on the GPU's
    NUMA node."""

    def __init__(self, w, cfg: Config, pin_budget: Optional[int] = None, numa: Optional[bool] = None):
        import synth

        self.w, self.cfg = w, cfg
        budget = DEFAULT_PIN_BUDGET if pin_budget is None else pin_budget
        L = lib()
        if numa is None:
            numa = os.environ.get("PIPEBOOST_NUMA", "1") != "0"
        self.numa_node = gpu_numa_node() if numa else -1
        check(L.pb_set_host_numa_node(self.numa_node))
        kind = w.dtype
        self.layer_bytes = L.pb_layer_bytes(ctypes.byref(cfg))
        self.globals_bytes = L.pb_globals_bytes(ctypes.byref(cfg))
        if not self.layer_bytes or not self.globals_bytes:
            raise PbError(PB_EINVAL, "invalid config for %s" % w.name)
        self.globals = Pinned(self.globals_bytes)
        self.globals.view()[:] = 0
        for name in synth.GLOBAL_TENSORS:
            off, _ = globals_tensor(cfg, name)
            synth.fill_base_tensor(w, -1, name, kind, self.globals.ptr + 2 * off)
        self.layers: List[Pinned] = []
        self.pinned_layers = 0
        for layer in range(w.n_layers):
            if (layer + 1) * self.layer_bytes <= budget:
                blob = Pinned(self.layer_bytes)
                self.pinned_layers += 1
            else:
                blob = Pageable(self.layer_bytes, self.numa_node)
            self._zero_padding(blob, cfg)
            for name in synth.LAYER_TENSORS:
                off, _ = layer_tensor(cfg, name)
                synth.fill_base_tensor(w, layer, name, kind, blob.ptr + 2 * off)
            self.layers.append(blob)
        self.loras: Dict[int, List[Pinned]] = {}

    def _zero_padding(self, blob: Pinned, cfg: Config):
        # every byte of the blob is written by a tensor except the alignment
        # gaps between them: zero only those (the tensors' own fills touch the
        # rest first, from all of the generator's threads)
        import synth

        spans = sorted(layer_tensor(cfg, n) for n in synth.LAYER_TENSORS)
        pos = 0
        for off, n in spans:
            if 2 * off > pos:
                ctypes.memset(blob.ptr + pos, 0, 2 * off - pos)
            pos = max(pos, 2 * (off + n))
        if blob.nbytes > pos:
            ctypes.memset(blob.ptr + pos, 0, blob.nbytes - pos)

    def lora_mask(self) -> int:
        m = 0
        for t in self.w.lora_targets:
            m |= LORA_BITS[t]
        return m

    def add_lora(self, adapter: int) -> List[Pinned]:
        import synth

        w, cfg = self.w, self.cfg
        mask = self.lora_mask()
        nbytes = lib().pb_lora_layer_bytes(ctypes.byref(cfg), w.lora_rank, mask)
        if not nbytes:
            raise PbError(PB_EINVAL, "invalid LoRA shape")
        blobs = []
        for layer in range(w.n_layers):
            blob = Pinned(nbytes)
            for t in w.lora_targets:
                for which in ("A", "B"):
                    off, _ = lora_tensor(cfg, w.lora_rank, mask, t, which)
                    synth.fill_lora_tensor(w, adapter, layer, t, which, w.dtype,
                                           blob.ptr + 2 * off)
            blobs.append(blob)
        self.loras[adapter] = blobs
        return blobs

    def free(self):
        self.globals.free()
        for b in self.layers:
            b.free()
        for bl in self.loras.values():
            for b in bl:
                b.free()


class Model:
    """A pb_model over a torch-allocated arena and two torch streams."""

    def __init__(self, cfg: Config, device: str = "cuda:0"):
        import torch

        self.cfg = cfg
        L = lib()
        self.arena_bytes = L.pb_arena_bytes(ctypes.byref(cfg))
        if not self.arena_bytes:
            raise PbError(PB_EINVAL, "invalid config")
        self.device = torch.device(device)
        self.arena = torch.empty(self.arena_bytes + 256, dtype=torch.uint8, device=self.device)
        base = self.arena.data_ptr()
        self.base = (base + 255) // 256 * 256
        self.copy_stream = torch.cuda.Stream(device=self.device)
        self.compute_stream = torch.cuda.Stream(device=self.device)
        torch.cuda.synchronize(self.device)
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            check(L.pb_model_create(ctypes.byref(cfg), ctypes.c_void_p(self.base),
                                    self.arena_bytes, ctypes.c_void_p(self.copy_stream.cuda_stream),
                                    ctypes.c_void_p(self.compute_stream.cuda_stream),
                                    ctypes.byref(h)))
        self.h = h

    def stream_layers(self, hw: HostWeights, order: Optional[Sequence[int]] = None):
        n = self.cfg.n_layers
        order = list(range(n)) if order is None else list(order)
        arr = (ctypes.c_int32 * len(order))(*order)
        ptrs = (ctypes.c_void_p * n)(*[b.ptr for b in hw.layers])
        check(lib().pb_stream_layers(self.h, arr, len(order), ptrs, ctypes.c_void_p(hw.globals.ptr)))

    def attach_lora(self, slot: int, blobs: List[Pinned], rank: int, alpha: float, mask: int):
        ptrs = (ctypes.c_void_p * len(blobs))(*[b.ptr for b in blobs])
        check(lib().pb_attach_lora(self.h, slot, rank, alpha, mask, ptrs))

    def prefill(self, tokens: np.ndarray, adapter_of_seq: Optional[Sequence[int]] = None,
                want_logits: bool = True):
        tokens = np.ascontiguousarray(tokens, dtype=np.int32)
        B, T = tokens.shape
        out_tok = np.empty(B, dtype=np.int32)
        logits = np.empty((B, self.cfg.vocab), dtype=np.float32) if want_logits else None
        ad = None
        if adapter_of_seq is not None:
            ad_arr = np.ascontiguousarray(adapter_of_seq, dtype=np.int32)
            ad = ad_arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        check(lib().pb_prefill_first_token(
            self.h, tokens.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), B, T, ad,
            out_tok.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
            logits.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) if want_logits else None))
        return out_tok, logits

    def prefill_stage(self, tokens: np.ndarray, adapter_of_seq: Optional[Sequence[int]], layer_begin: int,
                      layer_end: int, hidden_in=None, hidden_out=None, want_logits: bool = True):
        """Layers [layer_begin, layer_end) of a prefill (pb_prefill_stage).  hidden_in /
        hidden_out: device fp32 tensors of [B*T, d_model] (or None at the ends).
        Returns (tokens, logits) from the last stage, None from the others."""
        tokens = np.ascontiguousarray(tokens, dtype=np.int32)
        B, T = tokens.shape
        last = layer_end == self.cfg.n_layers
        out_tok = np.empty(B, dtype=np.int32) if last else None
        logits = np.empty((B, self.cfg.vocab), dtype=np.float32) if (last and want_logits) else None
        ad = None
        if adapter_of_seq is not None:
            ad_arr = np.ascontiguousarray(adapter_of_seq, dtype=np.int32)
            ad = ad_arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        check(lib().pb_prefill_stage(
            self.h, tokens.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), B, T, ad, layer_begin, layer_end,
            ctypes.c_void_p(hidden_in.data_ptr()) if hidden_in is not None else None,
            ctypes.c_void_p(hidden_out.data_ptr()) if hidden_out is not None else None,
            out_tok.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)) if last else None,
            logits.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) if logits is not None else None))
        return (out_tok, logits) if last else None

    def decode(self, tokens: np.ndarray, adapter_of_seq: Optional[Sequence[int]] = None,
               want_logits: bool = True):
        """One decode step: tokens [B] (the newest token of each sequence)."""
        tokens = np.ascontiguousarray(tokens, dtype=np.int32).reshape(-1)
        B = tokens.shape[0]
        out_tok = np.empty(B, dtype=np.int32)
        logits = np.empty((B, self.cfg.vocab), dtype=np.float32) if want_logits else None
        ad = None
        if adapter_of_seq is not None:
            ad_arr = np.ascontiguousarray(adapter_of_seq, dtype=np.int32)
            ad = ad_arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        check(lib().pb_decode_step(
            self.h, tokens.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), B, ad,
            out_tok.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
            logits.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) if want_logits else None))
        return out_tok, logits

    def rebuild_kv(self, tokens: np.ndarray, layer_has_kv: Sequence[bool],
                   adapter_of_seq: Optional[Sequence[int]] = None, want_logits: bool = True):
        """KV-cache rebuild over tokens [B, T]; returns the next token of each sequence."""
        tokens = np.ascontiguousarray(tokens, dtype=np.int32)
        B, T = tokens.shape
        has = np.ascontiguousarray([1 if h else 0 for h in layer_has_kv], dtype=np.uint8)
        out_tok = np.empty(B, dtype=np.int32)
        logits = np.empty((B, self.cfg.vocab), dtype=np.float32) if want_logits else None
        ad = None
        if adapter_of_seq is not None:
            ad_arr = np.ascontiguousarray(adapter_of_seq, dtype=np.int32)
            ad = ad_arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        check(lib().pb_rebuild_kv(
            self.h, tokens.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), B, T, ad,
            has.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
            out_tok.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
            logits.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) if want_logits else None))
        return out_tok, logits

    def merge_lora(self, slot: int):
        check(lib().pb_merge_lora(self.h, slot))

    def unmerge_lora(self):
        check(lib().pb_unmerge_lora(self.h))

    def invalidate_kv(self, layer_lost: Sequence[bool], value: int = 0xFF):
        lost = np.ascontiguousarray([1 if x else 0 for x in layer_lost], dtype=np.uint8)
        check(lib().pb_invalidate_kv(self.h, lost.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)), value))

    def poison(self, value: int = 0xFF):
        check(lib().pb_poison_weights(self.h, value))

    def set_chunk_bytes(self, n: int):
        check(lib().pb_set_chunk_bytes(self.h, n))

    def set_stream_delay_us(self, us: int):
        check(lib().pb_set_stream_delay_us(self.h, us))

    def load_stats(self):
        b, ms = ctypes.c_double(), ctypes.c_double()
        check(lib().pb_last_load_stats(self.h, ctypes.byref(b), ctypes.byref(ms)))
        return b.value, ms.value

    def set_graph_replay(self, on: bool):
        """Record settled forward shapes as HIP graphs and replay them (default on)."""
        check(lib().pb_set_graph_replay(self.h, 1 if on else 0))

    def set_timing(self, on: bool):
        check(lib().pb_set_kernel_timing(self.h, 1 if on else 0))

    def reset_timing(self):
        check(lib().pb_reset_kernel_timing(self.h))

    def timing(self) -> Dict[str, tuple]:
        out = {}
        for i, k in enumerate(KERNEL_KINDS):
            ms, n = ctypes.c_double(), ctypes.c_int64()
            check(lib().pb_get_kernel_timing(self.h, i, ctypes.byref(ms), ctypes.byref(n)))
            out[k] = (ms.value, n.value)
        return out

    def destroy(self):
        if self.h:
            lib().pb_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def setup(w, device: str = "cuda:0", hw: Optional[HostWeights] = None, **cap):
    """Create the host blobs (layer blobs pinned up to the budget) and a model."""
    cfg = make_config(w, **cap)
    hw = hw or HostWeights(w, cfg)
    m = Model(cfg, device)
    return hw, m


def attach_all(m: Model, hw: HostWeights):
    """Attach adapter a of the workload into slot a, for every adapter it uses."""
    w = hw.w
    used = sorted({a for a in w.adapters() if a >= 0})
    for a in used:
        blobs = hw.loras.get(a) or hw.add_lora(a)
        m.attach_lora(a, blobs, w.lora_rank, w.lora_alpha, hw.lora_mask())


class Scheduler:
    """Epoch-based adapter switching (pb_sched_*): per-adapter request queues;
    epoch_batches = 0 is the eager, arrival-order baseline."""

    def __init__(self, n_adapters: int, epoch_batches: int):
        h = ctypes.c_void_p()
        check(lib().pb_sched_create(n_adapters, epoch_batches, ctypes.byref(h)))
        self.h = h

    def submit(self, request_id: int, adapter: int):
        check(lib().pb_sched_submit(self.h, request_id, adapter))

    def next(self, max_batch: int):
        """(request ids, adapter, switched), or None when every queue is empty."""
        ids = (ctypes.c_int64 * max_batch)()
        n, a, sw = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        check(lib().pb_sched_next(self.h, max_batch, ids, ctypes.byref(n), ctypes.byref(a), ctypes.byref(sw)))
        if n.value == 0:
            return None
        return list(ids[:n.value]), a.value, bool(sw.value)

    def stats(self):
        """(pending, switches, active adapter; -2 before the first batch)."""
        p, sw, a = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int32()
        check(lib().pb_sched_stats(self.h, ctypes.byref(p), ctypes.byref(sw), ctypes.byref(a)))
        return p.value, sw.value, a.value

    def close(self):
        if self.h:
            check(lib().pb_sched_destroy(self.h))
            self.h = None


def plan_loading(n_layers: int, alive: Sequence[bool]):
    """Per-GPU layer orders and owned blocks (pb_plan_loading): returns
    (orders [n_gpus][n_layers] with -1 rows for failed GPUs, [(first, len)] per GPU)."""
    G = len(alive)
    al = np.ascontiguousarray([1 if a else 0 for a in alive], dtype=np.uint8)
    order = np.empty((G, n_layers), dtype=np.int32)
    first = np.empty(G, dtype=np.int32)
    ln = np.empty(G, dtype=np.int32)
    p32 = ctypes.POINTER(ctypes.c_int32)
    check(lib().pb_plan_loading(n_layers, G, al.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
                                order.ctypes.data_as(p32), first.ctypes.data_as(p32), ln.ctypes.data_as(p32)))
    return order, list(zip(first.tolist(), ln.tolist()))


# ---- kernel-level entry points (include/pipeboost_ops.h) --------------------
# Arguments are torch tensors on the GPU; the call is enqueued on `stream`
# (a torch.cuda.Stream, default: the current stream).

# The wrappers cost host time that a one-token product feels (a qkv product of d
# 2048 called in a row: 5.7 us a call, 7.8 with an address object per operand and
# the stream looked up through its class): addresses go as plain integers (their
# argtypes are void pointers), the current stream's handle is asked for directly.

def _ptr(t):
    return None if t is None else t.data_ptr()


_current_raw_stream = None


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    global _current_raw_stream
    if _current_raw_stream is None:
        import torch

        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and dev is not None:
            torch.cuda.current_stream()  # initialises the runtime
            _current_raw_stream = lambda: raw(dev())
        else:
            _current_raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _current_raw_stream()


def op_gemm(dtype: int, epi: int, X, W, bias, C=None, R=None, qscale: float = 1.0,
            qcols: int = 0, workspace=None, stream=None):
    M, K = X.shape
    N = W.shape[0]
    check(lib().pb_op_gemm(dtype, epi, _ptr(X), _ptr(W), _ptr(bias), _ptr(C), _ptr(R), M, N, K,
                           qscale, qcols, _ptr(workspace),
                           0 if workspace is None else workspace.numel() * workspace.element_size(),
                           _stream(stream)))


def op_gemm_lora(dtype: int, epi: int, X, W, bias, Z, zs: int, W2, group: int, group_mask: int,
                 C=None, R=None, qscale: float = 1.0, qcols: int = 0, workspace=None, stream=None):
    """pb_op_gemm_lora: Z [M, ldz] scaled shrinks (group g's block at column g * zs), W2 [N, K2]."""
    M, K = X.shape
    N = W.shape[0]
    K2 = W2.shape[1]
    check(lib().pb_op_gemm_lora(dtype, epi, _ptr(X), _ptr(W), _ptr(bias), _ptr(C), _ptr(R), M, N, K,
                                _ptr(Z), Z.shape[1], zs, _ptr(W2), K2, group, group_mask, qscale, qcols,
                                _ptr(workspace),
                                0 if workspace is None else workspace.numel() * workspace.element_size(),
                                _stream(stream)))


def op_gemm_noalloc(dtype: int, epi: int, X, W, bias, C=None, R=None, qscale: float = 1.0,
                    qcols: int = 0, stream=None):
    """pb_op_gemm_noalloc: pb_op_gemm with the library's own split-K scratch."""
    M, K = X.shape
    N = W.shape[0]
    check(lib().pb_op_gemm_noalloc(dtype, epi, _ptr(X), _ptr(W), _ptr(bias), _ptr(C), _ptr(R), M, N,
                                   K, qscale, qcols, _stream(stream)))


def op_attention(dtype: int, qkv, out, B: int, T: int, H: int, hd: int, stream=None):
    check(lib().pb_op_attention(dtype, _ptr(qkv), _ptr(out), B, T, H, hd, _stream(stream)))


def op_layernorm(dtype: int, x, g, b, out, eps: float = 1e-5, stream=None):
    rows, d = x.shape
    import torch

    check(lib().pb_op_layernorm(dtype, _ptr(x), _ptr(g), _ptr(b), _ptr(out),
                                1 if out.dtype == torch.float32 else 0, rows, d, eps,
                                _stream(stream)))


# ---- a cache of pages, and beam search over it -----------------------------------
# A layer's pool is a tensor [n_pages, 2 (k, v), kv heads, page_size, head_dim] of any
# strides with unit last one: a page may hold cache rows [k | v] (a permuted view) or
# each head's tokens in a row.  What the C entry points cannot see (types, shapes,
# strides that no argument carries, the device) is checked here.

# (These checks run before every launch: plain comparisons, no helper per operand.
# A one-token append called in a row: 8.9 us with the helpers, 7.7 without.)

_torch = None


def _checked(op, stream, dtype, storage, ints, others=()):
    """The torch module, after: every tensor on the current device, where the call is
    enqueued (a stream that is given too); storage of dtype's type; (name, tensor,
    shape) of ints contiguous int32."""
    global _torch
    if _torch is None:
        import torch as _torch_module

        _torch = _torch_module
    torch = _torch
    i32 = torch.int32
    first = storage[0] if storage else others[0]
    dev = first.get_device()
    if storage:
        want = torch.float16 if dtype == PB_F16 else torch.bfloat16
        for t in storage:
            if t.dtype is not want:
                raise PbError(PB_EINVAL, "%s: %s operand with dtype %d" % (op, t.dtype, dtype))
            if t.get_device() != dev:
                raise PbError(PB_EINVAL, "%s: tensors on %s and on %s" % (op, first.device, t.device))
    for name, t, shape in ints:
        if t.dtype is not i32 or t.shape != shape or not t.is_contiguous():
            raise PbError(PB_EINVAL, "%s: %s must be contiguous int32 %s" % (op, name, list(shape)))
        if t.get_device() != dev:
            raise PbError(PB_EINVAL, "%s: tensors on %s and on %s" % (op, first.device, t.device))
    for t in others:
        if t is not None and t.get_device() != dev:
            raise PbError(PB_EINVAL, "%s: tensors on %s and on %s" % (op, first.device, t.device))
    if dev < 0 or dev != torch.cuda.current_device():
        raise PbError(PB_EINVAL, "%s: tensors on %s, which is not the current device" % (op, first.device))
    if stream is not None and stream.device_index != dev:
        raise PbError(PB_EINVAL, "%s: the stream is another device's" % op)
    return torch


def _heads(op, name, t):
    """Row stride of [rows, heads, head_dim] whose rows are contiguous."""
    rs, hs, es = t.stride()
    shape = t.shape
    if es != 1 or (hs != shape[2] and shape[1] > 1):
        raise PbError(PB_EINVAL, "%s: the heads of a row of %s must be contiguous" % (op, name))
    return rs


def kv_pool(pool) -> KvPool:
    """pb_kv_pool of a layer's pool tensor [n_pages, 2, kv heads, page_size, head_dim]."""
    shape, stride = pool.shape, pool.stride()
    if len(shape) != 5 or shape[1] != 2 or stride[4] != 1:
        raise PbError(PB_EINVAL, "a pool is [n_pages, 2, kv heads, page_size, head_dim] with unit last stride")
    return KvPool(pool.data_ptr(), *stride[:4], shape[0], shape[3], shape[2], shape[4])


def _tables(op, tables):
    """Rows, width and row stride of int32 page tables."""
    shape = tables.shape
    if len(shape) != 2:
        raise PbError(PB_EINVAL, "%s: tables must be int32 [rows, width]" % op)
    S, width = shape
    ld, es = tables.stride()
    if (es != 1 and width > 1 and S > 0) or tables.element_size() != 4 or tables.is_floating_point():
        raise PbError(PB_EINVAL, "%s: tables must be int32 [rows, width] with contiguous rows" % op)
    return S, width, ld if S > 1 else width


def _nbytes(workspace):
    if workspace is None:
        return 0
    if not workspace.is_contiguous():
        raise PbError(PB_EINVAL, "a workspace must be contiguous")
    return workspace.numel() * workspace.element_size()


def op_kv_append(dtype: int, k, v, pool, tables, start, lens, row0=None, max_rows: Optional[int] = None, stream=None):
    """pb_op_kv_append: tokens start[s] .. lens[s]-1 of every sequence from rows row0[s], row0[s] + 1, ... of
    k and v [rows, kv heads, head_dim] (views of a fused projection's rows fit).  Without row0 the rows are a
    padded batch of max_rows per sequence; max_rows defaults to rows / sequences then, to rows with row0."""
    op = "op_kv_append"
    c = kv_pool(pool)
    S, width, ld = _tables(op, tables)
    of = (S,)
    ints = [("start", start, of), ("lens", lens, of)]
    if row0 is not None:
        ints.append(("row0", row0, of))
    shape = k.shape
    if len(shape) != 3 or v.shape != shape or shape[1] != c.n_kv_heads or shape[2] != c.head_dim:
        raise PbError(PB_EINVAL, "%s: k and v must be [rows, %d, %d]" % (op, c.n_kv_heads, c.head_dim))
    n = shape[0]
    if max_rows is None:
        max_rows = n if row0 is not None else n // max(S, 1)
    _checked(op, stream, dtype, (pool, k, v), ints, (tables,))
    rc = lib().pb_op_kv_append(dtype, k.data_ptr(), _heads(op, "k", k), v.data_ptr(), _heads(op, "v", v), n,
                               ctypes.byref(c), tables.data_ptr(), width, ld, start.data_ptr(), lens.data_ptr(),
                               _ptr(row0), S, max_rows, _stream(stream))
    if rc:
        check(rc)


def paged_attention_workspace(n_seqs: int, n_heads: int, pool, width: int) -> int:
    """Bytes of workspace with which op_paged_attention splits as it likes."""
    return lib().pb_op_paged_attention_workspace(n_seqs, n_heads, ctypes.byref(kv_pool(pool)), width)


def op_paged_attention(dtype: int, q, pool, tables, lens, out, scale: float = 1.0, window: int = 0, workspace=None,
                       shared: bool = False, stream=None):
    """pb_op_paged_attention: q and out [sequences, heads, head_dim] (rows may be strided); scale 1 for a q that is
    divided by sqrt(head_dim) already; shared: rows next to each other share pages (beams)."""
    op = "op_paged_attention"
    c = kv_pool(pool)
    S, width, ld = _tables(op, tables)
    shape = q.shape
    if len(shape) != 3 or out.shape != shape or shape[0] != S or shape[2] != c.head_dim:
        raise PbError(PB_EINVAL, "%s: q and out must be [%d, heads, %d]" % (op, S, c.head_dim))
    _checked(op, stream, dtype, (pool, q, out), (("lens", lens, (S,)),), (tables, workspace))
    rc = lib().pb_op_paged_attention(dtype, q.data_ptr(), _heads(op, "q", q), ctypes.byref(c), tables.data_ptr(), width,
                                     ld, lens.data_ptr(), S, shape[1], scale, window, shared, out.data_ptr(),
                                     _heads(op, "out", out), _ptr(workspace), _nbytes(workspace), _stream(stream))
    if rc:
        check(rc)


def beam_select_workspace(B: int, W: int, V: int) -> int:
    """Bytes of workspace of op_beam_select."""
    return lib().pb_op_beam_select_workspace(B, W, V)


def op_beam_select(logits, scores, alive, out_scores, out_tokens, out_parents, out_alive, eos: int, pad: int,
                   workspace, stream=None):
    """pb_op_beam_select: logits fp32 [B W, V] (rows may be strided), scores fp32 and alive int32 [B, W], outputs
    [B, W] (out_scores and out_alive may be scores and alive)."""
    op = "op_beam_select"
    of = scores.shape
    if len(of) != 2:
        raise PbError(PB_EINVAL, "%s: scores must be [B, W]" % op)
    B, W = of
    torch = _checked(op, stream, 0, (), (("alive", alive, of), ("out_tokens", out_tokens, of),
                                         ("out_parents", out_parents, of), ("out_alive", out_alive, of)),
                     (logits, scores, out_scores, workspace))
    f32 = torch.float32
    for name, t in (("scores", scores), ("out_scores", out_scores)):
        if t.dtype is not f32 or t.shape != of or not t.is_contiguous():
            raise PbError(PB_EINVAL, "%s: %s must be contiguous float32 [%d, %d]" % (op, name, B, W))
    shape = logits.shape
    if logits.dtype is not f32 or len(shape) != 2 or shape[0] != B * W or (logits.stride(1) != 1 and shape[1] > 1):
        raise PbError(PB_EINVAL, "%s: logits must be float32 [%d, V] with contiguous rows" % (op, B * W))
    rc = lib().pb_op_beam_select(logits.data_ptr(), logits.stride(0), scores.data_ptr(), alive.data_ptr(), B, W,
                                 shape[1], eos, pad, out_scores.data_ptr(), out_tokens.data_ptr(),
                                 out_parents.data_ptr(), out_alive.data_ptr(), _ptr(workspace), _nbytes(workspace),
                                 _stream(stream))
    if rc:
        check(rc)


def page_fork_workspace(out_rows: int, n_pages: int) -> int:
    """Bytes of workspace of op_page_fork."""
    return lib().pb_op_page_fork_workspace(out_rows, n_pages)


def op_page_fork(dtype: int, pools, parents, tables, lens, refs, grow, out_tables, out_start, out_lens, out_refs, short_of,
                 workspace, stream=None):
    """pb_op_page_fork: pools [layers, n_pages, 2, kv heads, page_size, head_dim]; parents, grow, out_start, out_lens
    int32 [out rows]; tables int32 [in rows, width], out_tables [out rows, width]; lens int32 [in rows]; refs,
    out_refs int32 [n_pages]; short_of int32 [2]."""
    op = "op_page_fork"
    if pools.dim() != 6 or pools.shape[0] < 1:
        raise PbError(PB_EINVAL, "%s: pools must be [layers, n_pages, 2, kv heads, page_size, head_dim]" % op)
    shape, stride = pools.shape, pools.stride()
    if shape[2] != 2 or stride[5] != 1:
        raise PbError(PB_EINVAL, "%s: pools must be [layers, n_pages, 2, kv heads, page_size, head_dim]" % op)
    c = KvPool(pools.data_ptr(), *stride[1:5], shape[1], shape[4], shape[3], shape[5])
    S, width, _ = _tables(op, tables)
    R = parents.shape[0]
    of, pages = (R,), (shape[1],)
    _checked(op, stream, dtype, (pools,),
             (("tables", tables, (S, width)), ("out_tables", out_tables, (R, width)), ("lens", lens, (S,)),
              ("parents", parents, of), ("grow", grow, of), ("out_start", out_start, of), ("out_lens", out_lens, of),
              ("refs", refs, pages), ("out_refs", out_refs, pages), ("short_of", short_of, (2,))), (workspace,))
    rc = lib().pb_op_page_fork(dtype, ctypes.byref(c), shape[0], stride[0], parents.data_ptr(), R,
                               tables.data_ptr(), width, lens.data_ptr(), S, refs.data_ptr(), grow.data_ptr(),
                               out_tables.data_ptr(), out_start.data_ptr(), out_lens.data_ptr(), out_refs.data_ptr(),
                               short_of.data_ptr(), _ptr(workspace), _nbytes(workspace), _stream(stream))
    if rc:
        check(rc)


# ---- linear layers in 8 bits ------------------------------------------------------
# 8-bit rows are int8 [rows, cols] with contiguous rows; their scales float32 [rows].
#
# A call of one token waits for its host work.  The conditions on its tensors are asked by a
# small extension module (q8/py_q8.cpp), which hands them to the C entry point; a call that does
# not meet them goes through the checks below, which find and name what is wrong.

ARGS_PATH = os.path.join(HERE, "lib", "pipeboost_q8_args.so")
_q8 = None


def _q8_ready():
    """The extension module, with the loaded library's entry points."""
    global _q8, _torch
    L = lib()
    import importlib.machinery
    import importlib.util

    import torch

    if not os.path.exists(ARGS_PATH):
        raise RuntimeError("pipeboost_q8_args.so is not built (%s); run __graft_entry__.build()" % ARGS_PATH)
    loader = importlib.machinery.ExtensionFileLoader("pipeboost_q8_args", ARGS_PATH)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("pipeboost_q8_args", loader))
    loader.exec_module(m)
    if getattr(m, "TORCH", None) != str(torch.__version__):  # tensors are read by that version's headers
        raise RuntimeError("pipeboost_q8_args.so is for torch %s, not %s; run __graft_entry__.build()" % (getattr(m, "TORCH", "?"), torch.__version__))
    m.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (L.pb_op_norm_q8, L.pb_op_quant_q8, L.pb_op_gemm_q8)))
    _torch = torch
    torch.cuda.is_available() and torch.cuda.current_stream()  # initialises the runtime
    _q8 = m
    return m


def _kinds(dtype):
    return (_torch.bfloat16, _torch.float16)[dtype]


def _refuse(op, why, *args):
    raise PbError(PB_EINVAL, "%s: %s" % (op, why % args))


def _rows_wrong(op, name, t, dtypes, shape):
    if (t.layout is not _torch.strided or t.dtype not in dtypes or tuple(t.shape) != tuple(shape)
            or (t.stride(1) != 1 and shape[1] > 1)):
        _refuse(op, "%s must be %s %s with contiguous rows", name, " or ".join(str(d) for d in dtypes), list(shape))


def _vector_wrong(op, name, t, dtype, n):
    if t.layout is not _torch.strided or t.dtype is not dtype or tuple(t.shape) != (n,) or not t.is_contiguous():
        _refuse(op, "%s must be contiguous %s [%d]", name, dtype, n)


def _device_wrong(op, tensors, stream):
    first = tensors[0]
    for t in tensors:
        if t is not None and t.device != first.device:
            _refuse(op, "tensors on %s and on %s", first.device, t.device)
    if not first.is_cuda or first.get_device() != _torch.cuda.current_device():
        _refuse(op, "tensors on %s, which is not the current device", first.device)
    if stream is not None and stream.device_index != first.get_device():
        _refuse(op, "the stream is another device's")
    _refuse(op, "a size past 32 bits, or a tensor that is no plain memory")


def _norm_q8_failed(rc, dtype, x, g, q, scale, delta, sum, b, out, stream):
    if rc != _q8.LOOK:
        check(rc)
    op = "op_norm_q8"
    i8, f32 = _torch.int8, _torch.float32
    if dtype not in (0, 1):
        _refuse(op, "bad dtype %s", dtype)
    if x.dim() != 2:
        _refuse(op, "x must be [rows, d]")
    rows, d = of = x.shape
    kind = _kinds(dtype)
    _rows_wrong(op, "x", x, (f32, kind), of)
    if (q is None) != (scale is None):
        _refuse(op, "q and scale go together")
    for name, t, types in (("delta", delta, (kind,)), ("sum", sum, (x.dtype,)), ("out", out, (kind,)), ("q", q, (i8,))):
        if t is not None:
            _rows_wrong(op, name, t, types, of)
    if scale is not None:
        _vector_wrong(op, "scale", scale, f32, rows)
    _vector_wrong(op, "g", g, kind, d)
    if b is not None:
        _vector_wrong(op, "b", b, kind, d)
    _device_wrong(op, [x, g, q, scale, delta, sum, b, out], stream)


def op_norm_q8(dtype: int, x, g, q=None, scale=None, delta=None, sum=None, b=None, out=None, layer: bool = False,
               eps: float = 1e-5, stream=None):
    """pb_op_norm_q8: x [rows, d] float32 or dtype's type; delta (dtype's type) is added and the sum stored in `sum`
    (x's type; may be x); its RMS norm (layer: layer norm) with gain g and bias b [d] goes to q int8 [rows, d] with
    scale float32 [rows], and to out (dtype's type) where given.  Rows may be strided."""
    rc = (_q8 or _q8_ready()).norm(dtype, layer, x, g, q, scale, delta, sum, b, out, eps, -1 if stream is None else stream.device_index,
                                   0 if stream is None else stream.cuda_stream)
    if rc:
        _norm_q8_failed(rc, dtype, x, g, q, scale, delta, sum, b, out, stream)


def _quant_q8_failed(rc, dtype, x, q, scale, stream):
    if rc != _q8.LOOK:
        check(rc)
    op = "op_quant_q8"
    i8, f32 = _torch.int8, _torch.float32
    if dtype not in (0, 1):
        _refuse(op, "bad dtype %s", dtype)
    if x.dim() != 2:
        _refuse(op, "x must be [rows, cols]")
    _rows_wrong(op, "x", x, (f32, _kinds(dtype)), x.shape)
    _rows_wrong(op, "q", q, (i8,), x.shape)
    _vector_wrong(op, "scale", scale, f32, x.shape[0])
    _device_wrong(op, [x, q, scale], stream)


def op_quant_q8(dtype: int, x, q, scale, stream=None):
    """pb_op_quant_q8: x [rows, cols] (float32 or dtype's type) to q int8 [rows, cols] and scale float32 [rows]."""
    rc = (_q8 or _q8_ready()).quant(dtype, x, q, scale, -1 if stream is None else stream.device_index,
                                    0 if stream is None else stream.cuda_stream)
    if rc:
        _quant_q8_failed(rc, dtype, x, q, scale, stream)


def gemm_q8_workspace(M: int, N: int, K: int) -> int:
    """Bytes of workspace with which op_gemm_q8 splits K as it likes, for up to M tokens and rows of any stride."""
    return lib().pb_op_gemm_q8_workspace(M, N, K)


def _gemm_q8_failed(rc, dtype, epi, X, sx, W, sw, bias, out, workspace, stream):
    if rc != _q8.LOOK:
        check(rc)
    op = "op_gemm_q8"
    i8, f32 = _torch.int8, _torch.float32
    if dtype not in (0, 1) or epi not in (0, 1, 2, 3):
        _refuse(op, "bad dtype %s or epilogue %s", dtype, epi)
    if X.dim() != 2 or W.dim() != 2:
        _refuse(op, "X must be [M, K] and W [N, K]")
    (M, K), N = X.shape, W.shape[0]
    _rows_wrong(op, "X", X, (i8,), (M, K))
    _rows_wrong(op, "W", W, (i8,), (N, K))
    _vector_wrong(op, "sx", sx, f32, M)
    _vector_wrong(op, "sw", sw, f32, N)
    if bias is not None:
        _vector_wrong(op, "bias", bias, _kinds(dtype), N)
    if out is None:
        _refuse(op, "epilogues 0 and 1 write C, 2 and 3 R")
    _rows_wrong(op, "R" if epi >= 2 else "C", out, (f32 if epi >= 2 else _kinds(dtype),), (M, N))
    if workspace is not None and not workspace.is_contiguous():
        _refuse(op, "a workspace must be contiguous")
    _device_wrong(op, [X, sx, W, sw, bias, out, workspace], stream)


def op_gemm_q8(dtype: int, epi: int, X, sx, W, sw, bias=None, C=None, R=None, qscale: float = 1.0, qcols: int = 0,
               workspace=None, stream=None):
    """pb_op_gemm_q8: X int8 [M, K] with sx [M], W int8 [N, K] with sw [N], bias [N] of dtype's type or None; epilogues 0
    and 1 write C [M, N] (dtype's type), 2 adds to R [M, N] (float32), 3 writes it.  Rows may be strided."""
    rc = (_q8 or _q8_ready()).gemm(dtype, epi, X, sx, W, sw, bias, C, R, qscale, qcols, workspace,
                                   -1 if stream is None else stream.device_index, 0 if stream is None else stream.cuda_stream)
    if rc:
        _gemm_q8_failed(rc, dtype, epi, X, sx, W, sw, bias, R if epi >= 2 else C, workspace, stream)
