"""ctypes binding of libpsd.so: same call names as include/psd.h, torch tensors in and out.

Nothing here computes: tensors are allocated with torch, their device pointers and the
current HIP stream are handed to the library, and every step of the PSD path runs in its
kernels.  Loading fails loudly when the library has not been built; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass, field
from typing import List, Optional, Sequence, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
MAX_NODES = 32
MAX_BLOCK = 64
HIST = MAX_NODES + MAX_BLOCK + 1


class PsdError(RuntimeError):
    pass


class _Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("d_head", C.c_int32), ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("mask_id", C.c_int32),
                ("rms_eps", C.c_float), ("qkv_bias", C.c_int32), ("dtype", C.c_int32), ("logit_scale", C.c_float),
                ("max_seq", C.c_int32), ("attention", C.c_int32)]


_PP = C.POINTER(C.c_void_p)


class _Weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p), ("rope_cos", C.c_void_p),
                ("rope_sin", C.c_void_p), ("attn_norm", _PP), ("wq", _PP), ("wk", _PP), ("wv", _PP), ("bq", _PP),
                ("bk", _PP), ("bv", _PP), ("wo", _PP), ("ffn_norm", _PP), ("w_gate", _PP), ("w_up", _PP), ("w_down", _PP),
                ("w_down_stride", C.c_int32)]


class _Policy(C.Structure):
    _fields_ = [("tau", C.c_float), ("k_min", C.c_int32), ("k_max", C.c_int32), ("eos_stop", C.c_int32),
                ("eos_id", C.c_int32), ("single_forward", C.c_int32)]


class _Graph(C.Structure):
    _fields_ = [("K", C.c_int32), ("rank_set", C.c_uint64 * MAX_NODES)]


class _Stats(C.Structure):
    _fields_ = [("invocations", C.c_int64), ("tokens_policy", C.c_int64), ("tokens_draft", C.c_int64),
                ("tokens_postverify", C.c_int64), ("depth_hist", C.c_int32 * HIST), ("tokens_counted", C.c_int64),
                ("stopped", C.c_int32), ("eos_pos", C.c_int32)]


class _GraphScore(C.Structure):
    _fields_ = [("seconds", C.c_double), ("tokens_per_s", C.c_double), ("tpf", C.c_double), ("tokens", C.c_int64),
                ("invocations", C.c_int64)]


class _Work(C.Structure):
    _fields_ = [("gemm_flops", C.c_double), ("attn_flops", C.c_double), ("head_flops", C.c_double),
                ("head_bytes", C.c_double), ("weight_bytes", C.c_double)]


class _Segment(C.Structure):
    _fields_ = [("k", C.c_void_p), ("vt", C.c_void_p), ("lens", C.c_void_p), ("weights", C.c_void_p), ("stride_k", C.c_int64),
                ("stride_vt", C.c_int64), ("stride_w", C.c_int64), ("ld_k", C.c_int32), ("ld_vt", C.c_int32), ("ld_w", C.c_int32),
                ("len", C.c_int32), ("seqs_per_unit", C.c_int32), ("reserved", C.c_int32)]


class _AttentionShape(C.Structure):
    _fields_ = [("S", C.c_int32), ("L", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32),
                ("dtype", C.c_int32), ("ld_q", C.c_int64), ("ld_out", C.c_int64)]


class _KvShared(C.Structure):
    _fields_ = [("prefix", C.c_void_p), ("cache", C.c_void_p), ("prefix_weights", C.c_void_p), ("cache_weights", C.c_void_p),
                ("prefix_capacity", C.c_int32), ("prefix_len", C.c_int32), ("capacity", C.c_int32), ("len", C.c_int32),
                ("seqs_per_cache", C.c_int32), ("reserved", C.c_int32)]


class _DebugLayout(C.Structure):
    _fields_ = [("off_a", C.c_int64), ("off_qkv", C.c_int64), ("off_vt", C.c_int64), ("off_o", C.c_int64),
                ("off_act", C.c_int64), ("ld_qkv", C.c_int32), ("ld_act", C.c_int32), ("ld_vt", C.c_int32),
                ("reserved", C.c_int32)]


class _RotaryScaling(C.Structure):
    _fields_ = [("theta", C.c_double), ("stretch", C.c_double), ("trained", C.c_double), ("slow", C.c_double), ("fast", C.c_double),
                ("kind", C.c_int32), ("reserved", C.c_int32)]


class _RotaryShape(C.Structure):
    _fields_ = [("n_tokens", C.c_int64), ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_q_out", C.c_int64), ("ld_k_out", C.c_int64),
                ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32), ("rotated", C.c_int32), ("interleaved", C.c_int32),
                ("first", C.c_int32), ("rows_per_seq", C.c_int32), ("dtype", C.c_int32), ("factor", C.c_float), ("eps", C.c_float),
                ("reserved", C.c_int32)]


class _Kv8Cache(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("lens", C.c_void_p), ("stride_codes", C.c_int64), ("stride_scales", C.c_int64),
                ("capacity", C.c_int32), ("len", C.c_int32), ("block", C.c_int32), ("format", C.c_int32), ("n_kv_heads", C.c_int32),
                ("d_head", C.c_int32), ("seqs_per_unit", C.c_int32), ("reserved", C.c_int32)]


_lib = None


def library_path() -> str:
    return os.environ.get("PSD_LIBRARY", os.path.join(_HERE, "libpsd.so"))


def load_library():
    """Loads libpsd.so (built by paper_2605_15609_amd/build.py).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise PsdError(f"{path} not found: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    sig = {
        "psd_status_string": (C.c_char_p, [i32]),
        "psd_last_error": (C.c_char_p, []),
        "psd_create": (i32, [C.POINTER(_Config), C.POINTER(_Weights), C.POINTER(vp)]),
        "psd_destroy": (i32, [vp]),
        "psd_debug_set_plain": (i32, [vp, i32]),
        "psd_debug_workspace_layout": (i32, [C.POINTER(_Config), i32, i32, i32, C.POINTER(_DebugLayout)]),
        "psd_debug_layer": (i32, [vp, i32, vp, i32, i32, i32, i32, vp, i64, vp]),
        "psd_workspace_bytes": (i64, [C.POINTER(_Config), i32, i32, i32]),
        "psd_decode_scratch_bytes": (i64, [i32, i32, i32, i32]),
        "psd_struct_sizes": (i32, [C.POINTER(i32), i32]),
        "psd_graph_chain": (i32, [i32, i32, C.POINTER(_Graph)]),
        "psd_graph_lattice": (i32, [i32, C.POINTER(_Graph)]),
        "psd_calibrate_graph": (i32, [vp, vp, vp, i32, i32, i32, i32, C.POINTER(_Policy), C.POINTER(_Graph), i32,
                                      C.POINTER(_GraphScore), C.POINTER(i32), vp, i32, vp, i64, vp]),
        "psd_forward_confidence": (i32, [vp, vp, i32, i32, i32, i32, vp, vp, vp, i64, vp]),
        "psd_forward_logits": (i32, [vp, vp, i32, i32, i32, i32, vp, vp, i64, vp]),
        "psd_select_unmask": (i32, [vp, vp, i32, i32, i32, i32, vp, vp, C.POINTER(_Policy), vp, vp, vp]),
        "psd_build_drafts": (i32, [vp, vp, i32, i32, i32, i32, vp, vp, C.POINTER(_Graph), vp, vp, vp, vp]),
        "psd_accept": (i32, [vp, vp, vp, i32, i32, i32, i32, vp, vp, C.POINTER(_Graph), C.POINTER(_Policy), vp, vp, vp,
                             vp, vp]),
        "psd_verify_accept": (i32, [vp, vp, vp, i32, i32, i32, i32, vp, vp, C.POINTER(_Graph), C.POINTER(_Policy), vp,
                                    vp, vp, vp, vp, i64, vp]),
        "psd_kv_cache_bytes": (i64, [C.POINTER(_Config), i32]),
        "psd_kv_reset": (i32, [vp, vp, i32, i32, vp]),
        "psd_kv_prefill": (i32, [vp, vp, i32, i32, i32, i32, vp, i32, vp, i64, vp]),
        "psd_forward_confidence_cached": (i32, [vp, vp, i32, i32, i32, i32, i32, vp, i32, vp, vp, vp, vp, i64, vp]),
        "psd_decode_block_cached": (i32, [vp, vp, i32, i32, i32, i32, C.POINTER(_Policy), C.POINTER(_Graph), C.POINTER(_Stats),
                                           vp, i32, vp, i64, vp]),
        "psd_decode_block": (i32, [vp, vp, i32, i32, C.POINTER(i32), i32, C.POINTER(_Policy), C.POINTER(_Graph), C.POINTER(_Stats),
                                   vp, i64, vp]),
        "psd_decode": (i32, [vp, vp, i32, i32, C.POINTER(i32), i32, C.POINTER(_Policy), C.POINTER(_Graph), C.POINTER(_Stats),
                             i32, C.POINTER(i32), vp, i64, vp]),
        "psd_forward_confidence_approx": (i32, [vp, vp, i32, i32, i32, i32, i32, i32, vp, i32, vp, vp, vp, vp, i64, vp]),
        "psd_decode_block_approx": (i32, [vp, vp, i32, i32, i32, i32, C.POINTER(_Policy), C.POINTER(_Graph), C.POINTER(_Stats),
                                          vp, i32, vp, i64, vp]),
        "psd_kernel_gemm_bf16": (i32, [vp, vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, vp, i32, vp]),
        "psd_kernel_gemm_residual_splitk": (i32, [vp, vp, i64, i32, i32, vp, vp, i64, i32, vp, vp]),
        "psd_kernel_attention_scratch_bytes": (i64, [i32, i32, i32, i32]),
        "psd_kernel_attention_bf16": (i32, [vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]),
        "psd_kernel_head_scratch_bytes": (i64, [i32, i32]),
        "psd_kernel_head_confidence_bf16": (i32, [vp, vp, i32, i32, i32, C.c_float, i32, vp, vp, vp, vp]),
        "psd_debug_force_gemm_tile": (i32, [i32]),
        "psd_debug_gemm_plan": (i32, [i64, i32, i32, i32, C.POINTER(i32)]),
        "psd_debug_gemm_cut": (i32, [i64, i32, i32, i32, C.POINTER(i64), C.POINTER(i64)]),
        "psd_debug_qkv_fused": (i32, [i64, i32, i32, i32, i32, i32, i32]),
        "psd_debug_gemm_ahead": (i32, [i64, i32, i32, i32]),
        "psd_debug_head_plan": (i32, [i32, i32, i32, C.POINTER(i32), C.POINTER(i32)]),
        "psd_debug_qkv_cut": (i32, [i64, i32, i32, i32, i32, i32]),
        "psd_debug_set_graphs": (i32, [vp, i32, C.POINTER(i64)]),
        "psd_kernel_packed_bytes": (i64, [i64, i32]),
        "psd_kernel_pack_rows": (i32, [vp, i64, i32, vp, vp]),
        "psd_kernel_head_stream_bf16": (i32, [vp, vp, i32, i32, i32, C.c_float, i32, vp, vp, vp, vp]),
        "psd_kernel_head_stream_static_bf16": (i32, [vp, vp, i32, i32, i32, C.c_float, i32, vp, vp, vp]),
        "psd_kernel_mfma_rate": (i32, [vp, i64, i32, vp, i64, C.POINTER(C.c_double), vp]),
        "psd_probe_begin": (i32, [vp, i32, i32, i32]),
        "psd_probe_end": (i32, [vp, i32, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.POINTER(C.c_double)]),
        "psd_probe_read": (i32, [vp, i32, i32, C.POINTER(C.c_float), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
        "psd_kernel_gemm_tile": (i32, [i64, i32, i32]),
        "psd_kernel_gemm_tile_count": (i32, []),
        "psd_kernel_gemm_tile_name": (C.c_char_p, [i32]),
        "psd_forward_work": (i32, [C.POINTER(_Config), i32, i32, i32, C.POINTER(_Work)]),
        "psd_shared_struct_sizes": (i32, [C.POINTER(i32), i32]),
        "psd_attention_shared_bytes": (i64, [vp, vp, i32]),
        "psd_attention_shared": (i32, [vp, vp, vp, i32, vp, vp, vp, i64, vp]),
        "psd_debug_attention_plan": (i32, [vp, vp, i32, C.POINTER(i32), i32]),
        "psd_attention_weights_bytes": (i64, [vp, vp, i32]),
        "psd_attention_weights": (i32, [vp, vp, vp, i32, vp, i32, vp, i64, vp]),
        "psd_shared_workspace_bytes": (i64, [C.POINTER(_Config), i32, i32, C.POINTER(_KvShared)]),
        "psd_forward_confidence_shared": (i32, [vp, vp, i32, i32, i32, i32, C.POINTER(_KvShared), vp, vp, vp, vp, i64, vp]),
        "psd_kv_extend_shared": (i32, [vp, vp, i32, i32, i32, i32, C.POINTER(_KvShared), vp, i64, vp]),
        "psd_decode_block_shared": (i32, [vp, vp, i32, i32, i32, i32, C.POINTER(_Policy), C.POINTER(_Graph), C.POINTER(_Stats),
                                          C.POINTER(_KvShared), vp, i64, vp]),
        "psd_kv_evict": (i32, [vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp]),
        "psd_kv8_struct_sizes": (i32, [C.POINTER(i32), i32]),
        "psd_rotary_frequencies": (i32, [C.POINTER(_RotaryScaling), i32, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
        "psd_rotary": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "psd_kv8_store": (i32, [vp, i32, vp, vp, i64, i64, i32, i32, i32, vp, vp, vp]),
        "psd_kv8_load": (i32, [vp, i32, i32, i32, vp, vp, i64, i64, i32, vp]),
        "psd_attention_kv8_bytes": (i64, [vp, vp, i32]),
        "psd_attention_kv8": (i32, [vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, i64, vp]),
        "psd_debug_force_attention_kv8": (i32, [i32, i32]),
        "psd_debug_attention_kv8_plan": (i32, [vp, vp, i32, C.POINTER(i32)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    # the structures declared here must be the ones the library was built with
    mine = [C.sizeof(t) for t in (_Config, _Weights, _Policy, _Graph, _Stats, _Work, _GraphScore, _DebugLayout)]
    theirs = (i32 * len(mine))()
    if lib.psd_struct_sizes(theirs, len(mine)) != len(mine) or list(theirs) != mine:
        raise PsdError(f"binding and libpsd.so disagree on the structure layouts: {mine} vs {list(theirs)} (rebuild the library)")
    mine = [C.sizeof(t) for t in (_Segment, _AttentionShape, _KvShared)]
    theirs = (i32 * len(mine))()
    if lib.psd_shared_struct_sizes(theirs, len(mine)) != len(mine) or list(theirs) != mine:
        raise PsdError(f"binding and libpsd.so disagree on the segment layouts: {mine} vs {list(theirs)} (rebuild the library)")
    mine = [C.sizeof(t) for t in (_RotaryShape, _RotaryScaling, _Kv8Cache)]
    theirs = (i32 * len(mine))()
    if lib.psd_kv8_struct_sizes(theirs, len(mine)) != len(mine) or list(theirs) != mine:
        raise PsdError(f"binding and libpsd.so disagree on the layouts of 8-bit caches: {mine} vs {list(theirs)} (rebuild the library)")
    _lib = lib
    return lib


def _check(rc: int):
    if rc < 0:
        lib = load_library()
        raise PsdError(f"{lib.psd_status_string(int(rc)).decode()} ({int(rc)}): {lib.psd_last_error().decode()}")
    return rc


@dataclass(frozen=True)
class Policy:
    tau: float = 0.9
    k_min: int = 1
    k_max: int = 0
    eos_id: Optional[int] = None     # EOS early stopping of the block loop (App. B.1); None = off
    # block loops: the post-verification commit doubles as the next stage-1 commit and the next drafts come from the
    # accepted draft's verifier output -- one model call per iteration; not the literal Alg. 1
    single_forward: bool = False

    def c(self) -> _Policy:
        return _Policy(float(np.float32(self.tau)), int(self.k_min), int(self.k_max),
                       0 if self.eos_id is None else 1, 0 if self.eos_id is None else int(self.eos_id),
                       1 if self.single_forward else 0)


@dataclass(frozen=True)
class Graph:
    rank_sets: tuple      # K ints, bit r set <-> rank r speculated; rank_sets[0] == 0

    @property
    def K(self) -> int:
        return len(self.rank_sets)

    def c(self) -> _Graph:
        g = _Graph()
        g.K = self.K
        for k, bits in enumerate(self.rank_sets):
            g.rank_set[k] = int(bits)
        return g


def chain_graph(K: int, width: int = 1) -> Graph:
    g = _Graph()
    _check(load_library().psd_graph_chain(K, width, C.byref(g)))
    return Graph(tuple(int(g.rank_set[k]) for k in range(g.K)))


def lattice_graph(depth: int) -> Graph:
    g = _Graph()
    _check(load_library().psd_graph_lattice(depth, C.byref(g)))
    return Graph(tuple(int(g.rank_set[k]) for k in range(g.K)))


@dataclass
class Stats:
    invocations: int = 0
    tokens_policy: int = 0
    tokens_draft: int = 0
    tokens_postverify: int = 0
    depth_hist: List[int] = field(default_factory=lambda: [0] * HIST)
    tokens_counted: int = 0      # resolved positions at or before the EOS position (App. B.1)
    stopped: bool = False
    eos_pos: int = -1

    @property
    def tokens(self) -> int:
        return self.tokens_policy + self.tokens_draft + self.tokens_postverify

    @property
    def tpf(self) -> float:
        return self.tokens / max(1, self.invocations)

    @property
    def tpf_counted(self) -> float:
        return self.tokens_counted / max(1, self.invocations)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev_i32(t, device):
    return torch.as_tensor(np.ascontiguousarray(t, dtype=np.int32) if not torch.is_tensor(t) else t, device=device) \
        .to(torch.int32).contiguous()


def pack_qkv(lt: dict) -> None:
    """Re-homes wq | wk | wv (and bq | bk | bv) of one layer back to back in one allocation, so the
    library can run the three projections as a single contraction, and w_down into padded rows.
    Views keep the storage alive."""
    w = torch.cat([lt["wq"], lt["wk"], lt["wv"]], dim=0).contiguous()
    nq, nk = lt["wq"].shape[0], lt["wk"].shape[0]
    lt["wq"], lt["wk"], lt["wv"] = w[:nq], w[nq:nq + nk], w[nq + nk:]
    if lt.get("bq") is not None:
        b = torch.cat([lt["bq"], lt["bk"], lt["bv"]]).contiguous()
        lt["bq"], lt["bk"], lt["bv"] = b[:nq], b[nq:nq + nk], b[nq + nk:]
    # w_down [d_model, d_ffn] with rows padded by 64 elements: dense rows of a multiple of 8 KB would all start
    # in the same cache channel (see psd_weights.w_down_stride)
    wd = lt["w_down"]
    if wd.dtype == torch.bfloat16 and wd.stride(0) == wd.shape[1]:
        padded = torch.zeros((wd.shape[0], wd.shape[1] + 64), dtype=wd.dtype, device=wd.device)
        padded[:, :wd.shape[1]] = wd
        lt["w_down"] = padded[:, :wd.shape[1]]


class Model:
    """Device-resident weights plus the library handle.  ``Model.from_host(host_model)``
    uploads a psd_inputs.HostModel; matrices go up in the model dtype, the rest as fp32."""

    def __init__(self, shape, max_seq: int, tensors: dict, layer_tensors: list, device="cuda:0"):
        self.lib = load_library()
        self.shape = shape
        self.max_seq = int(max_seq)
        self.device = torch.device(device)
        self._tensors = tensors            # keep alive: the handle borrows the pointers
        self._layers = layer_tensors
        self._ws = None
        cfg = _Config(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.d_head, shape.d_ffn,
                      shape.vocab, shape.mask_id, shape.rms_eps, int(shape.qkv_bias), 1 if shape.dtype == "bf16" else 0,
                      float(shape.logit_scale), self.max_seq, 1 if getattr(shape, "attention", "bidirectional") == "block_causal" else 0)
        self.cfg = cfg
        self._check_tensors(shape, mat_dtype=torch.bfloat16 if shape.dtype == "bf16" else torch.float32)
        w = _Weights()
        for name in ("tok_emb", "final_norm", "lm_head", "rope_cos", "rope_sin"):
            setattr(w, name, tensors[name].data_ptr())
        self._arrays = {}
        for name in ("attn_norm", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "ffn_norm", "w_gate", "w_up", "w_down"):
            if layer_tensors[0].get(name) is None:
                setattr(w, name, None)
                continue
            arr = (C.c_void_p * shape.n_layers)(*[lt[name].data_ptr() for lt in layer_tensors])
            self._arrays[name] = arr
            setattr(w, name, C.cast(arr, _PP))
        strides = {lt["w_down"].stride(0) for lt in layer_tensors}
        assert len(strides) == 1 and all(lt["w_down"].stride(1) == 1 for lt in layer_tensors)
        w.w_down_stride = strides.pop()
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.psd_create(C.byref(cfg), C.byref(w), C.byref(handle)))
        self.handle = handle

    def _check_tensors(self, shape, mat_dtype):
        """The library takes raw pointers: a tensor of the wrong dtype or extent would be read as garbage or past its
        end.  Matrices [out, in] in the model dtype; norm gains, biases and rotary tables fp32."""
        d, hq, hkv, f, v = shape.d_model, shape.n_heads * shape.d_head, shape.n_kv_heads * shape.d_head, shape.d_ffn, shape.vocab
        want = {"tok_emb": ((v, d), mat_dtype), "lm_head": ((v, d), mat_dtype), "final_norm": ((d,), torch.float32),
                "rope_cos": ((self.max_seq, shape.d_head // 2), torch.float32),
                "rope_sin": ((self.max_seq, shape.d_head // 2), torch.float32)}
        per_layer = {"attn_norm": ((d,), torch.float32), "ffn_norm": ((d,), torch.float32), "wq": ((hq, d), mat_dtype),
                     "wk": ((hkv, d), mat_dtype), "wv": ((hkv, d), mat_dtype), "wo": ((d, hq), mat_dtype),
                     "w_gate": ((f, d), mat_dtype), "w_up": ((f, d), mat_dtype), "w_down": ((d, f), mat_dtype),
                     "bq": ((hq,), torch.float32), "bk": ((hkv,), torch.float32), "bv": ((hkv,), torch.float32)}

        def check(name, t, dims, dtype, dense=True):
            if tuple(t.shape) != tuple(dims) or t.dtype != dtype or t.device.type != self.device.type or t.stride(-1) != 1 \
                    or (dense and not t.is_contiguous()):
                raise PsdError(f"{name}: expected a {'dense ' if dense else ''}{dtype} tensor of shape {tuple(dims)} on {self.device}, "
                               f"got {t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}")
        for name, (dims, dtype) in want.items():
            check(name, self._tensors[name], dims, dtype)
        for l, lt in enumerate(self._layers):
            for name, (dims, dtype) in per_layer.items():
                if lt.get(name) is None:
                    if name in ("bq", "bk", "bv") and not shape.qkv_bias:
                        continue
                    raise PsdError(f"layer {l}: {name} is missing")
                check(f"layer {l} {name}", lt[name], dims, dtype, dense=(name != "w_down"))

    @classmethod
    def from_host(cls, host_model, device="cuda:0") -> "Model":
        shape = host_model.shape
        mat_dtype = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        dev = torch.device(device)

        def up(a, dtype):
            return torch.from_numpy(np.ascontiguousarray(a)).to(device=dev, dtype=dtype).contiguous()

        tensors = {"tok_emb": up(host_model.tok_emb, mat_dtype), "lm_head": up(host_model.lm_head, mat_dtype),
                   "final_norm": up(host_model.final_norm, torch.float32),
                   "rope_cos": up(host_model.rope_cos, torch.float32), "rope_sin": up(host_model.rope_sin, torch.float32)}
        layers = []
        for lw in host_model.layers:
            lt = {}
            for k, v in lw.items():
                if v is None:
                    lt[k] = None
                else:
                    lt[k] = up(v, mat_dtype if v.ndim == 2 else torch.float32)
            pack_qkv(lt)
            layers.append(lt)
        return cls(shape, host_model.max_seq, tensors, layers, device)

    def close(self):
        if getattr(self, "handle", None):
            self.lib.psd_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_plain(self, mask: int):
        _check(self.lib.psd_debug_set_plain(self.handle, int(mask)))

    def set_graphs(self, enabled: Optional[bool] = None) -> int:
        """Switches the HIP-graph replay of the block loops' model calls on / off (None: leave); returns the number of
        graph launches so far."""
        n = C.c_int64()
        _check(self.lib.psd_debug_set_graphs(self.handle, -1 if enabled is None else int(bool(enabled)), C.byref(n)))
        return int(n.value)

    def probe_begin(self, epilogue: int, tile: int, max_launches: int = 65536):
        _check(self.lib.psd_probe_begin(self.handle, epilogue, tile, max_launches))

    def probe_end(self, epilogue: int):
        ms, n, fl = C.c_double(), C.c_int64(), C.c_double()
        _check(self.lib.psd_probe_end(self.handle, epilogue, C.byref(ms), C.byref(n), C.byref(fl)))
        return ms.value, n.value, fl.value

    def probe_read(self, epilogue: int, max_n: int = 1 << 16):
        """Per timed launch of the last probe of this kind: (milliseconds, a, b) -- see psd_probe_read."""
        ms, a, b = (C.c_float * max_n)(), (C.c_int64 * max_n)(), (C.c_int64 * max_n)()
        n = self.lib.psd_probe_read(self.handle, epilogue, max_n, ms, a, b)
        _check(n)
        return [(float(ms[i]), int(a[i]), int(b[i])) for i in range(n)]

    def workspace(self, n_bytes: int) -> torch.Tensor:
        if self._ws is None or self._ws.numel() < n_bytes:
            self._ws = None
            self._ws = torch.empty(int(n_bytes) + 256, dtype=torch.uint8, device=self.device)
        return self._ws

    def forward_ws(self, S: int, N: int, L: int, extra: int = 0):
        need = self.lib.psd_workspace_bytes(C.byref(self.cfg), S, N, L)
        _check(need)
        ws = self.workspace(need + extra)
        return ws, need + extra


def forward_work(model: Model, S: int, N: int, L: int) -> dict:
    w = _Work()
    _check(model.lib.psd_forward_work(C.byref(model.cfg), S, N, L, C.byref(w)))
    return {k: getattr(w, k) for k, _ in _Work._fields_}


# ------------------------------------------------------------------------------------------
# the calls of include/psd.h
# ------------------------------------------------------------------------------------------


def psd_forward_confidence(model: Model, tokens: torch.Tensor, block_start: int, L: int):
    """tokens int32 [S, N] on the device -> (top1 int32 [S, L], conf float32 [S, L])."""
    assert tokens.dtype == torch.int32 and tokens.is_contiguous() and tokens.dim() == 2
    S, N = tokens.shape
    top1 = torch.empty((S, L), dtype=torch.int32, device=tokens.device)
    conf = torch.empty((S, L), dtype=torch.float32, device=tokens.device)
    ws, nb = model.forward_ws(S, N, L)
    _check(model.lib.psd_forward_confidence(model.handle, _ptr(tokens), S, N, block_start, L, _ptr(top1), _ptr(conf),
                                            _ptr(ws), nb, _stream()))
    return top1, conf


def psd_forward_logits(model: Model, tokens: torch.Tensor, block_start: int, L: int) -> torch.Tensor:
    assert tokens.dtype == torch.int32 and tokens.is_contiguous() and tokens.dim() == 2
    S, N = tokens.shape
    logits = torch.empty((S * L, model.shape.vocab), dtype=torch.float32, device=tokens.device)
    ws, nb = model.forward_ws(S, N, L)
    _check(model.lib.psd_forward_logits(model.handle, _ptr(tokens), S, N, block_start, L, _ptr(logits), _ptr(ws), nb,
                                        _stream()))
    return logits


def psd_select_unmask(model: Model, tokens: torch.Tensor, block_start: int, L: int, top1: torch.Tensor,
                      conf: torch.Tensor, policy: Policy):
    """In place on tokens [B, N]; returns (transfer_mask uint8 [B, L], n_selected int32 [B])."""
    B, N = tokens.shape
    tm = torch.empty((B, L), dtype=torch.uint8, device=tokens.device)
    ns = torch.empty((B,), dtype=torch.int32, device=tokens.device)
    pol = policy.c()
    _check(model.lib.psd_select_unmask(model.handle, _ptr(tokens), B, N, block_start, L, _ptr(top1), _ptr(conf),
                                       C.byref(pol), _ptr(tm), _ptr(ns), _stream()))
    return tm, ns


def psd_build_drafts(model: Model, tokens: torch.Tensor, block_start: int, L: int, top1: torch.Tensor,
                     conf: torch.Tensor, graph: Graph):
    """-> (sigma int32 [B, L], m int32 [B], drafts int32 [B, K, N])."""
    B, N = tokens.shape
    sigma = torch.empty((B, L), dtype=torch.int32, device=tokens.device)
    m = torch.empty((B,), dtype=torch.int32, device=tokens.device)
    drafts = torch.empty((B, graph.K, N), dtype=torch.int32, device=tokens.device)
    g = graph.c()
    _check(model.lib.psd_build_drafts(model.handle, _ptr(tokens), B, N, block_start, L, _ptr(top1), _ptr(conf),
                                      C.byref(g), _ptr(sigma), _ptr(m), _ptr(drafts), _stream()))
    return sigma, m, drafts


def psd_accept(model: Model, tokens: torch.Tensor, drafts: torch.Tensor, block_start: int, L: int, sigma: torch.Tensor,
               m: torch.Tensor, graph: Graph, policy: Policy, v_top1: torch.Tensor, v_conf: torch.Tensor):
    """In place on tokens; returns (k_star int32 [B], accepted uint8 [B, K])."""
    B, N = tokens.shape
    k_star = torch.empty((B,), dtype=torch.int32, device=tokens.device)
    accepted = torch.empty((B, graph.K), dtype=torch.uint8, device=tokens.device)
    g, pol = graph.c(), policy.c()
    _check(model.lib.psd_accept(model.handle, _ptr(tokens), _ptr(drafts), B, N, block_start, L, _ptr(sigma), _ptr(m),
                                C.byref(g), C.byref(pol), _ptr(v_top1), _ptr(v_conf), _ptr(k_star), _ptr(accepted),
                                _stream()))
    return k_star, accepted


def psd_verify_accept(model: Model, tokens: torch.Tensor, drafts: torch.Tensor, block_start: int, L: int,
                      sigma: torch.Tensor, m: torch.Tensor, graph: Graph, policy: Policy):
    """One batched forward over the drafts + acceptance; in place on tokens.
    Returns (k_star, accepted, v_top1 [B, K, L], v_conf [B, K, L])."""
    B, N = tokens.shape
    K = graph.K
    k_star = torch.empty((B,), dtype=torch.int32, device=tokens.device)
    accepted = torch.empty((B, K), dtype=torch.uint8, device=tokens.device)
    v_top1 = torch.empty((B, K, L), dtype=torch.int32, device=tokens.device)
    v_conf = torch.empty((B, K, L), dtype=torch.float32, device=tokens.device)
    g, pol = graph.c(), policy.c()
    ws, nb = model.forward_ws(B * K, N, L)
    _check(model.lib.psd_verify_accept(model.handle, _ptr(tokens), _ptr(drafts), B, N, block_start, L, _ptr(sigma),
                                       _ptr(m), C.byref(g), C.byref(pol), _ptr(k_star), _ptr(accepted), _ptr(v_top1),
                                       _ptr(v_conf), _ptr(ws), nb, _stream()))
    return k_star, accepted, v_top1, v_conf


def _add_stats(stats, cstats, B) -> List[Stats]:
    out = list(stats) if stats is not None else [Stats() for _ in range(B)]
    for b in range(B):
        out[b].invocations += cstats[b].invocations
        out[b].tokens_policy += cstats[b].tokens_policy
        out[b].tokens_draft += cstats[b].tokens_draft
        out[b].tokens_postverify += cstats[b].tokens_postverify
        out[b].tokens_counted += cstats[b].tokens_counted
        if cstats[b].stopped:
            out[b].stopped, out[b].eos_pos = True, int(cstats[b].eos_pos)
        for i in range(HIST):
            out[b].depth_hist[i] += cstats[b].depth_hist[i]
    return out


def _starts(block_start, B: int):
    """One block start for the whole batch, or one per sequence -> int32[B] for the C call."""
    vals = [int(block_start)] * B if np.isscalar(block_start) else [int(v) for v in block_start]
    if len(vals) != B:
        raise PsdError(f"{len(vals)} block starts for a batch of {B}")
    return (C.c_int32 * B)(*vals)


def psd_decode_block(model: Model, tokens: torch.Tensor, block_start, L: int, policy: Policy, graph: Graph,
                     stats: Optional[Sequence[Stats]] = None) -> List[Stats]:
    """Alg. 1 on one block of every sequence of tokens [B, N], in place; block_start is one position for the batch or one
    per sequence.  Blocks until done."""
    B, N = tokens.shape
    K = graph.K
    extra = model.lib.psd_decode_scratch_bytes(B, N, L, K)
    _check(extra)
    ws, nb = model.forward_ws(B * K, N, L, extra=extra)
    cstats = (_Stats * B)()
    g, pol = graph.c(), policy.c()
    _check(model.lib.psd_decode_block(model.handle, _ptr(tokens), B, N, _starts(block_start, B), L, C.byref(pol), C.byref(g),
                                      cstats, _ptr(ws), nb, _stream()))
    return _add_stats(stats, cstats, B)


def psd_decode(model: Model, tokens: torch.Tensor, block_start, L: int, policy: Policy, graph: Graph,
               stats: Optional[Sequence[Stats]] = None, max_iterations: int = 0):
    """The whole generation behind one call: every sequence walks through its own blocks (see psd.h).  block_start as for
    psd_decode_block.  Returns (stats, block starts on return, iterations run); with max_iterations > 0 the call returns
    after that many iterations and can be continued from the returned block starts."""
    B, N = tokens.shape
    K = graph.K
    extra = model.lib.psd_decode_scratch_bytes(B, N, L, K)
    _check(extra)
    ws, nb = model.forward_ws(B * K, N, L, extra=extra)
    cstats = (_Stats * B)()
    g, pol = graph.c(), policy.c()
    starts = _starts(block_start, B)
    done = C.c_int32(0)
    _check(model.lib.psd_decode(model.handle, _ptr(tokens), B, N, starts, L, C.byref(pol), C.byref(g), cstats,
                                int(max_iterations), C.byref(done), _ptr(ws), nb, _stream()))
    return _add_stats(stats, cstats, B), [int(v) for v in starts], int(done.value)


class KvCache:
    """Device memory for the prefix KV caches of n_seqs sequences of a context-causal block model (zeroed)."""

    def __init__(self, model: Model, n_seqs: int, capacity: int):
        per_seq = model.lib.psd_kv_cache_bytes(C.byref(model.cfg), capacity)
        _check(per_seq)
        self.model, self.n_seqs, self.capacity = model, n_seqs, capacity
        self.mem = torch.empty(per_seq * n_seqs + 256, dtype=torch.uint8, device=model.device)
        self.reset()

    def reset(self):
        _check(self.model.lib.psd_kv_reset(self.model.handle, _ptr(self.mem), self.n_seqs, self.capacity, _stream()))

    def new_weights(self) -> torch.Tensor:
        """fp32 zeros [n_seqs, n_layers, n_kv_heads, capacity]: what the positions draw (SharedKv, segment)."""
        s = self.model.shape
        return torch.zeros((self.n_seqs, s.n_layers, s.n_kv_heads, self.capacity), dtype=torch.float32, device=self.mem.device)

    def segment(self, length: int, weights: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None) -> "KvSegment":
        """The layers of all caches as the units of one segment (sequence by sequence), `length` positions each: what psd_kv_evict
        takes from and gives to.  weights as new_weights makes them; lens int32 [n_seqs * n_layers]."""
        s = self.model.shape
        dtype = torch.bfloat16 if s.dtype == "bf16" else torch.float32
        width, ld_vt, units = s.n_kv_heads * s.d_head, (self.capacity + 63) // 64 * 64, self.n_seqs * s.n_layers
        unit = self.capacity * width + width * ld_vt
        flat = self.mem[:self.mem.numel() // 16 * 16].view(dtype)
        if weights is not None:
            want = (self.n_seqs, s.n_layers, s.n_kv_heads, self.capacity)
            if tuple(weights.shape) != want or not weights.is_contiguous():
                raise PsdError(f"weights: dense float32 {want}, not {tuple(weights.shape)}")
            weights = weights.view(units, s.n_kv_heads, self.capacity)
        return KvSegment(flat.as_strided((units, self.capacity, width), (unit, width, 1)),
                         flat.as_strided((units, width, ld_vt), (unit, ld_vt, 1), self.capacity * width), s.d_head, length=length, lens=lens,
                         weights=weights)


# A prompt's rows go into the cache in passes of up to PREFILL_ROWS rows whose workspace, which the model keeps, stays within
# PREFILL_WORKSPACE bytes.  16 sequences of 1024: 8B shape, 8 layers 43.0 ms with 4096 rows (664 MB) and with 16384 (1.8 GB);
# the small one 2.95 ms with 4096, 1.94 with 16384 (252 MB).
PREFILL_ROWS, PREFILL_WORKSPACE = 16384, 768 << 20


def _prefill_rows(model: Model, B: int, n_prompt: int, L: int) -> int:
    """Rows per sequence and pass."""
    if B < 1 or L < 1:
        return L               # refused by the library
    rows = max(L, min(n_prompt, PREFILL_ROWS // (B * L) * L))
    while rows > L and model.lib.psd_workspace_bytes(C.byref(model.cfg), B, rows, L) > PREFILL_WORKSPACE:
        rows = max(L, rows // (2 * L) * L)
    return rows


def psd_kv_prefill(model: Model, tokens: torch.Tensor, n_prompt: int, L: int, cache: KvCache) -> None:
    B, N = tokens.shape
    try:
        ws, nb = model.forward_ws(B, _prefill_rows(model, B, n_prompt, L), L)
    except torch.cuda.OutOfMemoryError:
        ws, nb = model.forward_ws(B, L, L)      # block by block
    _check(model.lib.psd_kv_prefill(model.handle, _ptr(tokens), B, N, n_prompt, L, _ptr(cache.mem), cache.capacity, _ptr(ws), nb,
                                    _stream()))


def psd_forward_confidence_cached(model: Model, tokens: torch.Tensor, block_start: int, L: int, cache: KvCache,
                                  seqs_per_cache: int = 1, want_logits: bool = False):
    """tokens int32 [S, N]; the block rows against the caches -> (top1 [S, L], conf [S, L][, logits [S*L, V]])."""
    S, N = tokens.shape
    top1 = torch.empty((S, L), dtype=torch.int32, device=tokens.device)
    conf = torch.empty((S, L), dtype=torch.float32, device=tokens.device)
    logits = torch.empty((S * L, model.shape.vocab), dtype=torch.float32, device=tokens.device) if want_logits else None
    ws, nb = model.forward_ws(S, L, L)
    _check(model.lib.psd_forward_confidence_cached(model.handle, _ptr(tokens), S, N, block_start, L, seqs_per_cache,
                                                   _ptr(cache.mem), cache.capacity, _ptr(top1), _ptr(conf), _ptr(logits),
                                                   _ptr(ws), nb, _stream()))
    return (top1, conf, logits) if want_logits else (top1, conf)


def psd_decode_block_cached(model: Model, tokens: torch.Tensor, block_start: int, L: int, policy: Policy, graph: Graph,
                            cache: KvCache, stats: Optional[Sequence[Stats]] = None) -> List[Stats]:
    """psd_decode_block with cached model calls; the finished block is appended to the caches."""
    B, N = tokens.shape
    K = graph.K
    extra = model.lib.psd_decode_scratch_bytes(B, N, L, K)
    _check(extra)
    ws, nb = model.forward_ws(B * K, L, L, extra=extra)
    cstats = (_Stats * B)()
    g, pol = graph.c(), policy.c()
    _check(model.lib.psd_decode_block_cached(model.handle, _ptr(tokens), B, N, block_start, L, C.byref(pol), C.byref(g), cstats,
                                             _ptr(cache.mem), cache.capacity, _ptr(ws), nb, _stream()))
    return _add_stats(stats, cstats, B)


def psd_forward_confidence_approx(model: Model, tokens: torch.Tensor, block_start: int, L: int, cache: KvCache, refresh: bool,
                                  seqs_per_cache: int = 1, want_logits: bool = False):
    """Model call of a bidirectional model under the approximate prefix + suffix cache: refresh = exact call over the whole
    sequences that fills the caches; otherwise the block rows against them.  Returns (top1, conf[, logits])."""
    S, N = tokens.shape
    ws, nb = model.forward_ws(S, N if refresh else L, L)
    top1 = torch.empty((S, L), dtype=torch.int32, device=tokens.device)
    conf = torch.empty((S, L), dtype=torch.float32, device=tokens.device)
    logits = torch.empty((S * L, model.cfg.vocab), dtype=torch.float32, device=tokens.device) if want_logits else None
    _check(model.lib.psd_forward_confidence_approx(model.handle, _ptr(tokens), S, N, block_start, L, 1 if refresh else 0,
                                                   seqs_per_cache, _ptr(cache.mem), cache.capacity, _ptr(top1), _ptr(conf),
                                                   _ptr(logits), _ptr(ws), nb, _stream()))
    return (top1, conf, logits) if want_logits else (top1, conf)


def psd_decode_block_approx(model: Model, tokens: torch.Tensor, block_start: int, L: int, policy: Policy, graph: Graph,
                            cache: KvCache, stats: Optional[Sequence[Stats]] = None) -> List[Stats]:
    """psd_decode_block under the approximate cache: the first model call on the block is exact and fills the caches."""
    B, N = tokens.shape
    K = graph.K
    extra = model.lib.psd_decode_scratch_bytes(B, N, L, K)
    _check(extra)
    full = model.lib.psd_workspace_bytes(C.byref(model.cfg), B, N, L)
    rows = model.lib.psd_workspace_bytes(C.byref(model.cfg), B * K, L, L)
    _check(full)
    _check(rows)
    if full >= rows:
        ws, nb = model.forward_ws(B, N, L, extra=extra)
    else:
        ws, nb = model.forward_ws(B * K, L, L, extra=extra)
    cstats = (_Stats * B)()
    g, pol = graph.c(), policy.c()
    _check(model.lib.psd_decode_block_approx(model.handle, _ptr(tokens), B, N, block_start, L, C.byref(pol), C.byref(g), cstats,
                                             _ptr(cache.mem), cache.capacity, _ptr(ws), nb, _stream()))
    return _add_stats(stats, cstats, B)


# ---- keys that a batch shares, the weights they draw, eviction by those weights (see psd.h) ----

_DTYPES = {torch.bfloat16: 1, torch.float32: 0}


def _int32(value, what: str) -> int:
    """A count for a 32-bit argument (ctypes would cut what is larger)."""
    n = int(value)
    if not -2 ** 31 <= n < 2 ** 31:
        raise PsdError(f"{what} {n} is no 32-bit number")
    return n


class KvSegment:
    """Keys that the sequences of a batch attend to, one unit of them for every seqs_per_unit consecutive sequences.

    k [units, positions, n_kv_heads * d_head] and vt [units, n_kv_heads * d_head, at least the positions rounded up to 16] (values
    transposed, keys of every group of 16 in the order 0-3, 8-11, 4-7, 12-15), bf16 or fp32, dense along the last dimension; the
    first `length` positions are keys (default: all), or lens[unit] of them (int32 [units]; what is outside 0 .. length is cut).
    weights fp32 [units, n_kv_heads, positions]: what psd_attention_weights writes and psd_kv_evict goes by."""

    def __init__(self, k: torch.Tensor, vt: torch.Tensor, d_head: int, length: Optional[int] = None, seqs_per_unit: int = 1,
                 lens: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None):
        if k.dim() != 3 or vt.dim() != 3 or k.dtype not in _DTYPES or vt.dtype != k.dtype or k.shape[0] != vt.shape[0] \
                or k.shape[2] != vt.shape[1] or d_head < 1 or k.shape[2] % d_head or k.stride(2) != 1 or vt.stride(2) != 1:
            raise PsdError(f"keys [units, positions, heads * d_head] and values [units, heads * d_head, slots] of one type, dense along the "
                           f"last dimension, not {k.dtype} {tuple(k.shape)} {k.stride()} and {vt.dtype} {tuple(vt.shape)} {vt.stride()}")
        units, positions, width = k.shape
        n = positions if length is None else int(length)
        if not 0 <= n <= positions or (n + 15) // 16 * 16 > vt.shape[2]:
            raise PsdError(f"{n} keys of {positions} positions, value rows of {vt.shape[2]}")
        if lens is not None and (lens.dtype != torch.int32 or tuple(lens.shape) != (units,) or not lens.is_contiguous()):
            raise PsdError(f"lens: dense int32 [{units}], not {lens.dtype} {tuple(lens.shape)}")
        if weights is not None and (weights.dtype != torch.float32 or weights.dim() != 3 or tuple(weights.shape[:2]) != (units, width // d_head)
                                    or weights.shape[2] < n or weights.stride(2) != 1):
            raise PsdError(f"weights: float32 [{units}, {width // d_head}, at least {n}] dense along the last dimension, not "
                           f"{weights.dtype} {tuple(weights.shape)} {weights.stride()}")
        for t in (vt, lens, weights):
            if t is not None and t.device != k.device:
                raise PsdError(f"a segment on {k.device} and {t.device}")
        self.k, self.vt, self.lens, self.weights = k, vt, lens, weights
        self.units, self.length, self.d_head, self.n_kv_heads = units, n, int(d_head), width // d_head
        self.seqs_per_unit, self.device, self.dtype = int(seqs_per_unit), k.device, k.dtype
        def address(t):
            return None if t is None or t.numel() == 0 else t.data_ptr()
        # (strides of dimensions of one entry mean nothing, and torch gives any)
        ld_k, ld_vt = k.stride(1) if positions > 1 else width, vt.stride(1) if width > 1 else vt.shape[2]
        ld_w = 0 if weights is None else weights.stride(1) if self.n_kv_heads > 1 else weights.shape[2]
        self.c = _Segment(address(k), address(vt), address(lens), address(weights), k.stride(0) if units > 1 else 0,
                          vt.stride(0) if units > 1 else 0, 0 if weights is None or units == 1 else weights.stride(0), _int32(ld_k, "key row stride"),
                          _int32(ld_vt, "value row stride"), _int32(ld_w, "weight row stride"), _int32(n, "length"),
                          _int32(self.seqs_per_unit, "seqs_per_unit"), 0)


class KvSegments:
    """The segments of a batch, coarse to fine, as the calls take them (built once, used by many calls)."""

    def __init__(self, segments: Sequence[KvSegment]):
        self.segments = list(segments)
        if not self.segments:
            raise PsdError("no segments")
        first = self.segments[0]
        for s in self.segments:
            if (s.device, s.dtype, s.d_head, s.n_kv_heads) != (first.device, first.dtype, first.d_head, first.n_kv_heads):
                raise PsdError("segments of different devices, types or heads")
        self.c = (_Segment * len(self.segments))(*[s.c for s in self.segments])
        self.shapes: dict = {}      # (see _attention_shape)
        self.n, self.device, self.dtype, self.d_head, self.n_kv_heads = len(self.segments), first.device, first.dtype, first.d_head, first.n_kv_heads


def _rows(t: torch.Tensor, what: str) -> int:
    """Row stride of [S, L, heads, d_head] whose S * L rows are evenly spaced and hold their heads densely."""
    S, L, H, d = t.shape
    row = t.stride(1) if L > 1 else t.stride(0) if S > 1 else H * d
    if (d > 1 and t.stride(3) != 1) or (H > 1 and t.stride(2) != d) or (S > 1 and t.stride(0) != L * row):
        raise PsdError(f"{what}: heads of a row one behind the other, rows evenly spaced, not {tuple(t.shape)} with strides {t.stride()}")
    return row


def _attention_shape(q: torch.Tensor, keys: KvSegments, out: Optional[torch.Tensor] = None) -> _AttentionShape:
    """The shape of a call, checked.  A program makes the same call over and over: what was checked once for tensors of these shapes,
    strides, types and devices is not checked again (it says nothing about their contents or addresses)."""
    key = (q.shape, q.stride(), q.dtype, q.device) if out is None else (q.shape, q.stride(), q.dtype, q.device, out.shape, out.stride(), out.dtype, out.device)
    found = keys.shapes.get(key)
    if found is not None:
        return found
    if q.dim() != 4 or q.dtype != keys.dtype or q.device != keys.device or q.shape[3] != keys.d_head:
        raise PsdError(f"q [S, L, heads, {keys.d_head}] {keys.dtype} on {keys.device}, not {q.dtype} {tuple(q.shape)} on {q.device}")
    S, L, H, d = q.shape
    if out is not None and (out.shape != q.shape or out.dtype != q.dtype or out.device != q.device):
        raise PsdError(f"out like q, not {out.dtype} {tuple(out.shape)} on {out.device}")
    for s in keys.segments:
        if s.seqs_per_unit < 1 or s.units * s.seqs_per_unit != S:
            raise PsdError(f"{s.units} units of {s.seqs_per_unit} sequences for a batch of {S}")
    if S * L * H >= 2 ** 31:
        raise PsdError(f"{S} sequences of {L} rows of {H} heads are too many")
    shape = _AttentionShape(S, L, H, keys.n_kv_heads, d, _DTYPES[q.dtype], _rows(q, "q"), H * d if out is None else _rows(out, "out"))
    if len(keys.shapes) >= 64:
        keys.shapes.clear()
    keys.shapes[key] = shape
    return shape


def _check_lse(lse: torch.Tensor, q: torch.Tensor) -> None:
    if lse.dtype != torch.float32 or lse.shape != q.shape[:3] or not lse.is_contiguous() or lse.device != q.device:
        raise PsdError(f"lse: dense float32 {tuple(q.shape[:3])} on {q.device}, not {lse.dtype} {tuple(lse.shape)} on {lse.device}")


def _workspace(need, device, given: Optional[torch.Tensor]):
    """(address, bytes, the tensor that has to live until the call is enqueued) of a call's workspace, `given` or new."""
    if given is None:
        if need == 0:
            return None, 0, None
        given = torch.empty((need,), dtype=torch.uint8, device=device)
    elif given.device != device or not given.is_contiguous():
        raise PsdError(f"a dense workspace on {device}, not on {given.device}")
    return given.data_ptr(), given.nbytes, given


class _on_device:
    """The current stream of a tensor's device, whichever device is current."""

    def __init__(self, device):
        if device.type != "cuda":
            raise PsdError(f"tensors on a GPU, not on {device}")
        self.device, self.guard = device, None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream if _raw_stream is None else _raw_stream(self.device.index)

    def __exit__(self, *what):
        if self.guard is not None:
            self.guard.__exit__(*what)


# (the address alone: torch.cuda.current_stream makes an object for it, 2.9 of the 15 us that a small call took)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def psd_attention_workspace(q: torch.Tensor, keys: KvSegments) -> torch.Tensor:
    """What psd_attention_shared needs for q and keys, to be kept and passed on as ws."""
    shape = _attention_shape(q, keys)
    return torch.empty((max(256, _check(load_library().psd_attention_shared_bytes(C.byref(shape), keys.c, keys.n))),), dtype=torch.uint8,
                       device=q.device)


def psd_attention_weights_bytes(q: torch.Tensor, keys: KvSegments) -> int:
    """Bytes of workspace that psd_attention_weights needs for q and keys (possibly 0)."""
    shape = _attention_shape(q, keys)
    return int(_check(load_library().psd_attention_weights_bytes(C.byref(shape), keys.c, keys.n)))


def attention_plan(q: torch.Tensor, keys: KvSegments) -> List[Tuple[int, ...]]:
    """psd_debug_attention_plan: (first segment, segments, form, units, tiles, parts, rows of a unit and KV head) of every job."""
    shape, jobs = _attention_shape(q, keys), (C.c_int32 * 28)()
    n = _check(load_library().psd_debug_attention_plan(C.byref(shape), keys.c, keys.n, jobs, 4))
    return [tuple(jobs[7 * i:7 * i + 7]) for i in range(n)]


def psd_attention_shared(q: torch.Tensor, keys: KvSegments, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of q [S, L, n_heads, d_head] over the keys of all segments -> out [S, L, n_heads, d_head]; lse fp32 [S, L, n_heads]
    receives the log of each row's sum of exponentials."""
    lib = load_library()
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    shape = _attention_shape(q, keys, out)
    if lse is not None:
        _check_lse(lse, q)
    with _on_device(q.device) as stream:
        need = 0 if ws is not None else _check(lib.psd_attention_shared_bytes(C.byref(shape), keys.c, keys.n))
        at, n, ws = _workspace(need, q.device, ws)
        _check(lib.psd_attention_shared(C.byref(shape), q.data_ptr(), keys.c, keys.n, out.data_ptr(), None if lse is None else lse.data_ptr(),
                                        at, n, stream))
    return out


def psd_attention_weights(q: torch.Tensor, keys: KvSegments, lse: torch.Tensor, accumulate: bool = True,
                          ws: Optional[torch.Tensor] = None) -> None:
    """What every key of the segments with weights drew from the rows of q under the lse of psd_attention_shared, added to their
    weights (accumulate) or in their place."""
    lib = load_library()
    shape = _attention_shape(q, keys)
    _check_lse(lse, q)
    with _on_device(q.device) as stream:
        need = 0 if ws is not None else _check(lib.psd_attention_weights_bytes(C.byref(shape), keys.c, keys.n))
        at, n, ws = _workspace(need, q.device, ws)
        _check(lib.psd_attention_weights(C.byref(shape), q.data_ptr(), keys.c, keys.n, lse.data_ptr(), int(bool(accumulate)), at, n, stream))


def psd_kv_evict(src: KvSegment, dst: KvSegment, keep: int, first: int = 0, last: int = 0, kept: Optional[torch.Tensor] = None,
                 kept_lens: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The `keep` positions of every unit and KV head of src that drew most (the first and last ones always) into dst, in ascending
    order -> kept int32 [units, n_kv_heads, keep], their positions in src, -1 behind the last; kept_lens int32 [units]."""
    shape = (src.units, src.n_kv_heads, int(keep))
    if (dst.units, dst.n_kv_heads, dst.d_head, dst.dtype, dst.device) != (src.units, src.n_kv_heads, src.d_head, src.dtype, src.device):
        raise PsdError("source and destination differ in units, heads, type or device")
    if not 1 <= _int32(keep, "keep") or _int32(first, "first") < 0 or _int32(last, "last") < 0:
        raise PsdError(f"keep {keep}, first {first}, last {last}")
    if kept is None:
        kept = torch.empty(shape, dtype=torch.int32, device=src.device)
    for name, t, want in (("kept", kept, shape), ("kept_lens", kept_lens, shape[:1])):
        if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != want or not t.is_contiguous() or t.device != src.device):
            raise PsdError(f"{name}: dense int32 {want} on {src.device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    with _on_device(src.device) as stream:
        _check(load_library().psd_kv_evict(C.byref(src.c), C.byref(dst.c), src.units, src.n_kv_heads, src.d_head, _DTYPES[src.dtype], int(keep),
                                           int(first), int(last), kept.data_ptr(), _ptr(kept_lens), stream))
    return kept


_ROTARY_KINDS = {"plain": 0, "linear": 1, "base": 2, "parts": 3}
_KV8_FORMATS = {"int8": 0, "e4m3": 1}


def rotary_frequencies(rotated: int, theta: float, kind: str = "plain", stretch: float = 1.0, trained: float = 0.0, slow: float = 1.0,
                       fast: float = 32.0) -> Tuple[torch.Tensor, float]:
    """psd_rotary_frequencies: (float64 [rotated / 2] on the CPU, the factor for psd_rotary) of theta^(-2j / rotated), plain or scaled for contexts
    `stretch` times as long ("linear", "base", "parts" with the trained length and the turns over it below / above which a frequency is
    stretched / kept)."""
    if kind not in _ROTARY_KINDS:
        raise PsdError(f"scaling {kind!r}, not one of {sorted(_ROTARY_KINDS)}")
    n = _int32(rotated, "rotated")
    out, factor = torch.empty((max(0, min(n, 1 << 16)) // 2,), dtype=torch.float64), C.c_double(1.0)
    scaling = _RotaryScaling(float(theta), float(stretch), float(trained), float(slow), float(fast), _ROTARY_KINDS[kind], 0)
    _check(load_library().psd_rotary_frequencies(C.byref(scaling), n, C.cast(out.data_ptr(), C.POINTER(C.c_double)), C.byref(factor)))
    return out, factor.value


def _address(t: Optional[torch.Tensor]):
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _layout(t: Optional[torch.Tensor]):
    # (the device's number, not the device, whose hash is slow; whatever is not on a GPU is -1 and never passes a check beside what is)
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


def _dense_on(t: torch.Tensor, what: str, dtype, shape, device) -> None:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != device:
        raise PsdError(f"{what}: dense {dtype} {tuple(shape)} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def psd_rotary(q: torch.Tensor, k: Optional[torch.Tensor], frequencies: torch.Tensor, positions: Optional[torch.Tensor] = None, first: int = 0,
               interleaved: bool = False, factor: float = 1.0, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None,
               eps: float = 1e-6, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None
               ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """q [S, L, n_heads, d_head] and k [S, L, n_kv_heads, d_head] (or None), normed where there are gains (float32 [d_head]), their first
    2 * len(frequencies) channels (float64) turned by positions int32 [S, L] (None: first + row) -> (q_out, k_out), new or given; q_out = q
    and k_out = k work in place."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is not None and k_out is None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    shape = _rotary_shape(q, k, frequencies, positions, first, interleaved, factor, q_gain, k_gain, eps, q_out, k_out)
    with _on_device(q.device) as stream:
        _check(load_library().psd_rotary(C.byref(shape), q.data_ptr(), None if k is None else k.data_ptr(), frequencies.data_ptr(),
                                         None if positions is None else positions.data_ptr(), None if q_gain is None else q_gain.data_ptr(),
                                         None if k_gain is None else k_gain.data_ptr(), q_out.data_ptr(), None if k is None else k_out.data_ptr(), stream))
    return q_out, k_out


_rotary_shapes: dict = {}


def _rotary_shape(q, k, frequencies, positions, first, interleaved, factor, q_gain, k_gain, eps, q_out, k_out) -> _RotaryShape:
    """The shape of a call, checked once for tensors of these shapes, strides, types and devices (as _attention_shape)."""
    key = (first, interleaved, factor, eps, _layout(q), _layout(k), _layout(frequencies), _layout(positions), _layout(q_gain), _layout(k_gain), _layout(q_out),
           _layout(k_out))
    found = _rotary_shapes.get(key)
    if found is not None:
        return found
    if q.dim() != 4 or q.dtype not in _DTYPES or (k is not None and (k.dim() != 4 or k.dtype != q.dtype or k.device != q.device
                                                                     or (k.shape[0], k.shape[1], k.shape[3]) != (q.shape[0], q.shape[1], q.shape[3]))):
        raise PsdError(f"q [S, L, heads, d] and k [S, L, KV heads, d], bf16 or fp32, not {q.dtype} {tuple(q.shape)} and "
                       f"{None if k is None else (k.dtype, tuple(k.shape), k.device)}")
    if k is None and (k_gain is not None or k_out is not None):
        raise PsdError("a gain or an output of no keys")
    S, L, H, d = q.shape
    for name, t, like in (("q_out", q_out, q), ("k_out", k_out, k)):
        if t is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
            raise PsdError(f"{name}: {like.dtype} {tuple(like.shape)} on {like.device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    if frequencies.dim() != 1:
        raise PsdError(f"frequencies: float64 [pairs], not {tuple(frequencies.shape)}")
    _dense_on(frequencies, "frequencies", torch.float64, frequencies.shape, q.device)
    if positions is not None:
        _dense_on(positions, "positions", torch.int32, (S, L), q.device)
    for name, t in (("q_gain", q_gain), ("k_gain", k_gain)):
        if t is not None:
            _dense_on(t, name, torch.float32, (d,), q.device)
    shape = _RotaryShape(S * L, _rows(q, "q"), 0 if k is None else _rows(k, "k"), _rows(q_out, "q_out"), 0 if k is None else _rows(k_out, "k_out"),
                         _int32(H, "heads"), 0 if k is None else _int32(k.shape[2], "KV heads"), _int32(d, "d_head"), _int32(2 * frequencies.numel(), "rotated"),
                         int(bool(interleaved)), _int32(first, "first"), _int32(L, "rows"), _DTYPES[q.dtype], float(factor), float(eps), 0)
    if len(_rotary_shapes) >= 256:
        _rotary_shapes.clear()
    _rotary_shapes[key] = shape
    return shape


class Kv8Cache:
    """Keys and values in 8 bits with a scale for every block of positions and KV head.

    codes uint8 [units, n_kv_heads, positions / 32, 2, 32 * d_head] and scales float32 [units, n_kv_heads, positions / block, 2], each unit dense
    (include/psd.h has the order of the codes); format "int8" or "e4m3".  The first `length` positions (default: all) of a unit are held, or lens[unit]
    of them (int32 [units], what is outside 0 .. length is cut); seqs_per_unit consecutive sequences attend to a unit.  These three may be set anew (a
    workspace kept for a shorter length may then be too small, which the call says); everything else stays as the cache was made."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, d_head: int, format: str = "int8", length: Optional[int] = None,
                 lens: Optional[torch.Tensor] = None, seqs_per_unit: int = 1):
        if format not in _KV8_FORMATS:
            raise PsdError(f"format {format!r}, not one of {sorted(_KV8_FORMATS)}")
        if codes.dim() != 5 or codes.dtype != torch.uint8 or d_head < 1 or tuple(codes.shape[3:]) != (2, 32 * d_head) or scales.dim() != 4 \
                or scales.dtype != torch.float32 or scales.shape[:2] != codes.shape[:2] or scales.shape[3] != 2 \
                or not codes[:1].is_contiguous() or not scales[:1].is_contiguous():
            raise PsdError(f"codes uint8 [units, heads, positions / 32, 2, {32 * d_head}] and scales float32 [units, heads, blocks, 2], dense, not "
                           f"{codes.dtype} {tuple(codes.shape)} {codes.stride()} and {scales.dtype} {tuple(scales.shape)} {scales.stride()}")
        units, heads, tiles = codes.shape[:3]
        positions, blocks = 32 * tiles, scales.shape[2]
        block = positions // blocks if blocks else 32
        if block * blocks != positions:
            raise PsdError(f"{blocks} scales for {positions} positions")
        if scales.device != codes.device:
            raise PsdError(f"a cache on {codes.device} and {scales.device}")
        self.codes, self.scales, self.format, self.device = codes, scales, format, codes.device
        self.units, self.n_kv_heads, self.d_head, self.capacity, self.block = units, heads, int(d_head), positions, block
        self.c = _Kv8Cache(_address(codes), _address(scales), None, codes.stride(0) if units > 1 else 0, scales.stride(0) if units > 1 else 0,
                           _int32(positions, "positions"), 0, _int32(block, "block"), _KV8_FORMATS[format], _int32(heads, "KV heads"),
                           _int32(d_head, "d_head"), 1, 0)
        self.shapes: dict = {}      # (see rows and _kv8_shape)
        self.length, self.lens, self.seqs_per_unit = positions if length is None else length, lens, seqs_per_unit

    def __setattr__(self, name, value):
        """What the calls read is self.c, so that says what the attributes say (anew: a copy of the cache has its own)."""
        if name == "length":
            value = int(value)
            if not 0 <= value <= self.capacity:
                raise PsdError(f"{value} positions of {self.capacity}")
            self._describe("len", value)
        elif name == "lens":
            if value is not None:
                _dense_on(value, "lens", torch.int32, (self.units,), self.device)
            self._describe("lens", _address(value))
        elif name == "seqs_per_unit":
            value = _int32(value, "seqs_per_unit")
            self._describe("seqs_per_unit", value)
            self.__dict__["shapes"] = {}
        elif name in self.__dict__:
            raise PsdError(f"{name} stays as the cache was made")
        super().__setattr__(name, value)

    def _describe(self, field, value):
        c = _Kv8Cache.from_buffer_copy(self.c)
        setattr(c, field, value)
        self.__dict__["c"] = c

    @classmethod
    def empty(cls, units: int, n_kv_heads: int, d_head: int, positions: int, block: int = 32, format: str = "int8", device="cuda:0",
              lens: Optional[torch.Tensor] = None, seqs_per_unit: int = 1) -> "Kv8Cache":
        """A cache of at least `positions` positions, not written yet."""
        if block not in (16, 32, 64, 128) or min(units, n_kv_heads, d_head) < 1 or positions < 0:
            raise PsdError(f"{units} units of {n_kv_heads} x {d_head}, {positions} positions, {block} to a scale (16, 32, 64, 128)")
        n = -(-positions // max(block, 32)) * max(block, 32)
        return cls(torch.empty((units, n_kv_heads, n // 32, 2, 32 * d_head), dtype=torch.uint8, device=device),
                   torch.empty((units, n_kv_heads, n // block, 2), dtype=torch.float32, device=device), d_head, format, None, lens, seqs_per_unit)

    def rows(self, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None,
             counts: Optional[torch.Tensor] = None) -> Tuple[int, int, int, int]:
        """(rows of a unit, row stride of k, of v, dtype) of [units, n, n_kv_heads, d_head] and what goes with them, checked once for tensors of
        these shapes, strides, types and devices (as _attention_shape)."""
        key = ("rows", _layout(k), _layout(v), _layout(starts), _layout(counts))
        found = self.shapes.get(key)
        if found is not None:
            return found
        want = (self.units, self.n_kv_heads, self.d_head)
        for name, t in (("k", k), ("v", v)):
            if t.dim() != 4 or t.dtype not in _DTYPES or t.dtype != k.dtype or (t.shape[0], t.shape[2], t.shape[3]) != want or t.shape != k.shape \
                    or t.device != self.device:
                raise PsdError(f"{name}: [{want[0]}, n, {want[1]}, {want[2]}] bf16 or fp32 on {self.device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
        for name, t in (("starts", starts), ("counts", counts)):
            if t is not None:
                _dense_on(t, name, torch.int32, (self.units,), self.device)
        _int32(self.units, "units")
        return self.remember(key, (_int32(k.shape[1], "rows"), _rows(k, "k"), _rows(v, "v"), _DTYPES[k.dtype]))

    def remember(self, key, found):
        if len(self.shapes) >= 64:
            self.shapes.clear()
        self.shapes[key] = found
        return found


def psd_kv8_store(cache: Kv8Cache, k: torch.Tensor, v: torch.Tensor, first: int = 0, starts: Optional[torch.Tensor] = None,
                  counts: Optional[torch.Tensor] = None) -> None:
    """Rows k, v [units, n, n_kv_heads, d_head] into the cache, at positions first .. of every unit or from starts int32 [units] on; counts
    int32 [units]: only the first of a unit's rows.  cache.lens is left as it is."""
    n, ld_k, ld_v, dtype = cache.rows(k, v, starts, counts)
    with _on_device(cache.device) as stream:
        _check(load_library().psd_kv8_store(C.byref(cache.c), cache.units, k.data_ptr(), v.data_ptr(), ld_k, ld_v, dtype, n, _int32(first, "first"),
                                            None if starts is None else starts.data_ptr(), None if counts is None else counts.data_ptr(), stream))


def psd_kv8_load(cache: Kv8Cache, first: int = 0, n: Optional[int] = None, dtype=torch.bfloat16, k_out: Optional[torch.Tensor] = None,
                 v_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """What positions first .. first + n - 1 (default: up to cache.length) of every unit stand for -> k, v [units, n, n_kv_heads, d_head], new (of dtype, zero behind
    a unit's length) or given (left as they are there)."""
    n = max(cache.length - _int32(first, "first"), 0) if n is None else _int32(n, "n")
    if (k_out is None) != (v_out is None):
        raise PsdError("k_out and v_out, or neither")
    if k_out is None:
        if n < 0 or dtype not in _DTYPES:
            raise PsdError(f"{n} positions as {dtype}")
        k_out, v_out = (torch.zeros((cache.units, n, cache.n_kv_heads, cache.d_head), dtype=dtype, device=cache.device) for _ in range(2))
    rows, ld_k, ld_v, kind = cache.rows(k_out, v_out)
    if rows != n:
        raise PsdError(f"{rows} rows for {n} positions")
    with _on_device(cache.device) as stream:
        _check(load_library().psd_kv8_load(C.byref(cache.c), cache.units, _int32(first, "first"), n, k_out.data_ptr(), v_out.data_ptr(), ld_k, ld_v, kind, stream))
    return k_out, v_out


def _kv8_shape(q: torch.Tensor, cache: Kv8Cache, k: Optional[torch.Tensor], v: Optional[torch.Tensor], out: Optional[torch.Tensor]):
    """(shape, row strides of k and v) of a call, checked once for tensors of these shapes, strides, types and devices (as _attention_shape)."""
    key = (_layout(q), _layout(k), _layout(v), _layout(out))
    found = cache.shapes.get(key)
    if found is not None:
        return found
    if q.dim() != 4 or q.dtype not in _DTYPES or q.device != cache.device or q.shape[3] != cache.d_head:
        raise PsdError(f"q [S, L, heads, {cache.d_head}] bf16 or fp32 on {cache.device}, not {q.dtype} {tuple(q.shape)} on {q.device}")
    S, L, H, d = q.shape
    if (k is None) != (v is None):
        raise PsdError("keys and values of the rows' own blocks, or neither")
    for name, t in (("k", k), ("v", v)):
        if t is not None and (t.dtype != q.dtype or t.device != q.device or tuple(t.shape) != (S, L, cache.n_kv_heads, d)):
            raise PsdError(f"{name}: {q.dtype} {(S, L, cache.n_kv_heads, d)} on {q.device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    if out is not None and (out.shape != q.shape or out.dtype != q.dtype or out.device != q.device):
        raise PsdError(f"out like q, not {out.dtype} {tuple(out.shape)} on {out.device}")
    if cache.seqs_per_unit < 1 or cache.units * cache.seqs_per_unit != S:
        raise PsdError(f"{cache.units} units of {cache.seqs_per_unit} sequences for a batch of {S}")
    if S * L * H >= 2 ** 31:
        raise PsdError(f"{S} sequences of {L} rows of {H} heads are too many")
    shape = _AttentionShape(S, L, H, cache.n_kv_heads, d, _DTYPES[q.dtype], _rows(q, "q"), H * d if out is None else _rows(out, "out"))
    return cache.remember(key, (shape, 0 if k is None else _rows(k, "k"), 0 if v is None else _rows(v, "v")))


def psd_attention_kv8_workspace(q: torch.Tensor, cache: Kv8Cache, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None) -> torch.Tensor:
    """What psd_attention_kv8 needs for q and cache, to be kept and passed on as ws."""
    shape = _kv8_shape(q, cache, k, v, None)[0]
    need = _check(load_library().psd_attention_kv8_bytes(C.byref(shape), C.byref(cache.c), int(k is not None)))
    return torch.empty((max(256, need),), dtype=torch.uint8, device=q.device)


def attention_kv8_plan(q: torch.Tensor, cache: Kv8Cache, own_rows: bool = False) -> Tuple[int, ...]:
    """psd_debug_attention_kv8_plan: (form, tiles of rows of a unit and KV head, parts of the keys, keys of a part)."""
    plan = (C.c_int32 * 4)()
    _check(load_library().psd_debug_attention_kv8_plan(C.byref(_kv8_shape(q, cache, None, None, None)[0]), C.byref(cache.c), int(bool(own_rows)), plan))
    return tuple(plan)


def psd_attention_kv8(q: torch.Tensor, cache: Kv8Cache, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of q [S, L, n_heads, d_head] over the cache and, where given, the rows k, v [S, L, n_kv_heads, d_head] of each sequence's own
    block -> out like q; lse fp32 [S, L, n_heads] receives the log of each row's sum of exponentials."""
    lib = load_library()
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    shape, ld_k, ld_v = _kv8_shape(q, cache, k, v, out)
    if lse is not None:
        _check_lse(lse, q)
    with _on_device(q.device) as stream:
        need = 0 if ws is not None else _check(lib.psd_attention_kv8_bytes(C.byref(shape), C.byref(cache.c), int(k is not None)))
        at, n, ws = _workspace(need, q.device, ws)
        _check(lib.psd_attention_kv8(C.byref(shape), q.data_ptr(), C.byref(cache.c), None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
                                     ld_k, ld_v, out.data_ptr(), None if lse is None else lse.data_ptr(), at, n, stream))
    return out


@dataclass
class SharedKv:
    """What the block rows of a shared call attend to besides their block: prefix_len positions of `prefix` (a cache of one sequence), then
    `length` positions of their sequence's cache.  prefix_weights / cache_weights (KvCache.new_weights): collect what the positions draw."""
    prefix: Optional[KvCache] = None
    prefix_len: int = 0
    cache: Optional[KvCache] = None
    length: int = 0
    prefix_weights: Optional[torch.Tensor] = None
    cache_weights: Optional[torch.Tensor] = None

    def c(self, model: Model, n_caches: int, seqs_per_cache: int = 1) -> _KvShared:
        device = _device_of(model)
        for what, cache, weights, n in (("prefix", self.prefix, self.prefix_weights, 1), ("cache", self.cache, self.cache_weights, n_caches)):
            if cache is not None and cache.n_seqs < n:
                raise PsdError(f"{what}: {cache.n_seqs} sequences, {n} needed")
            if cache is not None and (cache.model.shape, cache.mem.device) != (model.shape, device):
                raise PsdError(f"{what}: the cache of another model or device")
            if weights is not None:
                want = None if cache is None else (cache.n_seqs, model.shape.n_layers, model.shape.n_kv_heads, cache.capacity)
                if tuple(weights.shape) != want or weights.dtype != torch.float32 or not weights.is_contiguous() or weights.device != device:
                    raise PsdError(f"{what} weights: dense float32 {want} on {device}, not {weights.dtype} {tuple(weights.shape)} on {weights.device}")

        def address(t):
            return None if t is None else t.data_ptr()
        return _KvShared(None if self.prefix is None else self.prefix.mem.data_ptr(), None if self.cache is None else self.cache.mem.data_ptr(),
                         address(self.prefix_weights), address(self.cache_weights), 0 if self.prefix is None else self.prefix.capacity,
                         _int32(self.prefix_len, "prefix_len"), 0 if self.cache is None else self.cache.capacity, _int32(self.length, "length"),
                         _int32(seqs_per_cache, "seqs_per_cache"), 0)


def _device_of(model: Model) -> torch.device:
    """Where the weights are, with its index (model.device is what the caller named, "cuda" for one)."""
    return model._tensors["tok_emb"].device


def _check_tokens(model: Model, tokens: torch.Tensor) -> torch.device:
    """The device of the model, where its token rows have to be."""
    device = _device_of(model)
    if tokens.dim() != 2 or tokens.dtype != torch.int32 or not tokens.is_contiguous() or tokens.device != device:
        raise PsdError(f"tokens: dense int32 [sequences, positions] on {device}, not {tokens.dtype} {tuple(tokens.shape)} {tokens.stride()} on {tokens.device}")
    return device


def _shared_ws(model: Model, S: int, L: int, kv: _KvShared, extra: int = 0):
    need = _check(model.lib.psd_shared_workspace_bytes(C.byref(model.cfg), S, L, C.byref(kv))) + extra
    return model.workspace(need), need


def psd_forward_confidence_shared(model: Model, tokens: torch.Tensor, block_start: int, L: int, kv: SharedKv, seqs_per_cache: int = 1,
                                  want_logits: bool = False):
    """tokens int32 [S, N]; the block rows against a prefix of the whole batch and their caches -> (top1 [S, L], conf [S, L][, logits])."""
    block_start, L = _int32(block_start, "block_start"), _int32(L, "L")
    with _on_device(_check_tokens(model, tokens)) as stream:
        S, N = tokens.shape
        if seqs_per_cache < 1 or S % seqs_per_cache:
            raise PsdError(f"{S} sequences, {seqs_per_cache} to a cache")
        c = kv.c(model, S // seqs_per_cache, seqs_per_cache)
        ws, nb = _shared_ws(model, S, L, c)
        top1 = torch.empty((S, L), dtype=torch.int32, device=tokens.device)
        conf = torch.empty((S, L), dtype=torch.float32, device=tokens.device)
        logits = torch.empty((S * L, model.shape.vocab), dtype=torch.float32, device=tokens.device) if want_logits else None
        _check(model.lib.psd_forward_confidence_shared(model.handle, _ptr(tokens), S, N, block_start, L, C.byref(c), _ptr(top1), _ptr(conf),
                                                       _ptr(logits), _ptr(ws), nb, stream))
    return (top1, conf, logits) if want_logits else (top1, conf)


def psd_kv_extend_shared(model: Model, tokens: torch.Tensor, block_start: int, L: int, kv: SharedKv) -> None:
    """The block of every sequence of tokens [B, N] behind the first kv.length positions of its cache (kv.length is then L more: the
    caller's to count)."""
    block_start, L = _int32(block_start, "block_start"), _int32(L, "L")
    with _on_device(_check_tokens(model, tokens)) as stream:
        B, N = tokens.shape
        c = kv.c(model, B)
        ws, nb = _shared_ws(model, B, L, c)
        _check(model.lib.psd_kv_extend_shared(model.handle, _ptr(tokens), B, N, block_start, L, C.byref(c), _ptr(ws), nb, stream))


def psd_decode_block_shared(model: Model, tokens: torch.Tensor, block_start: int, L: int, policy: Policy, graph: Graph, kv: SharedKv,
                            stats: Optional[Sequence[Stats]] = None) -> List[Stats]:
    """psd_decode_block with shared model calls; the finished block is appended to the caches (kv.length is then L more)."""
    block_start, L = _int32(block_start, "block_start"), _int32(L, "L")
    with _on_device(_check_tokens(model, tokens)) as stream:
        B, N = tokens.shape
        K = graph.K
        c = kv.c(model, B)
        extra = _check(model.lib.psd_decode_scratch_bytes(B, N, L, K))
        ws, nb = _shared_ws(model, B * K, L, kv.c(model, B, K), extra=extra)
        cstats = (_Stats * B)()
        g, pol = graph.c(), policy.c()
        _check(model.lib.psd_decode_block_shared(model.handle, _ptr(tokens), B, N, block_start, L, C.byref(pol), C.byref(g),
                                                 cstats, C.byref(c), _ptr(ws), nb, stream))
    return _add_stats(stats, cstats, B)


def psd_calibrate_graph(model: Model, tokens: torch.Tensor, prompt_len: int, L: int, policy: Policy,
                        candidates: Sequence[Graph], cache: Optional[KvCache] = None):
    """Offline choice of the draft graph: decodes the calibration batch tokens [B, N] (left untouched) once per
    candidate and returns (index of the candidate with the highest tokens/s, list of score dicts)."""
    B, N = tokens.shape
    K = max(g.K for g in candidates)
    extra = model.lib.psd_decode_scratch_bytes(B, N, L, K)
    _check(extra)
    ws, nb = model.forward_ws(B * K, N, L, extra=extra)
    work = torch.empty_like(tokens)
    cg = (_Graph * len(candidates))(*[g.c() for g in candidates])
    scores = (_GraphScore * len(candidates))()
    best = C.c_int32(-1)
    pol = policy.c()
    _check(model.lib.psd_calibrate_graph(model.handle, _ptr(tokens), _ptr(work), B, N, prompt_len, L, C.byref(pol), cg,
                                         len(candidates), scores, C.byref(best), None if cache is None else _ptr(cache.mem),
                                         0 if cache is None else cache.capacity, _ptr(ws), nb, _stream()))
    return int(best.value), [{k: getattr(sc, k) for k, _ in _GraphScore._fields_} for sc in scores]


def decode(model: Model, tokens: torch.Tensor, prompt_len: int, L: int, policy: Policy, graph: Graph) -> List[Stats]:
    """Semi-autoregressive generation of everything behind the prompt: one psd_decode call (every sequence walks through
    its own blocks; with EOS early stopping a sequence ends with the block that produced the EOS token).  A generated
    part that is not whole blocks is decoded block by block with a shorter last block."""
    B, N = tokens.shape
    if (N - prompt_len) % L == 0:
        return psd_decode(model, tokens, prompt_len, L, policy, graph)[0]
    stats = [Stats() for _ in range(B)]
    for block_start in range(prompt_len, N, L):
        if all(s.stopped for s in stats):
            break
        if any(s.stopped for s in stats):
            raise PsdError("a ragged last block after an EOS stop of part of the batch: decode those sequences separately")
        stats = psd_decode_block(model, tokens, block_start, min(L, N - block_start), policy, graph, stats)
    return stats


# ------------------------------------------------------------------------------------------
# kernel-level hooks (parity tests and timing at full shapes without a model)
# ------------------------------------------------------------------------------------------

EPI_STORE, EPI_BIAS, EPI_RESIDUAL, EPI_SWIGLU = 0, 1, 2, 3


def debug_layer(model: Model, layer: int, hidden: torch.Tensor, S: int, N: int, L: int, stop_after: int = 0) -> dict:
    """psd_debug_layer: one layer of the model on the caller's residual stream hidden fp32 [S*N, d_model] (in place).
    Returns views of the intermediates the layer left in the workspace (valid until the next call on this model):
    a [S*N, d], qkv [S*N, qkv_w] (rotary applied), o [S*N, H*dh], act [S*N, d_ffn] (stop_after = 0 only)."""
    assert hidden.dtype == torch.float32 and hidden.is_contiguous() and hidden.shape == (S * N, model.shape.d_model)
    ws, nb = model.forward_ws(S, N, L)
    lay = _DebugLayout()
    _check(model.lib.psd_debug_workspace_layout(C.byref(model.cfg), S, N, L, C.byref(lay)))
    _check(model.lib.psd_debug_layer(model.handle, layer, _ptr(hidden), S, N, L, stop_after, _ptr(ws), nb, _stream()))
    sh = model.shape
    dt = torch.bfloat16 if sh.dtype == "bf16" else torch.float32
    esz = 2 if sh.dtype == "bf16" else 4
    T = S * N
    qkv_w = (sh.n_heads + 2 * sh.n_kv_heads) * sh.d_head

    def view(off, rows, ld, width):
        return ws[off: off + rows * ld * esz].view(dt).view(rows, ld)[:, :width]

    out = {"a": view(lay.off_a, T, sh.d_model, sh.d_model), "qkv": view(lay.off_qkv, T, lay.ld_qkv, qkv_w),
           "o": view(lay.off_o, T, sh.n_heads * sh.d_head, sh.n_heads * sh.d_head)}
    if stop_after == 0:
        out["act"] = view(lay.off_act, T, lay.ld_act, sh.d_ffn)
    return out


# ------------------------------------------------------------------------------------------
# kernel-level hooks (parity tests and timing at full shapes without a model)
# ------------------------------------------------------------------------------------------

EPI_STORE, EPI_BIAS, EPI_RESIDUAL, EPI_SWIGLU = 0, 1, 2, 3


def kernel_gemm_bf16(A: torch.Tensor, W: torch.Tensor, epilogue: int = EPI_STORE, W2: Optional[torch.Tensor] = None,
                     bias: Optional[torch.Tensor] = None, resid: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None):
    """A bf16 [M, K], W bf16 [N, K] -> out bf16 [M, N] (or resid fp32 [M, N] += for EPI_RESIDUAL).
    A and W (W2 like W) may be row-strided views (unit stride along K)."""
    lib = load_library()
    M, K = A.shape
    Nout = W.shape[0]
    assert A.stride(1) == 1 and W.stride(1) == 1 and (W2 is None or W2.stride() == W.stride())
    lda, ldw = A.stride(0), W.stride(0)
    if epilogue == EPI_RESIDUAL:
        assert resid is not None and resid.dtype == torch.float32
        _check(lib.psd_kernel_gemm_bf16(_ptr(A), _ptr(W), None, M, Nout, K, lda, ldw, epilogue, None, None, _ptr(resid),
                                        resid.stride(0), _stream()))
        return resid
    if out is None:
        out = torch.empty((M, Nout), dtype=torch.bfloat16, device=A.device)
    _check(lib.psd_kernel_gemm_bf16(_ptr(A), _ptr(W), _ptr(W2), M, Nout, K, lda, ldw, epilogue, _ptr(bias), _ptr(out), None,
                                    out.stride(0), _stream()))
    return out


def kernel_gemm_residual_splitk(A: torch.Tensor, W: torch.Tensor, resid: torch.Tensor, k_splits: int = 0,
                                partial: Optional[torch.Tensor] = None) -> int:
    """resid fp32 [M, N] += A W^T with the K range cut into k_splits parts (0 = the forward's choice);
    returns the number of parts used."""
    lib = load_library()
    M, K = A.shape
    Nout = W.shape[0]
    assert A.is_contiguous() and W.is_contiguous()
    assert resid.dtype == torch.float32 and resid.is_contiguous() and resid.shape == (M, Nout)
    if partial is None:
        partial = torch.empty((7 * M * Nout,), dtype=torch.float32, device=A.device)
    used = C.c_int32(0)
    _check(lib.psd_kernel_gemm_residual_splitk(_ptr(A), _ptr(W), M, Nout, K, _ptr(resid), _ptr(partial),
                                               partial.numel() * 4, k_splits, C.byref(used), _stream()))
    return used.value


def kernel_attention_bf16(qkv: torch.Tensor, S: int, N: int, n_heads: int, n_kv_heads: int, d_head: int,
                          out: Optional[torch.Tensor] = None, vT: Optional[torch.Tensor] = None):
    """qkv bf16 [S*N, (n_heads + 2 n_kv_heads) * d_head], possibly a row-strided view -> out bf16 [S*N, n_heads*d_head]."""
    lib = load_library()
    assert qkv.stride(1) == 1
    if vT is None:
        vT = torch.empty((lib.psd_kernel_attention_scratch_bytes(S, N, n_kv_heads, d_head) // 2,), dtype=torch.bfloat16,
                         device=qkv.device)
    if out is None:
        out = torch.empty((S * N, n_heads * d_head), dtype=torch.bfloat16, device=qkv.device)
    _check(lib.psd_kernel_attention_bf16(_ptr(qkv), qkv.stride(0), S, N, n_heads, n_kv_heads, d_head, _ptr(vT), _ptr(out),
                                         _stream()))
    return out


def kernel_head_confidence_bf16(y: torch.Tensor, W: torch.Tensor, scale: float, mask_id: int, scratch=None):
    """y bf16 [rows, d], W bf16 [V, d] -> (row_sum fp32 [rows], row_arg int32 [rows])."""
    lib = load_library()
    rows, d = y.shape
    V = W.shape[0]
    if scratch is None:
        scratch = torch.empty((int(lib.psd_kernel_head_scratch_bytes(rows, V)),), dtype=torch.uint8, device=y.device)
    row_sum = torch.empty((rows,), dtype=torch.float32, device=y.device)
    row_arg = torch.empty((rows,), dtype=torch.int32, device=y.device)
    _check(lib.psd_kernel_head_confidence_bf16(_ptr(y), _ptr(W), rows, V, d, float(scale), int(mask_id), _ptr(scratch),
                                               _ptr(row_sum), _ptr(row_arg), _stream()))
    return row_sum, row_arg


def kernel_mfma_rate(operands: torch.Tensor, iters: int = 4000) -> float:
    """Sustained TFLOP/s of a pure-MFMA loop on the given bf16 operand data (see psd.h)."""
    lib = load_library()
    sink = torch.empty((4 << 20,), dtype=torch.uint8, device=operands.device)
    fl = C.c_double()
    nbytes = operands.numel() * operands.element_size()
    _check(lib.psd_kernel_mfma_rate(_ptr(operands), nbytes, 50, _ptr(sink), sink.numel(), C.byref(fl), _stream()))
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    _check(lib.psd_kernel_mfma_rate(_ptr(operands), nbytes, iters, _ptr(sink), sink.numel(), C.byref(fl), _stream()))
    e1.record()
    torch.cuda.synchronize()
    return fl.value / (e0.elapsed_time(e1) * 1e-3) / 1e12


def kernel_pack_rows(src: torch.Tensor) -> torch.Tensor:
    """Row-major bf16 [R, K] -> its MFMA-fragment-order copy (flat bf16 tensor)."""
    lib = load_library()
    R, K = src.shape
    n = int(lib.psd_kernel_packed_bytes(R, K))
    _check(n)
    dst = torch.empty((n // 2,), dtype=torch.bfloat16, device=src.device)
    _check(lib.psd_kernel_pack_rows(_ptr(src), R, K, _ptr(dst), _stream()))
    return dst


def kernel_head_stream_bf16(y: torch.Tensor, W_packed: torch.Tensor, V: int, scale: float, mask_id: int, scratch=None,
                            y_packed=None):
    """Streaming LM-head on a pre-packed weight copy; y row-major bf16 [rows, d] is packed here."""
    lib = load_library()
    rows, d = y.shape
    if y_packed is None:
        y_packed = kernel_pack_rows(y)
    if scratch is None:
        scratch = torch.empty((int(lib.psd_kernel_head_scratch_bytes(rows, V)),), dtype=torch.uint8, device=y.device)
    row_sum = torch.empty((rows,), dtype=torch.float32, device=y.device)
    row_arg = torch.empty((rows,), dtype=torch.int32, device=y.device)
    _check(lib.psd_kernel_head_stream_bf16(_ptr(y_packed), _ptr(W_packed), rows, V, d, float(scale), int(mask_id),
                                           _ptr(scratch), _ptr(row_sum), _ptr(row_arg), _stream()))
    return row_sum, row_arg


def kernel_head_stream_static_bf16(y_packed: torch.Tensor, W_packed: torch.Tensor, rows: int, V: int, d: int, scale: float,
                                   mask_id: int, row_sum: torch.Tensor, row_arg: torch.Tensor) -> None:
    """psd_kernel_head_stream_static_bf16: every buffer comes from the caller, the library's static array serves as
    scratch; nothing is allocated here or in the library."""
    _check(load_library().psd_kernel_head_stream_static_bf16(_ptr(y_packed), _ptr(W_packed), rows, V, d, float(scale),
                                                             int(mask_id), _ptr(row_sum), _ptr(row_arg), _stream()))
