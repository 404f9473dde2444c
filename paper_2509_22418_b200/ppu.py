"""ctypes binding of libppu.so: the same calls as include/ppu.h, argument marshalling only.

PyTorch is used for device memory (the arena, token buffers) and the CUDA stream.  Every step
of the training path runs inside the library's kernels; if the library or a CUDA device is
missing the calls raise - there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libppu.so")

PPU_OK = 0
STATUS = {0: "PPU_OK", -1: "PPU_EINVAL", -2: "PPU_ESHAPE", -3: "PPU_ESUBSET", -4: "PPU_ENOMEM",
          -5: "PPU_ESTATE", -6: "PPU_ECUDA", -7: "PPU_ETIMEOUT", -8: "PPU_ETOKEN"}
SUBSET_FFN_SLICE, SUBSET_FFN_LAYERS, SUBSET_EXPLICIT = 0, 1, 2


class PpuError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class ModelCfg(C.Structure):
    _fields_ = [("n_layer", C.c_int32), ("d_model", C.c_int32), ("n_head", C.c_int32),
                ("d_ff", C.c_int32), ("vocab", C.c_int32), ("max_batch", C.c_int32),
                ("max_seq", C.c_int32), ("ln_eps", C.c_float), ("rope_base", C.c_float),
                ("adam_lr", C.c_float), ("adam_beta1", C.c_float), ("adam_beta2", C.c_float),
                ("adam_eps", C.c_float), ("adam_wd", C.c_float), ("outer_lr", C.c_float),
                ("outer_momentum", C.c_float)]


class SubsetSpec(C.Structure):
    _fields_ = [("n_replicas", C.c_int32), ("mode", C.c_int32), ("n_slices", C.c_int32),
                ("layer_stride", C.c_int32), ("ranges", C.POINTER(C.c_int32)),
                ("train_non_mlp", C.c_int32), ("n_head_slices", C.c_int32),
                ("head_ranges", C.POINTER(C.c_int32))]


class Stats(C.Structure):
    _fields_ = [("param_count", C.c_int64), ("arena_bytes", C.c_int64), ("state_bytes", C.c_int64),
                ("activation_bytes", C.c_int64), ("launches_last_step", C.c_int64),
                ("launches_last_sync", C.c_int64), ("flops_fwd", C.c_double),
                ("flops_dgrad", C.c_double), ("flops_wgrad", C.c_double), ("outer_bytes", C.c_double),
                ("saved_bytes_last_step", C.c_int64)]


CLS_GEMM, CLS_ATTN, CLS_LN, CLS_XENT, CLS_ADAMW, CLS_OUTER, CLS_OTHER, CLS_COUNT = 0, 1, 2, 3, 4, 5, 6, 8
CLS_NAMES = {CLS_GEMM: "gemm", CLS_ATTN: "attention", CLS_LN: "layernorm", CLS_XENT: "cross_entropy",
             CLS_ADAMW: "adamw", CLS_OUTER: "outer", CLS_OTHER: "other"}


class Profile(C.Structure):
    _fields_ = [("ms", C.c_double * CLS_COUNT), ("work", C.c_double * CLS_COUNT),
                ("launches", C.c_int64 * CLS_COUNT), ("dropped", C.c_int64)]

    # the two classes bench.py's roofline is built from
    gemm_ms = property(lambda self: self.ms[CLS_GEMM])
    gemm_flops = property(lambda self: self.work[CLS_GEMM])
    gemm_launches = property(lambda self: self.launches[CLS_GEMM])
    attn_ms = property(lambda self: self.ms[CLS_ATTN])
    attn_flops = property(lambda self: self.work[CLS_ATTN])
    attn_launches = property(lambda self: self.launches[CLS_ATTN])


_lib = None


def lib():
    """Loads libppu.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise PpuError(-6, f"{LIB_PATH} is missing: run paper_2509_22418_b200/build.py")
        _lib = C.CDLL(LIB_PATH)
        _lib.ppu_last_error.restype = C.c_char_p
    return _lib


def _check(rc):
    if rc != PPU_OK:
        raise PpuError(rc, lib().ppu_last_error().decode())


def make_cfg(n_layer, d_model, n_head, d_ff, vocab, max_batch, max_seq, ln_eps=1e-5,
             rope_base=1e4, adam_lr=1e-3, adam_beta1=0.9, adam_beta2=0.95, adam_eps=1e-8,
             adam_wd=0.1, outer_lr=0.7, outer_momentum=0.9) -> ModelCfg:
    return ModelCfg(n_layer, d_model, n_head, d_ff, vocab, max_batch, max_seq, ln_eps, rope_base,
                    adam_lr, adam_beta1, adam_beta2, adam_eps, adam_wd, outer_lr, outer_momentum)


def make_spec(n_replicas, mode=SUBSET_FFN_SLICE, n_slices=1, layer_stride=1, ranges=None,
              train_non_mlp=0, n_head_slices=0, head_ranges=None):
    """ranges: int array [K][L][2] for SUBSET_EXPLICIT; head_ranges: optional int array [K][2].
    Returns (spec, keepalive)."""
    keep = []
    ptr = C.POINTER(C.c_int32)()
    hptr = C.POINTER(C.c_int32)()
    if ranges is not None:
        keep.append(np.ascontiguousarray(ranges, dtype=np.int32))
        ptr = keep[-1].ctypes.data_as(C.POINTER(C.c_int32))
    if head_ranges is not None:
        keep.append(np.ascontiguousarray(head_ranges, dtype=np.int32))
        assert keep[-1].shape == (n_replicas, 2)
        hptr = keep[-1].ctypes.data_as(C.POINTER(C.c_int32))
    return SubsetSpec(n_replicas, mode, n_slices, layer_stride, ptr, int(train_non_mlp),
                      int(n_head_slices), hptr), keep


def ppu_query_bytes(cfg: ModelCfg, spec: SubsetSpec) -> int:
    n = C.c_size_t(0)
    _check(lib().ppu_query_bytes(C.byref(cfg), C.byref(spec), C.byref(n)))
    return n.value


def _np_ptr(a, ctype):
    return a.ctypes.data_as(C.POINTER(ctype))


class Context:
    """Owns the torch arena and the ppu_ctx handle; methods mirror the C calls."""

    def __init__(self, cfg: ModelCfg, spec: SubsetSpec, keepalive=None, device="cuda:0", stream=None):
        import torch
        if not torch.cuda.is_available():
            raise PpuError(-6, "no CUDA device: this library has no CPU path")
        self.torch = torch
        self.cfg, self.spec, self._keep = cfg, spec, keepalive
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        nbytes = ppu_query_bytes(cfg, spec)
        self.arena = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.arena.data_ptr() + 255) & ~255
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._h = C.c_void_p()
        _check(lib().ppu_create(C.byref(cfg), C.byref(spec), C.c_void_p(base), C.c_size_t(nbytes),
                                C.c_void_p(self.stream.cuda_stream), C.byref(self._h)))
        n = C.c_int64()
        _check(lib().ppu_param_count(self._h, C.byref(n)))
        self.param_count = n.value

    def close(self):
        if self._h:
            lib().ppu_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the four calls of the path ----
    def ppu_local_step(self, replica: int, tokens_dev) -> None:
        assert tokens_dev.is_cuda and tokens_dev.dtype == self.torch.int32 and tokens_dev.is_contiguous()
        b, s = tokens_dev.shape
        _check(lib().ppu_local_step(self._h, replica, C.c_void_p(tokens_dev.data_ptr()), b, s))

    def ppu_local_step_host(self, replica: int, tokens_host: np.ndarray) -> float:
        t = np.ascontiguousarray(tokens_host, dtype=np.int32)
        out = C.c_double()
        _check(lib().ppu_local_step_host(self._h, replica, _np_ptr(t, C.c_int32), t.shape[0],
                                         t.shape[1], C.byref(out)))
        return out.value

    def ppu_outer_sync(self, replicas) -> None:
        r = np.ascontiguousarray(list(replicas), dtype=np.int32)
        _check(lib().ppu_outer_sync(self._h, _np_ptr(r, C.c_int32), len(r)))

    def ppu_outer_sync_group(self, replicas, group: int, n_groups: int) -> None:
        r = np.ascontiguousarray(list(replicas), dtype=np.int32)
        _check(lib().ppu_outer_sync_group(self._h, _np_ptr(r, C.c_int32), len(r), group, n_groups))

    def ppu_loss(self, replica: int) -> float:
        out = C.c_double()
        _check(lib().ppu_loss(self._h, replica, C.byref(out)))
        return out.value

    def ppu_eval_loss(self, replica: int, tokens_dev) -> float:
        b, s = tokens_dev.shape
        out = C.c_double()
        _check(lib().ppu_eval_loss(self._h, replica, C.c_void_p(tokens_dev.data_ptr()), b, s,
                                   C.byref(out)))
        return out.value

    # ---- accessors ----
    def tensors(self):
        n = C.c_int32()
        _check(lib().ppu_tensor_count(self._h, C.byref(n)))
        recs = []
        for i in range(n.value):
            name = C.create_string_buffer(64)
            off, nd = C.c_int64(), C.c_int32()
            shape = (C.c_int64 * 2)()
            _check(lib().ppu_tensor_info(self._h, i, name, 64, C.byref(off), C.byref(nd), shape))
            recs.append((name.value.decode(), off.value, tuple(shape[:nd.value])))
        return recs

    def ppu_set_params(self, theta: np.ndarray, replica: int = -1) -> None:
        t = np.ascontiguousarray(theta, dtype=np.float32)
        _check(lib().ppu_set_params(self._h, replica, _np_ptr(t, C.c_float), C.c_int64(t.size)))

    def ppu_get_params(self, replica: int = -1) -> np.ndarray:
        out = np.empty(self.param_count, dtype=np.float32)
        _check(lib().ppu_get_params(self._h, replica, _np_ptr(out, C.c_float), C.c_int64(out.size)))
        return out

    def ppu_get_working_bf16(self) -> np.ndarray:
        out = np.empty(self.param_count, dtype=np.uint16)
        _check(lib().ppu_get_working_bf16(self._h, _np_ptr(out, C.c_uint16), C.c_int64(out.size)))
        return out

    def ppu_get_outer_momentum(self) -> np.ndarray:
        out = np.empty(self.param_count, dtype=np.float32)
        _check(lib().ppu_get_outer_momentum(self._h, _np_ptr(out, C.c_float), C.c_int64(out.size)))
        return out

    def ppu_set_outer_momentum(self, buf: np.ndarray) -> None:
        t = np.ascontiguousarray(buf, dtype=np.float32)
        _check(lib().ppu_set_outer_momentum(self._h, _np_ptr(t, C.c_float), C.c_int64(t.size)))

    def ppu_subset_count(self, replica: int) -> int:
        n = C.c_int64()
        _check(lib().ppu_subset_count(self._h, replica, C.byref(n)))
        return n.value

    def ppu_subset_index(self, replica: int) -> np.ndarray:
        out = np.empty(self.ppu_subset_count(replica), dtype=np.int64)
        _check(lib().ppu_subset_index(self._h, replica, _np_ptr(out, C.c_int64), C.c_int64(out.size)))
        return out

    def ppu_get_subset_grads(self, replica: int) -> np.ndarray:
        out = np.empty(self.ppu_subset_count(replica), dtype=np.float32)
        _check(lib().ppu_get_subset_grads(self._h, replica, _np_ptr(out, C.c_float),
                                          C.c_int64(out.size)))
        return out

    def ppu_get_subset_state(self, replica: int):
        n = self.ppu_subset_count(replica)
        m, v = np.empty(n, dtype=np.float32), np.empty(n, dtype=np.float32)
        step = C.c_int32()
        _check(lib().ppu_get_subset_state(self._h, replica, _np_ptr(m, C.c_float),
                                          _np_ptr(v, C.c_float), C.byref(step), C.c_int64(n)))
        return m, v, step.value

    def ppu_set_subset_state(self, replica: int, m, v, step: int) -> None:
        n = self.ppu_subset_count(replica)
        mm = None if m is None else np.ascontiguousarray(m, dtype=np.float32)
        vv = None if v is None else np.ascontiguousarray(v, dtype=np.float32)
        _check(lib().ppu_set_subset_state(self._h, replica,
                                          None if mm is None else _np_ptr(mm, C.c_float),
                                          None if vv is None else _np_ptr(vv, C.c_float),
                                          C.c_int32(step), C.c_int64(n)))

    def ppu_replica_values(self, replica: int):
        """The replica's packed trained values as a torch view into the arena (no copy)."""
        ptr, n = C.c_void_p(), C.c_int64()
        _check(lib().ppu_replica_values(self._h, replica, C.byref(ptr), C.byref(n)))
        off = ptr.value - self.arena.data_ptr()
        return self.arena[off:off + 4 * n.value].view(self.torch.float32)

    def ppu_set_backends(self, gemm: int = 0, attention: int = 0) -> None:
        _check(lib().ppu_set_backends(self._h, gemm, attention))

    def ppu_check_guards(self) -> int:
        n = C.c_int64()
        _check(lib().ppu_check_guards(self._h, C.byref(n)))
        return n.value

    def ppu_set_adam_lr(self, lr: float) -> None:
        _check(lib().ppu_set_adam_lr(self._h, C.c_float(lr)))

    def ppu_sync(self) -> None:
        _check(lib().ppu_sync(self._h))

    def ppu_profile_enable(self, enable: bool) -> None:
        _check(lib().ppu_profile_enable(self._h, int(enable)))

    def ppu_profile_read(self) -> Profile:
        p = Profile()
        _check(lib().ppu_profile_read(self._h, C.byref(p)))
        return p

    def ppu_stats(self) -> Stats:
        s = Stats()
        _check(lib().ppu_stats(self._h, C.byref(s)))
        return s


# ---- single-operator entry points (device tensors from torch) ----
def ppu_gemm(A, a_kmajor, B, b_kmajor, M, N, K, out_f32=False, backend=0):
    """A, B: bf16 CUDA tensors, 2-D row-major as stored.  Returns C [M,N]."""
    import torch
    out = torch.empty((M, N), dtype=torch.float32 if out_f32 else torch.bfloat16, device=A.device)
    st = torch.cuda.current_stream(A.device).cuda_stream
    _check(lib().ppu_gemm(C.c_void_p(A.data_ptr()), C.c_int64(A.stride(0)), int(a_kmajor),
                          C.c_void_p(B.data_ptr()), C.c_int64(B.stride(0)), int(b_kmajor),
                          C.c_void_p(out.data_ptr()), C.c_int64(out.stride(0)), int(out_f32),
                          M, N, K, backend, C.c_void_p(st)))
    return out


def ppu_attention_fwd(qkv, batch, seq, n_head, d_head, backend=0):
    import torch
    d = n_head * d_head
    U = torch.empty((batch * seq, d), dtype=torch.bfloat16, device=qkv.device)
    lse = torch.empty((batch, n_head, seq), dtype=torch.float32, device=qkv.device)
    st = torch.cuda.current_stream(qkv.device).cuda_stream
    _check(lib().ppu_attention_fwd(C.c_void_p(qkv.data_ptr()), C.c_void_p(U.data_ptr()),
                                   C.c_void_p(lse.data_ptr()), batch, seq, n_head, d_head, backend,
                                   C.c_void_p(st)))
    return U, lse


def ppu_attention_bwd(qkv, U, lse, dU, batch, seq, n_head, d_head, backend=0):
    import torch
    dqkv = torch.empty_like(qkv)
    scratch = torch.empty((batch * n_head * seq,), dtype=torch.float32, device=qkv.device)
    st = torch.cuda.current_stream(qkv.device).cuda_stream
    _check(lib().ppu_attention_bwd(C.c_void_p(qkv.data_ptr()), C.c_void_p(U.data_ptr()),
                                   C.c_void_p(lse.data_ptr()), C.c_void_p(dU.data_ptr()),
                                   C.c_void_p(dqkv.data_ptr()), C.c_void_p(scratch.data_ptr()),
                                   batch, seq, n_head, d_head, backend, C.c_void_p(st)))
    return dqkv


STATIC_SCRATCH_FLOATS = 1 << 20


def ppu_attention_bwd_static(qkv, U, lse, dU, batch, seq, n_head, d_head, backend=0):
    """Attention backward without caller scratch: for users who cannot allocate device memory
    at the point of the call.  Limited to batch * n_head * seq <= STATIC_SCRATCH_FLOATS."""
    import torch
    dqkv = torch.empty_like(qkv)
    st = torch.cuda.current_stream(qkv.device).cuda_stream
    _check(lib().ppu_attention_bwd_static(C.c_void_p(qkv.data_ptr()), C.c_void_p(U.data_ptr()),
                                          C.c_void_p(lse.data_ptr()), C.c_void_p(dU.data_ptr()),
                                          C.c_void_p(dqkv.data_ptr()), batch, seq, n_head, d_head,
                                          backend, C.c_void_p(st)))
    return dqkv


# ---- losses of hidden states against the vocabulary ------------------------------------------
# These and the operators below take their operands as values: where one requires a gradient, outputs carry no graph all the
# same (a torch.autograd.Function calls the forward and the backward one).
MAX_TEACHER_ENTRIES = 128
NORM_LAYER, NORM_RMS = 0, 1
_ops = None


def _binding():
    """The compiled binding (_ops.so): checks, outputs, workspaces, streams and the C calls."""
    global _ops
    if _ops is None:
        import torch  # noqa: F401  (its libraries have to be loaded first)
        lib()
        try:
            from . import _ops as m
        except ImportError as e:
            raise PpuError(-6, f"_ops.so does not load ({e}): run paper_2509_22418_b200/build.py") from e
        m.set_error(PpuError)
        _ops = m
    return _ops


def _int32(*values):
    """The values, or an error where one does not fit the C argument (ctypes keeps its low bits)."""
    for v in values:
        if not -2 ** 31 <= v < 2 ** 31:
            raise PpuError(-2, f"{v} is too large")
    return values


def ppu_head_query_bytes(T, d, V, grads=3, chunk_rows=0, k=1) -> int:
    """Bytes of workspace of a head loss; grads: 1 (dX) + 2 (dE); k: entries a row (1 for xent)."""
    n = C.c_size_t(0)
    _check(lib().ppu_head_query_bytes(*_int32(T, d, V, grads, chunk_rows, k), C.byref(n)))
    return n.value


_GRAD_WORDS = {"x": 1, "e": 2, "xe": 3, "ex": 3}


def _grads(grad):
    if isinstance(grad, str):
        if grad not in _GRAD_WORDS:
            raise PpuError(-1, f"grad must be True, False or one of {sorted(_GRAD_WORDS)}, got {grad!r}")
        return _GRAD_WORDS[grad]
    return 3 if grad else 0


def ppu_head_xent(X, E, target, row_weight=None, grad=True, chunk_rows=0, workspace=None, flags=None):
    """Softmax cross entropy of hidden states X [T, d] against the vocabulary matrix E [V, d] (bf16;
    rows may be strided), in chunks of rows: the logits of more rows than a chunk's never exist.  target: int32 [T], negative: the row does not
    count.  row_weight: fp32 [T], or None for the mean over the rows that count.  grad: True, False, or "x" /
    "e" for one gradient only (E frozen, X frozen).  workspace: uint8 tensor of ppu_head_query_bytes, or None.
    Returns (loss, row_loss [T], lse [T], dX, dE).  flags: int32 [8] zeros, which ppu_op_status reads later.  Without flags NOTHING
    is reported: rows whose id is V or more are left out as if they had none, and results are returned, though not
    valid, where a bounded wait inside a kernel ran out."""
    return (_ops or _binding()).head_xent(X, E, target, row_weight, _grads(grad), chunk_rows, workspace, flags)


def ppu_head_distill(X, E, teacher_ids, teacher_logits, temperature=1.0, teacher_lse=None, row_weight=None,
                     grad=True, chunk_rows=0, workspace=None, flags=None):
    """Distillation of X [T, d], E [V, d] (bf16) from a teacher's top logits: teacher_ids int32 [T, k]
    (negative: absent) and teacher_logits fp32 [T, k]; teacher_lse fp32 [T]: the log-sum-exp of all of the
    teacher's logits / temperature, or None for the softmax over the k entries.  Loss and gradients are those of
    sum_j q_j (log q_j - log p_j); multiply row_weight by temperature ** 2 for gradients of the
    same size at every temperature.  The rest, flags among it, as ppu_head_xent."""
    return (_ops or _binding()).head_distill(X, E, teacher_ids, teacher_logits, temperature, teacher_lse, row_weight, _grads(grad), chunk_rows,
                                             workspace, flags)


def ppu_op_status(flags) -> None:
    """Waits for the current stream; raises what a call given `flags` (int32 [8], zeros at first) reported."""
    import torch
    if not (isinstance(flags, torch.Tensor) and flags.is_cuda and flags.dtype == torch.int32 and flags.shape == (8,) and flags.is_contiguous()):
        raise PpuError(-1, "flags must be a contiguous int32 CUDA tensor of 8 values")
    with torch.cuda.device(flags.device):
        _check(lib().ppu_op_status(C.c_void_p(flags.data_ptr()), C.c_void_p(torch.cuda.current_stream(flags.device).cuda_stream)))


# ---- norms before and after a block, with its gate and the residual scale --------------------
_KINDS = {"layer": NORM_LAYER, "rms": NORM_RMS}


def _kind(kind):
    if kind not in _KINDS:
        raise PpuError(-1, f"kind must be one of {sorted(_KINDS)}")
    return _KINDS[kind]


def ppu_norm_gate_fwd(y, r, post_gain, pre_gain, post_shift=None, pre_shift=None, gate=None, gate_rows=0,
                      kind="layer", res_scale=1.0, eps=1e-5, in_place=False):
    """n = N(y) post_gain + post_shift; r_out = res_scale r + gate n; h = N(r_out) pre_gain + pre_shift for
    a block's output y [T, d] (bf16) and the residual stream r [T, d] (fp32); kind "layer" or "rms";
    gate fp32 [ceil(T / gate_rows), d] (gate_rows 0: one row for all).  in_place: r_out is r (refused where r requires a
    gradient and gradients are recorded).
    Returns (r_out fp32, h bf16, stats fp32 [T, 4])."""
    return (_ops or _binding()).norm_gate_fwd(y, r, post_gain, pre_gain, post_shift, pre_shift, gate, gate_rows, _kind(kind), res_scale, eps, in_place)


def ppu_norm_gate_query_bytes(T, d, gate_rows=0) -> int:
    """Bytes of workspace of ppu_norm_gate_bwd (gate_rows 0: no gate)."""
    n = C.c_size_t(0)
    _check(lib().ppu_norm_gate_query_bytes(*_int32(T, d, gate_rows), C.byref(n)))
    return n.value


def ppu_norm_gate_bwd(dh, dr_out, y, r_out, stats, post_gain, pre_gain, post_shift=None, pre_shift=None, gate=None,
                      gate_rows=0, kind="layer", res_scale=1.0, workspace=None):
    """Gradients of ppu_norm_gate_fwd from dh [T, d] (bf16) and dr_out [T, d] (fp32, or None), with the saved
    r_out and stats.  Returns (dy bf16, dr fp32, dpost_gain, dpost_shift, dpre_gain, dpre_shift,
    dgate); those of absent operands are None."""
    return (_ops or _binding()).norm_gate_bwd(dh, dr_out, y, r_out, stats, post_gain, pre_gain, post_shift, pre_shift, gate, gate_rows, _kind(kind),
                                              res_scale, workspace)


# ---- embedding lookup and the table's gradient -----------------------------------------------
_TYPES = {"bf16": 0, "fp32": 1}


def _dtype(word):
    if word not in _TYPES:
        raise PpuError(-1, f"dtype must be one of {sorted(_TYPES)}, got {word!r}")
    return _TYPES[word]


def ppu_embed_fwd(ids, E, scale=1.0, dtype="fp32", flags=None):
    """out[t] = scale E[ids[t]] for ids [T] (int32) and the table E [V, d] (bf16 or fp32; rows may be strided).  Negative ids
    are absent and give a row of zeros; ids of V or more as well, which ppu_op_status reports from flags (int32 [8] zeros; without them
    nothing is reported).  dtype: the result's, "fp32" (the residual stream) or "bf16".  Returns out [T, d]."""
    return (_ops or _binding()).embed_fwd(ids, E, scale, _dtype(dtype), flags)


def ppu_embed_query_bytes(T, d, V) -> int:
    """Bytes of workspace of ppu_embed_bwd."""
    n = C.c_size_t(0)
    _check(lib().ppu_embed_query_bytes(*_int32(T, d, V), C.byref(n)))
    return n.value


def ppu_embed_bwd(ids, dout, V, scale=1.0, dtype=None, add=None, in_place=False, workspace=None, flags=None):
    """The table's gradient, dE[v] = add[v] + scale sum of dout[t] over the tokens with ids[t] = v, from dout [T, d] (bf16 or fp32; rows may be
    strided); sums are fp32 in a fixed order.  dtype: dE's, "bf16" (the default) or "fp32".  add [V, d], of that type: a gradient to form it on top
    of, such as ppu_head_xent's dE of a tied table; in_place: dE is add, whose rows without tokens are not touched (refused where add
    requires a gradient and gradients are recorded).  workspace: uint8 tensor of ppu_embed_query_bytes, or None.  Ids as ppu_embed_fwd.
    Returns dE [V, d]."""
    return (_ops or _binding()).embed_bwd(ids, dout, V, scale, -1 if dtype is None else _dtype(dtype), add, in_place, workspace, flags)


# ---- norms of queries and keys for each head, with the rotation by position ------------------
PAIRS_ADJACENT, PAIRS_HALVES = 0, 1
_PAIRS = {"adjacent": PAIRS_ADJACENT, "halves": PAIRS_HALVES}


def _pairs(pairs):
    if pairs not in _PAIRS:
        raise PpuError(-1, f"pairs must be one of {sorted(_PAIRS)}")
    return _PAIRS[pairs]


def ppu_qk_norm_fwd(qkv, n_q, n_k, n_v, q_gain=None, k_gain=None, positions=None, seq=0, kind="rms", eps=1e-6, rope_base=1e4, inv_freq=None,
                    rot_dim=None, pairs="adjacent", in_place=False):
    """Norms each query and key head of qkv [T, (n_q + n_k + n_v) d_head] (bf16; rows may be strided), multiplies by its gain and rotates it by
    position; value heads are copied.  kind "rms" or "layer"; gains fp32 [d_head], shared by the heads, or [heads, d_head], or None (ones).
    positions int32 [T], or None: t mod seq (seq 0: t).  The first rot_dim columns of a head (None: all) are rotated, "adjacent" pairs (2i, 2i + 1) or
    "halves" (i, i + rot_dim / 2), by position rope_base ** (-2i / rot_dim), or position inv_freq[i] (fp32 [rot_dim / 2]).  in_place: the
    result is qkv (refused where it requires a gradient and gradients are recorded).  With n_q = n_k = n_v the result is what
    ppu_attention_fwd reads."""
    return (_ops or _binding()).qk_norm_fwd(qkv, n_q, n_k, n_v, q_gain, k_gain, positions, seq, _kind(kind), eps, rope_base, inv_freq, rot_dim, _pairs(pairs), in_place)


def ppu_qk_norm_query_bytes(T, n_q, n_k, n_v, d_head, gain_per_head=False) -> int:
    """Bytes of workspace of ppu_qk_norm_bwd."""
    n = C.c_size_t(0)
    _check(lib().ppu_qk_norm_query_bytes(*_int32(T, n_q, n_k, n_v, d_head), int(bool(gain_per_head)), C.byref(n)))
    return n.value


def ppu_qk_norm_bwd(dout, qkv, n_q, n_k, n_v, q_gain=None, k_gain=None, positions=None, seq=0, kind="rms", eps=1e-6, rope_base=1e4, inv_freq=None,
                    rot_dim=None, pairs="adjacent", in_place=False, workspace=None):
    """Gradients of ppu_qk_norm_fwd from dout (shape of qkv, bf16; what ppu_attention_bwd returns) and the qkv it was given (not its
    result).  in_place: dqkv is dout.  Returns (dqkv, dq_gain, dk_gain); those of absent gains are None."""
    return (_ops or _binding()).qk_norm_bwd(qkv, n_q, n_k, n_v, q_gain, k_gain, positions, seq, _kind(kind), eps, rope_base, inv_freq, rot_dim, _pairs(pairs), dout,
                                            in_place, workspace)


# ---- orthogonalised update of matrices --------------------------------------------------------
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


def ppu_orthogonalize_query_bytes(batch, m, n, steps=5) -> int:
    """Bytes of workspace of ppu_orthogonalize."""
    k = C.c_size_t(0)
    _check(lib().ppu_orthogonalize_query_bytes(*_int32(batch, m, n, steps), C.byref(k)))
    return k.value


def ppu_orthogonalize(G, momentum=None, beta=0.95, weight=1.0, nesterov=True, steps=5, coef=NEWTON_SCHULZ, eps=1e-7, scale=1.0, in_place=False, workspace=None,
                      flags=None):
    """The update of matrices G [m, n] or [batch, m, n] (bf16 or fp32; rows and matrices may be strided: one matrix of every layer of a parameter
    vector is a batch, and so are the heads of one projection, whose rows lie beside one another) whose singular values are brought to about one: m' = beta momentum + weight G, u = weight G + beta m' (nesterov) or m'
    (without a momentum u = G); X = u / (|u| + eps); `steps` times A = X X^T, X = a X + (b A + c A A) X; O = scale X.  coef: (a, b, c), or a
    sequence of one such triple for each step.  momentum fp32, G's shape; in_place: m' is written over it (refused where it requires a gradient
    and gradients are recorded).  flags: int32 [8] zeros for ppu_op_status, which reports a bounded wait inside a kernel that ran out; without them the
    result is returned, though not valid.  Returns (O bf16, m' fp32 or None)."""
    flat = coef if coef is NEWTON_SCHULZ else tuple(float(x) for c in coef for x in (c if hasattr(c, "__len__") else (c,)))
    return (_ops or _binding()).orthogonalize(G, momentum, beta, weight, nesterov, flat, steps, eps, scale, in_place, workspace, flags)
