"""Python binding of libfdhvp (include/fdhvp.h): argument marshalling only.

Every computation runs in the HIP library; PyTorch supplies device memory and
the current stream.  Loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libfdhvp.so")

# enums (include/fdhvp.h)
OK, BREAKDOWN = 0, 1
ERR = {-1: "INVALID_ARG", -2: "WORKSPACE", -3: "HIP", -4: "NONFINITE", -5: "STATE", -6: "UNSUPPORTED"}
FAMILY = {"gpt2": 0, "llama": 1, "quad_diag": 2}
DTYPE = {"f32": 0, "bf16": 1}
REORTH = {"none": 0, "full": 1, "window": 2}
TOKENS = {"uniform": 0, "zipf": 1}
VEC = {"rademacher": 0, "gaussian": 1}
REDUCTION = {"mean": 0, "sum": 1}
IGNORE = -100


class FdhError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"fdhvp error {ERR.get(status, status)}: {msg}")
        self.status = status


class ModelConfig(C.Structure):
    _fields_ = [("family", C.c_int32), ("n_layers", C.c_int32), ("d_model", C.c_int32),
                ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_ff", C.c_int32),
                ("vocab", C.c_int32), ("max_seq", C.c_int32), ("dtype", C.c_int32),
                ("norm_eps", C.c_float), ("rope_base", C.c_float), ("reserved", C.c_int32),
                ("quad_n", C.c_int64)]


class QkConfig(C.Structure):
    _fields_ = [("norm", C.c_int32), ("n_axes", C.c_int32), ("sections", C.c_int32 * 4), ("interleaved", C.c_int32),
                ("reserved", C.c_int32)]


class QkGains(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v_q", C.c_void_p), ("v_k", C.c_void_p), ("eps", C.c_double)]


class EmbedTables(C.Structure):
    _fields_ = [("e", C.c_void_p), ("v_e", C.c_void_p), ("p", C.c_void_p), ("v_p", C.c_void_p), ("eps", C.c_double)]


class HeadInputs(C.Structure):
    _fields_ = [("x_m", C.c_void_p), ("x_d", C.c_void_p), ("ldx", C.c_int64), ("w_m", C.c_void_p), ("w_d", C.c_void_p),
                ("targets", C.c_void_p), ("T", C.c_int32), ("piece", C.c_int32), ("reserved", C.c_int32)]


class HeadGrads(C.Structure):
    _fields_ = [("dx_m", C.c_void_p), ("dx_d", C.c_void_p), ("lddx", C.c_int64), ("dw", C.c_void_p), ("scale", C.c_double),
                ("eps", C.c_double), ("dtype", C.c_int32), ("accumulate", C.c_int32)]


class LanczosOpts(C.Structure):
    _fields_ = [("reorth", C.c_int32), ("window", C.c_int32), ("basis_dtype", C.c_int32),
                ("breakdown_tol", C.c_float)]


class Batch(C.Structure):
    _fields_ = [("tokens", C.c_void_p), ("labels", C.c_void_p), ("B", C.c_int32), ("S", C.c_int32)]


class Block(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("offset", C.c_int64), ("numel", C.c_int64),
                ("rows", C.c_int64), ("cols", C.c_int64), ("layer", C.c_int32), ("kind", C.c_int32)]


_lib = None


def lib():
    """The loaded shared library (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_00816_amd.build`")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, u64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_double
    pd, pi = C.POINTER(C.c_double), C.POINTER(C.c_int32)
    sig = {
        "fdh_api_version": (i32, []),
        "fdh_create": (i32, [C.POINTER(ModelConfig), vp, C.POINTER(vp)]),
        "fdh_create_qk": (i32, [C.POINTER(ModelConfig), C.POINTER(QkConfig), vp, C.POINTER(vp)]),
        "fdh_destroy": (None, [vp]),
        "fdh_num_params": (i64, [vp]),
        "fdh_num_blocks": (i32, [vp]),
        "fdh_param_layout": (i32, [vp, C.POINTER(Block), i32, pi]),
        "fdh_workspace_bytes": (i32, [vp, i32, i32, i32, C.POINTER(LanczosOpts), C.POINTER(C.c_size_t)]),
        "fdh_set_workspace": (i32, [vp, vp, C.c_size_t, i32, i32, i32, C.POINTER(LanczosOpts)]),
        "fdh_set_recompute": (i32, [vp, i32]),
        "fdh_set_vocab_piece": (i32, [vp, i32]),
        "fdh_init_params": (i32, [vp, vp, u64]),
        "fdh_make_tokens": (i32, [vp, vp, i32, i32, u64, i32]),
        "fdh_random_vector": (i32, [vp, vp, u64, i32]),
        "fdh_set_quad_diag": (i32, [vp, vp]),
        "fdh_hvp": (i32, [vp, vp, vp, f64, vp, i32, i32, vp]),
        "fdh_last_losses": (i32, [vp, pd, pd]),
        "fdh_bind": (i32, [vp, vp, vp, i32, i32, f64]),
        "fdh_bind_dataset": (i32, [vp, vp, C.POINTER(Batch), i32, f64, i32, C.POINTER(i64)]),
        "fdh_bind_dataset_positions": (i32, [vp, vp, C.POINTER(Batch), C.POINTER(vp), i32, f64, i32, C.POINTER(i64)]),
        "fdh_qk_scratch_bytes": (i32, [vp, i32, i32, C.POINTER(C.c_size_t)]),
        "fdh_qk_forward": (i32, [vp, C.POINTER(QkGains), vp, i32, i32, vp, vp, i64, vp, vp, i64]),
        "fdh_qk_backward": (i32, [vp, C.POINTER(QkGains), vp, i32, i32, vp, vp, i64, vp, vp, i64, vp, vp, i64, vp, vp,
                                  i32, vp, C.c_size_t]),
        "fdh_set_embed_scale": (i32, [vp, f64]),
        "fdh_embed_scratch_bytes": (i32, [vp, i32, i32, C.POINTER(C.c_size_t)]),
        "fdh_embed_forward": (i32, [vp, C.POINTER(EmbedTables), vp, i32, i32, vp, vp, i64]),
        "fdh_embed_backward": (i32, [vp, vp, i32, i32, vp, i64, f64, vp, vp, i32, vp, C.c_size_t]),
        "fdh_head_scratch_bytes": (i32, [vp, i32, i32, i32, C.POINTER(C.c_size_t)]),
        "fdh_head_loss": (i32, [vp, C.POINTER(HeadInputs), vp, vp, vp, C.c_size_t]),
        "fdh_head_grad": (i32, [vp, C.POINTER(HeadInputs), vp, vp, C.POINTER(HeadGrads), vp, C.c_size_t]),
        "fdh_hvp_bound": (i32, [vp, vp, vp]),
        "fdh_set_basis_offload": (i32, [vp, i32, vp, C.c_size_t]),
        "fdh_lanczos": (i32, [vp, i32, u64, C.POINTER(LanczosOpts), pd, pd, pi]),
        "fdh_slq_density": (i32, [vp, i32, i32, u64, C.POINTER(LanczosOpts), pd, pd, pi, pd]),
        "fdh_block_stats": (i32, [vp, vp, vp, pd]),
        "fdh_block_stats_noalloc": (i32, [vp, vp, vp, pd]),
        "fdh_block_diagonal": (i32, [vp, vp, pd]),
        "fdh_cg_solve": (i32, [vp, vp, C.c_double, i32, C.c_double, vp, pd, C.POINTER(C.c_int32)]),
        "fdh_last_error": (C.c_char_p, [vp]),
        "fdh_ritz_diagnostics": (i32, [pd, pd, i32, f64, pd, pd, pd, pi, pi, pi]),
        "fdh_testing_gemm": (i32, [i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, C.c_float, i32, vp]),
        "fdh_testing_gemm_pair": (i32, [i32, i32, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp,
                                        vp, vp, C.c_float, i32, vp]),
        "fdh_testing_gemm_channels": (i32, [i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, C.c_float, vp,
                                            C.c_size_t, vp]),
        "fdh_testing_gemm_epilogue": (i32, [i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, i64, i32, C.c_float, C.c_float,
                                            vp, vp, C.c_float, vp, i32, i32, vp, C.c_size_t, vp]),
        "fdh_testing_gemm_plan": (i32, [i32, i32, i32, i32, i32, C.c_size_t, C.POINTER(i32)]),
        "fdh_testing_qk_split": (i32, [i32, i64, i32, i32, i32, i32, i32, i32, C.POINTER(i64)]),
        "fdh_testing_unfused_attention": (i32, [vp, i32]),
        "fdh_testing_unsplit_wgrad": (i32, [vp, i32]),
        "fdh_testing_head_route": (i32, [vp, i32, i32, i32, pi]),
        "fdh_testing_timing": (i32, [vp, i32]),
        "fdh_testing_timing_read": (i32, [vp, pd]),
        "fdh_testing_copy": (i32, [vp, vp, C.c_size_t, vp]),
        "fdh_testing_layout_digest": (i32, [vp, C.POINTER(C.c_uint64)]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _check_tokens(t):
    import torch
    if t is not None and (t.dtype != torch.int32 or t.dim() != 2 or not t.is_cuda or not t.is_contiguous()):
        raise ValueError("tokens must be a contiguous int32 [B, S] tensor on the device")


def _check_vec(t, n: int, what: str, dtypes=("float32",), optional=False):
    """A parameter-sized device operand: the kernels read or write exactly n
    elements of the given type through its pointer, so anything else (another
    dtype, a short or strided tensor, host memory) is refused here, before any
    launch."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{what} is required")
    if not hasattr(t, "data_ptr") or not hasattr(t, "is_cuda"):
        raise ValueError(f"{what} must be a torch tensor on the device")
    dt = str(t.dtype).replace("torch.", "")
    if dt not in dtypes:
        raise ValueError(f"{what} must have dtype {' or '.join(dtypes)}, not {dt}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be on the device")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if t.numel() != n:
        raise ValueError(f"{what} must have {n} elements, not {t.numel()}")


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _current_stream(dev: int) -> int:
    """The current stream of a device (torch's own shortcut where it has one: the
    stream object costs some 3 us)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(dev) if raw else torch.cuda.current_stream(dev).cuda_stream


def opts(reorth="full", window=0, basis="f32", tol=0.0) -> LanczosOpts:
    return LanczosOpts(REORTH[reorth], int(window), DTYPE[basis], float(tol))


@dataclass
class Entry:
    name: str
    offset: int
    numel: int
    rows: int
    cols: int
    layer: int
    kind: int


class Model:
    """One fdh_ctx: a model (or the quadratic test operator) on the current GPU.

    Llama family: qk_norm norms every query and key head before the rotation;
    rope_sections (rotated pairs per position axis, together head_dim / 2)
    rotates over several axes, rope_interleaved deals the axes' pairs in turn.
    embed_scale: factor of the token embedding (set_embed_scale).
    stream: a hipStream_t (torch's ``stream.cuda_stream``); None is the default
    stream."""

    def __init__(self, family: str, n_layers=0, d_model=0, n_heads=1, n_kv_heads=0, d_ff=0, vocab=0,
                 max_seq=0, dtype="f32", norm_eps=1e-5, rope_base=10000.0, quad_n=0, stream=None, qk_norm=False,
                 rope_sections=None, rope_interleaved=False, embed_scale=1.0):
        self._L = lib()
        self.cfg = ModelConfig(FAMILY[family], n_layers, d_model, n_heads, n_kv_heads or n_heads, d_ff, vocab,
                               max_seq, DTYPE[dtype], norm_eps, rope_base, 0, quad_n)
        self.family, self.dtype = family, dtype
        h = C.c_void_p()
        sec = [] if rope_sections is None else [int(s) for s in rope_sections]
        if len(sec) > 4:
            raise ValueError("rope_sections: at most 4 axes")
        qk = QkConfig(int(bool(qk_norm)), len(sec), (C.c_int32 * 4)(*sec), int(bool(rope_interleaved)), 0)
        st = self._L.fdh_create_qk(C.byref(self.cfg), C.byref(qk), stream if stream is not None else C.c_void_p(0),
                                   C.byref(h))
        if st != OK:
            raise FdhError(st, "fdh_create rejected the configuration")
        self.qk_norm, self.n_axes = bool(qk_norm), max(1, len(sec))
        self._stream = int(getattr(stream, "value", stream) or 0)
        self._qk_dh = d_model // max(1, n_heads)
        self._qk_cols = (n_heads + 2 * (n_kv_heads or n_heads)) * self._qk_dh
        self._h = h
        self._ws = None
        self._keep = []        # tensors the bound operator points to
        self._diag = None      # QUAD_DIAG diagonal the context points to
        self._d, self._vocab, self._max_seq = d_model, vocab, max_seq
        if embed_scale != 1.0:
            self.set_embed_scale(embed_scale)

    @classmethod
    def from_workload(cls, w: dict, stream=None):
        return cls(w["family"], w["n_layers"], w["d_model"], w["n_heads"], w["n_kv_heads"], w["d_ff"],
                   w["vocab"], w["max_seq"], w["dtype"], rope_base=w["rope_base"], stream=stream,
                   qk_norm=w.get("qk_norm", False), rope_sections=w.get("rope_sections"),
                   rope_interleaved=w.get("rope_interleaved", False), embed_scale=w.get("embed_scale", 1.0))

    def close(self):
        if getattr(self, "_h", None):
            self._L.fdh_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _param_dtypes(self):
        return ("float32",) if self.dtype == "f32" else ("bfloat16", "uint16", "int16")

    def _check_params(self, p):
        _check_vec(p, self.num_params, "params", self._param_dtypes())

    def _check_vec(self, t, what, optional=False):
        _check_vec(t, self.num_params, what, optional=optional)

    def _check(self, st: int, what: str) -> int:
        if st < 0:
            msg = self._L.fdh_last_error(self._h)
            raise FdhError(st, f"{what}: {msg.decode() if msg else ''}")
        return st

    # ---- description ----
    @property
    def num_params(self) -> int:
        return int(self._L.fdh_num_params(self._h))

    @property
    def num_blocks(self) -> int:
        return int(self._L.fdh_num_blocks(self._h))

    def layout(self) -> list[Entry]:
        n = C.c_int32()
        self._check(self._L.fdh_param_layout(self._h, None, 0, C.byref(n)), "fdh_param_layout")
        arr = (Block * n.value)()
        self._check(self._L.fdh_param_layout(self._h, arr, n.value, C.byref(n)), "fdh_param_layout")
        return [Entry(b.name.decode(), b.offset, b.numel, b.rows, b.cols, b.layer, b.kind) for b in arr]

    def workspace_bytes(self, B=0, S=0, m=0, o: LanczosOpts | None = None) -> int:
        out = C.c_size_t()
        self._check(self._L.fdh_workspace_bytes(self._h, B, S, m, C.byref(o) if o else None, C.byref(out)),
                    "fdh_workspace_bytes")
        return int(out.value)

    def set_recompute(self, on: bool = True):
        """Activation recomputation for the following workspace_bytes /
        set_workspace: keep only each layer's input pair and rerun the layer's
        forward before its backward (same results, less memory)."""
        self._check(self._L.fdh_set_recompute(self._h, 1 if on else 0), "fdh_set_recompute")

    def set_vocab_piece(self, columns: int):
        """Run the HVP's head `columns` of the vocabulary at a time from the next workspace_bytes /
        set_workspace on, without logits that stay (0: whole logits)."""
        self._check(self._L.fdh_set_vocab_piece(self._h, int(columns)), "fdh_set_vocab_piece")

    def set_embed_scale(self, scale: float):
        """Factor of the token embedding in every following call (1 by default)."""
        self._check(self._L.fdh_set_embed_scale(self._h, float(scale)), "fdh_set_embed_scale")

    # ---- memory ----
    def set_workspace(self, B=0, S=0, m=0, o: LanczosOpts | None = None):
        import torch
        n = self.workspace_bytes(B, S, m, o)
        # detach before the old buffer goes back to torch, so that the context
        # never points at freed memory (also when the new size is refused)
        self._check(self._L.fdh_set_workspace(self._h, None, 0, 0, 0, 0, None), "fdh_set_workspace")
        self._ws = None
        buf = torch.empty(max(n, 256) + 256, dtype=torch.uint8, device="cuda")
        base = buf.data_ptr()
        off = (-base) % 256
        self._ws = buf
        self._check(self._L.fdh_set_workspace(self._h, C.c_void_p(base + off), n, B, S, m,
                                              C.byref(o) if o else None), "fdh_set_workspace")
        return n

    def empty_params(self):
        import torch
        dt = torch.float32 if self.dtype == "f32" else torch.uint16 if hasattr(torch, "uint16") else torch.int16
        if self.dtype == "bf16":
            dt = torch.bfloat16
        return torch.empty(self.num_params, dtype=dt, device="cuda")

    def init_params(self, seed: int):
        p = self.empty_params()
        self._check_params(p)
        self._check(self._L.fdh_init_params(self._h, _ptr(p), seed), "fdh_init_params")
        return p

    def make_tokens(self, B: int, S: int, seed: int, dist="uniform"):
        import torch
        t = torch.empty((B, S), dtype=torch.int32, device="cuda")
        self._check(self._L.fdh_make_tokens(self._h, _ptr(t), B, S, seed, TOKENS[dist]), "fdh_make_tokens")
        return t

    def random_vector(self, seed: int, kind="rademacher", out=None):
        import torch
        v = torch.empty(self.num_params, dtype=torch.float32, device="cuda") if out is None else out
        self._check_vec(v, "out")
        self._check(self._L.fdh_random_vector(self._h, _ptr(v), seed, VEC[kind]), "fdh_random_vector")
        return v

    def set_quad_diag(self, diag):
        self._check_vec(diag, "diag")
        self._diag = diag
        self._check(self._L.fdh_set_quad_diag(self._h, _ptr(diag)), "fdh_set_quad_diag")

    # ---- the hot path ----
    def hvp(self, params, v, eps: float, tokens=None, out=None):
        """Hv (float32 [P]) of the FD-HVP at step eps; enqueued on the context stream."""
        import torch
        if out is None:
            out = torch.empty(self.num_params, dtype=torch.float32, device="cuda")
        self._check_params(params)
        self._check_vec(v, "v")
        self._check_vec(out, "out")
        _check_tokens(tokens)
        B, S = (tokens.shape if tokens is not None else (0, 0))
        self._check(self._L.fdh_hvp(self._h, _ptr(params), _ptr(v), float(eps), _ptr(tokens), B, S, _ptr(out)),
                    "fdh_hvp")
        return out

    def last_losses(self):
        lp, lm = C.c_double(), C.c_double()
        self._check(self._L.fdh_last_losses(self._h, C.byref(lp), C.byref(lm)), "fdh_last_losses")
        return lp.value, lm.value

    def bind(self, params, tokens, eps: float):
        self._check_params(params)
        _check_tokens(tokens)
        B, S = (tokens.shape if tokens is not None else (0, 0))
        self._check(self._L.fdh_bind(self._h, _ptr(params), _ptr(tokens), B, S, float(eps)), "fdh_bind")
        self._keep = [params, tokens]   # (a refused call leaves the operator bound before, and its tensors)

    def bind_dataset(self, params, batches, eps: float, reduction: str = "mean", positions=None) -> int:
        """Bind the token-weighted dataset operator over ``batches``: a list of
        int32 [B, S] token tensors or (tokens, labels) pairs on the device
        (labels aligned with the tokens, -100 = no target).  positions (Llama
        family): one int32 [axes, B, S] tensor or None (0 .. S - 1 on every
        axis) per batch.  Returns the number of kept targets."""
        import torch
        self._check_params(params)
        items = [b if isinstance(b, tuple) else (b, None) for b in batches]
        for tok, lab in items:
            for x in (tok, lab):
                if x is not None and (x.dtype != torch.int32 or x.dim() != 2 or not x.is_cuda or not x.is_contiguous()):
                    raise ValueError("tokens and labels must be contiguous int32 [B, S] tensors on the device")
            if lab is not None and lab.shape != tok.shape:
                raise ValueError("labels must have the shape of their tokens")
        pos = [None] * len(items) if positions is None else list(positions)
        if len(pos) != len(items):
            raise ValueError("positions must have one entry per batch")
        for p, (tok, _) in zip(pos, items):
            if p is not None and (p.dtype != torch.int32 or not p.is_cuda or not p.is_contiguous()
                                  or tuple(p.shape) != (self.n_axes, *tok.shape)):
                raise ValueError(f"positions must be contiguous int32 [{self.n_axes}, B, S] tensors on the device")
        parr = (C.c_void_p * len(items))(*[_ptr(p) for p in pos])
        arr = (Batch * len(items))(*[Batch(_ptr(t), _ptr(l), t.shape[0], t.shape[1]) for t, l in items])
        n = C.c_int64()
        if positions is None:
            st = self._L.fdh_bind_dataset(self._h, _ptr(params), arr, len(items), float(eps), REDUCTION[reduction],
                                          C.byref(n))
        else:
            st = self._L.fdh_bind_dataset_positions(self._h, _ptr(params), arr, parr, len(items), float(eps),
                                                    REDUCTION[reduction], C.byref(n))
        self._check(st, "fdh_bind_dataset")
        self._keep = [params] + [x for it in items for x in it if x is not None] + [p for p in pos if p is not None]
        return int(n.value)

    # ---- the q/k front of a layer ----
    # (these run in a few microseconds on the device, so their checks are kept short)
    def _qk_pair(self, pair, what, dtype, T, dev):
        """Pointers and row stride of a pair of [T, (n_heads + 2 n_kv_heads) head_dim] tensors."""
        m, d = pair
        shape, n = m.shape, self._qk_cols
        if len(shape) != 2 or shape[1] != n or shape[0] != T or d.shape != shape:
            raise ValueError(f"{what} must be two [{T}, {n}] tensors")
        if m.dtype is not dtype or d.dtype is not dtype:
            raise ValueError(f"{what} must have dtype {dtype}")
        (ld, one), (ld_d, one_d) = m.stride(), d.stride()
        if one != 1 or one_d != 1:
            raise ValueError(f"{what}: the elements of a row must be contiguous")
        if T <= 1:
            ld = n
        elif ld != ld_d:
            raise ValueError(f"{what}: both tensors must have the same row stride")
        if m.get_device() != dev or d.get_device() != dev:
            raise ValueError("tensors must lie on the current device")
        return m.data_ptr(), d.data_ptr(), ld

    def _qk_args(self, t, seq, gains, eps, positions):
        """(device, gains, positions pointer, B) of a call whose rows are those of t;
        refuses a current device or stream that is not the call's."""
        import torch
        dev, T = t.get_device(), t.shape[0] if t.dim() else 0
        if dev < 0 or dev != torch.cuda.current_device():
            raise ValueError("tensors must lie on the current device")
        if seq < 1 or T % seq:
            raise ValueError("seq must be positive and divide the number of tokens")
        if _current_stream(dev) != self._stream:
            raise ValueError("the current stream is not the model's: build the model with stream=<the current stream>")
        g = None
        if gains is not None:
            q, k, vq, vk = gains
            for x, what, dt in ((q, "gains", self._qk_dtype), (k, "gains", self._qk_dtype),
                                (vq, "gain directions", torch.float32), (vk, "gain directions", torch.float32)):
                if x is None and dt is torch.float32 and what != "gains":
                    continue
                if x is None or x.dtype is not dt or x.numel() != self._qk_dh or not x.is_contiguous():
                    raise ValueError(f"{what} must be contiguous {dt} tensors of {self._qk_dh} elements")
                if x.get_device() != dev:
                    raise ValueError("tensors must lie on the current device")
            g = C.byref(QkGains(q.data_ptr(), k.data_ptr(), _ptr(vq), _ptr(vk), eps))
        pos = 0
        if positions is not None:
            if positions.dtype is not torch.int32 or positions.numel() != self.n_axes * T or not positions.is_contiguous():
                raise ValueError(f"positions must be a contiguous int32 tensor of {self.n_axes} x tokens elements")
            if positions.get_device() != dev:
                raise ValueError("tensors must lie on the current device")
            pos = positions.data_ptr()
        return dev, g, pos, T // seq

    def _call_device(self, t):
        """The device of a call on caller-owned tensors; refuses a current device or stream
        that is not the call's."""
        import torch
        dev = t.get_device()
        if dev < 0 or dev != torch.cuda.current_device():
            raise ValueError("tensors must lie on the current device")
        if _current_stream(dev) != self._stream:
            raise ValueError("the current stream is not the model's: build the model with stream=<the current stream>")
        return dev

    @staticmethod
    def _rows(t, what, dtype, T, n, dev):
        """Pointer and row stride of a [T, n] tensor with contiguous rows."""
        if t.dim() != 2 or t.shape[0] != T or t.shape[1] != n or t.dtype is not dtype:
            raise ValueError(f"{what} must be a [{T}, {n}] tensor of {dtype}")
        ld, one = t.stride()
        if one != 1 and n > 1:
            raise ValueError(f"{what}: the elements of a row must be contiguous")
        if t.get_device() != dev:
            raise ValueError("tensors must lie on the current device")
        return t.data_ptr(), n if T <= 1 else ld

    def _row_pair(self, pair, what, dtype, T, n, dev):
        """Pointers and the common row stride of a pair of them."""
        m, d = pair
        pm, lm = self._rows(m, what, dtype, T, n, dev)
        pd, ld = self._rows(d, what, dtype, T, n, dev)
        if lm != ld:
            raise ValueError(f"{what}: both tensors must have the same row stride")
        return pm, pd, lm

    @staticmethod
    def _whole(t, what, dtype, n, dev, cols=0):
        """Pointer of a contiguous tensor of n elements; with cols a table whose rows have so many (or
        its elements in one dimension)."""
        if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous {dtype} tensor of {n} elements")
        if cols and t.dim() > 1 and t.shape[-1] != cols:
            raise ValueError(f"{what} must have rows of {cols} elements")
        if t.get_device() != dev:
            raise ValueError("tensors must lie on the current device")
        return t.data_ptr()

    @staticmethod
    def _scratch_arg(t, dev):
        if t is None:
            return 0, 0
        if not t.is_contiguous() or t.get_device() != dev:
            raise ValueError("scratch must be contiguous and lie on the current device")
        return t.data_ptr(), t.numel() * t.element_size()

    @functools.cached_property
    def _qk_dtype(self):
        import torch
        return torch.float32 if self.dtype == "f32" else torch.bfloat16

    def qk_scratch(self, B: int, S: int):
        """A device buffer for qk_backward on B x S tokens (None where it needs none)."""
        import torch
        n = C.c_size_t()
        self._check(self._L.fdh_qk_scratch_bytes(self._h, B, S, C.byref(n)), "fdh_qk_scratch_bytes")
        return torch.empty(n.value, dtype=torch.uint8, device="cuda") if n.value else None

    def qk_forward(self, x, seq: int, gains=None, eps: float = 1.0, positions=None, out=None):
        """Per-head norm (with qk_norm) and rotation of the query and key columns of
        the pair x = (mean, half difference), each [tokens, (n_heads + 2 n_kv_heads)
        head_dim] of the model's dtype in rows of any stride; value columns are
        copied.  tokens = B * seq.  gains = (q, k, v_q, v_k): the gains and their
        directions (or None), taken at q +- eps v_q.  positions: int32 [axes,
        tokens], None for 0 .. seq - 1.  out: a pair to write (x itself for in
        place).  Enqueued on the model's stream, which must be the current one."""
        import torch
        dev, g, pos, B = self._qk_args(x[0], seq, gains, eps, positions)
        T, dt = B * seq, self._qk_dtype
        xm, xd, ldx = self._qk_pair(x, "x", dt, T, dev)
        if out is None:
            out = tuple(torch.empty((T, self._qk_cols), dtype=dt, device=x[0].device) for _ in range(2))
        ym, yd, ldy = self._qk_pair(out, "out", dt, T, dev)
        st = self._L.fdh_qk_forward(self._h, g, pos, B, seq, xm, xd, ldx, ym, yd, ldy)
        if st < 0:
            self._check(st, "fdh_qk_forward")
        return out

    def qk_backward(self, dy, seq: int, x=None, gains=None, eps: float = 1.0, positions=None, out=None, gain_grads=None,
                    accumulate: bool = False, scratch=None):
        """Backward of qk_forward: dx (a pair of the model's dtype) from the float32
        pair dy.  With qk_norm also x (the forward's input) and gains, and the
        result is (dx, (dq, dk)) with the gains' entries of Hv, float32
        [head_dim] (added to gain_grads with accumulate).  scratch: qk_scratch(B,
        seq), made here if None; calls that may overlap on the device need one
        each."""
        import torch
        dev, g, pos, B = self._qk_args(dy[0], seq, gains, eps, positions)
        T, dt = B * seq, self._qk_dtype
        gm, gd, lddy = self._qk_pair(dy, "dy", torch.float32, T, dev)
        if out is None:
            out = tuple(torch.empty((T, self._qk_cols), dtype=dt, device=dy[0].device) for _ in range(2))
        om, od, lddx = self._qk_pair(out, "out", dt, T, dev)
        xm = xd = ldx = 0
        dg = (None, None)
        if self.qk_norm:
            if x is None:
                raise ValueError("a model with qk_norm needs x")
            xm, xd, ldx = self._qk_pair(x, "x", dt, T, dev)
            if gain_grads is None:
                if accumulate:
                    raise ValueError("accumulate needs gain_grads")
                gain_grads = tuple(torch.empty(self._qk_dh, device=dy[0].device) for _ in range(2))
            dg = gain_grads
            for t in dg:
                if t.dtype is not torch.float32 or t.numel() != self._qk_dh or not t.is_contiguous():
                    raise ValueError(f"gain_grads must be contiguous float32 tensors of {self._qk_dh} elements")
            if scratch is None:
                scratch = self.qk_scratch(B, seq)
            elif not scratch.is_contiguous():
                raise ValueError("scratch must be contiguous")
            for t in (*dg, scratch):
                if t is not None and t.get_device() != dev:
                    raise ValueError("tensors must lie on the current device")
        nb = 0 if scratch is None else scratch.numel() * scratch.element_size()
        st = self._L.fdh_qk_backward(self._h, g, pos, B, seq, xm, xd, ldx, gm, gd, lddy, om, od, lddx, _ptr(dg[0]), _ptr(dg[1]),
                                     int(accumulate), _ptr(scratch), nb)
        if st < 0:
            self._check(st, "fdh_qk_backward")
        return (out, gain_grads) if self.qk_norm else out

    # ---- the two ends of the model ----
    def _embed_tokens(self, tokens):
        import torch
        if tokens.dtype is not torch.int32 or tokens.dim() != 2 or not tokens.is_contiguous():
            raise ValueError("tokens must be a contiguous int32 [B, S] tensor on the device")
        dev = self._call_device(tokens)
        B, S = tokens.shape
        return dev, B, S

    def embed_scratch(self, B: int, S: int):
        """A device buffer for embed_backward on B x S tokens (None where it needs none)."""
        import torch
        n = C.c_size_t()
        self._check(self._L.fdh_embed_scratch_bytes(self._h, B, S, C.byref(n)), "fdh_embed_scratch_bytes")
        return torch.empty(n.value, dtype=torch.uint8, device="cuda") if n.value else None

    def embed_forward(self, tokens, table, eps: float = 1.0, positions=None, out=None):
        """The token embedding of int32 [B, S] tokens at both points: the float32 pair (mean,
        half difference) of [B S, d_model] rows embed_scale * e[token] (+ p[position]).
        table = (e, v): [vocab, d_model] of the model's dtype and its float32 direction (or
        None), taken at e +- eps v; positions = (p, v_p) likewise, [>= S, d_model], for the
        GPT-2 family.  out: a pair to write, rows of any stride.  A token outside the
        vocabulary gives a row of NaN.  Enqueued on the model's stream, which must be the
        current one."""
        import torch
        dev, B, S = self._embed_tokens(tokens)
        T, d, dt, f32 = B * S, self._d, self._qk_dtype, torch.float32
        e, ve = table
        pe, pve = self._whole(e, "table", dt, self._vocab * d, dev, d), 0
        if ve is not None:
            pve = self._whole(ve, "the table's direction", f32, self._vocab * d, dev, d)
        pp = pvp = 0
        if positions is not None:
            p, vp = positions
            if p.dim() != 2 or p.shape[0] < S:
                raise ValueError(f"positions must have at least {S} rows")
            pp = self._whole(p, "positions", dt, p.shape[0] * d, dev, d)
            if vp is not None:
                pvp = self._whole(vp, "the positions' direction", f32, p.shape[0] * d, dev, d)
        if out is None:
            out = tuple(torch.empty((T, d), dtype=f32, device=tokens.device) for _ in range(2))
        xm, xd, ldx = self._row_pair(out, "out", f32, T, d, dev)
        st = self._L.fdh_embed_forward(self._h, C.byref(EmbedTables(pe, pve, pp, pvp, eps)), tokens.data_ptr(), B, S, xm, xd, ldx)
        if st < 0:
            self._check(st, "fdh_embed_forward")
        return out

    def embed_backward(self, dx, tokens, eps: float = 1.0, out=None, out_positions=None, accumulate: bool = False, scratch=None):
        """The tables' entries of Hv from dx, the float32 [B S, d_model] half difference of the
        gradient of embed_forward's rows: float32 [vocab, d_model], for the GPT-2 family a
        tuple with [max_seq, d_model] positions.  With accumulate they are added to out (and
        out_positions).  scratch: embed_scratch(B, S), made here if None; calls that may
        overlap on the device need one each."""
        import torch
        dev, B, S = self._embed_tokens(tokens)
        d, f32 = self._d, torch.float32
        pd, ldd = self._rows(dx, "dx", f32, B * S, d, dev)
        gpt2 = self.family == "gpt2"
        if accumulate and (out is None or (gpt2 and out_positions is None)):
            raise ValueError("accumulate needs out (and out_positions)")
        if out is None:
            out = torch.empty((self._vocab, d), dtype=f32, device=tokens.device)
        if gpt2 and out_positions is None:
            out_positions = torch.empty((self._max_seq, d), dtype=f32, device=tokens.device)
        po, pp = self._whole(out, "out", f32, self._vocab * d, dev, d), 0
        if out_positions is not None:
            pp = self._whole(out_positions, "out_positions", f32, self._max_seq * d, dev, d)
        if scratch is None:
            scratch = self.embed_scratch(B, S)
        ps, ns = self._scratch_arg(scratch, dev)
        st = self._L.fdh_embed_backward(self._h, tokens.data_ptr(), B, S, pd, ldd, eps, po, pp, int(accumulate), ps, ns)
        if st < 0:
            self._check(st, "fdh_embed_backward")
        return (out, out_positions) if gpt2 else out

    def head_scratch(self, T: int, piece: int = 0, grads: bool = True):
        """A device buffer for head_grad (or, without grads, head_loss) on T rows (None where
        it needs none)."""
        import torch
        n = C.c_size_t()
        self._check(self._L.fdh_head_scratch_bytes(self._h, T, piece, int(grads), C.byref(n)), "fdh_head_scratch_bytes")
        return torch.empty(n.value, dtype=torch.uint8, device="cuda") if n.value else None

    def _head_inputs(self, x, w, targets, piece):
        import torch
        dev = self._call_device(targets)
        T, d, dt = targets.numel(), self._d, self._qk_dtype
        xm, xd, ldx = self._row_pair(x, "x", dt, T, d, dev)
        wm, wd = (self._whole(t, "w", dt, self._vocab * d, dev, d) for t in w)
        tg = self._whole(targets, "targets", torch.int32, T, dev)
        return dev, T, HeadInputs(xm, xd, ldx, wm, wd, tg, T, piece, 0)

    def _head_loss_out(self, loss, T, dev):
        import torch
        return tuple(self._whole(t, "loss", torch.float32, T, dev) for t in loss)

    def head_loss(self, x, w, targets, piece: int = 0, out=None, scratch=None):
        """Softmax cross-entropy of every row of the pair x ([T, d_model] of the model's dtype, rows
        of any stride) times the pair w ([vocab, d_model]; (theta, eps v) in the model's dtype)
        against targets (int32 [T], -100: none): the float32 pair [T] of its mean and half
        difference over the two points.  The logits are formed `piece` columns of the vocabulary at a
        time (0: chosen) and not kept.  scratch: head_scratch(T, piece, grads=False), made here if
        None.  Enqueued on the model's stream, which must be the current one."""
        import torch
        dev, T, inp = self._head_inputs(x, w, targets, piece)
        if out is None:
            out = tuple(torch.empty(T, dtype=torch.float32, device=targets.device) for _ in range(2))
        lm, ld = self._head_loss_out(out, T, dev)
        if scratch is None:
            scratch = self.head_scratch(T, piece, grads=False)
        ps, ns = self._scratch_arg(scratch, dev)
        st = self._L.fdh_head_loss(self._h, C.byref(inp), lm, ld, ps, ns)
        if st < 0:
            self._check(st, "fdh_head_loss")
        return out

    def head_grad(self, x, w, targets, scale: float = 1.0, eps: float = 1.0, piece: int = 0, loss=None, dx=None, dw=None,
                  accumulate: bool = False, scratch=None):
        """head_loss with the gradients of scale * sum(loss): (loss, dx, dw), dx a pair like x and dw
        [vocab, d_model] the half difference of w's gradient over eps (its entries of Hv).  dx and
        dw are of the model's dtype, or float32 where they are given so; with accumulate dw is added
        to what it holds (float32).  scratch: head_scratch(T, piece)."""
        import torch
        dev, T, inp = self._head_inputs(x, w, targets, piece)
        d, dt, f32 = self._d, self._qk_dtype, torch.float32
        if accumulate and dw is None:
            raise ValueError("accumulate needs dw")
        given = dw if dw is not None else dx[0] if dx is not None else None
        gt = dt if given is None else given.dtype
        if gt is not dt and gt is not f32:
            raise ValueError(f"gradients must have dtype {dt} or {f32}")
        if loss is None:
            loss = tuple(torch.empty(T, dtype=torch.float32, device=targets.device) for _ in range(2))
        if dx is None:
            dx = tuple(torch.empty((T, d), dtype=gt, device=targets.device) for _ in range(2))
        if dw is None:
            dw = torch.empty((self._vocab, d), dtype=gt, device=targets.device)
        lm, ld = self._head_loss_out(loss, T, dev)
        dm, dd, lddx = self._row_pair(dx, "dx", gt, T, d, dev)
        pw = self._whole(dw, "dw", gt, self._vocab * d, dev, d)
        if scratch is None:
            scratch = self.head_scratch(T, piece)
        ps, ns = self._scratch_arg(scratch, dev)
        g = HeadGrads(dm, dd, lddx, pw, scale, eps, DTYPE["f32"] if gt is f32 else self.cfg.dtype, int(accumulate))
        st = self._L.fdh_head_grad(self._h, C.byref(inp), lm, ld, C.byref(g), ps, ns)
        if st < 0:
            self._check(st, "fdh_head_grad")
        return loss, dx, dw

    def hvp_bound(self, v, out=None):
        """H v of the bound operator (float32 [P]); enqueued on the context stream."""
        import torch
        if out is None:
            out = torch.empty(self.num_params, dtype=torch.float32, device="cuda")
        self._check_vec(v, "v")
        self._check_vec(out, "out")
        self._check(self._L.fdh_hvp_bound(self._h, _ptr(v), _ptr(out)), "fdh_hvp_bound")
        return out

    def set_basis_offload(self, device_rows: int, host_rows=None):
        """Keep at most device_rows Lanczos rows on the device and the rest in
        host_rows (a pinned host tensor, e.g. torch.empty(n, dtype=torch.uint8,
        pin_memory=True)); device_rows < 0 undoes it.  Call before set_workspace."""
        self._host_rows = host_rows
        nbytes = 0 if host_rows is None else host_rows.numel() * host_rows.element_size()
        self._check(self._L.fdh_set_basis_offload(self._h, int(device_rows), _ptr(host_rows), nbytes),
                    "fdh_set_basis_offload")

    def lanczos(self, m: int, probe_seed: int, o: LanczosOpts):
        a = np.zeros(m)
        b = np.zeros(m)
        s = C.c_int32()
        st = self._check(self._L.fdh_lanczos(self._h, m, probe_seed, C.byref(o),
                                             a.ctypes.data_as(C.POINTER(C.c_double)),
                                             b.ctypes.data_as(C.POINTER(C.c_double)), C.byref(s)), "fdh_lanczos")
        return a, b, int(s.value), st

    def slq_density(self, probes: int, m: int, seed: int, o: LanczosOpts):
        nodes = np.zeros((probes, m))
        weights = np.zeros((probes, m))
        steps = np.zeros(probes, dtype=np.int32)
        tr = C.c_double()
        st = self._check(self._L.fdh_slq_density(
            self._h, probes, m, seed, C.byref(o), nodes.ctypes.data_as(C.POINTER(C.c_double)),
            weights.ctypes.data_as(C.POINTER(C.c_double)), steps.ctypes.data_as(C.POINTER(C.c_int32)),
            C.byref(tr)), "fdh_slq_density")
        return nodes, weights, steps, tr.value, st

    def cg_solve(self, b, lam: float, max_iters: int, rel_tol: float = 0.0, x=None):
        """CG for (H + lam I) x = b on the bound operator (b: float32 [P] on device).
        Returns (x, residual norms ||r_0|| .. ||r_s||, s, status)."""
        import torch
        self._check_vec(b, "b")
        if x is None:
            x = torch.empty_like(b)
        self._check_vec(x, "x")
        res = np.zeros(max_iters + 1)
        s = C.c_int32()
        st = self._check(self._L.fdh_cg_solve(self._h, _ptr(b), float(lam), int(max_iters), float(rel_tol), _ptr(x),
                                              res.ctypes.data_as(C.POINTER(C.c_double)), C.byref(s)), "fdh_cg_solve")
        return x, res[:int(s.value) + 1], int(s.value), st

    def unfused_attention(self, on: bool):
        """Plan the unfused attention path at the next set_workspace (testing)."""
        self._check(self._L.fdh_testing_unfused_attention(self._h, int(on)), "fdh_testing_unfused_attention")

    def unsplit_wgrad(self, on):
        """Weight-gradient launch form (testing): False/0 default (token slices,
        shared launches), True/1 one launch over all tokens per weight, 2 token
        slices without shared launches."""
        self._check(self._L.fdh_testing_unsplit_wgrad(self._h, int(on)), "fdh_testing_unsplit_wgrad")

    def layout_digest(self) -> int:
        """Digest of the workspace carve in use (testing; host only)."""
        out = C.c_uint64()
        self._check(self._L.fdh_testing_layout_digest(self._h, C.byref(out)), "fdh_testing_layout_digest")
        return int(out.value)

    def timing(self, enable: bool):
        self._check(self._L.fdh_testing_timing(self._h, int(enable)), "fdh_testing_timing")

    def timing_read(self) -> dict:
        out = np.zeros(16)
        self._check(self._L.fdh_testing_timing_read(self._h, out.ctypes.data_as(C.POINTER(C.c_double))),
                    "fdh_testing_timing_read")
        cats = ["gemm", "lanczos", "attention", "c3"]
        return {c: dict(launches=out[4 * i], ms=out[4 * i + 1], flops=out[4 * i + 2], bytes=out[4 * i + 3])
                for i, c in enumerate(cats)}

    def block_diagonal(self, v):
        """Exp I statistics per layer: columns abs diff, relative error, cosine, ||(Hv)^(b)||."""
        self._check_vec(v, "v")
        out = np.zeros((max(self.num_blocks, 0), 4))
        self._check(self._L.fdh_block_diagonal(self._h, _ptr(v), out.ctypes.data_as(C.POINTER(C.c_double))),
                    "fdh_block_diagonal")
        return out

    def block_stats_noalloc(self, a, b):
        """fdh_block_stats without the workspace (fixed device scratch; no allocation)."""
        self._check_vec(a, "a")
        self._check_vec(b, "b")
        out = np.zeros((max(self.num_blocks, 0), 3))
        self._check(self._L.fdh_block_stats_noalloc(self._h, _ptr(a), _ptr(b),
                                                    out.ctypes.data_as(C.POINTER(C.c_double))),
                    "fdh_block_stats_noalloc")
        return out

    def block_stats(self, a, b):
        self._check_vec(a, "a")
        self._check_vec(b, "b")
        out = np.zeros((max(self.num_blocks, 0), 3))
        self._check(self._L.fdh_block_stats(self._h, _ptr(a), _ptr(b), out.ctypes.data_as(C.POINTER(C.c_double))),
                    "fdh_block_stats")
        return out


def ritz_diagnostics(alpha, beta, tol: float = 1e-8):
    """Ritz-value diagnostics of T_s (include/fdhvp.h: fdh_ritz_diagnostics).
    Returns (nodes, weights, resid, copies, spurious, n_ghosts)."""
    a = np.ascontiguousarray(alpha, dtype=np.float64)
    b = np.ascontiguousarray(beta, dtype=np.float64)
    s = a.size
    if b.size < s:
        raise ValueError("beta needs as many entries as alpha")
    nodes, weights, resid = np.zeros(s), np.zeros(s), np.zeros(s)
    copies, spurious, ng = np.zeros(s, np.int32), np.zeros(s, np.int32), C.c_int32()
    dp = lambda x: x.ctypes.data_as(C.POINTER(C.c_double))
    ip = lambda x: x.ctypes.data_as(C.POINTER(C.c_int32))
    st = lib().fdh_ritz_diagnostics(dp(a), dp(b), s, float(tol), dp(nodes), dp(weights), dp(resid), ip(copies),
                                    ip(spurious), C.byref(ng))
    if st != OK:
        raise FdhError(st, "fdh_ritz_diagnostics")
    return nodes, weights, resid, copies, spurious.astype(bool), int(ng.value)


def testing_copy(dst, src, nbytes: int):
    st = lib().fdh_testing_copy(_ptr(dst), _ptr(src), int(nbytes), _stream())
    if st != OK:
        raise FdhError(st, "fdh_testing_copy")


def testing_gemm(dtype: str, M, N, K, batch, a_kmajor, b_kmajor, A, B, A2, B2, Cout, causal=0, alpha=1.0, tile=0):
    st = lib().fdh_testing_gemm(DTYPE[dtype], M, N, K, batch, int(a_kmajor), int(b_kmajor), _ptr(A), _ptr(B),
                                _ptr(A2), _ptr(B2), _ptr(Cout), causal, float(alpha), int(tile), _stream())
    if st != OK:
        raise FdhError(st, "fdh_testing_gemm")


def testing_gemm_channels(dtype: str, M, N, K, batch, a_kmajor, b_kmajor, A, B, A2, B2, C2, C1, alpha=1.0, scratch=None):
    """C2 = alpha (A B^T + A2 B2^T) and C1 = alpha A B^T (None: not formed) as an HVP launches them (testing)."""
    st = lib().fdh_testing_gemm_channels(DTYPE[dtype], M, N, K, batch, int(a_kmajor), int(b_kmajor), _ptr(A), _ptr(B),
                                         _ptr(A2), _ptr(B2), _ptr(C2), _ptr(C1), float(alpha), _ptr(scratch),
                                         0 if scratch is None else scratch.numel() * scratch.element_size(), _stream())
    if st != OK:
        raise FdhError(st, "fdh_testing_gemm_channels")


def testing_gemm_epilogue(dtype: str, M, N, K, batch, a_kmajor, b_kmajor, A, B, A2, B2, out, ldc=None, alpha=1.0, beta=0.0,
                          bias_theta=None, bias_v=None, bias_v_scale=1.0, resid=None, causal=0, tile=0, scratch=None):
    """One product with the whole epilogue (testing); out float32 or of the operand type, A2/B2 may be None."""
    import torch
    st = lib().fdh_testing_gemm_epilogue(DTYPE[dtype], M, N, K, batch, int(a_kmajor), int(b_kmajor), _ptr(A), _ptr(B),
                                         _ptr(A2), _ptr(B2), _ptr(out), N if ldc is None else ldc,
                                         int(out.dtype != torch.float32), float(alpha), float(beta), _ptr(bias_theta),
                                         _ptr(bias_v), float(bias_v_scale), _ptr(resid), int(causal), int(tile), _ptr(scratch),
                                         0 if scratch is None else scratch.numel() * scratch.element_size(),
                                         _stream())
    if st != OK:
        raise FdhError(st, "fdh_testing_gemm_epilogue")


def testing_gemm_plan(dtype: str, M, N, K, batch=1, scratch_bytes=0):
    """(tile width, slices of 32 k per part, parts of the two-pair and the one-pair product) of a launch (testing)."""
    out = (C.c_int32 * 4)()
    st = lib().fdh_testing_gemm_plan(DTYPE[dtype], M, N, K, batch, scratch_bytes, out)
    if st != OK:
        raise FdhError(st, "fdh_testing_gemm_plan")
    return tuple(out)


def testing_gemm_pair(M0, N0, K0, M1, N1, K1, a_kmajor, b_kmajor, P0, P1, alpha=1.0, tile=6, batch0=1, batch1=1):
    """Two bf16 products in one launch (testing); P_q = (A, B, A2, B2, C), A2/B2 may be None."""
    import torch
    A0, B0, A20, B20, C0 = P0
    A1, B1, A21, B21, C1 = P1
    for (M, N, K, z, (A, B, A2, B2, Cq)) in ((M0, N0, K0, batch0, P0), (M1, N1, K1, batch1, P1)):
        for t, n, dt in ((A, z * M * K, torch.bfloat16), (B, z * N * K, torch.bfloat16), (A2, z * M * K, torch.bfloat16),
                         (B2, z * N * K, torch.bfloat16), (Cq, z * M * N, torch.float32)):
            if t is not None and (not t.is_cuda or not t.is_contiguous() or t.dtype != dt or t.numel() != n):
                raise ValueError("testing_gemm_pair: operand of the wrong device, layout, type or size")
    st = lib().fdh_testing_gemm_pair(M0, N0, K0, int(batch0), M1, N1, K1, int(batch1), int(a_kmajor), int(b_kmajor),
                                     _ptr(A0), _ptr(B0),
                                     _ptr(A20), _ptr(B20), _ptr(C0), _ptr(A1), _ptr(B1), _ptr(A21), _ptr(B21),
                                     _ptr(C1), float(alpha), int(tile), _stream())
    if st != OK:
        raise FdhError(st, "fdh_testing_gemm_pair")
