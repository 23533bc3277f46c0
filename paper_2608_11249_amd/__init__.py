"""Python binding of libdlmc.so: DLM-based lossless compression on MI355X.

Argument marshalling only -- every step of the masked-diffusion pass runs in
the library's HIP kernels and host runtime.  The library is built in-tree by
``paper_2608_11249_amd.build.build()``; importing this module does not need a
GPU, but every call that does GPU work fails loudly when the library is
missing or no GPU is present.  torch is used only to hand device buffers and
streams to the stage hooks.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Callable, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdlmc.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "dlmc.h")

FFN = {"gelu": 0, "swiglu": 1}
NORM = {"layernorm": 0, "rmsnorm": 1}
DTYPE = {"f32": 0, "bf16": 1, "bf16-mx4head": 2}  # bf16-mx4head: the LM head in E2M1
MX_FORMAT = {"fp4": 0, "fp8": 1}  # E2M1, E4M3
MAX_ROWS = 2 ** 31 - 1  # of a matrix that a call takes
FLAG_CRC = 1
STAGES = ["embed", "norm", "qkv", "attn", "oproj", "ffn_in", "ffn_out", "head", "entropy",
          "select", "cdf", "reveal", "compact"]
PROFILE_ONE_LAYER = 1 << 31  # DLMC_PROFILE_ONE_LAYER
DEFAULT_STREAM = 1  # DLMC_DEFAULT_STREAM


class LibraryMissing(RuntimeError):
    pass


class DlmcError(RuntimeError):
    def __init__(self, code: int, what: str, detail: str):
        super().__init__(f"dlmc error {code} ({what}): {detail}")
        self.code = code


class ModelConfig(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_layers", ctypes.c_int32),
                ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("d_ffn", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("ffn_kind", ctypes.c_int32), ("norm_kind", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("rope_theta", ctypes.c_float),
                ("norm_eps", ctypes.c_float), ("embed_exp", ctypes.c_int32),
                ("attn_exp", ctypes.c_int32), ("ffn_in_exp", ctypes.c_int32),
                ("ffn_out_exp", ctypes.c_int32), ("head_exp", ctypes.c_int32),
                ("max_chunk", ctypes.c_int32), ("max_batch", ctypes.c_int32)]


class CodecParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("chunk_len", ctypes.c_int32),
                ("tau_bits", ctypes.c_float), ("m_min", ctypes.c_int32),
                ("m_max", ctypes.c_int32), ("cdf_bits", ctypes.c_int32),
                ("coder_bits", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("flags", ctypes.c_int32), ("schedule", ctypes.c_int32),
                ("blocks", ctypes.c_int32), ("u1", ctypes.c_int32),
                ("growth", ctypes.c_double), ("coder", ctypes.c_int32),
                ("context", ctypes.c_int32), ("context_kind", ctypes.c_int32),
                ("rank_compressor", ctypes.c_int32), ("context_seed", ctypes.c_uint64),
                ("rank_level", ctypes.c_int32), ("reserved", ctypes.c_int32)]


SCHEDULE = {"entropy": 0, "uniform": 1, "progressive": 2}
CODER = {"range": 0, "rans": 1, "rank": 2}
RANK_COMPRESSOR = {"none": 0, "zlib": 1, "lzma": 2, "zstd": 3}
CONTEXT = {"contiguous": 0, "random": 1, "attention": 2}


TRACE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64,
                            ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                            ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_uint32),
                            ctypes.c_uint64)

_lib = None
P = ctypes.POINTER
vp, i32, u32, u64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float
i64 = ctypes.c_int64
_SIGS = {
    "dlmc_model_create": (i32, [P(ModelConfig), u64, i32, P(vp)]),
    "dlmc_model_destroy": (None, [vp]),
    "dlmc_set_stream": (i32, [vp, vp]),
    "dlmc_encode_bound": (i32, [vp, P(CodecParams), u64, P(u64)]),
    "dlmc_encode": (i32, [vp, P(CodecParams), vp, u64, vp, u64, P(u64)]),
    "dlmc_decode_size": (i32, [vp, u64, P(u64)]),
    "dlmc_decode": (i32, [vp, vp, u64, i32, vp, u64, P(u64)]),
    "dlmc_encoder_begin": (i32, [vp, P(CodecParams), vp, u64, P(vp)]),
    "dlmc_encoder_step": (i32, [vp, P(i32), P(u64)]),
    "dlmc_encoder_finish": (i32, [vp, vp, u64, P(u64)]),
    "dlmc_session_destroy": (None, [vp]),
    "dlmc_set_trace": (i32, [vp, TRACE_FN, vp]),
    "dlmc_forward_logits": (i32, [vp, vp, i32, i32, vp, vp, vp]),
    "dlmc_entropy_cdf": (i32, [vp, vp, i32, i32, vp, vp, vp, vp]),
    "dlmc_entropy_cdf_noalloc": (i32, [vp, vp, i32, i32, vp, vp, vp, vp]),
    "dlmc_select": (i32, [vp, vp, vp, i32, i32, i32, f32, i32, i32, vp, vp, vp]),
    "dlmc_weight_copy": (i32, [vp, i32, vp, u64]),
    "dlmc_profile_enable": (i32, [vp, ctypes.c_uint32]),
    "dlmc_profile_read": (i32, [vp, i32, P(ctypes.c_double), P(u64), P(ctypes.c_double)]),
    "dlmc_rc_encode": (i32, [vp, vp, u64, i32, i32, vp, u64, P(u64)]),
    "dlmc_rc_decode": (i32, [vp, u64, vp, u64, i32, i32, i32, vp]),
    "dlmc_rans_encode": (i32, [vp, vp, u64, i32, vp, u64, P(u64)]),
    "dlmc_rank_rows": (i32, [vp, vp, i32, vp, vp]),
    "dlmc_context_scores": (i32, [vp, vp, i32, vp]),
    "dlmc_select_rank_rows": (i32, [vp, vp, i32, vp, vp]),
    "dlmc_rans_decode": (i32, [vp, u64, vp, u64, i32, i32, vp]),
    "dlmc_encode_range": (i32, [vp, P(CodecParams), vp, u64, u64, u64, vp, u64, P(u64)]),
    "dlmc_encode_range_bound": (i32, [vp, P(CodecParams), u64, u64, u64, P(u64)]),
    "dlmc_merge": (i32, [P(vp), P(u64), i32, vp, u64, P(u64)]),
    "dlmc_numerics_id": (i32, [P(u64)]),
    "dlmc_test_inject_nonfinite": (i32, [vp, i32]),
    "dlmc_test_head_logits": (i32, [vp, i32]),
    "dlmc_test_gemm_tiles": (i32, [i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_int32),
                                   ctypes.POINTER(ctypes.c_int32)]),
    "dlmc_set_operator_stream": (i32, [vp, vp]),
    "dlmc_mx_bytes": (i32, [i32, i32, i32, P(u64), P(u64)]),
    "dlmc_mx_quantize": (i32, [vp, vp, i32, i64, i32, i32, i32, vp, vp]),
    "dlmc_mx_dequantize": (i32, [vp, vp, vp, i32, i32, i32, vp, i32, i64]),
    "dlmc_add_norm_mx": (i32, [vp, vp, i32, i64, vp, i32, i64, vp, i64, vp, i32, f32, i32, i32, i32,
                               vp, vp]),
    "dlmc_mx_matmul": (i32, [vp, vp, vp, i32, vp, vp, i32, i32, i32, vp, i32, i64]),
    "dlmc_token_scores": (i32, [vp, vp, i32, i64, i32, vp, i32, vp, vp, vp, vp, vp, u64]),
    "dlmc_token_scores_ws": (i32, [vp, i32, i32, P(u64)]),
    "dlmc_test_mx_tiles": (i32, [i32, i32, i32, i32, i32, P(i32)]),
    "dlmc_test_score_launch": (i32, [i32, i32, i32, i32, P(i32), P(i32), P(u64)]),
    "dlmc_status_string": (ctypes.c_char_p, [i32]),
    "dlmc_last_error": (ctypes.c_char_p, []),
}


def lib():
    """The loaded libdlmc.so (raises LibraryMissing if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise LibraryMissing(f"{LIB_PATH} is not built; run paper_2608_11249_amd.build.build()")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def header_symbols():
    """Function names declared in include/dlmc.h."""
    txt = open(HEADER).read()
    return sorted(set(re.findall(r"\b(dlmc_[a-z_0-9]+)\s*\(", txt)) - {"dlmc_trace_fn"})


def _check(st: int):
    if st != 0:
        L = lib()
        raise DlmcError(st, L.dlmc_status_string(st).decode(), L.dlmc_last_error().decode())


def _ptr(a) -> int:
    """Address of a numpy array or a torch tensor."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        return a.ctypes.data
    return a.data_ptr()


def _refuse(why: str):
    raise DlmcError(-1, lib().dlmc_status_string(-1).decode(), why)


class MXMatrix:
    """A matrix [rows, cols] held with block scales (include/dlmc.h gives the
    layout): torch uint8 tensors codes [rows, pitch] and scales [groups, slots, 8]
    on one GPU; fmt "fp4" (E2M1) or "fp8" (E4M3)."""

    __slots__ = ("fmt", "rows", "cols", "device", "_codes", "_scales", "_both", "_ptrs")

    def __init__(self, codes, scales, fmt: str, rows: int, cols: int):
        shapes = MXMatrix._shapes(fmt, rows, cols)
        for t, shape in zip((codes, scales), shapes):
            if not _torch().is_tensor(t) or t.shape != shape or t.element_size() != 1 or not t.is_contiguous():
                _refuse(f"codes or scales do not fit {rows} x {cols} in {fmt}")
        self.fmt, self.rows, self.cols, self.device = fmt, rows, cols, codes.get_device()
        if scales.get_device() != self.device:
            _refuse("codes and scales must be on one GPU")
        self._codes, self._scales, self._both = codes, scales, None
        self._ptrs = codes.data_ptr(), scales.data_ptr()

    @staticmethod
    def _shapes(fmt: str, rows: int, cols: int):
        if fmt not in MX_FORMAT:
            _refuse(f"format must be fp4 or fp8, not {fmt!r}")
        if not 0 <= rows <= MAX_ROWS or not 1 <= cols <= 1 << 24:
            _refuse(f"no matrix of {rows} x {cols} values is held")
        groups = (cols + 255) >> 8
        return (rows, groups << (7 if fmt == "fp4" else 8)), (groups, (rows + 31) & -32, 8)

    @staticmethod
    def like(t, fmt: str, rows: int, cols: int) -> "MXMatrix":
        """One to be filled, on the device of tensor t (both arrays in one allocation:
        an allocation is a fifth of what a short call costs the host)."""
        (n, pitch), (groups, slots, _) = MXMatrix._shapes(fmt, rows, cols)
        q = MXMatrix.__new__(MXMatrix)
        size = (n * pitch + 255) & -256
        both = t.new_empty(size + groups * slots * 8, dtype=_torch().uint8)
        q.fmt, q.rows, q.cols, q.device = fmt, rows, cols, both.get_device()
        q._codes = q._scales = None
        q._both = both
        at = both.data_ptr()
        q._ptrs = at, at + size
        return q

    @staticmethod
    def empty(fmt: str, rows: int, cols: int, device) -> "MXMatrix":
        """One to be filled, on `device`."""
        return MXMatrix.like(_torch().empty(0, device=device), fmt, rows, cols)

    def _part(self, which: int):
        shape = MXMatrix._shapes(self.fmt, self.rows, self.cols)[which]
        n = 1
        for e in shape:
            n *= e
        at = self._ptrs[which] - self._ptrs[0] if n else 0
        return self._both[at: at + n].view(shape)

    def _new(self, dtype, rows: int, cols: int):
        return (self._codes if self._both is None else self._both).new_empty((rows, cols), dtype=dtype)

    @property
    def codes(self):
        if self._codes is None:
            self._codes = self._part(0)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            self._scales = self._part(1)
        return self._scales


_torch_module = _types = _raw = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _type_codes():
    """Element types of the calls on block-scaled values and scores."""
    global _types
    if _types is None:
        _types = {_torch().float32: DTYPE["f32"], _torch().bfloat16: DTYPE["bf16"]}
    return _types


def _raw_stream(device: int) -> int:
    """The handle of torch's current stream on GPU `device` (0: the default one)."""
    global _raw
    if _raw is None:
        torch = _torch()
        # without the Stream object, where torch offers that: 2 us a call
        _raw = getattr(torch._C, "_cuda_getCurrentRawStream",
                       lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw(device)


def model_config(shape, max_chunk: int, max_batch: int) -> ModelConfig:
    return ModelConfig(ctypes.sizeof(ModelConfig), shape.n_layers, shape.d_model, shape.n_heads,
                       shape.d_ffn, shape.vocab, FFN[shape.ffn], NORM[shape.norm], DTYPE[shape.dtype],
                       shape.rope_theta, shape.norm_eps, shape.embed_exp, shape.attn_exp,
                       shape.ffn_in_exp, shape.ffn_out_exp, shape.head_exp, max_chunk, max_batch)


def codec_params(codec, batch: Optional[int] = None, crc: bool = False) -> CodecParams:
    return CodecParams(ctypes.sizeof(CodecParams), codec.chunk_len, codec.tau_bits, codec.m_min,
                       codec.m_max, codec.cdf_bits, codec.coder_bits,
                       codec.batch if batch is None else batch, FLAG_CRC if crc else 0,
                       SCHEDULE[codec.schedule], codec.blocks, codec.u1, float(codec.growth),
                       CODER[codec.coder], codec.context, CONTEXT[codec.context_kind],
                       RANK_COMPRESSOR[codec.rank_compressor], codec.context_seed,
                       codec.rank_level, 0)


class Encoder:
    """Streaming encoder: ``step()`` runs exactly one masked-diffusion pass."""

    def __init__(self, model: "Model", codec, tokens: np.ndarray, batch=None, crc=False):
        self.model = model
        self._tok = np.ascontiguousarray(tokens, dtype=np.int32)
        self._cp = codec_params(codec, batch, crc)
        h = vp()
        model._off_default_stream()
        _check(lib().dlmc_encoder_begin(model.handle, ctypes.byref(self._cp), _ptr(self._tok),
                                        len(self._tok), ctypes.byref(h)))
        self.handle = h
        self.coded = 0
        self.done = False

    def step(self) -> bool:
        done, coded = i32(0), u64(0)
        self.model._off_default_stream()
        _check(lib().dlmc_encoder_step(self.handle, ctypes.byref(done), ctypes.byref(coded)))
        self.coded += coded.value
        self.done = bool(done.value)
        return self.done

    def finish(self) -> bytes:
        bound = self.model.encode_bound(self._cp, len(self._tok))
        out = np.empty(bound, dtype=np.uint8)
        n = u64(0)
        self.model._off_default_stream()
        _check(lib().dlmc_encoder_finish(self.handle, _ptr(out), bound, ctypes.byref(n)))
        return out[: n.value].tobytes()

    def close(self):
        if self.handle:
            lib().dlmc_session_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Model:
    """A masked diffusion LM with seeded random weights on one GPU."""

    def __init__(self, shape, max_chunk: int, max_batch: int = 1, device: int = 0):
        self.shape = shape
        self.cfg = model_config(shape, max_chunk, max_batch)
        h = vp()
        _check(lib().dlmc_model_create(ctypes.byref(self.cfg), shape.seed, device, ctypes.byref(h)))
        self.handle = h
        self.device = device
        self._trace_cb = None
        self._ws_sizes = {}
        self._stream = None  # what set_stream was last given
        self._op_stream = None  # the stream of the calls that return without waiting
        self._hook_stream = False  # whether that was a stage hook's default stream

    def close(self):
        if getattr(self, "handle", None):
            lib().dlmc_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # ---- compression
    def encode_bound(self, cp: CodecParams, n: int) -> int:
        out = u64(0)
        _check(lib().dlmc_encode_bound(self.handle, ctypes.byref(cp), n, ctypes.byref(out)))
        return out.value

    def encode(self, tokens, codec, batch=None, crc=False) -> bytes:
        tok = np.ascontiguousarray(tokens, dtype=np.int32)
        cp = codec_params(codec, batch, crc)
        bound = self.encode_bound(cp, len(tok))
        out = np.empty(max(bound, 1), dtype=np.uint8)
        n = u64(0)
        self._off_default_stream()
        _check(lib().dlmc_encode(self.handle, ctypes.byref(cp), _ptr(tok), len(tok), _ptr(out),
                                 bound, ctypes.byref(n)))
        return out[: n.value].tobytes()

    def encode_range(self, tokens, codec, first_chunk: int, n_chunks: int, batch=None,
                     crc=False) -> bytes:
        """A partial container of chunks [first_chunk, first_chunk + n_chunks)."""
        tok = np.ascontiguousarray(tokens, dtype=np.int32)
        cp = codec_params(codec, batch, crc)
        bound = u64(0)
        _check(lib().dlmc_encode_range_bound(self.handle, ctypes.byref(cp), len(tok), first_chunk,
                                             n_chunks, ctypes.byref(bound)))
        out = np.empty(max(bound.value, 1), dtype=np.uint8)
        n = u64(0)
        self._off_default_stream()
        _check(lib().dlmc_encode_range(self.handle, ctypes.byref(cp), _ptr(tok), len(tok),
                                       first_chunk, n_chunks, _ptr(out), bound.value,
                                       ctypes.byref(n)))
        return out[: n.value].tobytes()

    def inject_nonfinite(self, on: bool):
        """Test hook: every forward writes a NaN into its first logit while on."""
        _check(lib().dlmc_test_inject_nonfinite(self.handle, 1 if on else 0))

    def head_logits_mode(self, mode: int):
        """Test hook: 0 deferred logits chosen by cost, 1 always, 2 never."""
        _check(lib().dlmc_test_head_logits(self.handle, int(mode)))

    def decode(self, data: bytes, batch: int = 0) -> np.ndarray:
        buf = np.frombuffer(data, dtype=np.uint8).copy()
        n = decode_size(data)
        out = np.empty(max(n, 1), dtype=np.int32)
        got = u64(0)
        self._off_default_stream()
        _check(lib().dlmc_decode(self.handle, _ptr(buf), len(buf), batch, _ptr(out), n,
                                 ctypes.byref(got)))
        return out[: got.value]

    def encoder(self, codec, tokens, batch=None, crc=False) -> Encoder:
        return Encoder(self, codec, tokens, batch, crc)

    def set_trace(self, fn: Optional[Callable], coded: bool = False):
        """fn(dir, chunk, pass, positions: list, entropies: list, cdf_hash) or
        None; with coded=True fn(dir, chunk, pass, positions, entropies,
        coded_pairs: list of (start, freq) / (rank, symbol), cdf_hash)."""
        if fn is None:
            self._trace_cb = None
            _check(lib().dlmc_set_trace(self.handle, TRACE_FN(), None))
            return

        def cb(_user, d, chunk, pas, n, pos, ent, iv, hsh):
            p = [pos[i] for i in range(n)]
            e = [ent[i] for i in range(n)]
            if coded:
                fn(int(d), int(chunk), int(pas), p, e,
                   [(int(iv[2 * i]), int(iv[2 * i + 1])) for i in range(n)], int(hsh))
            else:
                fn(int(d), int(chunk), int(pas), p, e, int(hsh))

        self._trace_cb = TRACE_FN(cb)
        _check(lib().dlmc_set_trace(self.handle, self._trace_cb, None))

    def profile(self, on: bool = True, stages: Optional[Sequence[str]] = None,
                one_layer: bool = False):
        """Enable (all stages, or the named ones) / disable per-stage event
        timing; every call resets the counters.  one_layer: time the per-layer
        stages in one layer per forward pass (rotating), not in every layer."""
        if not on:
            mask = 0
        elif stages is None:
            mask = (1 << len(STAGES)) - 1
        else:
            mask = 0
            for name in stages:
                mask |= 1 << STAGES.index(name)
        if on and one_layer:
            mask |= PROFILE_ONE_LAYER
        _check(lib().dlmc_profile_enable(self.handle, mask))

    def profile_read(self) -> dict:
        """{stage: (ms_total, launches, work)} since profiling was enabled."""
        out = {}
        for i, name in enumerate(STAGES):
            ms, n, wk = ctypes.c_double(0), u64(0), ctypes.c_double(0)
            _check(lib().dlmc_profile_read(self.handle, i, ctypes.byref(ms), ctypes.byref(n),
                                           ctypes.byref(wk)))
            out[name] = (ms.value, n.value, wk.value)
        return out

    def set_stream(self, stream_handle: Optional[int]):
        _check(lib().dlmc_set_stream(self.handle, stream_handle))
        self._stream = self._op_stream = stream_handle or None
        self._hook_stream = False

    def _off_default_stream(self):
        """Calls without tensors run on the library's own stream again after a
        stage hook on the default one."""
        if self._hook_stream:
            self.set_stream(None)

    # ---- stage hooks on torch device tensors
    def _on_current_stream(self, device, fn, *args):
        """One call on torch's current stream, so that it follows the work that
        fills its tensors (which live until it returns).  The default stream's
        handle is 0, for which the library would take its own stream."""
        import torch
        stream = torch.cuda.current_stream(device).cuda_stream or DEFAULT_STREAM
        if stream != self._stream or stream != self._op_stream:
            self.set_stream(stream)
            self._hook_stream = stream == DEFAULT_STREAM
        _check(fn(self.handle, *(_ptr(a) if torch.is_tensor(a) else a for a in args)))

    def forward_logits(self, state):
        """state: int32 cuda tensor [B, T].  Returns (logits [n, V], rows [n])."""
        import torch
        B, T = state.shape
        V = self.shape.vocab
        logits = torch.empty(B * T * V, dtype=torch.float32, device=state.device)
        rows = torch.empty(B * T, dtype=torch.int32, device=state.device)
        n = torch.zeros(1, dtype=torch.int32, device=state.device)
        self._on_current_stream(state.device, lib().dlmc_forward_logits, state.contiguous(), B, T,
                                logits, rows, n)
        k = int(n.item())
        return logits[: k * V].view(k, V), rows[:k]

    def entropy_cdf(self, logits, cdf_bits: int, want_cdf: bool = True):
        """Per row of logits [n, V]: (H bits, max, g, cdf) (g, cdf None if not wanted)."""
        import torch
        n, V = logits.shape
        dev = logits.device
        H = torch.empty(n, dtype=torch.float32, device=dev)
        mx = torch.empty(n, dtype=torch.float32, device=dev)
        g = cdf = None
        if want_cdf:
            g = torch.empty(n * V, dtype=torch.int32, device=dev)
            cdf = torch.empty(n * (V + 1), dtype=torch.int32, device=dev)
        self._on_current_stream(dev, lib().dlmc_entropy_cdf, logits.contiguous(), n, cdf_bits, H,
                                mx, g, cdf)
        if want_cdf:
            g, cdf = g.view(n, V), cdf.view(n, V + 1)
        return H, mx, g, cdf


    def entropy_cdf_noalloc(self, logits, cdf_bits: int, want_cdf: bool = True):
        """entropy_cdf through the allocation-free entry point (the library's
        static scratch); the outputs are torch tensors allocated here."""
        import torch
        n, V = logits.shape
        dev = logits.device
        H = torch.empty(n, dtype=torch.float32, device=dev)
        mx = torch.empty(n, dtype=torch.float32, device=dev)
        g = cdf = None
        if want_cdf:
            g = torch.empty(n * V, dtype=torch.int32, device=dev)
            cdf = torch.empty(n * (V + 1), dtype=torch.int32, device=dev)
        self._on_current_stream(dev, lib().dlmc_entropy_cdf_noalloc, logits.contiguous(), n,
                                cdf_bits, H, mx, g, cdf)
        if want_cdf:
            g, cdf = g.view(n, V), cdf.view(n, V + 1)
        return H, mx, g, cdf

    def context_scores(self, tokens) -> np.ndarray:
        """Attention-based context score of every position of one chunk."""
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        out = np.empty(len(t), dtype=np.float32)
        self._off_default_stream()
        _check(lib().dlmc_context_scores(self.handle, _ptr(t), len(t), _ptr(out)))
        return out

    def rank_rows(self, logits, sym):
        """Ranks of sym[i] in device logits row i (torch tensors on cuda)."""
        import torch
        n = int(sym.shape[0])
        out = torch.empty(n, dtype=torch.int32, device=logits.device)
        self._on_current_stream(logits.device, lib().dlmc_rank_rows, logits.contiguous(), n,
                                sym.contiguous(), out)
        return out

    def select_rank_rows(self, logits, rank):
        """The symbol of rank[i] in device logits row i."""
        import torch
        n = int(rank.shape[0])
        out = torch.empty(n, dtype=torch.int32, device=logits.device)
        self._on_current_stream(logits.device, lib().dlmc_select_rank_rows, logits.contiguous(), n,
                                rank.contiguous(), out)
        return out

    def select(self, H, rows, B: int, T: int, tau: float, m_min: int, m_max: int):
        """Schedule on device entropies; returns (sel_pos [B, m_max], sel_row, n_sel [B])."""
        import torch
        dev = H.device
        sel_pos = torch.full((B, m_max), -1, dtype=torch.int32, device=dev)
        sel_row = torch.full((B, m_max), -1, dtype=torch.int32, device=dev)
        n_sel = torch.zeros(B, dtype=torch.int32, device=dev)
        self._on_current_stream(dev, lib().dlmc_select, H.contiguous(), rows.contiguous(),
                                int(rows.numel()), B, T, tau, m_min, m_max, sel_pos, sel_row,
                                n_sel)
        return sel_pos, sel_row, n_sel

    # ---- block-scaled values and token scores (torch device tensors; the calls
    # return without waiting for the GPU, nor for other streams when the current one
    # changes, so what they cost a short launch is the host's time: one pass of checks, no
    # copies, raw pointers.  They compute no gradients: what they compute requires none,
    # whatever the inputs do, and an `out` that does is refused, but under torch.no_grad())
    def _call(self, fn, *args):
        stream = _raw_stream(self.device) or DEFAULT_STREAM
        if stream != self._op_stream:
            _check(lib().dlmc_set_operator_stream(self.handle, stream))
            self._op_stream = stream
        st = fn(self.handle, *args)
        if st:
            _check(st)

    def _here(self, t, what: str):
        if t.get_device() != self.device:
            _refuse(f"{what} must be on the model's GPU (cuda:{self.device}), not on {t.device}")

    def _rows(self, t, what: str, cols: Optional[int] = None):
        """(type code, row distance, pointer) of a 2-d fp32 or bf16 tensor on this
        GPU whose rows are contiguous; `cols` if it has to have that many columns."""
        code = _type_codes().get(getattr(t, "dtype", None))
        if code is None:
            _refuse(f"{what} must be a float32 or bfloat16 tensor")
        if t.dim() != 2:
            _refuse(f"{what} must be 2-d")
        if t.get_device() != self.device:
            self._here(t, what)
        n, c = t.shape
        if n > MAX_ROWS:
            _refuse(f"{what} has more rows than {MAX_ROWS}")
        if cols is not None and c != cols:
            _refuse(f"{what} must have {cols} columns, not {c}")
        ld, step = t.stride()
        if c > 1 and step != 1:
            _refuse(f"{what} must have contiguous rows")
        if n <= 1:
            ld = c
        elif ld < c:
            _refuse(f"{what}: rows overlap")
        return code, ld, t.data_ptr()

    def _out(self, t, cols: int):
        """As _rows, of a tensor that is to be written."""
        if getattr(t, "requires_grad", False) and _torch().is_grad_enabled():
            _refuse("out requires a gradient, and these calls compute none")
        return self._rows(t, "out", cols)

    @staticmethod
    def _wrote(t):
        """Lets autograd see that t has other values (a graph that saved them refuses to
        go on)."""
        _torch().autograd.graph.increment_version(t)

    def _vector(self, t, what: str, n: int, dtype):
        if getattr(t, "dtype", None) != dtype or t.dim() != 1 or t.shape[0] != n:
            _refuse(f"{what} must be a tensor of {n} {dtype} values")
        self._here(t, what)
        return t.contiguous()

    def _held(self, q, what: str):
        """(codes, scales) pointers of an MXMatrix on this GPU."""
        if not isinstance(q, MXMatrix):
            _refuse(f"{what} must be an MXMatrix")
        if q.device != self.device:
            _refuse(f"{what} must be on the model's GPU (cuda:{self.device})")
        return q._ptrs

    @staticmethod
    def _out_type(dtype) -> int:
        code = _type_codes().get(dtype)
        return _refuse(f"output type must be float32 or bfloat16, not {dtype}") if code is None else code

    def mx_quantize(self, x, fmt: str = "fp4") -> MXMatrix:
        """x [rows, cols] (fp32 or bf16) in E2M1 ("fp4") or E4M3 ("fp8") with a
        power-of-two scale for each 32 columns; nothing saturates."""
        code, ld, ptr = self._rows(x, "x")
        rows, cols = x.shape
        q = MXMatrix.like(x, fmt, rows, cols)
        self._call(lib().dlmc_mx_quantize, ptr, code, ld, rows, cols, MX_FORMAT[fmt], *q._ptrs)
        return q

    def mx_dequantize(self, q: MXMatrix, dtype=None):
        """The values that q holds, bf16 (the default: exact) or fp32 [rows, cols]."""
        torch = _torch()
        dtype = torch.bfloat16 if dtype is None else dtype
        code = self._out_type(dtype)
        codes, scales = self._held(q, "q")
        out = q._new(dtype, q.rows, q.cols)
        self._call(lib().dlmc_mx_dequantize, codes, scales, MX_FORMAT[q.fmt], q.rows, q.cols, out.data_ptr(), code,
                   q.cols)
        return out

    def add_norm_mx(self, x, delta=None, gain=None, fmt: str = "fp8", norm: Optional[str] = None,
                    eps: Optional[float] = None, out=None):
        """(r, q): r = x + delta [rows, cols] in x's type (x itself without a delta;
        written to `out`, which may be x or delta, if given) and its norm times gain (fp32)
        as an MXMatrix.  norm ("rmsnorm" or "layernorm") and eps: the model's."""
        code, ld, ptr = self._rows(x, "x")
        rows, cols = x.shape
        kind = NORM.get(self.shape.norm if norm is None else norm)
        if kind is None:
            _refuse(f"norm must be rmsnorm or layernorm, not {norm!r}")
        if not 1 <= cols <= 8192:
            _refuse("a norm takes 1 to 8192 columns")
        dcode = ldd = lds = 0
        dptr = gptr = sptr = None
        if delta is not None:
            dcode, ldd, dptr = self._rows(delta, "delta", cols)
            if delta.shape[0] != rows:
                _refuse(f"delta must have {rows} rows, not {delta.shape[0]}")
        if gain is not None:
            gain = self._vector(gain, "gain", cols, _torch().float32)
            gptr = gain.data_ptr()
        if out is not None:
            r = out
            ocode, lds, sptr = self._out(out, cols)
            if ocode != code or out.shape[0] != rows:
                _refuse("out must have x's shape and type")
        elif delta is None:
            r = x
        else:
            r = x.new_empty((rows, cols))
            lds, sptr = cols, r.data_ptr()
        q = MXMatrix.like(x, fmt, rows, cols)
        self._call(lib().dlmc_add_norm_mx, ptr, code, ld, dptr, dcode, ldd, sptr, lds, gptr, kind,
                   self.shape.norm_eps if eps is None else eps, rows, cols, MX_FORMAT[fmt],
                   *q._ptrs)
        if out is not None:
            self._wrote(out)
        return r, q

    def mx_matmul(self, a: MXMatrix, b: MXMatrix, out_dtype=None, out=None):
        """a b^T [a.rows, b.rows] of a in either format and b in E2M1, as fp32 (the
        default) or bf16, into `out` if given.  Sums are fp32; with a in E4M3 each
        product loses what lies 2^13 below the largest of its block of 32 columns."""
        ac, asc = self._held(a, "a")
        bc, bsc = self._held(b, "b")
        if b.fmt != "fp4":
            _refuse(f"b must be held in fp4, not in {b.fmt}")
        M, N, K = a.rows, b.rows, a.cols
        if K != b.cols:
            _refuse(f"a has {K} columns, b {b.cols}")
        given = out is not None
        if not given:
            dtype = _torch().float32 if out_dtype is None else out_dtype
            code, ldo = self._out_type(dtype), N
            out = a._new(dtype, M, N)
            optr = out.data_ptr()
        else:
            code, ldo, optr = self._out(out, N)
            if out.shape[0] != M or (out_dtype is not None and out.dtype != out_dtype):
                _refuse("out does not have the product's shape and type")
        self._call(lib().dlmc_mx_matmul, ac, asc, MX_FORMAT[a.fmt], bc, bsc, M, N, K, optr, code, ldo)
        if given:
            self._wrote(out)
        return out

    def _scores_ws(self, n: int, top: int) -> int:
        """Bytes of workspace, which go by the sizes alone (asked for once each)."""
        need = self._ws_sizes.get((n, top))
        if need is None:
            size = u64(0)
            _check(lib().dlmc_token_scores_ws(self.handle, n, top, ctypes.byref(size)))
            if len(self._ws_sizes) >= 64:
                self._ws_sizes.clear()
            need = self._ws_sizes[n, top] = size.value
        return need

    def token_scores(self, logits, tokens=None, top: int = 0):
        """Of logits [n, vocab] (fp32 or bf16): (log2 probability of tokens[i] in row
        i (None without tokens), entropy in bits, ids [n, top] of the most probable
        symbols, their log2 probabilities)."""
        torch = _torch()
        V = self.shape.vocab
        code, ld, ptr = self._rows(logits, "logits", V)
        n = logits.shape[0]
        if not 0 <= top <= min(64, V):
            _refuse("top must be in 0..64, at most the vocabulary")
        logp = tptr = lptr = None
        f32t, i32t = torch.float32, torch.int32
        if tokens is not None:
            tokens = self._vector(tokens, "tokens", n, i32t)
            logp = logits.new_empty(n, dtype=f32t)
            tptr, lptr = tokens.data_ptr(), logp.data_ptr()
        H = logits.new_empty(n, dtype=f32t)
        ids = logits.new_empty((n, top), dtype=i32t)
        tlp = logits.new_empty((n, top), dtype=f32t)
        need = self._scores_ws(n, top)
        ws = logits.new_empty(need, dtype=torch.uint8) if need else None
        self._call(lib().dlmc_token_scores, ptr, code, ld, n, tptr, top, lptr, H.data_ptr(), ids.data_ptr(),
                   tlp.data_ptr(), ws.data_ptr() if need else None, need)
        return logp, H, ids, tlp

    def weight(self, tensor_id: int, rows: int, cols: int) -> np.ndarray:
        """A weight tensor in canonical [out, in] layout (uint16 bf16 bits or float32)."""
        dt = np.float32 if self.shape.dtype == "f32" else np.uint16
        out = np.empty((rows, cols), dtype=dt)
        _check(lib().dlmc_weight_copy(self.handle, tensor_id, _ptr(out), out.nbytes))
        return out


GEMM_EPI = {"store": 0, "residual": 1, "qkv": 2, "gelu": 3, "swiglu": 4}


def gemm_tiles(M: int, N: int, K: int, epi: str, d_model: int = 0):
    """(kind, split) the bf16 GEMM chooses (host only): kind "128x128",
    "192x128", "4wave" with columns [0, split) on 256 x 256 tiles, "64x64" or
    "128x64" (split: 1 with the deeper ring) or "128x128deep"."""
    kind, split = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().dlmc_test_gemm_tiles(M, N, K, GEMM_EPI[epi], d_model, ctypes.byref(kind),
                                      ctypes.byref(split)))
    return ("128x128", "192x128", "4wave", "64x64", "128x64", "128x128deep")[kind.value], split.value


MX_TILES = ("32x64", "32x128", "64x64", "64x128", "128x256", "256x256", "128x256deep")


def mx_tiles(fmt: str, M: int, N: int, K: int, live_rows: int = -1) -> str:
    """The tiles that mx_matmul takes of a [M, K] in fmt and b [N, K] (host only), or a
    model's head with so many masked rows of M; "128x256deep": with the whole LDS of
    a CU."""
    kind = i32()
    _check(lib().dlmc_test_mx_tiles(MX_FORMAT[fmt], M, N, K, live_rows, ctypes.byref(kind)))
    return MX_TILES[kind.value]


def score_launches(n_rows: int, vocab: int, top: int):
    """(rows, splits, workspace bytes) of each launch that token_scores makes of
    n_rows rows (host only)."""
    out = []
    while True:
        rows, splits, ws = i32(), i32(), u64()
        _check(lib().dlmc_test_score_launch(n_rows, vocab, top, len(out), ctypes.byref(rows), ctypes.byref(splits),
                                            ctypes.byref(ws)))
        if rows.value == 0:
            return out
        out.append((rows.value, splits.value, ws.value))


def decode_size(data: bytes) -> int:
    buf = np.frombuffer(data, dtype=np.uint8)
    n = u64(0)
    _check(lib().dlmc_decode_size(_ptr(buf) if len(buf) else None, len(buf), ctypes.byref(n)))
    return n.value


def merge(parts: Sequence[bytes]) -> bytes:
    """One complete container from partial containers of the same input."""
    bufs = [np.frombuffer(p, dtype=np.uint8).copy() for p in parts]
    ptrs = (vp * len(bufs))(*[b.ctypes.data if len(b) else None for b in bufs])
    lens = (u64 * len(bufs))(*[len(b) for b in bufs])
    n = u64(0)
    L = lib()
    st = L.dlmc_merge(ptrs, lens, len(bufs), None, 0, ctypes.byref(n))
    if st != -6:
        _check(st)
    out = np.empty(max(n.value, 1), dtype=np.uint8)
    _check(L.dlmc_merge(ptrs, lens, len(bufs), _ptr(out), n.value, ctypes.byref(n)))
    return out[: n.value].tobytes()


def numerics_id() -> int:
    """This build's numerics identity (recorded in every container)."""
    out = u64(0)
    _check(lib().dlmc_numerics_id(ctypes.byref(out)))
    return out.value


def rc_encode(start, freq, cdf_bits: int, coder_bits: int) -> bytes:
    s = np.ascontiguousarray(start, dtype=np.uint32)
    f = np.ascontiguousarray(freq, dtype=np.uint32)
    cap = len(s) * 8 + 64
    out = np.empty(cap, dtype=np.uint8)
    n = u64(0)
    _check(lib().dlmc_rc_encode(_ptr(s), _ptr(f), len(s), cdf_bits, coder_bits, _ptr(out), cap,
                                ctypes.byref(n)))
    return out[: n.value].tobytes()


def rc_decode(data: bytes, cdfs: np.ndarray, cdf_bits: int, coder_bits: int) -> np.ndarray:
    c = np.ascontiguousarray(cdfs, dtype=np.uint32)
    n, V1 = c.shape
    buf = np.frombuffer(data, dtype=np.uint8).copy()
    out = np.empty(max(n, 1), dtype=np.int32)
    _check(lib().dlmc_rc_decode(_ptr(buf), len(buf), _ptr(c), n, V1 - 1, cdf_bits, coder_bits,
                                _ptr(out)))
    return out[:n]


def rans_encode(start, freq, cdf_bits: int) -> bytes:
    s = np.ascontiguousarray(start, dtype=np.uint32)
    f = np.ascontiguousarray(freq, dtype=np.uint32)
    cap = len(s) * 4 + 16
    out = np.empty(cap, dtype=np.uint8)
    n = u64(0)
    _check(lib().dlmc_rans_encode(_ptr(s), _ptr(f), len(s), cdf_bits, _ptr(out), cap,
                                  ctypes.byref(n)))
    return out[: n.value].tobytes()


def rans_decode(data: bytes, cdfs: np.ndarray, cdf_bits: int) -> np.ndarray:
    c = np.ascontiguousarray(cdfs, dtype=np.uint32)
    n, V1 = c.shape
    buf = np.frombuffer(data, dtype=np.uint8).copy()
    out = np.empty(max(n, 1), dtype=np.int32)
    _check(lib().dlmc_rans_decode(_ptr(buf) if len(buf) else None, len(buf), _ptr(c), n, V1 - 1,
                                  cdf_bits, _ptr(out)))
    return out[:n]
