"""Python binding of libpsc.so (include/psc.h): argument marshalling only.

Every step of the mask path runs in the library's HIP kernels; torch is used
for device memory and streams.  There is no fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpsc.so")

PSC_F32, PSC_BF16 = 0, 1
FORM_F32, FORM_BF16, FORM_I8, FORM_MX4 = range(4)
ADV_OK, ADV_REJECTED, ADV_EOS, ADV_OVERFLOW, ADV_BAD_INPUT, ADV_SKIPPED = range(6)
_STATUS = {0: "PSC_OK", -1: "PSC_E_INVALID_ARG", -2: "PSC_E_GRAMMAR", -3: "PSC_E_NOT_LALR1", -4: "PSC_E_OOM",
           -5: "PSC_E_DEVICE", -6: "PSC_E_NOT_BOUND", -7: "PSC_E_LIMIT", -8: "PSC_E_IO", -9: "PSC_E_FORMAT",
           -10: "PSC_E_NOT_VIABLE"}

EXPORTED = ["psc_build", "psc_info", "psc_device_bytes", "psc_bind_device", "psc_compute_masks",
            "psc_apply_mask", "psc_compute_and_apply", "psc_state_reset", "psc_advance",
            "psc_compute_masks_dense", "psc_compute_and_apply_dense", "psc_compute_and_argmax",
            "psc_compute_and_argmax_dense", "psc_compute_classes", "psc_compute_classes_dense", "psc_decode_step",
            "psc_save", "psc_load", "psc_device_error_count", "psc_classify_host", "psc_class_mask_host",
            "psc_host_state", "psc_free", "psc_last_error", "psc_device_bytes_ex", "psc_bind_device_ex",
            "psc_compute_masks_n", "psc_compute_classes_n", "psc_compute_and_apply_n", "psc_compute_and_argmax_n",
            "psc_predictor_fill", "psc_predictor_updates", "psc_timeline_records", "psc_compute_and_apply_timeline",
            "psc_set_options", "psc_compute_and_argmax_noalloc", "psc_grammar_compile", "psc_grammar_view",
            "psc_grammar_symbol_name", "psc_grammar_free", "psc_build_from_text", "psc_quantize_rows",
            "psc_head_workspace", "psc_head_logits", "psc_head_logits_quantized", "psc_quantize_mx", "psc_lookup_rows",
            "psc_add_rms_norm", "psc_head_mx_workspace", "psc_head_logits_mx", "psc_penalize", "psc_append_tokens", "psc_sample_workspace",
            "psc_sample"]

BIND_FLAT, BIND_SLICED = 1, 2
OPT_SPECULATE = 1
_LAYOUTS = {None: 0, "default": 0, "flat": BIND_FLAT, "sliced": BIND_SLICED}


class PscError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


# Argument checks (not asserts, so that python -O keeps them): the library
# trusts the sizes it is given, so a tensor of the wrong shape, dtype or
# device must never reach it.  (The lengths of ragged stacks live on the
# device: the calls pass stacks.numel() to the *_n entry points, which
# reject a sequence whose stack would reach past it.)
def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(f"psc: expected {what}")


_T = {}   # torch types, looked up once


def _torch_types():
    if not _T:
        import torch
        raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        _T.update(tensor=torch.Tensor, i32=torch.int32,
                  codes={torch.float32: PSC_F32, torch.bfloat16: PSC_BF16},
                  stream=(lambda: raw(device())) if raw and device
                  else lambda: torch.cuda.current_stream().cuda_stream,
                  f32=torch.float32, bf16=torch.bfloat16, i8=torch.int8, u8=torch.uint8, empty=torch.empty,
                  device=device or torch.cuda.current_device)
    return _T


def _i32(t, name: str, dev: int, numel: int | None = None, shape: tuple | None = None):
    """t as a contiguous int32 tensor on device index `dev` (get_device(): -1
    for host memory), with numel elements or the given shape."""
    T = _T or _torch_types()
    # one cheap test on the common path; the message is built only on failure
    if (type(t) is T["tensor"] and t.dtype is T["i32"] and t.get_device() == dev and t.is_contiguous()
            and (numel is None or t.numel() == numel) and (shape is None or t.shape == shape)):
        return t
    _require(isinstance(t, T["tensor"]) and t.dtype is T["i32"] and t.is_contiguous(),
             f"{name} to be a contiguous int32 tensor")
    _require(t.get_device() == dev, f"{name} on device {dev} (the bound device), not {t.get_device()}")
    _require(numel is None or t.numel() == numel, f"{name} to hold {numel} elements, not {t.numel()}")
    _require(shape is None or tuple(t.shape) == tuple(shape),
             f"{name} of shape {shape and tuple(shape)}, not {tuple(t.shape)}")
    return t


def _logits(t, dev: int, B: int, V: int) -> int:
    """The dtype code of contiguous logits [B, V] on device index `dev`."""
    T = _T or _torch_types()
    code = T["codes"].get(getattr(t, "dtype", None))
    if (code is not None and type(t) is T["tensor"] and t.get_device() == dev and t.is_contiguous()
            and t.shape == (B, V)):
        return code
    _require(isinstance(t, T["tensor"]) and t.is_contiguous() and tuple(t.shape) == (B, V),
             f"logits to be a contiguous tensor of shape ({B}, {V})")
    _require(t.get_device() == dev, f"logits on device {dev} (the bound device), not {t.get_device()}")
    _require(code is not None, f"float32 or bfloat16 logits, not {t.dtype}")
    return code


def _step_args(dev: int, stacks, lens, qs, logits=None, V: int = 0, out=None, out_cols: int = 0):
    """The checks of one mask-step call in one test on the common path:
    ragged states, optional logits [B, V], optional int32 out ([B, out_cols],
    or [B] when out_cols is 0).  Returns (B, logits dtype code or None)."""
    T = _T or _torch_types()
    i32 = T["i32"]
    try:
        B = lens.numel()
        code = T["codes"].get(logits.dtype) if logits is not None else None
        ok = (lens.dtype is i32 and lens.get_device() == dev and lens.is_contiguous()
              and qs.dtype is i32 and qs.get_device() == dev and qs.is_contiguous() and qs.numel() == B
              and stacks.dtype is i32 and stacks.get_device() == dev and stacks.is_contiguous()
              and (logits is None or (code is not None and logits.get_device() == dev and logits.is_contiguous()
                                      and logits.shape == (B, V)))
              and (out is None or (out.dtype is i32 and out.get_device() == dev and out.is_contiguous()
                                   and out.shape == ((B, out_cols) if out_cols else (B,)))))
    except AttributeError:
        ok = False
    if ok:
        return B, code
    # the slow path names what is wrong
    B = int(_i32(lens, "stack_lens", dev).numel())
    _i32(qs, "lexer_states", dev, numel=B)
    _i32(stacks, "stacks", dev)
    code = _logits(logits, dev, B, V) if logits is not None else None
    if out is not None:
        _i32(out, "out", dev, shape=(B, out_cols) if out_cols else (B,))
    return B, code


class _Grammar(C.Structure):
    _fields_ = [
        ("n_lex_states", C.c_int32), ("lex_next", C.c_void_p), ("lex_accept", C.c_void_p),
        ("n_terminals", C.c_int32), ("terminal_ignored", C.c_void_p), ("end_terminal", C.c_int32),
        ("n_lr_states", C.c_int32), ("n_nonterminals", C.c_int32), ("action", C.c_void_p),
        ("goto_table", C.c_void_p), ("n_productions", C.c_int32), ("prod_lhs", C.c_void_p),
        ("prod_len", C.c_void_p),
    ]


class _Vocab(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("bytes", C.c_void_p), ("offsets", C.c_void_p),
                ("eos_id", C.c_int32)]


class Info(C.Structure):
    _fields_ = [
        ("vocab_size", C.c_int32), ("mask_words", C.c_int32), ("mask_stride_words", C.c_int32),
        ("n_lex_states", C.c_int32), ("n_lr_states", C.c_int32), ("n_classes", C.c_int32),
        ("dfa_states_built", C.c_int64), ("dfa_states", C.c_int32), ("dfa_rows", C.c_int32),
        ("dense_rows", C.c_int32), ("max_sparse_edges", C.c_int32), ("table_bytes", C.c_int64),
        ("mask_table_bytes", C.c_int64), ("device_bytes", C.c_int64), ("build_seconds", C.c_double),
        ("chain_states", C.c_int32), ("chains", C.c_int32), ("mask_slices_unique", C.c_int32),
        ("bound_mask_layout", C.c_int32), ("sliced_mask_bytes", C.c_int64),
        ("skip_edges", C.c_int64),
    ]

    def as_dict(self) -> dict:
        return {k: getattr(self, k) for k, _ in self._fields_}


class _Penalties(C.Structure):
    _fields_ = [("history", C.c_void_p), ("lens", C.c_void_p), ("prompt_lens", C.c_void_p), ("cap", C.c_int32),
                ("n_bias", C.c_int32), ("repetition", C.c_void_p), ("presence", C.c_void_p),
                ("frequency", C.c_void_p), ("bias_ids", C.c_void_p), ("bias_values", C.c_void_p)]


class _Sampling(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p),
                ("noise", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """Load libpsc.so; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run __graft_entry__.build() "
                              "(or python paper_2608_03065_amd/build.py) first")
        L = C.CDLL(LIB_PATH)
        P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
        L.psc_build.argtypes = [P, P, C.POINTER(P)]
        L.psc_info.argtypes = [P, P]
        L.psc_device_bytes.argtypes = [P]
        L.psc_device_bytes.restype = C.c_size_t
        L.psc_bind_device.argtypes = [P, P, C.c_size_t, P]
        L.psc_compute_masks.argtypes = [P, P, P, P, I32, P, P]
        L.psc_apply_mask.argtypes = [P, C.c_int, P, I32, I32, P]
        L.psc_compute_and_apply.argtypes = [P, P, P, P, I32, P, P, C.c_int, I32, P]
        L.psc_compute_and_argmax.argtypes = [P, P, P, P, I32, P, C.c_int, I32, P, P]
        L.psc_compute_and_argmax_dense.argtypes = [P, P, I32, P, P, I32, P, C.c_int, I32, P, P]
        L.psc_compute_classes.argtypes = [P, P, P, P, I32, P, P]
        L.psc_compute_classes_dense.argtypes = [P, P, I32, P, P, I32, P, P]
        L.psc_decode_step.argtypes = [P, P, P, P, P, P, P, I32, I32, P, P, P, P, C.c_int, I32, P]
        L.psc_save.argtypes = [P, C.c_char_p]
        L.psc_load.argtypes = [C.c_char_p, C.POINTER(P)]
        L.psc_state_reset.argtypes = [P, P, I32, P, P, I32, P]
        L.psc_advance.argtypes = [P, P, I32, P, P, I32, P, P, P]
        L.psc_compute_masks_dense.argtypes = [P, P, I32, P, P, I32, P, P]
        L.psc_compute_and_apply_dense.argtypes = [P, P, I32, P, P, I32, P, P, C.c_int, I32, P]
        L.psc_device_error_count.argtypes = [P, P, I32, P]
        L.psc_classify_host.argtypes = [P, P, P, P, I32, P]
        L.psc_class_mask_host.argtypes = [P, I32, P]
        L.psc_host_state.argtypes = [P, C.c_char_p, C.c_size_t, P, P, I32, P]
        L.psc_device_bytes_ex.argtypes = [P, C.c_uint32]
        L.psc_device_bytes_ex.restype = C.c_size_t
        L.psc_bind_device_ex.argtypes = [P, P, C.c_size_t, C.c_uint32, P]
        L.psc_compute_masks_n.argtypes = [P, P, I64, P, P, I32, P, P]
        L.psc_compute_classes_n.argtypes = [P, P, I64, P, P, I32, P, P]
        L.psc_compute_and_apply_n.argtypes = [P, P, I64, P, P, I32, P, P, C.c_int, I32, P]
        L.psc_compute_and_argmax_n.argtypes = [P, P, I64, P, P, I32, P, C.c_int, I32, P, P]
        L.psc_compute_and_argmax_noalloc.argtypes = [P, P, I64, P, P, I32, P, C.c_int, I32, P, P]
        L.psc_grammar_compile.argtypes = [C.c_char_p, C.c_size_t, C.POINTER(P)]
        L.psc_grammar_view.argtypes = [P, P]
        L.psc_grammar_symbol_name.argtypes = [P, I32, I32]
        L.psc_grammar_symbol_name.restype = C.c_char_p
        L.psc_grammar_free.argtypes = [P]
        L.psc_grammar_free.restype = None
        L.psc_build_from_text.argtypes = [C.c_char_p, C.c_size_t, P, C.POINTER(P)]
        L.psc_predictor_fill.argtypes = [P, I32, P]
        L.psc_set_options.argtypes = [P, C.c_uint32]
        L.psc_predictor_updates.argtypes = [P, P, I32, P]
        L.psc_timeline_records.argtypes = [P, I32, C.c_int]
        L.psc_timeline_records.restype = I64
        L.psc_compute_and_apply_timeline.argtypes = [P, P, I64, P, P, I32, P, P, C.c_int, I32, P, I64, P]
        L.psc_quantize_rows.argtypes = [P, C.c_int, I64, I64, I32, P, I64, P, P]
        L.psc_head_workspace.argtypes = [I32, I32, I32]
        L.psc_head_workspace.restype = C.c_size_t
        L.psc_head_logits.argtypes = [P, C.c_int, I64, I32, I32, P, I64, P, I32, P, P, P, C.c_int, I64, P,
                                      C.c_size_t, P]
        L.psc_head_logits_quantized.argtypes = [P, I64, P, I32, I32, P, I64, P, I32, P, P, P, C.c_int, I64, P, C.c_size_t, P]
        L.psc_quantize_mx.argtypes = [P, C.c_int, I64, I64, I32, P, I64, P, I64, P]
        L.psc_lookup_rows.argtypes = [C.c_int, P, I64, P, I64, I64, I32, P, I64, P, C.c_int, I64, P]
        L.psc_add_rms_norm.argtypes = [P, C.c_int, I64, P, C.c_int, I64, I64, I32, P, C.c_float, C.c_int, P, I64, P, I64, P]
        L.psc_head_mx_workspace.argtypes = [I32, I32, I32, C.c_int]
        L.psc_head_mx_workspace.restype = C.c_size_t
        L.psc_head_logits_mx.argtypes = [P, C.c_int, I64, P, I64, I32, I32, C.c_int, P, I64, P, I64, I32, P, P, P, C.c_int,
                                         I64, P, C.c_size_t, P]
        L.psc_penalize.argtypes = [P, C.c_int, I64, I32, I32, P, P, P]
        L.psc_append_tokens.argtypes = [P, I32, P, I32, P, P, P]
        L.psc_sample_workspace.argtypes = [I32, I32, C.c_int]
        L.psc_sample_workspace.restype = C.c_size_t
        L.psc_sample.argtypes = [P, C.c_int, I64, I32, I32, P, P, I32, P, P, P, P, P, C.c_size_t, P]
        L.psc_free.argtypes = [P]
        L.psc_free.restype = None
        L.psc_last_error.restype = C.c_char_p
        for name in ("psc_build", "psc_info", "psc_bind_device", "psc_compute_masks", "psc_apply_mask",
                     "psc_compute_and_apply", "psc_state_reset", "psc_advance", "psc_compute_masks_dense",
                     "psc_compute_and_apply_dense", "psc_compute_and_argmax", "psc_compute_and_argmax_dense",
                     "psc_compute_classes", "psc_compute_classes_dense", "psc_decode_step", "psc_save", "psc_load", "psc_device_error_count",
                     "psc_classify_host", "psc_class_mask_host", "psc_host_state", "psc_bind_device_ex",
                     "psc_compute_masks_n", "psc_compute_classes_n", "psc_compute_and_apply_n",
                     "psc_compute_and_argmax_n", "psc_predictor_fill", "psc_predictor_updates",
                     "psc_compute_and_apply_timeline", "psc_set_options", "psc_compute_and_argmax_noalloc",
                     "psc_grammar_compile", "psc_grammar_view", "psc_build_from_text", "psc_quantize_rows",
                     "psc_head_logits", "psc_head_logits_quantized", "psc_quantize_mx", "psc_lookup_rows", "psc_add_rms_norm",
                     "psc_head_logits_mx", "psc_penalize", "psc_append_tokens", "psc_sample"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise PscError(status, lib().psc_last_error().decode(errors="replace"))


def _stream_ptr(stream):
    """The hipStream_t of `stream`, or of the current device's current stream.
    The latter is asked for by its handle, 0.2 us: building the Stream object
    for it took 3.2 of a call's 9.0 us, and a call of few sequences takes the
    GPU 5 to 6."""
    if stream is not None:
        return stream.cuda_stream
    return (_T or _torch_types())["stream"]()


def pack_states(states, device=None):
    """[(q, stack bottom->top), ...] -> (stacks int32 [sum len], lens int32 [B], qs int32 [B]),
    numpy on the host, or torch tensors on `device` when given."""
    lens = np.array([len(s[1]) for s in states], dtype=np.int32)
    qs = np.array([s[0] for s in states], dtype=np.int32)
    stacks = (np.concatenate([np.asarray(s[1], dtype=np.int32) for s in states])
              if len(states) else np.zeros(0, np.int32))
    if device is None:
        return stacks, lens, qs
    import torch
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    return t(stacks if stacks.size else np.zeros(1, np.int32)), t(lens), t(qs)


class CompiledGrammar:
    """Grammar text compiled by the library (psc_grammar_compile): the lexer
    and LALR(1) tables psc_build takes, as numpy arrays, with the symbol
    names.  Raises PscError (PSC_E_NOT_LALR1 on a conflict)."""

    def __init__(self, text):
        data = text.encode("latin-1") if isinstance(text, str) else bytes(text)
        h = C.c_void_p()
        _check(lib().psc_grammar_compile(data, len(data), C.byref(h)))
        try:
            v = _Grammar()
            _check(lib().psc_grammar_view(h, C.addressof(v)))

            def arr(ptr, n, ct, dt):
                return np.ctypeslib.as_array(C.cast(ptr, C.POINTER(ct)), shape=(n,)).astype(dt).copy() \
                    if n else np.zeros(0, dt)
            nq, nt, ns, nn, npr = v.n_lex_states, v.n_terminals, v.n_lr_states, v.n_nonterminals, v.n_productions
            self.lex_next = arr(v.lex_next, nq * 256, C.c_int32, np.int32).reshape(nq, 256)
            self.lex_accept = arr(v.lex_accept, nq, C.c_int32, np.int32)
            self.terminal_ignored = arr(v.terminal_ignored, nt, C.c_uint8, np.uint8)
            self.end_terminal = int(v.end_terminal)
            self.action = arr(v.action, ns * nt, C.c_int32, np.int32).reshape(ns, nt)
            self.goto = arr(v.goto_table, ns * nn, C.c_int32, np.int32).reshape(ns, nn)
            self.prod_lhs = arr(v.prod_lhs, npr, C.c_int32, np.int32)
            self.prod_len = arr(v.prod_len, npr, C.c_int32, np.int32)
            name = lambda term, i: lib().psc_grammar_symbol_name(h, term, i).decode("latin-1")
            self.terminal_names = [name(1, i) for i in range(nt)]
            self.nonterminal_names = [name(0, i) for i in range(nn)]
        finally:
            lib().psc_grammar_free(h)


def _vocab_struct(vocab):
    toks = vocab.tokens
    offs = np.zeros(len(toks) + 1, dtype=np.int64)
    np.cumsum([len(t) for t in toks], out=offs[1:])
    blob = np.frombuffer(b"".join(toks) + b"\0", dtype=np.uint8).copy()
    return _Vocab(len(toks), blob.ctypes.data, offs.ctypes.data, int(vocab.eos_id)), (blob, offs)


class Classifier:
    """A built (grammar, vocabulary) classifier: psc_build .. psc_free; one
    built from grammar text with Classifier.from_text; or one read back with
    Classifier.load(path)."""

    @classmethod
    def from_text(cls, text, vocab) -> "Classifier":
        """psc_build_from_text: compile the grammar text, then build."""
        data = text.encode("latin-1") if isinstance(text, str) else bytes(text)
        vs, keep = _vocab_struct(vocab)
        h = C.c_void_p()
        _check(lib().psc_build_from_text(data, len(data), C.addressof(vs), C.byref(h)))
        self = cls.__new__(cls)
        self._h = h
        self._dev = None
        self.V = len(vocab.tokens)
        self.W = (self.V + 31) // 32
        return self

    @classmethod
    def load(cls, path: str) -> "Classifier":
        h = C.c_void_p()
        _check(lib().psc_load(os.fsencode(path), C.byref(h)))
        self = cls.__new__(cls)
        self._h = h
        self._dev = None
        inf = self.info()
        self.V = inf["vocab_size"]
        self.W = inf["mask_words"]
        return self

    def save(self, path: str) -> None:
        _check(lib().psc_save(self._h, os.fsencode(path)))

    def __init__(self, grammar, vocab):
        g = grammar
        arrs = dict(
            lex_next=np.ascontiguousarray(g.lexer.next, dtype=np.int32),
            lex_accept=np.ascontiguousarray(g.lexer.accept, dtype=np.int32),
            ignored=np.ascontiguousarray(g.terminal_ignored, dtype=np.uint8),
            action=np.ascontiguousarray(g.action, dtype=np.int32),
            goto=np.ascontiguousarray(g.goto, dtype=np.int32),
            lhs=np.ascontiguousarray(g.prod_lhs, dtype=np.int32),
            plen=np.ascontiguousarray(g.prod_len, dtype=np.int32),
        )
        toks = vocab.tokens
        offs = np.zeros(len(toks) + 1, dtype=np.int64)
        np.cumsum([len(t) for t in toks], out=offs[1:])
        blob = np.frombuffer(b"".join(toks) + b"\0", dtype=np.uint8).copy()
        gs = _Grammar(arrs["lex_next"].shape[0], arrs["lex_next"].ctypes.data, arrs["lex_accept"].ctypes.data,
                      arrs["action"].shape[1], arrs["ignored"].ctypes.data, int(g.end_terminal),
                      arrs["action"].shape[0], arrs["goto"].shape[1], arrs["action"].ctypes.data,
                      arrs["goto"].ctypes.data, arrs["lhs"].shape[0], arrs["lhs"].ctypes.data,
                      arrs["plen"].ctypes.data)
        vs = _Vocab(len(toks), blob.ctypes.data, offs.ctypes.data, int(vocab.eos_id))
        h = C.c_void_p()
        _check(lib().psc_build(C.addressof(gs), C.addressof(vs), C.byref(h)))
        self._h = h
        self._dev = None
        self.V = len(toks)
        self.W = (self.V + 31) // 32

    def __del__(self):
        if getattr(self, "_h", None) is not None and _lib is not None:
            _lib.psc_free(self._h)
            self._h = None

    # ---------------------------------------------------------------- host
    def info(self) -> dict:
        inf = Info()
        _check(lib().psc_info(self._h, C.byref(inf)))
        return inf.as_dict()

    def classify_host(self, states) -> np.ndarray:
        stacks, lens, qs = pack_states(states)
        out = np.zeros(len(states), np.int32)
        st = stacks if stacks.size else np.zeros(1, np.int32)
        _check(lib().psc_classify_host(self._h, st.ctypes.data, lens.ctypes.data, qs.ctypes.data,
                                       len(states), out.ctypes.data))
        return out

    def class_mask(self, cls: int) -> np.ndarray:
        row = np.zeros(self.W, np.uint32)
        _check(lib().psc_class_mask_host(self._h, int(cls), row.ctypes.data))
        return row

    def host_state(self, text: bytes, cap: int = 1 << 16):
        """psc_host_state: the prefix state (q, stack bottom->top) of `text`."""
        _require(isinstance(text, (bytes, bytearray)), "text as bytes")
        stack = np.zeros(max(int(cap), 1), np.int32)
        q, n = C.c_int32(0), C.c_int32(0)
        _check(lib().psc_host_state(self._h, bytes(text), len(text), C.byref(q), stack.ctypes.data, len(stack),
                                    C.byref(n)))
        return int(q.value), stack[:n.value].copy()

    def masks_host(self, states) -> np.ndarray:
        """Host walk + mask lookup (triage; not a device path)."""
        cls = self.classify_host(states)
        out = np.zeros((len(states), self.W), np.uint32)
        for i, c in enumerate(cls):
            if c >= 0:
                out[i] = self.class_mask(c)
        return out

    # -------------------------------------------------------------- device
    def bind(self, device="cuda", stream=None, layout=None):
        """Copy the tables to `device`; layout "flat" or "sliced" chooses the
        mask table's layout (psc_bind_device_ex), None the library default."""
        import torch
        _require(layout in _LAYOUTS, "layout None, 'flat' or 'sliced'")
        flags = _LAYOUTS[layout]
        n = int(lib().psc_device_bytes_ex(self._h, flags))
        buf = torch.empty(n + 256, dtype=torch.uint8, device=device)
        off = (-buf.data_ptr()) % 256
        ptr = buf.data_ptr() + off
        _check(lib().psc_bind_device_ex(self._h, ptr, n, flags, _stream_ptr(stream)))
        self._dev = buf
        self._device = buf.device
        self._dev_index = buf.get_device()
        self._dev_ptr = ptr
        return self

    def set_options(self, speculate: bool = False):
        """psc_set_options: PSC_OPT_SPECULATE when `speculate`."""
        _check(lib().psc_set_options(self._h, OPT_SPECULATE if speculate else 0))
        return self

    def predictor_fill(self, cls: int = -1, stream=None):
        """Every class-predictor entry to `cls` (-1: no prediction)."""
        _check(lib().psc_predictor_fill(self._h, int(cls), _stream_ptr(stream)))

    def predictor_updates(self, reset: bool = False, stream=None) -> int:
        """Walks whose class differed from the prediction since the last reset."""
        v = C.c_uint32()
        _check(lib().psc_predictor_updates(self._h, C.byref(v), int(reset), _stream_ptr(stream)))
        return int(v.value)

    def timeline_records(self, B: int, dtype) -> int:
        code = (_T or _torch_types())["codes"][dtype]
        return int(lib().psc_timeline_records(self._h, int(B), code))

    def compute_and_apply_timeline(self, stacks, stack_lens, lexer_states, logits, records, out=None, stream=None):
        """psc_compute_and_apply_timeline: the fused step with per-wavefront
        clock records (records: int64 device tensor [n, 4])."""
        B, dt = _step_args(self._idx, stacks, stack_lens, lexer_states, logits, self.V, out, self.W)
        T = _T or _torch_types()
        import torch
        _require(isinstance(records, T["tensor"]) and records.dtype == torch.int64 and records.is_contiguous()
                 and records.dim() == 2 and records.shape[1] == 4 and records.get_device() == self._idx,
                 "records as a contiguous int64 device tensor [n, 4]")
        out_ptr = None if out is None else out.data_ptr()
        _check(lib().psc_compute_and_apply_timeline(self._h, stacks.data_ptr(), stacks.numel(),
                                                    stack_lens.data_ptr(), lexer_states.data_ptr(), B, out_ptr,
                                                    logits.data_ptr(), dt, self.V, records.data_ptr(),
                                                    records.shape[0], _stream_ptr(stream)))
        return logits

    @property
    def device(self):
        """The device the tables are bound to (PSC_E_NOT_BOUND before bind)."""
        dev = getattr(self, "_device", None)
        if dev is None:
            raise PscError(-6, "the classifier is not bound to a device (call bind first)")
        return dev

    @property
    def _idx(self) -> int:
        idx = getattr(self, "_dev_index", None)
        if idx is None:
            raise PscError(-6, "the classifier is not bound to a device (call bind first)")
        return idx

    def compute_masks(self, stacks, stack_lens, lexer_states, out=None, stream=None):
        """Device int32 tensors -> uint32 bitmask [B, W] (torch.int32 view)."""
        import torch
        if out is None:
            out = torch.empty((int(stack_lens.shape[0]), self.W), dtype=torch.int32, device=self.device)
        B, _ = _step_args(self._idx, stacks, stack_lens, lexer_states, out=out, out_cols=self.W)
        _check(lib().psc_compute_masks_n(self._h, stacks.data_ptr(), stacks.numel(), stack_lens.data_ptr(),
                                         lexer_states.data_ptr(), B, out.data_ptr(), _stream_ptr(stream)))
        return out

    def compute_classes(self, stacks, stack_lens, lexer_states, out=None, stream=None):
        """Device int32 tensors -> class ids int32 [B] (-1 for a rejected input)."""
        import torch
        if out is None:
            out = torch.empty(int(stack_lens.shape[0]), dtype=torch.int32, device=self.device)
        B, _ = _step_args(self._idx, stacks, stack_lens, lexer_states, out=out)
        _check(lib().psc_compute_classes_n(self._h, stacks.data_ptr(), stacks.numel(), stack_lens.data_ptr(),
                                           lexer_states.data_ptr(), B, out.data_ptr(), _stream_ptr(stream)))
        return out

    def compute_and_apply(self, stacks, stack_lens, lexer_states, logits, out=None, stream=None):
        """One launch: masks for the B prefix states applied to logits [B, V] in
        place; the bitmask is also written to `out` when given.  Returns logits."""
        B, dt = _step_args(self._idx, stacks, stack_lens, lexer_states, logits, self.V, out, self.W)
        out_ptr = None if out is None else out.data_ptr()
        _check(lib().psc_compute_and_apply_n(self._h, stacks.data_ptr(), stacks.numel(), stack_lens.data_ptr(),
                                             lexer_states.data_ptr(), B, out_ptr, logits.data_ptr(), dt,
                                             self.V, _stream_ptr(stream)))
        return logits

    def compute_and_argmax(self, stacks, stack_lens, lexer_states, logits, out=None, stream=None):
        """Greedy token per sequence under its mask (int32 [B]; -1 = none
        allowed); the logits are only read."""
        import torch
        if out is None:
            out = torch.empty(int(stack_lens.shape[0]), dtype=torch.int32, device=self.device)
        B, dt = _step_args(self._idx, stacks, stack_lens, lexer_states, logits, self.V, out)
        _check(lib().psc_compute_and_argmax_n(self._h, stacks.data_ptr(), stacks.numel(), stack_lens.data_ptr(),
                                              lexer_states.data_ptr(), B, logits.data_ptr(), dt, self.V,
                                              out.data_ptr(), _stream_ptr(stream)))
        return out

    def compute_and_argmax_noalloc(self, stacks, stack_lens, lexer_states, logits, out, stream=None):
        """compute_and_argmax whose records live in the library's fixed
        per-GPU array (the call allocates nothing; B <= 4096; calls on one
        GPU must not overlap).  `out` is required: int32 [B]."""
        B, dt = _step_args(self._idx, stacks, stack_lens, lexer_states, logits, self.V, out)
        _check(lib().psc_compute_and_argmax_noalloc(self._h, stacks.data_ptr(), stacks.numel(),
                                                    stack_lens.data_ptr(), lexer_states.data_ptr(), B,
                                                    logits.data_ptr(), dt, self.V, out.data_ptr(),
                                                    _stream_ptr(stream)))
        return out

    def error_count(self, reset: bool = False, stream=None) -> int:
        v = C.c_uint32()
        _check(lib().psc_device_error_count(self._h, C.byref(v), int(reset), _stream_ptr(stream)))
        return int(v.value)


class DecodeStates:
    """B device-resident prefix states in the dense layout of psc_advance:
    stacks int32 [B, cap], lens int32 [B], qs int32 [B] (torch tensors)."""

    def __init__(self, clf: Classifier, B: int, cap: int, device="cuda", stream=None):
        import torch
        self.clf, self.B, self.cap = clf, int(B), int(cap)
        self.stacks = torch.zeros((self.B, self.cap), dtype=torch.int32, device=device)
        self.lens = torch.zeros(self.B, dtype=torch.int32, device=device)
        self.qs = torch.zeros(self.B, dtype=torch.int32, device=device)
        self.status = torch.zeros(self.B, dtype=torch.int32, device=device)
        _require(self.stacks.device == clf.device, f"the states on the classifier's device {clf.device}")
        self.reset(stream)

    def reset(self, stream=None):
        """Every sequence to the empty prefix (q0, stack [0])."""
        _check(lib().psc_state_reset(self.clf._h, self.stacks.data_ptr(), self.cap, self.lens.data_ptr(),
                                     self.qs.data_ptr(), self.B, _stream_ptr(stream)))
        return self

    def load(self, states):
        """Set the states from host (q, stack bottom->top) pairs."""
        import torch
        _require(len(states) == self.B, f"{self.B} states, not {len(states)}")
        st = np.zeros((self.B, self.cap), np.int32)
        for b, (q, a) in enumerate(states):
            _require(1 <= len(a) <= self.cap, f"stacks of 1 to {self.cap} symbols, not {len(a)}")
            st[b, :len(a)] = a
        self.stacks.copy_(torch.from_numpy(st))
        self.lens.copy_(torch.tensor([len(a) for _, a in states], dtype=torch.int32))
        self.qs.copy_(torch.tensor([q for q, _ in states], dtype=torch.int32))
        return self

    def advance(self, tokens, stream=None):
        """One token per sequence (int32 device tensor [B], < 0 = skip);
        returns the status tensor (ADV_*)."""
        _i32(tokens, "tokens", self.clf._idx, numel=self.B)
        _check(lib().psc_advance(self.clf._h, self.stacks.data_ptr(), self.cap, self.lens.data_ptr(),
                                 self.qs.data_ptr(), self.B, tokens.data_ptr(), self.status.data_ptr(),
                                 _stream_ptr(stream)))
        return self.status

    def compute_masks(self, out=None, stream=None):
        import torch
        if out is None:
            out = torch.empty((self.B, self.clf.W), dtype=torch.int32, device=self.lens.device)
        _i32(out, "out", self.clf._idx, shape=(self.B, self.clf.W))
        _check(lib().psc_compute_masks_dense(self.clf._h, self.stacks.data_ptr(), self.cap, self.lens.data_ptr(),
                                             self.qs.data_ptr(), self.B, out.data_ptr(), _stream_ptr(stream)))
        return out

    def compute_classes(self, out=None, stream=None):
        import torch
        if out is None:
            out = torch.empty(self.B, dtype=torch.int32, device=self.lens.device)
        _i32(out, "out", self.clf._idx, numel=self.B)
        _check(lib().psc_compute_classes_dense(self.clf._h, self.stacks.data_ptr(), self.cap, self.lens.data_ptr(),
                                               self.qs.data_ptr(), self.B, out.data_ptr(), _stream_ptr(stream)))
        return out

    def compute_and_apply(self, logits, out=None, stream=None):
        dt = _logits(logits, self.clf._idx, self.B, self.clf.V)
        out_ptr = None
        if out is not None:
            out_ptr = _i32(out, "out", self.clf._idx, shape=(self.B, self.clf.W)).data_ptr()
        _check(lib().psc_compute_and_apply_dense(self.clf._h, self.stacks.data_ptr(), self.cap,
                                                 self.lens.data_ptr(), self.qs.data_ptr(), self.B, out_ptr,
                                                 logits.data_ptr(), dt, self.clf.V, _stream_ptr(stream)))
        return logits

    def argmax(self, logits, out=None, stream=None):
        """Greedy token per sequence under its mask (int32 [B]; -1 = none)."""
        import torch
        dt = _logits(logits, self.clf._idx, self.B, self.clf.V)
        if out is None:
            out = torch.empty(self.B, dtype=torch.int32, device=logits.device)
        _i32(out, "out", self.clf._idx, numel=self.B)
        _check(lib().psc_compute_and_argmax_dense(self.clf._h, self.stacks.data_ptr(), self.cap,
                                                  self.lens.data_ptr(), self.qs.data_ptr(), self.B,
                                                  logits.data_ptr(), dt, self.clf.V, out.data_ptr(),
                                                  _stream_ptr(stream)))
        return out

    def decode_step(self, tokens, logits, out=None, stream=None):
        """psc_decode_step: advance by `tokens` (int32 [B], < 0 = skip), then
        mask `logits` [B, V] for the new states in place, in one launch.  The
        new states go to a second set of buffers, which then become this
        object's; returns the status tensor (ADV_*)."""
        import torch
        dev, T = self.clf._idx, (_T or _torch_types())
        dt = T["codes"].get(getattr(logits, "dtype", None))
        try:
            ok = (tokens.dtype is T["i32"] and tokens.get_device() == dev and tokens.is_contiguous()
                  and tokens.numel() == self.B and dt is not None and logits.get_device() == dev
                  and logits.is_contiguous() and logits.shape == (self.B, self.clf.V))
        except AttributeError:
            ok = False
        if not ok:      # names what is wrong
            _i32(tokens, "tokens", dev, numel=self.B)
            dt = _logits(logits, dev, self.B, self.clf.V)
        if getattr(self, "_spare", None) is None:
            self._spare = (torch.empty_like(self.stacks), torch.empty_like(self.lens), torch.empty_like(self.qs))
        so, lo, qo = self._spare
        out_ptr = None
        if out is not None:
            out_ptr = _i32(out, "out", self.clf._idx, shape=(self.B, self.clf.W)).data_ptr()
        _check(lib().psc_decode_step(self.clf._h, self.stacks.data_ptr(), self.lens.data_ptr(), self.qs.data_ptr(),
                                     so.data_ptr(), lo.data_ptr(), qo.data_ptr(), self.cap, self.B,
                                     tokens.data_ptr(), self.status.data_ptr(), out_ptr, logits.data_ptr(), dt,
                                     self.clf.V, _stream_ptr(stream)))
        self._spare = (self.stacks, self.lens, self.qs)
        self.stacks, self.lens, self.qs = so, lo, qo
        return self.status

    def host_states(self):
        """The states as host (q, stack) pairs (synchronises)."""
        st = self.stacks.cpu().numpy()
        lens = self.lens.cpu().numpy()
        qs = self.qs.cpu().numpy()
        return [(int(qs[b]), st[b, :lens[b]].copy()) for b in range(self.B)]


def apply_mask(logits, bitmask, stream=None):
    """In place: logits[b, v] = -inf where bit v of bitmask[b] is 0."""
    import torch
    _require(isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 2,
             "logits to be a 2-D device tensor")
    B, V = logits.shape
    dt = _logits(logits, logits.get_device(), B, V)
    _i32(bitmask, "bitmask", logits.get_device(), shape=(B, (V + 31) // 32))
    _check(lib().psc_apply_mask(logits.data_ptr(), dt, bitmask.data_ptr(), B, V, _stream_ptr(stream)))
    return logits


# ---------------------------------------------------------------- operators around the logits

SAMPLE_MAX_K = 64


def _rows(t, name: str, dev: int | None = None, shape: tuple | None = None):
    """(dtype code, row stride) of t, a float32 or bfloat16 matrix on the
    current device whose rows do not overlap and whose elements are adjacent."""
    T = _T or _torch_types()
    if type(t) is T["tensor"] and t.dim() == 2:      # no message is put together on the common path
        (rows, cols), (apart, step) = t.shape, t.stride()
        code, at = T["codes"].get(t.dtype), t.get_device()
        if (code is not None and (shape is None or (rows, cols) == shape) and step == 1 and apart >= cols
                and at >= 0 and at == T["device"]() and (dev is None or at == dev)):
            return code, apart if rows > 1 else cols
    _require(isinstance(t, T["tensor"]) and t.dim() == 2, f"{name} to be a matrix")
    code = T["codes"].get(t.dtype)
    _require(code is not None, f"float32 or bfloat16 {name}, not {t.dtype}")
    _require(shape is None or tuple(t.shape) == tuple(shape), f"{name} of shape {shape and tuple(shape)}, not {tuple(t.shape)}")
    rows, cols = t.shape
    _require(cols <= 1 or t.stride(1) == 1, f"{name} whose rows' elements are adjacent")
    stride = t.stride(0) if rows > 1 else cols
    _require(rows <= 1 or stride >= cols, f"{name} whose rows do not overlap")
    at = t.get_device()
    _require(at >= 0 and at == T["device"]() and (dev is None or at == dev), f"{name} on the current device")
    return code, stride


def _vector(t, name: str, dtype: str, dev: int, shape: tuple):
    """The address of t, a contiguous tensor of `shape`; None for None."""
    if t is None:
        return None
    T = _T or _torch_types()
    if not (type(t) is T["tensor"] and t.dtype is T[dtype] and t.shape == shape and t.get_device() == dev
            and t.is_contiguous()):
        _require(isinstance(t, T["tensor"]) and t.dtype is T[dtype] and tuple(t.shape) == tuple(shape)
                 and t.is_contiguous(), f"{name} to be a contiguous {T[dtype]} tensor of shape {tuple(shape)}")
        _require(t.get_device() == dev, f"{name} on device {dev}, not {t.get_device()}")
    return t.data_ptr()


def _new(shape, dtype: str, device, stream):
    """An uninitialised tensor for a call on `stream` (None: the current one),
    out of that stream's memory."""
    T = _T or _torch_types()
    if stream is None:
        return T["empty"](shape, dtype=T[dtype], device=device)
    import torch
    with torch.cuda.stream(stream):
        return T["empty"](shape, dtype=T[dtype], device=device)


def quantize_rows(x, stream=None):
    """(q, scales): the rows of x [N, D] in 8 bits, int8 [N, D] whose rows start
    at multiples of 16 bytes, with a scale each, float32 [N] (psc_quantize_rows)."""
    code, stride = _rows(x, "x")
    n, D = x.shape
    q_stride = (D + 15) // 16 * 16
    q, scales = _new((n, q_stride), "i8", x.device, stream), _new(n, "f32", x.device, stream)
    _check(lib().psc_quantize_rows(x.data_ptr(), code, stride, n, D, q.data_ptr(), q_stride, scales.data_ptr(),
                                   _stream_ptr(stream)))
    return q[:, :D], scales


def _logits_out(out, dtype, default, B: int, V: int, device, stream):
    """(out, its dtype code and row stride): logits [B, V], new ones of `dtype` (or `default`) where out is None."""
    T = _T or _torch_types()
    if out is not None:
        _require(dtype is None or dtype == out.dtype, "dtype to be that of out")
        code, stride = _rows(out, "out", device.index, (B, V))
        return out, code, stride
    code = T["codes"].get(default if dtype is None else dtype)
    if code is None:
        _require(False, f"float32 or bfloat16 logits, not {dtype}")
    return _new((B, V), ("f32", "bf16")[code], device, stream), code, V


def _matrix(t, name: str) -> None:
    T = _T or _torch_types()
    if not (isinstance(t, T["tensor"]) and t.dim() == 2):
        _require(False, f"{name} to be a matrix")


def _wide(t, cols: int):
    """The first `cols` columns of t."""
    return t if t.shape[1] == cols else t.narrow(1, 0, cols)


def _packed(t, name: str, dtype: str, cols: int, align: int, dev: int | None = None, rows: int | None = None):
    """(row stride, rows, device index) of t, a matrix of bytes of `dtype` on the current device with `cols` adjacent
    columns and rows that start at multiples of `align` bytes."""
    T = _T or _torch_types()
    if type(t) is T["tensor"] and t.dtype is T[dtype] and t.dim() == 2:      # no message is put together on the common path
        (n, wide), (apart, step), at = t.shape, t.stride(), t.get_device()
        if n <= 1:
            apart = (cols + align - 1) // align * align
        if (wide == cols > 0 and step == 1 and apart % align == 0 and apart >= cols and t.data_ptr() % align == 0
                and at >= 0 and at == (T["device"]() if dev is None else dev) and (rows is None or n == rows)):
            return apart, n, at
    _require(isinstance(t, T["tensor"]) and t.dtype is T[dtype] and t.dim() == 2 and t.shape[1] == cols and cols > 0,
             f"{name} to be a matrix of {T[dtype]} with {cols} columns")
    n = t.shape[0]
    _require(rows is None or n == rows, f"{name} of {rows} rows, not {n}")
    apart = t.stride(0) if n > 1 else (cols + align - 1) // align * align
    at = t.get_device()
    _require(at >= 0 and at == (T["device"]() if dev is None else dev), f"{name} on the current device")
    _require((cols == 1 or t.stride(1) == 1) and apart >= cols and apart % align == 0 and t.data_ptr() % align == 0,
             f"{name} with adjacent elements and rows that start at multiples of {align} bytes")
    return apart, n, at


def head_logits(x, w, w_scales, dtype=None, bias=None, bitmask=None, out=None, stream=None, x_scales=None):
    """Logits [B, V] of hidden states x [B, D] by 8-bit weights w [V, D] with a
    scale per token (quantize_rows), forbidden tokens -inf (psc_head_logits).
    `out`: where to write them (its rows may lie apart); else a new tensor of
    `dtype`, that of x by default.  States that are in 8 bits already (x int8
    with x_scales float32 [B], as quantize_rows and add_rms_norm return them)
    are taken as they are, to bfloat16 logits by default (psc_head_logits_quantized)."""
    T = _T or _torch_types()
    if x_scales is None:
        x_code, x_stride = _rows(x, "x")
        default = x.dtype
    else:
        _matrix(x, "x")
        x_stride, default = _packed(x, "x", "i8", x.shape[1], 16)[0], T["bf16"]
    B, D = x.shape
    dev = x.get_device()
    if not (isinstance(w, T["tensor"]) and w.dtype is T["i8"] and w.dim() == 2 and w.shape[1] == D and D > 0):
        _require(False, f"w to be an int8 matrix of rows of {D} elements")
    V = w.shape[0]
    w_stride = w.stride(0) if V > 1 else (D + 15) // 16 * 16
    _require(w.get_device() == dev and (D == 1 or w.stride(1) == 1) and w_stride >= D and w_stride % 16 == 0
             and w.data_ptr() % 16 == 0, "w on x's device, with adjacent elements and rows that start at 16 bytes")
    out, code, y_stride = _logits_out(out, dtype, default, B, V, x.device, stream)
    L = lib()
    scales = _vector(w_scales, "w_scales", "f32", dev, (V,))
    _require(scales is not None, "w_scales")
    bias = _vector(bias, "bias", "f32", dev, (V,))
    words = _vector(bitmask, "bitmask", "i32", dev, (B, (V + 31) // 32))
    given = _vector(x_scales, "x_scales", "f32", dev, (B,))
    n = L.psc_head_workspace(B, D, V)
    ws = _new(n, "u8", x.device, stream)
    rest = (B, D, w.data_ptr(), w_stride, scales, V, bias, words, out.data_ptr(), code, y_stride, ws.data_ptr(), n,
            _stream_ptr(stream))
    _check(L.psc_head_logits(x.data_ptr(), x_code, x_stride, *rest) if given is None
           else L.psc_head_logits_quantized(x.data_ptr(), x_stride, given, *rest))
    return out


MX_BLOCK = 32
_STATES = {"bf16": FORM_BF16, "mx4": FORM_MX4}


def quantize_mx(x, stream=None):
    """(q, scales): the rows of x [N, D] in microscaled 4-bit floating point
    (psc_quantize_mx): uint8 [N, ceil(D / 2)], the even elements in the low
    halves, and of every 32 elements the power of two, uint8 [N, ceil(D / 32)];
    the rows of both start at multiples of 16 bytes."""
    code, stride = _rows(x, "x")
    n, D = x.shape
    blocks = (D + MX_BLOCK - 1) // MX_BLOCK
    q_stride, s_stride = blocks * 16, (blocks + 15) // 16 * 16
    q, scales = _new((n, q_stride), "u8", x.device, stream), _new((n, s_stride), "u8", x.device, stream)
    _check(lib().psc_quantize_mx(x.data_ptr(), code, stride, n, D, q.data_ptr(), q_stride, scales.data_ptr(), s_stride,
                                 _stream_ptr(stream)))
    return _wide(q, (D + 1) // 2), _wide(scales, blocks)


def lookup_rows(q, scales, ids=None, D=None, dtype=None, out=None, stream=None):
    """Rows `ids` (int32 [n]; None: all, in order) of a quantised table as
    numbers [n, D] (psc_lookup_rows): q and scales as quantize_rows or
    quantize_mx return them, D that of the table where it is odd and in 4 bits.
    A row whose id is outside the table is zeros.  `out`: where to write them;
    else a new tensor of `dtype`, bfloat16 by default."""
    T = _T or _torch_types()
    _matrix(q, "q")
    mx, cols = q.dtype is T["u8"], q.shape[1]
    if D is None:
        D = cols * 2 if mx else cols
    if D == 0:
        q_stride, rows, dev = 0, q.shape[0], q.get_device()
    else:
        q_stride, rows, dev = _packed(q, "q", "u8" if mx else "i8", (D + 1) // 2 if mx else D, 16)
    n = rows
    if ids is not None:
        if not (isinstance(ids, T["tensor"]) and ids.dim() == 1):
            _require(False, "ids to be a vector")
        n = ids.shape[0]
    if out is None:
        code, out_stride = T["codes"].get(T["bf16"] if dtype is None else dtype), D
        if code is None:
            _require(False, f"float32 or bfloat16 rows, not {dtype}")
        out = _new((n, D), ("f32", "bf16")[code], q.device, stream)
    else:
        _require(dtype is None or dtype == out.dtype, "dtype to be that of out")
        code, out_stride = _rows(out, "out", dev, (n, D))
    if D == 0 or n == 0:
        return out
    at_ids, s_stride = _vector(ids, "ids", "i32", dev, (n,)), 0
    if mx:
        s_stride = _packed(scales, "scales", "u8", (D + MX_BLOCK - 1) // MX_BLOCK, 4, dev, rows)[0]
        at = scales.data_ptr()
    else:
        at = _vector(scales, "scales", "f32", dev, (rows,))
        _require(at is not None, "scales")
    _check(lib().psc_lookup_rows(FORM_MX4 if mx else FORM_I8, q.data_ptr(), q_stride, at, s_stride, rows, D, at_ids, n,
                                 out.data_ptr(), code, out_stride, _stream_ptr(stream)))
    return out


def add_rms_norm(x, gain=None, residual=None, eps=1e-6, to=None, stream=None):
    """The root-mean-square norm of x [N, D], or of residual + x, which then
    becomes the residual [N, D], in place; times gain (float32 [D]) where given
    (psc_add_rms_norm).  `to`: float32 or bfloat16 (None: x's type), then the
    result is a matrix; "i8" or "mx4", then it is (q, scales) as quantize_rows
    or quantize_mx return them, for head_logits and head_logits_mx."""
    T = _T or _torch_types()
    code, stride = _rows(x, "x")
    (n, D), dev = x.shape, x.get_device()
    r_at, r_code, r_stride = None, PSC_F32, 0
    if residual is not None:
        r_code, r_stride = _rows(residual, "residual", dev, (n, D))
        r_at = residual.data_ptr()
    at_gain = _vector(gain, "gain", "f32", dev, (D,))
    eps = float(eps)
    _require(eps >= 0, "eps of at least 0")
    scales, s_at, s_stride = None, None, 0
    if to == "i8":
        form, o_stride = FORM_I8, (D + 15) // 16 * 16
        out, scales = _new((n, o_stride), "i8", x.device, stream), _new(n, "f32", x.device, stream)
        got = _wide(out, D), scales
    elif to == "mx4":
        blocks = (D + MX_BLOCK - 1) // MX_BLOCK
        form, o_stride, s_stride = FORM_MX4, blocks * 16, (blocks + 15) // 16 * 16
        out, scales = _new((n, o_stride), "u8", x.device, stream), _new((n, s_stride), "u8", x.device, stream)
        got = _wide(out, (D + 1) // 2), _wide(scales, blocks)
    else:
        form, o_stride = T["codes"].get(x.dtype if to is None else to), D
        if form is None:
            _require(False, f'to: float32, bfloat16, "i8" or "mx4", not {to}')
        out = got = _new((n, D), ("f32", "bf16")[form], x.device, stream)
    if scales is not None:
        s_at = scales.data_ptr()
    _check(lib().psc_add_rms_norm(x.data_ptr(), code, stride, r_at, r_code, r_stride, n, D, at_gain, eps, form,
                                  out.data_ptr(), o_stride, s_at, s_stride, _stream_ptr(stream)))
    return got


def head_logits_mx(x, w, w_scales, states="bf16", x_scales=None, dtype=None, bias=None, bitmask=None, out=None,
                   stream=None, D=None):
    """Logits [B, V] of hidden states x [B, D] by 4-bit weights w [V, ceil(D / 2)]
    with w_scales [V, ceil(D / 32)] (quantize_mx), forbidden tokens -inf
    (psc_head_logits_mx).  `states`: what the products take them in, "bf16", or
    "mx4", quantised as by quantize_mx.  States that are in 4 bits already (x
    uint8 with x_scales, as quantize_mx and add_rms_norm return them) are taken
    as they are; D is that of their rows where it is odd (else their last code
    counts too, a zero as the quantisers write it).  `out`: where to write the
    logits; else a new tensor of `dtype`, by default that of x, of states in
    4 bits bfloat16."""
    T = _T or _torch_types()
    form = _STATES.get(states)
    if form is None:
        _require(False, 'states: "bf16" or "mx4"')
    x_at, x_s_stride = None, 0
    if x_scales is None:
        x_code, x_stride = _rows(x, "x")
        if D is not None and D != x.shape[1]:
            _require(False, f"x of {D} columns")
        (B, D), dev, default = x.shape, x.get_device(), x.dtype
        cols, blocks = (D + 1) // 2, (D + MX_BLOCK - 1) // MX_BLOCK
    else:
        _matrix(x, "x")
        cols, default, form, x_code = x.shape[1], T["bf16"], FORM_MX4, FORM_MX4
        if D is None:
            D = cols * 2
        elif (D + 1) // 2 != cols:
            _require(False, f"x of {(D + 1) // 2} columns for D = {D}")
        blocks = (D + MX_BLOCK - 1) // MX_BLOCK
        x_stride, B, dev = _packed(x, "x", "u8", cols, 16)
        x_s_stride = _packed(x_scales, "x_scales", "u8", blocks, 1, dev, B)[0]
        x_at = x_scales.data_ptr()
    w_stride, V, _ = _packed(w, "w", "u8", cols, 16, dev)
    s_stride = _packed(w_scales, "w_scales", "u8", blocks, 4, dev, V)[0]
    out, code, y_stride = _logits_out(out, dtype, default, B, V, x.device, stream)
    L = lib()
    bias = _vector(bias, "bias", "f32", dev, (V,))
    words = _vector(bitmask, "bitmask", "i32", dev, (B, (V + 31) // 32))
    n = L.psc_head_mx_workspace(B, D, V, form)
    ws = _new(n, "u8", x.device, stream)
    _check(L.psc_head_logits_mx(x.data_ptr(), x_code, x_stride, x_at, x_s_stride, B, D, form, w.data_ptr(), w_stride,
                                w_scales.data_ptr(), s_stride, V, bias, words, out.data_ptr(), code, y_stride,
                                ws.data_ptr(), n, _stream_ptr(stream)))
    return out


def penalize(logits, history=None, lens=None, prompt_lens=None, repetition=None, presence=None, frequency=None,
             bias_ids=None, bias_values=None, bitmask=None, stream=None):
    """In place on logits [B, V]: penalties of the tokens in history [B, cap]
    (int32; lens [B] of them, the first prompt_lens [B] the prompt), biases
    (ids int32 [B, n], -1 for none; values float32), -inf where the bitmask
    forbids (psc_penalize).  Returns logits."""
    code, stride = _rows(logits, "logits")
    (B, V), dev = logits.shape, logits.get_device()
    cap = n_bias = 0
    if history is not None:
        _require(history.dim() == 2 and lens is not None, "history to be a matrix, with lens")
        cap = history.shape[1]
    if bias_ids is not None:
        _require(bias_ids.dim() == 2 and bias_values is not None, "bias_ids to be a matrix, with bias_values")
        n_bias = bias_ids.shape[1]
    rows = (B,)
    p = _Penalties(_vector(history, "history", "i32", dev, (B, cap)), _vector(lens, "lens", "i32", dev, rows),
                   _vector(prompt_lens, "prompt_lens", "i32", dev, rows), cap, n_bias,
                   _vector(repetition, "repetition", "f32", dev, rows),
                   _vector(presence, "presence", "f32", dev, rows),
                   _vector(frequency, "frequency", "f32", dev, rows),
                   _vector(bias_ids, "bias_ids", "i32", dev, (B, n_bias)),
                   _vector(bias_values, "bias_values", "f32", dev, (B, n_bias)))
    words = _vector(bitmask, "bitmask", "i32", dev, (B, (V + 31) // 32))
    _check(lib().psc_penalize(logits.data_ptr(), code, stride, B, V, C.byref(p), words, _stream_ptr(stream)))
    return logits


def append_tokens(history, lens, tokens, status=None, stream=None):
    """tokens [B] (int32, < 0: none) to the ends of the histories [B, cap], in
    place (psc_append_tokens); status [B], if given, receives ADV_OK,
    ADV_SKIPPED, ADV_OVERFLOW or ADV_BAD_INPUT."""
    T = _T or _torch_types()
    _require(isinstance(history, T["tensor"]) and history.dim() == 2 and history.get_device() >= 0
             and history.get_device() == T["device"](), "history to be a matrix on the current device")
    (B, cap), dev = history.shape, history.get_device()
    at = [_vector(t, name, "i32", dev, shape) for t, name, shape in
          ((history, "history", (B, cap)), (lens, "lens", (B,)), (tokens, "tokens", (B,)), (status, "status", (B,)))]
    _require(at[1] is not None and at[2] is not None, "lens and tokens")
    _check(lib().psc_append_tokens(at[0], cap, at[1], B, at[2], at[3], _stream_ptr(stream)))


def sample(logits, k, bitmask=None, temperature=None, top_k=None, top_p=None, min_p=None, noise=None, stream=None):
    """(tokens int32 [B], logprobs float32 [B], ids int32 [B, k], id_logprobs
    float32 [B, k]) of logits [B, V] under the bitmask: the k best tokens and
    one drawn from them (psc_sample).  temperature, top_p, min_p: float32 [B];
    top_k: int32 [B]; noise: float32 [B, k] of unit exponentials (None: the
    best token)."""
    code, stride = _rows(logits, "logits")
    (B, V), dev = logits.shape, logits.get_device()
    k = int(k)
    if not 1 <= k <= SAMPLE_MAX_K:
        _require(False, f"k in [1, {SAMPLE_MAX_K}]")
    _require(V > 0, "logits of at least one token")
    rows = (B,)
    p = _Sampling(_vector(temperature, "temperature", "f32", dev, rows), _vector(top_k, "top_k", "i32", dev, rows),
                  _vector(top_p, "top_p", "f32", dev, rows), _vector(min_p, "min_p", "f32", dev, rows),
                  _vector(noise, "noise", "f32", dev, (B, k)))
    words = _vector(bitmask, "bitmask", "i32", dev, (B, (V + 31) // 32))
    L, device = lib(), logits.device
    n = L.psc_sample_workspace(B, V, code)
    ws = _new(n, "u8", device, stream)
    tokens, ids = _new(B, "i32", device, stream), _new((B, k), "i32", device, stream)
    logprobs, id_logprobs = _new(B, "f32", device, stream), _new((B, k), "f32", device, stream)
    _check(L.psc_sample(logits.data_ptr(), code, stride, B, V, words, C.byref(p), k, tokens.data_ptr(),
                        logprobs.data_ptr(), ids.data_ptr(), id_logprobs.data_ptr(), ws.data_ptr(), n,
                        _stream_ptr(stream)))
    return tokens, logprobs, ids, id_logprobs
