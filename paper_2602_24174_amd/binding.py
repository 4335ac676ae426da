"""ctypes binding of libtasc.so: the same entry points as include/tasc.h, argument marshalling only.

PyTorch supplies device memory (`torch.empty(..., device="cuda")`) and the current stream; every step of
the path runs in the library's HIP kernels.  There is no CPU fallback: if the library is missing or a
call fails, TascError is raised.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtasc.so")

TASC_OK, TASC_EINVAL, TASC_ENOMEM, TASC_EHIP, TASC_ESTATE = 0, -1, -2, -3, -4
TASC_MEM_HOST, TASC_MEM_DEVICE = 0, 1
TASC_F32, TASC_BF16 = 0, 1
TASC_MAX_ORDER, TASC_MAX_K = 8, 15

EXPORTS = [
    "tasc_last_error", "tasc_ngram_build", "tasc_ngram_destroy", "tasc_ngram_export", "tasc_ngram_export_contexts",
    "tasc_ngram_unigram", "tasc_ngram_get_stats", "tasc_ngram_entropy", "tasc_ngram_entropy_noalloc", "tasc_model_bigram", "tasc_ngram_from_bigram", "tasc_tok_enrich", "tasc_model_create", "tasc_model_destroy", "tasc_session_kv_bytes",
    "tasc_session_workspace_bytes", "tasc_session_create", "tasc_session_destroy", "tasc_session_prefill", "tasc_draft",
    "tasc_verify_step", "tasc_generate", "tasc_session_get_tokens", "tasc_session_status", "tasc_profile_enable", "tasc_profile_read", "tasc_profile_durations", "tasc_config_set", "tasc_profile_phases", "tasc_calibration_copy", "tasc_calibration_mfma", "tasc_calibration_read", "tasc_calibration_handover", "tasc_calibration_gemm",
    "tasc_page_tables", "tasc_kv4_page_bytes", "tasc_kv4_append", "tasc_kv4_read", "tasc_kv4_attention_workspace_bytes",
    "tasc_kv4_attention", "tasc_accept_sampled_workspace_bytes", "tasc_accept_sampled", "tasc_sampled_scratch_bytes",
    "tasc_verify_step_sampled", "tasc_session_rewind", "tasc_generate_sampled", "tasc_session_kv4_bytes", "tasc_session_create_kv4",
    "tasc_sample_workspace_bytes", "tasc_sample", "tasc_filter_logits",
    "tasc_session_filter", "tasc_pages_fork", "tasc_pages_copy", "tasc_pages_workspace_bytes", "tasc_pages_free", "tasc_pages_compact",
]
KERNEL_CLASSES = ["draft", "prepare", "norm", "gemm_qkv", "rope_kv", "attn", "gemm_o", "gemm_gu", "gemm_d", "lmhead", "accept",
                  "verify", "layers"]


class TascError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"tasc status {status}: {message}")
        self.status = status


class NgramStats(C.Structure):
    _fields_ = [("n_tokens", C.c_int64), ("windows", C.c_int64 * (TASC_MAX_ORDER + 1)),
                ("distinct", C.c_int64 * (TASC_MAX_ORDER + 1)), ("kept", C.c_int64 * (TASC_MAX_ORDER + 1)),
                ("contexts", C.c_int64 * (TASC_MAX_ORDER + 1)), ("build_ms", C.c_double), ("count_ms", C.c_double)]


class TableEntropy(C.Structure):
    _fields_ = [("n_entries", C.c_int64), ("total", C.c_int64), ("n_cover", C.c_int64), ("shannon", C.c_double),
                ("renyi2", C.c_double)]


class ModelDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ffn", C.c_int32), ("vocab", C.c_int32),
                ("max_pos", C.c_int32), ("rope_theta", C.c_float), ("rms_eps", C.c_float)]


class WeightPtrs(C.Structure):
    _fields_ = [("where", C.c_int32), ("embed", C.c_void_p), ("lm_head", C.c_void_p), ("gf", C.c_void_p),
                ("wq", C.POINTER(C.c_void_p)), ("wk", C.POINTER(C.c_void_p)), ("wv", C.POINTER(C.c_void_p)),
                ("wo", C.POINTER(C.c_void_p)), ("wg", C.POINTER(C.c_void_p)), ("wu", C.POINTER(C.c_void_p)),
                ("wd", C.POINTER(C.c_void_p)), ("g1", C.POINTER(C.c_void_p)), ("g2", C.POINTER(C.c_void_p)),
                ("bias_rowptr", C.c_void_p), ("bias_col", C.c_void_p), ("bias_val", C.c_void_p), ("bias_base", C.c_void_p)]


class SpecParams(C.Structure):
    _fields_ = [("k", C.c_int32), ("lambda_q16", C.c_int32), ("p_min_ctx", C.c_int32), ("ctx_includes_generated", C.c_int32)]


class GenStats(C.Structure):
    _fields_ = [("steps", C.c_int64), ("emitted", C.c_int64), ("accepted", C.c_int64), ("proposed", C.c_int64),
                ("accept_hist", C.c_int64 * (TASC_MAX_K + 1)), ("prefill_ms", C.c_double), ("decode_ms", C.c_double),
                ("xcd_local_steps", C.c_int64)]


class Sampling(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("u", C.c_void_p), ("n_u", C.c_int64), ("scratch", C.c_void_p), ("scratch_bytes", C.c_size_t)]


class Kv4CacheDesc(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class Kv4Attn(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("q_stride", C.c_int64), ("out_stride", C.c_int64), ("table", C.c_void_p),
                ("row_off", C.c_void_p), ("kv_len", C.c_void_p), ("max_pages", C.c_int32), ("batch", C.c_int32), ("rows", C.c_int32),
                ("n_heads", C.c_int32), ("max_rows", C.c_int32), ("max_kv", C.c_int32), ("scale", C.c_float)]


_lib = None


def lib():
    """Loads libtasc.so (built by paper_2602_24174_amd/build.py or __graft_entry__.build())."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise TascError(TASC_EHIP, f"{LIB_PATH} is not built; run `python -m paper_2602_24174_amd.build`")
        # PyTorch first: it supplies the device memory and streams, and the process must end up with ONE HIP
        # runtime.  If libtasc.so pulled in the system's libamdhip64 before torch loaded its own, the runtime
        # that initialises second finds no device.
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        L.tasc_last_error.restype = C.c_char_p
        L.tasc_session_kv_bytes.restype = C.c_size_t
        L.tasc_session_workspace_bytes.restype = C.c_size_t
        L.tasc_session_kv_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        L.tasc_session_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
        L.tasc_ngram_build.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                       C.c_void_p, C.POINTER(C.c_void_p)]
        L.tasc_ngram_export.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(C.c_int64)]
        L.tasc_ngram_export_contexts.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                 C.POINTER(C.c_int64)]
        L.tasc_ngram_unigram.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_void_p]
        L.tasc_ngram_get_stats.argtypes = [C.c_void_p, C.POINTER(NgramStats)]
        L.tasc_tok_enrich.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
        L.tasc_model_bigram.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.tasc_ngram_from_bigram.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_void_p)]
        L.tasc_ngram_entropy.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(TableEntropy), C.c_void_p]
        L.tasc_ngram_entropy_noalloc.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.tasc_model_create.argtypes = [C.POINTER(ModelDesc), C.POINTER(WeightPtrs), C.POINTER(C.c_void_p)]
        L.tasc_session_create.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p,
                                          C.c_size_t, C.POINTER(C.c_void_p)]
        L.tasc_session_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]
        L.tasc_draft.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(SpecParams), C.c_void_p, C.c_void_p]
        L.tasc_verify_step.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_void_p]
        L.tasc_generate.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                    C.POINTER(SpecParams), C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(GenStats), C.c_void_p]
        L.tasc_session_get_tokens.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.c_void_p]
        L.tasc_session_status.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_void_p]
        L.tasc_config_set.argtypes = [C.c_int32, C.c_int32]
        L.tasc_profile_phases.argtypes = [C.c_void_p, C.c_int64]
        L.tasc_calibration_copy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.tasc_calibration_mfma.argtypes = [C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.tasc_calibration_read.argtypes = [C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.tasc_calibration_handover.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.tasc_calibration_gemm.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.tasc_profile_enable.argtypes = [C.c_uint32]
        L.tasc_profile_read.argtypes = [C.c_void_p, C.c_void_p]
        L.tasc_profile_durations.argtypes = [C.c_int32, C.c_void_p, C.c_int64, C.POINTER(C.c_int64)]
        L.tasc_page_tables.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        L.tasc_sampled_scratch_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        L.tasc_verify_step_sampled.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(Sampling), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.tasc_session_filter.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t]
        L.tasc_session_rewind.argtypes = [C.c_void_p, C.c_void_p]
        L.tasc_generate_sampled.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.POINTER(SpecParams),
                                            C.POINTER(Sampling), C.c_void_p, C.POINTER(GenStats), C.c_void_p]
        L.tasc_session_kv4_bytes.argtypes = [C.c_void_p, C.c_int32]
        L.tasc_session_create_kv4.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t,
                                              C.POINTER(C.c_void_p)]
        for name in ("tasc_kv4_page_bytes", "tasc_sampled_scratch_bytes", "tasc_session_kv4_bytes", "tasc_kv4_attention_workspace_bytes", "tasc_accept_sampled_workspace_bytes",
                     "tasc_pages_workspace_bytes", "tasc_sample_workspace_bytes"):
            getattr(L, name).restype = C.c_size_t
        L.tasc_kv4_page_bytes.argtypes = [C.c_int32] * 2
        L.tasc_sample_workspace_bytes.argtypes = [C.c_int32] * 2
        L.tasc_sample.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.tasc_filter_logits.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_int64, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.tasc_pages_workspace_bytes.argtypes = [C.c_int32]
        L.tasc_pages_fork.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_void_p]
        L.tasc_pages_copy.argtypes = [C.c_void_p, C.c_size_t, C.c_int32, C.c_int32, C.c_size_t, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.tasc_pages_free.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.tasc_pages_compact.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                         C.c_void_p, C.c_size_t, C.c_void_p]
        L.tasc_kv4_append.argtypes = [C.POINTER(Kv4CacheDesc), C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_void_p, C.c_int32, C.c_void_p]
        L.tasc_kv4_read.argtypes = [C.POINTER(Kv4CacheDesc), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.tasc_kv4_attention_workspace_bytes.argtypes = [C.c_int32] * 7
        L.tasc_kv4_attention.argtypes = [C.POINTER(Kv4CacheDesc), C.POINTER(Kv4Attn), C.c_void_p, C.c_size_t, C.c_void_p]
        L.tasc_accept_sampled_workspace_bytes.argtypes = [C.c_int32] * 3
        L.tasc_accept_sampled.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        for name in ("tasc_ngram_destroy", "tasc_model_destroy", "tasc_session_destroy"):
            getattr(L, name).argtypes = [C.c_void_p]
            getattr(L, name).restype = None
        _lib = L
    return _lib


def _check(status):
    if status != TASC_OK:
        raise TascError(status, lib().tasc_last_error().decode())


def _ptr(a):
    """Raw address of a numpy array (host), a torch tensor (host or device) or None."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        assert a.flags["C_CONTIGUOUS"]
        return a.ctypes.data
    assert a.is_contiguous()
    return a.data_ptr()


def _where(a):
    return TASC_MEM_HOST if isinstance(a, np.ndarray) or not a.is_cuda else TASC_MEM_DEVICE


def _stream(stream):
    if stream is not None:
        return stream
    import torch
    return torch.cuda.current_stream().cuda_stream


class Ngram:
    def __init__(self, handle, n_max):
        self.handle, self.n_max = handle, n_max

    def close(self):
        if self.handle:
            lib().tasc_ngram_destroy(self.handle)
            self.handle = None

    __del__ = close


def tasc_ngram_build(tokens, doc_offsets, vocab, n_max, p_min, stream=None) -> Ngram:
    """tokens: int32 numpy array (host) or cuda tensor; doc_offsets: int64 numpy array."""
    doc_offsets = np.ascontiguousarray(doc_offsets, dtype=np.int64)
    out = C.c_void_p()
    _check(lib().tasc_ngram_build(_ptr(tokens), _ptr(doc_offsets), len(doc_offsets) - 1, vocab, n_max, p_min, _where(tokens),
                                  _stream(stream), C.byref(out)))
    return Ngram(out.value, n_max)


def tasc_ngram_export(ng: Ngram, order: int):
    """Returns (ctx_next int32[R, order], counts uint32[R]), rows sorted by their tokens."""
    n = C.c_int64(0)
    _check(lib().tasc_ngram_export(ng.handle, order, None, None, C.byref(n)))
    rows = np.zeros((n.value, order), dtype=np.int32)
    counts = np.zeros(n.value, dtype=np.uint32)
    n = C.c_int64(n.value)
    _check(lib().tasc_ngram_export(ng.handle, order, _ptr(rows), _ptr(counts), C.byref(n)))
    return rows, counts


def tasc_ngram_export_contexts(ng: Ngram, order: int):
    n = C.c_int64(0)
    _check(lib().tasc_ngram_export_contexts(ng.handle, order, None, None, None, None, C.byref(n)))
    ctx = np.zeros((n.value, order - 1), dtype=np.int32)
    total = np.zeros(n.value, dtype=np.uint32)
    top = np.zeros(n.value, dtype=np.int32)
    top_count = np.zeros(n.value, dtype=np.uint32)
    n = C.c_int64(n.value)
    _check(lib().tasc_ngram_export_contexts(ng.handle, order, _ptr(ctx), _ptr(total), _ptr(top), _ptr(top_count), C.byref(n)))
    return ctx, total, top, top_count


def tasc_ngram_unigram(ng: Ngram, vocab: int):
    fb = C.c_int32(0)
    counts = np.zeros(vocab, dtype=np.uint32)
    _check(lib().tasc_ngram_unigram(ng.handle, C.byref(fb), _ptr(counts)))
    return fb.value, counts


def tasc_ngram_entropy(ng: Ngram, order: int, coverage_ppm: int = 800000, stream=None) -> TableEntropy:
    out = TableEntropy()
    _check(lib().tasc_ngram_entropy(ng.handle, order, coverage_ppm, C.byref(out), _stream(stream)))
    return out


def tasc_ngram_entropy_noalloc(ng: Ngram, order: int, coverage_ppm: int, out_device, stream=None):
    """out_device: cuda uint8 tensor of sizeof(TableEntropy) bytes, written on the stream (no synchronisation)."""
    assert out_device.is_cuda and out_device.numel() * out_device.element_size() >= C.sizeof(TableEntropy)
    _check(lib().tasc_ngram_entropy_noalloc(ng.handle, order, coverage_ppm, _ptr(out_device), _stream(stream)))


def tasc_tok_enrich(tokens, doc_offsets, vocab, n_max, budget, stream=None):
    """tokens: int32 numpy array (host) or cuda tensor.  Returns (merges [(ngram tuple, freq, new id)], final tokens
    (same kind as the input, trimmed), final offsets int64[D + 1], corpus lengths int64[n_merges + 1])."""
    doc_offsets = np.ascontiguousarray(doc_offsets, dtype=np.int64)
    n_docs = doc_offsets.shape[0] - 1
    rows = np.zeros((max(budget, 1), 1 + TASC_MAX_ORDER), dtype=np.int32)
    freq = np.zeros(max(budget, 1), dtype=np.int64)
    lens = np.zeros(budget + 1, dtype=np.int64)
    out_off = np.zeros(n_docs + 1, dtype=np.int64)
    if isinstance(tokens, np.ndarray):
        tokens = np.ascontiguousarray(tokens, dtype=np.int32)
        out = np.zeros(max(tokens.shape[0], 1), dtype=np.int32)
    else:
        import torch
        out = torch.zeros(max(tokens.shape[0], 1), dtype=torch.int32, device=tokens.device)
    n = C.c_int32(0)
    _check(lib().tasc_tok_enrich(_ptr(tokens), _ptr(doc_offsets), n_docs, vocab, n_max, budget, _where(tokens), _stream(stream),
                                 _ptr(rows), _ptr(freq), _ptr(lens), _ptr(out), _ptr(out_off), C.byref(n)))
    m = n.value
    merges = [(tuple(int(t) for t in rows[i, 1:1 + rows[i, 0]]), int(freq[i]), vocab + i) for i in range(m)]
    return merges, out[:int(lens[m])], out_off, lens[:m + 1]


def tasc_model_bigram(model: "Model", s: "Session", next_tok, stream=None):
    """next_tok: cuda int32 tensor [vocab], written in place."""
    _check(lib().tasc_model_bigram(model.handle, s.handle, _ptr(next_tok), _stream(stream)))


def tasc_ngram_from_bigram(next_tok, vocab, n_max, stream=None) -> Ngram:
    out = C.c_void_p()
    _check(lib().tasc_ngram_from_bigram(_ptr(next_tok), _where(next_tok), vocab, n_max, _stream(stream), C.byref(out)))
    return Ngram(out.value, n_max)


def tasc_ngram_get_stats(ng: Ngram) -> NgramStats:
    st = NgramStats()
    _check(lib().tasc_ngram_get_stats(ng.handle, C.byref(st)))
    return st


class Model:
    def __init__(self, handle, desc):
        self.handle, self.desc = handle, desc

    def close(self):
        if self.handle:
            lib().tasc_model_destroy(self.handle)
            self.handle = None

    __del__ = close


def tasc_model_create(cfg, weights, max_pos) -> Model:
    """cfg: object with the model fields of workload.WorkloadConfig; weights: the canonical dict of
    numpy arrays (host) from workload.make_model (uint16 arrays are bf16 bit patterns)."""
    desc = ModelDesc(TASC_BF16 if cfg.dtype == "bf16" else TASC_F32, cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.n_kv_heads,
                     cfg.head_dim, cfg.d_ffn, cfg.vocab, max_pos, cfg.rope_theta, cfg.rms_eps)
    L = cfg.n_layers

    alive = []

    def arr(name):
        mats = [np.ascontiguousarray(weights["layers"][l][name]) for l in range(L)]
        alive.append(mats)                                   # the library copies during the call
        a = (C.c_void_p * L)(*[_ptr(m) for m in mats])
        return C.cast(a, C.POINTER(C.c_void_p)), a

    keep = {n: arr(n) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")}
    b = weights.get("bias")
    w = WeightPtrs(TASC_MEM_HOST, _ptr(weights["embed"]), _ptr(weights["lm_head"]), _ptr(weights["gf"]),
                   *[keep[n][0] for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")],
                   _ptr(b["rowptr"]) if b else None, _ptr(b["col"]) if b else None, _ptr(b["val"]) if b else None,
                   _ptr(b["base"]) if b else None)
    out = C.c_void_p()
    _check(lib().tasc_model_create(C.byref(desc), C.byref(w), C.byref(out)))
    return Model(out.value, desc)


class Session:
    def __init__(self, handle, model, batch, max_len, max_rows, kv_pool, workspace):
        self.handle, self.model, self.batch, self.max_len, self.max_rows = handle, model, batch, max_len, max_rows
        self._kv_pool, self._workspace = kv_pool, workspace     # keep the caller-owned buffers alive
        self._filters = self._filter_workspace = None           # what tasc_session_filter was given, and a workspace made there
        self._scratch = {}                                      # of sampled steps, by k and stream

    def close(self):
        if self.handle:
            lib().tasc_session_destroy(self.handle)
            self.handle = None

    __del__ = close


def tasc_session_kv_bytes(model: Model, batch, max_len) -> int:
    return lib().tasc_session_kv_bytes(model.handle, batch, max_len)


def tasc_session_workspace_bytes(model: Model, batch, max_len, max_rows) -> int:
    return lib().tasc_session_workspace_bytes(model.handle, batch, max_len, max_rows)


def tasc_session_create(model: Model, batch, max_len, max_rows) -> Session:
    """Allocates the KV pool and the workspace through PyTorch and hands them to the library."""
    import torch
    kvb = tasc_session_kv_bytes(model, batch, max_len)
    wsb = tasc_session_workspace_bytes(model, batch, max_len, max_rows)
    kv = torch.empty(kvb, dtype=torch.uint8, device="cuda")
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = C.c_void_p()
    _check(lib().tasc_session_create(model.handle, batch, max_len, max_rows, kv.data_ptr(), kvb, ws.data_ptr(), wsb, C.byref(out)))
    return Session(out.value, model, batch, max_len, max_rows, kv, ws)


def tasc_session_prefill(model: Model, s: Session, prompts, prompt_offsets, max_new, stream=None):
    prompt_offsets = np.ascontiguousarray(prompt_offsets, dtype=np.int64)
    _check(lib().tasc_session_prefill(model.handle, s.handle, _ptr(prompts), _ptr(prompt_offsets), _where(prompts), max_new,
                                      _stream(stream)))


def spec_params(k, lambda_q16=49152, p_min_ctx=1, ctx_includes_generated=1) -> SpecParams:
    return SpecParams(k, lambda_q16, p_min_ctx, ctx_includes_generated)


def tasc_draft(ng: Ngram, s: Session, params: SpecParams, drafts, stream=None):
    """drafts: cuda int32 tensor [batch, k], written in place."""
    _check(lib().tasc_draft(ng.handle, s.handle, C.byref(params), _ptr(drafts), _stream(stream)))


def tasc_verify_step(model: Model, s: Session, drafts, k, accept_len=None, emitted=None, logits_dbg=None, stream=None):
    _check(lib().tasc_verify_step(model.handle, s.handle, _ptr(drafts), k, _ptr(accept_len), _ptr(emitted), _ptr(logits_dbg),
                                  _stream(stream)))


def tasc_generate(model: Model, ng, s: Session, prompts, prompt_offsets, max_new, params: SpecParams, out_tokens,
                  trace=None, trace_steps=0, stream=None) -> GenStats:
    prompt_offsets = np.ascontiguousarray(prompt_offsets, dtype=np.int64)
    st = GenStats()
    _check(lib().tasc_generate(model.handle, ng.handle if ng is not None else None, s.handle, _ptr(prompts), _ptr(prompt_offsets),
                               _where(prompts), max_new, C.byref(params), _ptr(out_tokens), _ptr(trace), trace_steps, C.byref(st),
                               _stream(stream)))
    return st


def tasc_session_status(s: Session, stream=None) -> bool:
    """True if a persistent-kernel step of this session ran into a wait time-out since its last prefill."""
    flag = C.c_int32(0)
    _check(lib().tasc_session_status(s.handle, C.byref(flag), _stream(stream)))
    return bool(flag.value)


def tasc_session_get_tokens(s: Session, b: int, stream=None) -> np.ndarray:
    n = C.c_int32(0)
    buf = np.zeros(s.max_len, dtype=np.int32)
    _check(lib().tasc_session_get_tokens(s.handle, b, _ptr(buf), s.max_len, C.byref(n), _stream(stream)))
    return buf[:n.value].copy()


def tasc_profile_enable(classes):
    """classes: iterable of names from KERNEL_CLASSES (empty = off)."""
    mask = 0
    for c in classes:
        mask |= 1 << KERNEL_CLASSES.index(c)
    _check(lib().tasc_profile_enable(mask))


def tasc_profile_read():
    """Returns {class name: (total_ms, launches)} for the classes that recorded something, and clears."""
    n = len(KERNEL_CLASSES)
    ms = np.zeros(n, dtype=np.float64)
    cnt = np.zeros(n, dtype=np.int64)
    _check(lib().tasc_profile_read(_ptr(ms), _ptr(cnt)))
    return {KERNEL_CLASSES[i]: (float(ms[i]), int(cnt[i])) for i in range(n) if cnt[i]}


def tasc_profile_durations(cls_name) -> np.ndarray:
    """Durations (ms) of every recorded launch of one class, in launch order; call before tasc_profile_read."""
    cls = KERNEL_CLASSES.index(cls_name)
    n = C.c_int64(0)
    _check(lib().tasc_profile_durations(cls, None, 0, C.byref(n)))
    out = np.zeros(max(n.value, 1), dtype=np.float64)
    _check(lib().tasc_profile_durations(cls, _ptr(out), out.shape[0], C.byref(n)))
    return out[:n.value]


TASC_CFG_SMALL_PATH, TASC_CFG_SMALL_GRID, TASC_CFG_SMALL_LAYER_WGS, TASC_CFG_SMALL_LAYER_STRIDE, TASC_CFG_TILED_PATH = 0, 1, 2, 3, 4
TASC_CFG_SMALL_XCD_LOCAL = 5
TASC_CFG_SMALL_LAYER_WORKERS = 6
TASC_CFG_SMALL_KERNEL = 7
TASC_CFG_PIPE_SHARE = 8
TASC_CFG_CHAINS = 9
TASC_CFG_STEP_GRAPH = 10
TASC_CFG_BUILD_LIST_KIB = 11
TASC_CFG_KEEP_SCRATCH_KIB = 12
TASC_CFG_ENRICH_WAIT = 13


def tasc_config_set(key: int, value: int):
    _check(lib().tasc_config_set(key, value))


def tasc_profile_phases(buf):
    """buf: cuda int64/uint64 tensor (or None to turn the per-phase timestamps off)."""
    _check(lib().tasc_profile_phases(_ptr(buf), 0 if buf is None else buf.numel()))


def tasc_calibration_mfma(iters=2000, stream=None) -> float:
    out = C.c_double(0.0)
    _check(lib().tasc_calibration_mfma(iters, _stream(stream), C.byref(out)))
    return out.value


def tasc_calibration_read(src, passes=1, stream=None) -> float:
    """Read rate (GB/s) of a stream of independent 16-byte loads over the device tensor src (a multiple of 64 KB)."""
    out = C.c_double(0.0)
    _check(lib().tasc_calibration_read(_ptr(src), src.numel() * src.element_size(), passes, _stream(stream), C.byref(out)))
    return out.value


def tasc_calibration_gemm(M, N, K, epilogue=0, slices=1, iters=20, stream=None) -> float:
    """Microseconds per launch of the tiled GEMM at this shape (epilogue 0 store, 1 residual, 2 SwiGLU, 4 partial sums)."""
    out = C.c_double(0.0)
    _check(lib().tasc_calibration_gemm(M, N, K, epilogue, slices, iters, _stream(stream), C.byref(out)))
    return out.value


def tasc_calibration_handover(n_workgroups, stride, nbytes, with_flags=False, stream=None) -> float:
    """Microseconds per hand-over of nbytes among n_workgroups resident workgroups (ids stride * j)."""
    out = C.c_double(0.0)
    _check(lib().tasc_calibration_handover(n_workgroups, stride, nbytes, 1 if with_flags else 0, _stream(stream), C.byref(out)))
    return out.value


def tasc_calibration_copy(dst, src, stream=None):
    """dst, src: cuda uint8 tensors of equal size (a multiple of 16 bytes)."""
    _check(lib().tasc_calibration_copy(_ptr(dst), _ptr(src), src.numel() * src.element_size(), _stream(stream)))


# ---------------------------------------------------------------- the operators of a serving step over a 4-bit cache
# (A call's checks are a good part of what a small one takes, so they are few and cheap: a device array costs 0.5 us here.)
def _refuse(message):
    raise TascError(TASC_EINVAL, message)


def _array(who, name, t, dtype, shape, dev):
    """Address of a contiguous tensor of device `dev` with this dtype and shape."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _refuse(f"{who}: {name} is not a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{dev}, the current device")


def _list(who, name, t, dtype, dev):
    """(address, length) of a contiguous one-dimensional tensor of any length."""
    if getattr(t, "ndim", 0) != 1:
        _refuse(f"{who}: {name} is not a one-dimensional {dtype} tensor on cuda:{dev}")
    return _array(who, name, t, dtype, t.shape, dev), t.shape[0]


def _rows(who, name, t, dtypes, shape, dev):
    """(address, elements from row to row) of a tensor [rows, heads, head_dim] whose rows are each side by side."""
    try:
        if t.dtype in dtypes and t.shape == shape and t.get_device() == dev:
            if t.is_contiguous():
                return t.data_ptr(), shape[1] * shape[2]
            row, head, one = t.stride()
            if (one == 1 or shape[2] == 1) and (head == shape[2] or shape[1] == 1):
                return t.data_ptr(), row
    except AttributeError:
        pass
    _refuse(f"{who}: {name} is not a {' or '.join(str(d) for d in dtypes)} tensor of shape {tuple(shape)} on cuda:{dev} whose rows are each side by side")


def _here(stream):
    """(the current device, stream of the call, whether that is the current one)"""
    import torch
    try:
        dev = torch.cuda.current_device()
    except (RuntimeError, AssertionError) as e:
        raise TascError(TASC_EHIP, f"no device: {e}") from None
    current = torch._C._cuda_getCurrentRawStream(dev)      # (what torch.cuda.current_stream(dev).cuda_stream is, without an object for it)
    return dev, current if stream is None else stream, stream is None or stream == current


def _workspace(who, workspace, need, dev, on_current):
    """(tensor kept alive, address, bytes).  A workspace made here belongs to the current stream."""
    import torch
    if workspace is None:
        if need == 0:
            return None, None, 0
        if not on_current:
            _refuse(f"{who}: a call on a stream other than the current one needs a workspace of {need} bytes")
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    elif not isinstance(workspace, torch.Tensor) or workspace.get_device() != dev or not workspace.is_contiguous():
        _refuse(f"{who}: the workspace is not a contiguous tensor of the current device")
    return workspace, workspace.data_ptr() or None, workspace.numel() * workspace.element_size()


def tasc_page_tables(kv_len, new_rows, held, free_pages, table, pages=None, row_off=None, slots=None, summary=None, n_free=None, stream=None):
    """int32 cuda tensors: kv_len, new_rows, held, pages [batch], free_pages [n_free] (None: the pages 0 .. n_free - 1), table [batch, max_pages],
    row_off [batch + 1], slots [any], summary [3]; table, pages, row_off, slots and summary are written in place."""
    import torch
    who, i32 = "page_tables", torch.int32
    dev, st, _ = _here(stream)
    kv, B = _list(who, "kv_len", kv_len, i32, dev)
    if getattr(table, "ndim", 0) != 2 or table.shape[0] != B:
        _refuse(f"{who}: table is not [{B}, max_pages]")
    per = kv_len.shape
    free = n = cap = 0
    if free_pages is not None:
        free, n = _list(who, "free_pages", free_pages, i32, dev)
    if n_free is not None:
        if free_pages is not None and n_free > n:
            _refuse(f"{who}: n_free {n_free} of {n} free pages")
        n = n_free
    at = 0
    if slots is not None:
        at, cap = _list(who, "slots", slots, i32, dev)
    _check(lib().tasc_page_tables(
        kv, None if new_rows is None else _array(who, "new_rows", new_rows, i32, per, dev), None if held is None else _array(who, "held", held, i32, per, dev), B,
        free or None, n, _array(who, "table", table, i32, table.shape, dev), table.shape[1], None if pages is None else _array(who, "pages", pages, i32, per, dev),
        None if row_off is None else _array(who, "row_off", row_off, i32, (B + 1,), dev), at or None, cap,
        None if summary is None else _array(who, "summary", summary, i32, (3,), dev), st))


def _tables(who, table, pages, dev):
    """(address of the table, of pages, batch, max_pages)"""
    import torch
    at, B = _list(who, "pages", pages, torch.int32, dev)
    if getattr(table, "ndim", 0) != 2 or table.shape[0] != B:
        _refuse(f"{who}: table is not [{B}, max_pages]")
    return _array(who, "table", table, torch.int32, table.shape, dev), at, B, table.shape[1]


def tasc_pages_fork(src, dst, kv_len, table, pages, new_pages, copy_from, copy_to, summary=None, stream=None):
    """int32 cuda tensors: src, dst, new_pages (or None), copy_from, copy_to [pairs], kv_len, pages [batch], table [batch, max_pages], summary [3]; kv_len, table,
    pages, copy_from, copy_to and summary are written in place."""
    import torch
    who, i32 = "pages_fork", torch.int32
    dev, st, _ = _here(stream)
    s, n = _list(who, "src", src, i32, dev)
    tab, at, B, cols = _tables(who, table, pages, dev)
    per = src.shape
    _check(lib().tasc_pages_fork(s or None, _array(who, "dst", dst, i32, per, dev) or None, n, None if new_pages is None else _array(who, "new_pages", new_pages, i32, per, dev) or None,
                                 _array(who, "kv_len", kv_len, i32, pages.shape, dev), tab, at, B, cols, _array(who, "copy_from", copy_from, i32, per, dev) or None,
                                 _array(who, "copy_to", copy_to, i32, per, dev) or None, None if summary is None else _array(who, "summary", summary, i32, (3,), dev), st))


def tasc_pages_copy(pool, page_bytes, n_pages, n_layers, copy_from, copy_to, layer_stride=None, stream=None):
    """pool: contiguous cuda tensor that holds n_layers layers of n_pages pages of page_bytes bytes, layer_stride bytes from one to the next (None: one behind the
    other); copy_from, copy_to int32 [any]."""
    import torch
    who, i32 = "pages_copy", torch.int32
    dev, st, _ = _here(stream)
    at, n = _list(who, "copy_from", copy_from, i32, dev)
    stride = n_pages * page_bytes if layer_stride is None else layer_stride
    if not isinstance(pool, torch.Tensor) or pool.get_device() != dev or not pool.is_contiguous():
        _refuse(f"{who}: the pool is not a contiguous tensor on cuda:{dev}, the current device")
    if min(page_bytes, n_pages, n_layers, stride) < 0 or (n_layers > 0 and (n_layers - 1) * stride + n_pages * page_bytes > pool.numel() * pool.element_size()):
        _refuse(f"{who}: the pool does not hold {n_layers} layers of {n_pages} pages of {page_bytes} bytes")
    _check(lib().tasc_pages_copy(pool.data_ptr(), page_bytes, n_pages, n_layers, stride, at or None, _array(who, "copy_to", copy_to, i32, copy_from.shape, dev) or None, n, st))


def tasc_pages_workspace_bytes(n_pages) -> int:
    return lib().tasc_pages_workspace_bytes(n_pages)


def tasc_pages_free(table, pages, n_pages, free_pages, summary=None, workspace=None, stream=None):
    """int32 cuda tensors: table [batch, max_pages], pages [batch]; free_pages [n_pages] and summary [3] are written in place."""
    import torch
    who, i32 = "pages_free", torch.int32
    dev, st, on_current = _here(stream)
    tab, at, B, cols = _tables(who, table, pages, dev)
    keep, ws, n = _workspace(who, workspace, 0 if workspace is not None else tasc_pages_workspace_bytes(n_pages), dev, on_current)
    _check(lib().tasc_pages_free(tab, at, B, cols, n_pages, _array(who, "free_pages", free_pages, i32, (n_pages,), dev),
                                 None if summary is None else _array(who, "summary", summary, i32, (3,), dev), ws, n, st))


def tasc_pages_compact(table, pages, n_pages, table_out, copy_from, copy_to, summary=None, workspace=None, stream=None):
    """int32 cuda tensors: table [batch, max_pages], pages [batch]; table_out [batch, max_pages] (it may be table), copy_from, copy_to [most moves] and
    summary [3] are written in place."""
    import torch
    who, i32 = "pages_compact", torch.int32
    dev, st, on_current = _here(stream)
    tab, at, B, cols = _tables(who, table, pages, dev)
    frm, cap = _list(who, "copy_from", copy_from, i32, dev)
    keep, ws, n = _workspace(who, workspace, 0 if workspace is not None else tasc_pages_workspace_bytes(n_pages), dev, on_current)
    _check(lib().tasc_pages_compact(tab, at, B, cols, n_pages, _array(who, "table_out", table_out, i32, table.shape, dev), frm or None,
                                    _array(who, "copy_to", copy_to, i32, copy_from.shape, dev) or None, cap,
                                    None if summary is None else _array(who, "summary", summary, i32, (3,), dev), ws, n, st))


def tasc_kv4_page_bytes(n_kv_heads, head_dim) -> int:
    return lib().tasc_kv4_page_bytes(n_kv_heads, head_dim)


class Kv4Cache:
    """A paged 4-bit cache of one layer: `pool` (made here unless given, of n_pages * tasc_kv4_page_bytes bytes) and its shape."""

    def __init__(self, n_pages, n_kv_heads, head_dim, pool=None):
        import torch
        page = tasc_kv4_page_bytes(n_kv_heads, head_dim)
        if page == 0 or n_pages < 1:
            _refuse(f"Kv4Cache: {n_pages} pages of {n_kv_heads} KV heads of {head_dim} channels")
        if pool is None:
            pool = torch.empty(n_pages * page, dtype=torch.uint8, device="cuda")
        elif not pool.is_cuda or not pool.is_contiguous() or pool.numel() * pool.element_size() < n_pages * page:
            _refuse(f"Kv4Cache: the pool does not hold {n_pages} pages of {page} bytes")
        self.pool, self.n_pages, self.n_kv_heads, self.head_dim = pool, n_pages, n_kv_heads, head_dim
        self.device = pool.get_device()
        self.desc = Kv4CacheDesc(pool.data_ptr(), n_pages, n_kv_heads, head_dim)
        self.ref = C.byref(self.desc)

    def on(self, who, dev):
        if self.device != dev:
            _refuse(f"{who}: the cache is on cuda:{self.device}, the current device is cuda:{dev}")
        return self.ref


def tasc_kv4_append(cache: Kv4Cache, k, v, slots, stream=None):
    """k, v: cuda tensors [rows, n_kv_heads, head_dim], fp32 or bf16 (both alike), a row's elements side by side; slots: int32 [rows]."""
    import torch
    who = "kv4_append"
    dev, st, _ = _here(stream)
    at, rows = _list(who, "slots", slots, torch.int32, dev)
    shape, dtype = (rows, cache.n_kv_heads, cache.head_dim), getattr(k, "dtype", None)
    ka, ks = _rows(who, "k", k, (torch.float32, torch.bfloat16), shape, dev)
    va, vs = _rows(who, "v", v, (dtype,), shape, dev)
    _check(lib().tasc_kv4_append(cache.on(who, dev), ka, va, TASC_F32 if dtype is torch.float32 else TASC_BF16, ks, vs, at, rows, st))


def tasc_kv4_read(cache: Kv4Cache, slots, k, v, stream=None):
    """k, v: cuda tensors [rows, n_kv_heads, head_dim], fp32 or bf16 (both alike), written in place; slots: int32 [rows]."""
    import torch
    who, dtype = "kv4_read", getattr(k, "dtype", None)
    if dtype is not torch.float32 and dtype is not torch.bfloat16:
        _refuse(f"{who}: {dtype} is neither float32 nor bfloat16")
    dev, st, _ = _here(stream)
    at, rows = _list(who, "slots", slots, torch.int32, dev)
    shape = (rows, cache.n_kv_heads, cache.head_dim)
    _check(lib().tasc_kv4_read(cache.on(who, dev), at, rows, TASC_F32 if dtype is torch.float32 else TASC_BF16, _array(who, "k", k, dtype, shape, dev),
                               _array(who, "v", v, dtype, shape, dev), st))


def tasc_kv4_attention_workspace_bytes(batch, rows, n_heads, n_kv_heads, head_dim, max_rows, max_kv) -> int:
    """Of this call: a smaller one may need more.  2^18 * (head_dim + 2) bytes are enough for all with rows <= batch * max_rows."""
    return lib().tasc_kv4_attention_workspace_bytes(batch, rows, n_heads, n_kv_heads, head_dim, max_rows, max_kv)


def tasc_kv4_attention(cache: Kv4Cache, q, table, row_off, kv_len, max_rows, max_kv, scale, out, workspace=None, stream=None):
    """q, out: bf16 cuda tensors [rows, n_heads, head_dim], a row's elements side by side; table int32 [batch, max_pages], row_off int32
    [batch + 1], kv_len int32 [batch].  out is written in place."""
    import torch
    who, i32 = "kv4_attention", torch.int32
    dev, st, on_current = _here(stream)
    if getattr(q, "ndim", 0) != 3 or q.shape[2] != cache.head_dim:
        _refuse(f"{who}: queries are not [rows, n_heads, {cache.head_dim}]")
    shape = q.shape
    rows, H, hd = shape
    qa, qs = _rows(who, "q", q, (torch.bfloat16,), shape, dev)
    oa, os = _rows(who, "out", out, (torch.bfloat16,), shape, dev)
    kv, B = _list(who, "kv_len", kv_len, i32, dev)
    if getattr(table, "ndim", 0) != 2 or table.shape[0] != B:
        _refuse(f"{who}: table is not [{B}, max_pages]")
    a = Kv4Attn(qa, oa, qs, os, _array(who, "table", table, i32, table.shape, dev), _array(who, "row_off", row_off, i32, (B + 1,), dev), kv, table.shape[1], B, rows, H,
                max_rows, max_kv, scale)
    need = 0 if workspace is not None else tasc_kv4_attention_workspace_bytes(B, rows, H, cache.n_kv_heads, hd, max_rows, max_kv)
    keep, ws, n = _workspace(who, workspace, need, dev, on_current)
    _check(lib().tasc_kv4_attention(cache.on(who, dev), a, ws, n, st))


def tasc_accept_sampled_workspace_bytes(batch, k, vocab) -> int:
    return lib().tasc_accept_sampled_workspace_bytes(batch, k, vocab)


def tasc_accept_sampled(logits, drafts, draft_probs, temperature, u, accept_len, emitted, logprob=None, workspace=None, stream=None):
    """logits: fp32 or bf16 cuda tensor [batch, k + 1, vocab], its rows evenly spaced; drafts int32 [batch, k], draft_probs fp32 [batch, k, vocab]
    or None, temperature fp32 [batch] or None, u fp32 [batch, k + 1, 2]; accept_len int32 [batch], emitted int32 [batch, k + 1] and
    logprob fp32 [batch, k + 1] (or None) are written in place."""
    import torch
    who, f32, i32 = "accept_sampled", torch.float32, torch.int32
    dev, st, on_current = _here(stream)
    dtype = getattr(logits, "dtype", None)
    if (dtype is not f32 and dtype is not torch.bfloat16) or logits.ndim != 3 or logits.get_device() != dev:
        _refuse(f"{who}: logits are not a float32 or bfloat16 tensor [batch, k + 1, vocab] on cuda:{dev}, the current device")
    B, nq, V = logits.shape
    stride = V
    if not logits.is_contiguous():
        far, near, one = logits.stride()
        stride = near if nq > 1 else far if B > 1 else V
        if one != 1 or (B > 1 and far != nq * stride):
            _refuse(f"{who}: the rows of logits are not evenly spaced")
    per_row = (B, nq)
    need = 0 if workspace is not None else tasc_accept_sampled_workspace_bytes(B, nq - 1, V)
    keep, ws, n = _workspace(who, workspace, need, dev, on_current)
    _check(lib().tasc_accept_sampled(
        logits.data_ptr(), TASC_F32 if dtype is f32 else TASC_BF16, stride, B, nq - 1, V,
        None if drafts is None and nq == 1 else _array(who, "drafts", drafts, i32, (B, nq - 1), dev),
        None if draft_probs is None else _array(who, "draft_probs", draft_probs, f32, (B, nq - 1, V), dev),
        None if temperature is None else _array(who, "temperature", temperature, f32, (B,), dev), _array(who, "u", u, f32, (B, nq, 2), dev),
        _array(who, "accept_len", accept_len, i32, (B,), dev), _array(who, "emitted", emitted, i32, per_row, dev),
        None if logprob is None else _array(who, "logprob", logprob, f32, per_row, dev), ws, n, st))


def tasc_sample_workspace_bytes(rows, vocab) -> int:
    """For tasc_filter_logits, too, with rows = batch * (k + 1)."""
    return lib().tasc_sample_workspace_bytes(rows, vocab)


def _filters(who, temperature, top_k, top_p, min_p, shape, dev):
    import torch
    f32 = torch.float32
    return (None if temperature is None else _array(who, "temperature", temperature, f32, shape, dev),
            None if top_k is None else _array(who, "top_k", top_k, torch.int32, shape, dev),
            None if top_p is None else _array(who, "top_p", top_p, f32, shape, dev),
            None if min_p is None else _array(who, "min_p", min_p, f32, shape, dev))


def tasc_sample(logits, u, token, temperature=None, top_k=None, top_p=None, min_p=None, logprob=None, kept=None, workspace=None, stream=None):
    """logits: fp32 or bf16 cuda tensor [rows, vocab], a row's side by side; u fp32 [rows]; temperature, top_p, min_p fp32 and top_k int32 [rows], or None;
    token int32, logprob fp32 and kept int32 [rows] (the last two may be None) are written in place."""
    import torch
    who, f32, i32 = "sample", torch.float32, torch.int32
    dev, st, on_current = _here(stream)
    dtype = getattr(logits, "dtype", None)
    if (dtype is not f32 and dtype is not torch.bfloat16) or logits.ndim != 2 or logits.get_device() != dev:
        _refuse(f"{who}: logits are not a float32 or bfloat16 tensor [rows, vocab] on cuda:{dev}, the current device")
    rows, V = logits.shape
    stride = V
    if not logits.is_contiguous():
        far, one = logits.stride()
        stride = far if rows > 1 else V
        if one != 1:
            _refuse(f"{who}: the rows of logits are not side by side")
    per = (rows,)
    keep, ws, n = _workspace(who, workspace, 0 if workspace is not None else tasc_sample_workspace_bytes(rows, V), dev, on_current)
    _check(lib().tasc_sample(logits.data_ptr(), TASC_F32 if dtype is f32 else TASC_BF16, stride, rows, V, *_filters(who, temperature, top_k, top_p, min_p, per, dev),
                             _array(who, "u", u, f32, per, dev), _array(who, "token", token, i32, per, dev),
                             None if logprob is None else _array(who, "logprob", logprob, f32, per, dev),
                             None if kept is None else _array(who, "kept", kept, i32, per, dev), ws, n, st))


def _evenly(who, name, t, dtype, shape, dev):
    """(address, elements from row to row) of a tensor [batch, k + 1, vocab] whose rows are evenly spaced"""
    if getattr(t, "dtype", None) is not dtype or t.shape != shape or t.get_device() != dev:
        _refuse(f"{who}: {name} is not a {dtype} tensor [batch, k + 1, vocab] on cuda:{dev}, the current device")
    B, nq, V = shape
    if t.is_contiguous():
        return t.data_ptr(), V
    far, near, one = t.stride()
    stride = near if nq > 1 else far if B > 1 else V
    if one != 1 or (B > 1 and far != nq * stride):
        _refuse(f"{who}: the rows of {name} are not evenly spaced")
    return t.data_ptr(), stride


def tasc_filter_logits(logits, out, temperature=None, top_k=None, top_p=None, min_p=None, kept=None, workspace=None, stream=None):
    """logits, out: fp32 or bf16 cuda tensors [batch, k + 1, vocab] (both alike; they may be one), their rows evenly spaced; temperature, top_p, min_p fp32
    and top_k int32 [batch], or None; kept int32 [batch, k + 1] or None; out and kept are written in place."""
    import torch
    who, f32 = "filter_logits", torch.float32
    dev, st, on_current = _here(stream)
    dtype = getattr(logits, "dtype", None)
    if (dtype is not f32 and dtype is not torch.bfloat16) or logits.ndim != 3:
        _refuse(f"{who}: logits are not a float32 or bfloat16 tensor [batch, k + 1, vocab]")
    B, nq, V = shape = logits.shape
    at, stride = _evenly(who, "logits", logits, dtype, shape, dev)
    to, out_stride = _evenly(who, "out", out, dtype, shape, dev)
    keep, ws, n = _workspace(who, workspace, 0 if workspace is not None else tasc_sample_workspace_bytes(B * nq, V), dev, on_current)
    _check(lib().tasc_filter_logits(at, TASC_F32 if dtype is f32 else TASC_BF16, stride, B, nq - 1, V, *_filters(who, temperature, top_k, top_p, min_p, (B,), dev),
                                    to, out_stride, None if kept is None else _array(who, "kept", kept, torch.int32, (B, nq), dev), ws, n, st))


# ---------------------------------------------------------------- sessions that sample, sessions over a 4-bit cache
def tasc_session_kv4_bytes(model: Model, n_pages) -> int:
    return lib().tasc_session_kv4_bytes(model.handle, n_pages)


def tasc_session_create_kv4(model: Model, batch, max_len, max_rows, n_pages) -> Session:
    """A session over a 4-bit cache of n_pages pages a layer; allocates the pool and the workspace through PyTorch."""
    import torch
    kvb = tasc_session_kv4_bytes(model, n_pages)
    wsb = tasc_session_workspace_bytes(model, batch, max_len, max_rows)
    kv = torch.empty(max(kvb, 1), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(wsb, 1), dtype=torch.uint8, device="cuda")
    out = C.c_void_p()
    _check(lib().tasc_session_create_kv4(model.handle, batch, max_len, max_rows, n_pages, kv.data_ptr(), kvb, ws.data_ptr(), wsb, C.byref(out)))
    return Session(out.value, model, batch, max_len, max_rows, kv, ws)


def tasc_sampled_scratch_bytes(model: Model, batch, k) -> int:
    return lib().tasc_sampled_scratch_bytes(model.handle, batch, k)


def _sampling(who, model, s, k, u, temperature, scratch, dev, st):
    """(what must stay alive, struct).  A scratch made here comes from the memory of the call's stream, where nothing that is still to run can
    write to it, and stays with the session, one for every k and stream, as recorded steps do (a program that steps on many streams gives its own)."""
    import torch
    if s._kv_pool.get_device() != dev:
        _refuse(f"{who}: the session is on cuda:{s._kv_pool.get_device()}, the current device is cuda:{dev}")
    if getattr(u, "ndim", 0) != 3:
        _refuse(f"{who}: u is not [batch, pairs, 2]")
    if scratch is None:
        if (k, st) not in s._scratch:
            with torch.cuda.stream(torch.cuda.ExternalStream(st, device=dev) if st else torch.cuda.default_stream(dev)):
                s._scratch[k, st] = torch.empty(max(tasc_sampled_scratch_bytes(model, s.batch, k), 1), dtype=torch.uint8, device="cuda")
        scratch = s._scratch[k, st]
    elif not isinstance(scratch, torch.Tensor) or scratch.get_device() != dev or not scratch.is_contiguous():
        _refuse(f"{who}: the scratch is not a contiguous tensor of the current device")
    return scratch, Sampling(None if temperature is None else _array(who, "temperature", temperature, torch.float32, (s.batch,), dev),
                             _array(who, "u", u, torch.float32, (s.batch, u.shape[1], 2), dev), u.shape[1], scratch.data_ptr(),
                             scratch.numel() * scratch.element_size())


def tasc_verify_step_sampled(model: Model, s: Session, drafts, k, u, temperature=None, accept_len=None, emitted=None, logprob=None, scratch=None, stream=None):
    """u: fp32 cuda tensor [batch, pairs, 2], pair e for a sequence's generated token e; temperature fp32 [batch] or None; accept_len int32 [batch],
    emitted int32 [batch, k + 1] and logprob fp32 [batch, k + 1] (or None) are written in place."""
    import torch
    who, i32 = "verify_step_sampled", torch.int32
    dev, st, _ = _here(stream)
    keep, p = _sampling(who, model, s, k, u, temperature, scratch, dev, st)
    per_row = (s.batch, k + 1)
    _check(lib().tasc_verify_step_sampled(model.handle, s.handle, None if drafts is None and k == 0 else _array(who, "drafts", drafts, i32, (s.batch, k), dev), k, C.byref(p),
                                          None if accept_len is None else _array(who, "accept_len", accept_len, i32, (s.batch,), dev),
                                          None if emitted is None else _array(who, "emitted", emitted, i32, per_row, dev),
                                          None if logprob is None else _array(who, "logprob", logprob, torch.float32, per_row, dev), st))


def tasc_session_filter(s: Session, top_k=None, top_p=None, min_p=None, workspace=None):
    """From the next sampled step on: top_k int32, top_p and min_p fp32 cuda tensors [batch] or None (all None: no filters); the session keeps them.  A workspace
    made here serves steps of every k and stays with the session.  Steps on any stream may still use what was in its place, or the filters that the session had
    before: they are waited for, except where the same tensors are given again."""
    import torch
    who = "session_filter"
    dev, _, _ = _here(None)
    if s._kv_pool.get_device() != dev:
        _refuse(f"{who}: the session is on cuda:{s._kv_pool.get_device()}, the current device is cuda:{dev}")
    _, k, p, m = _filters(who, None, top_k, top_p, min_p, (s.batch,), dev)
    wait = False
    if workspace is None and (k or p or m):
        if s._filter_workspace is None:
            s._filter_workspace = torch.empty(tasc_sample_workspace_bytes(min(s.batch * min(s.max_rows, TASC_MAX_K + 1), 65535), s.model.desc.vocab), dtype=torch.uint8, device="cuda")
            wait = True
        workspace = s._filter_workspace
    keep, ws, n = _workspace(who, workspace, 0, dev, True)
    had, has = s._filters or (), (top_k, top_p, min_p, workspace)
    if wait or any(t is not None and all(t is not x for x in has) for t in had):
        if torch.cuda.is_current_stream_capturing():
            _refuse(f"{who}: a call that has to wait for earlier steps cannot be captured")
        torch.cuda.synchronize()
    _check(lib().tasc_session_filter(s.handle, k, p, m, ws, n))
    s._filters = has


def tasc_session_rewind(s: Session, stream=None):
    _check(lib().tasc_session_rewind(s.handle, _stream(stream)))


def tasc_generate_sampled(model: Model, ng, s: Session, prompts, prompt_offsets, max_new, params: SpecParams, u, out_tokens, temperature=None, scratch=None,
                          stream=None) -> GenStats:
    """As tasc_generate; u: fp32 cuda tensor [batch, pairs, 2] (pairs = max_new gives every token its own)."""
    import torch
    who = "generate_sampled"
    dev, st, _ = _here(stream)
    prompt_offsets = np.ascontiguousarray(prompt_offsets, dtype=np.int64)
    keep, p = _sampling(who, model, s, params.k, u, temperature, scratch, dev, st)
    stats = GenStats()
    _check(lib().tasc_generate_sampled(model.handle, ng.handle if ng is not None else None, s.handle, _ptr(prompts), _ptr(prompt_offsets), _where(prompts), max_new,
                                       C.byref(params), C.byref(p), _array(who, "out_tokens", out_tokens, torch.int32, (s.batch, max_new), dev), C.byref(stats), st))
    return stats
