"""Thin ctypes binding over libst.so: same names as include/st.h, argument marshalling only.

PyTorch supplies device memory (weights, KV cache, workspace) and the stream handle; every
step of the path runs in the library's HIP kernels.  Loading fails loudly when the library has
not been built -- there is no fallback.
"""
import ctypes as C
import os

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libst.so")

ST_OK, ST_EINVAL, ST_ENOMEM, ST_ERANGE, ST_EHIP = 0, -1, -2, -3, -4
ST_BF16, ST_F16, ST_F32 = 0, 1, 2
ST_PAIRS_HALVES, ST_PAIRS_NEIGHBOURS = 0, 1
ST_TOKENS_DEVICE, ST_OUT_DEVICE, ST_TOKEN_CHAINED, ST_PREFILL_TWO_TERM, ST_PREFILL_FAST = 1, 2, 4, 8, 16

EXPORTS = ("st_query_sizes", "st_prefill_plan_check", "st_prefill_plan_forms", "st_model_create", "st_model_destroy", "st_kv_len",
           "st_kv_truncate", "st_prefill", "st_query_f16_bytes", "st_model_attach_f16", "st_batch_attach_f16",
           "st_decode_step", "st_decode_graph_state", "st_decode_step_kind", "st_decode_persist_plan",
           "st_decode_step_timed", "st_decode_greedy", "st_trigger_scan", "st_trigger_scan_static", "st_handoff",
           "st_generate", "st_generate_policy", "st_batch_query_sizes", "st_batch_create", "st_batch_destroy",
           "st_batch_kv_len", "st_batch_truncate", "st_batch_prefill", "st_batch_prefill_many", "st_batch_decode_step",
           "st_generate_batch", "st_kv4_query_sizes", "st_kv4_create", "st_kv4_destroy", "st_kv4_append", "st_kv4_attend",
           "st_kv4_attend_plan", "st_kv4_evict", "st_kv4_read", "st_paged_query_sizes", "st_paged_create", "st_paged_destroy",
           "st_paged_append", "st_paged_attend", "st_paged_attend_plan", "st_paged_keep", "st_verify_query_sizes", "st_verify_create",
           "st_verify_destroy", "st_verify_drafts", "st_verify_drafts64", "st_last_error")


class StError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"st error {code}: {msg}")
        self.code = code


class st_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "intermediate", "vocab")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float)] + \
               [(n, C.c_int32) for n in ("tie_embeddings", "qkv_bias", "max_seq", "max_chunk")]


_vpp = C.POINTER(C.c_void_p)


class st_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p)] + \
               [(n, _vpp) for n in ("wqkv", "bqkv", "wo", "w_gate_up", "w_down", "norm_attn", "norm_mlp")]


class st_trigger_rule(C.Structure):
    _fields_ = [("kw_bitmap", C.c_void_p), ("delim_bitmap", C.c_void_p), ("window", C.c_int32), ("vocab", C.c_int32)]


class st_spans(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("large_prefill_lo", "large_prefill_hi", "large_decode_lo", "large_decode_hi",
                                         "small_prefill_lo", "small_prefill_hi")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class st_gen_stats(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_out", "n_handoffs", "n_large", "n_spans")] + \
               [(n, C.c_double) for n in ("ms_small_decode", "ms_large_decode", "ms_small_prefill", "ms_large_prefill")]


class st_kv4_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_seq", "n_q_heads", "n_kv_heads", "head_dim", "max_seq", "max_rows",
                                         "max_pos")] + [("rms_eps", C.c_float)]


class st_kv4_span(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("seq", "len", "pos", "rows")]


class st_kv4_ledger(C.Structure):
    _fields_ = [("weights", C.c_void_p), ("positions", C.c_void_p)]


class st_paged_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_seq", "n_q_heads", "n_kv_heads", "head_dim", "n_pages", "page_size", "max_pages",
                                         "max_rows", "max_pos", "dtype", "rot_dim", "rot_pairs")] + [("rms_eps", C.c_float)]


class st_draft_tree(C.Structure):
    _fields_ = [("parent", C.c_void_p), ("depth", C.c_void_p), ("sees", C.c_void_p), ("words", C.c_int32), ("width", C.c_int32)]


class st_verify_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("vocab", "dtype", "max_rows", "max_width")]


_lib = None


def lib():
    """The loaded library; raises if it has not been built (python -m paper_2504_12329_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_12329_amd.build`")
        L = C.CDLL(LIB_PATH)
        i32p, f32p = C.POINTER(C.c_int32), C.POINTER(C.c_float)
        L.st_last_error.restype = C.c_char_p
        L.st_query_sizes.argtypes = [C.POINTER(st_config), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.st_prefill_plan_check.argtypes = [C.POINTER(st_config), C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.st_prefill_plan_forms.argtypes = [C.POINTER(st_config), C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
        L.st_model_create.argtypes = [C.POINTER(st_config), C.POINTER(st_weights), C.c_void_p, C.c_size_t,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]
        L.st_model_destroy.argtypes = [C.c_void_p]
        L.st_model_destroy.restype = None
        L.st_kv_len.argtypes = [C.c_void_p, i32p]
        L.st_kv_truncate.argtypes = [C.c_void_p, C.c_int32]
        L.st_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_uint32]
        L.st_decode_step.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_uint32]
        L.st_decode_step_timed.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double)]
        L.st_decode_graph_state.argtypes = [C.c_void_p, i32p, i32p]
        L.st_decode_step_kind.argtypes = [C.c_void_p, i32p]
        L.st_decode_persist_plan.argtypes = [C.POINTER(st_config), C.c_int32, C.POINTER(C.c_size_t),
                                             C.POINTER(C.c_size_t), i32p, i32p]
        L.st_query_f16_bytes.argtypes = [C.POINTER(st_config), C.POINTER(C.c_size_t)]
        L.st_model_attach_f16.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
        L.st_batch_attach_f16.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
        L.st_decode_greedy.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_uint32]
        L.st_trigger_scan.argtypes = [C.POINTER(st_trigger_rule), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                      C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint32]
        L.st_trigger_scan_static.argtypes = [C.POINTER(st_trigger_rule), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                             C.c_int32, C.c_void_p, C.c_void_p]
        L.st_handoff.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, i32p, C.c_int32, C.c_int32, C.c_void_p,
                                 i32p, C.POINTER(st_spans), C.c_uint32]
        L.st_generate.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(st_trigger_rule), C.c_int32, C.c_void_p,
                                  C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(st_spans),
                                  C.c_int32, C.POINTER(st_gen_stats)]
        L.st_generate_policy.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(st_policy), C.c_void_p, C.c_int32, C.c_int32,
                                         C.c_void_p, C.c_void_p, C.POINTER(st_action), C.c_int32,
                                         C.POINTER(st_gen_stats)]
        L.st_batch_query_sizes.argtypes = [C.POINTER(st_config), C.c_int32, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.st_batch_create.argtypes = [C.POINTER(st_config), C.POINTER(st_weights), C.c_int32, C.c_void_p, C.c_size_t,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]
        L.st_batch_destroy.argtypes = [C.c_void_p]
        L.st_batch_destroy.restype = None
        L.st_batch_kv_len.argtypes = [C.c_void_p, C.c_int32, i32p]
        L.st_batch_truncate.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        L.st_batch_prefill.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        L.st_batch_decode_step.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.st_batch_prefill_many.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                            C.c_void_p]
        L.st_generate_batch.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_int32,
                                        C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                        C.POINTER(st_gen_stats)]
        spans, ledger = C.POINTER(st_kv4_span), C.POINTER(st_kv4_ledger)
        L.st_kv4_query_sizes.argtypes = [C.POINTER(st_kv4_config), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.st_kv4_create.argtypes = [C.POINTER(st_kv4_config), C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t,
                                    C.c_void_p, C.POINTER(C.c_void_p)]
        L.st_kv4_destroy.argtypes = [C.c_void_p]
        L.st_kv4_destroy.restype = None
        L.st_kv4_append.argtypes = [C.c_void_p, C.c_int32, spans, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_int64, ledger]
        L.st_kv4_attend.argtypes = [C.c_void_p, C.c_int32, spans, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                    ledger]
        L.st_kv4_attend_plan.argtypes = [C.POINTER(st_kv4_config), spans, C.c_int32, C.c_int32] + [C.POINTER(C.c_int32)] * 3
        L.st_kv4_evict.argtypes = [C.c_void_p, C.c_int32, C.c_int32, spans, C.c_int32, C.c_int32, C.c_int32, ledger, ledger]
        L.st_kv4_read.argtypes = [C.c_void_p, C.c_int32, C.c_int32, spans, C.c_int32, C.c_void_p, C.c_void_p]
        L.st_paged_query_sizes.argtypes = [C.POINTER(st_paged_config), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.st_paged_create.argtypes = [C.POINTER(st_paged_config), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t,
                                      C.c_void_p, C.POINTER(C.c_void_p)]
        L.st_paged_destroy.argtypes = [C.c_void_p]
        L.st_paged_destroy.restype = None
        L.st_paged_append.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_int64]
        L.st_paged_attend.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64]
        L.st_paged_attend_plan.argtypes = [C.POINTER(st_paged_config), C.c_void_p, C.c_int32, C.c_int32, i32p, i32p, i32p]
        L.st_paged_keep.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p]
        L.st_verify_query_sizes.argtypes = [C.POINTER(st_verify_config), C.POINTER(C.c_size_t)]
        L.st_verify_create.argtypes = [C.POINTER(st_verify_config), C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]
        L.st_verify_destroy.argtypes = [C.c_void_p]
        L.st_verify_destroy.restype = None
        L.st_verify_drafts.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        L.st_verify_drafts64.argtypes = L.st_verify_drafts.argtypes
        _lib = L
    return _lib


def _check(rc):
    if rc != ST_OK:
        raise StError(rc, lib().st_last_error().decode())


def make_config(cfg):
    return st_config(*(cfg[n] for n, _ in st_config._fields_))


def st_query_sizes(cfg):
    kv, ws = C.c_size_t(), C.c_size_t()
    _check(lib().st_query_sizes(C.byref(make_config(cfg)), C.byref(kv), C.byref(ws)))
    return kv.value, ws.value


def st_prefill_plan_check(cfg, rows):
    """Host-only walk over the launch plan of a catch-up pass of `rows` rows; returns (launches, blocks) of a layer."""
    nl, nb = C.c_int32(), C.c_int32()
    _check(lib().st_prefill_plan_check(C.byref(make_config(cfg)), int(rows), C.byref(nl), C.byref(nb)))
    return nl.value, nb.value


def st_prefill_plan_forms(cfg, rows, pos0, two_term=True):
    """Kernel forms of a pass of `rows` rows at position `pos0`: for QKV, O, gate/up and down ("stream", weight tiles per block,
    K slices), ("ring", tile widths F (256 weight rows), Q (192), H (128) or two of them, sliced tail, K slices) or None
    (general kernel); then the attention's waves per block (None at head_dim 64) and key ranges."""
    f = (C.c_int32 * 6)()
    _check(lib().st_prefill_plan_forms(C.byref(make_config(cfg)), int(rows), int(pos0), int(two_term), f))
    gemms = [None if not v else ("stream", v >> 16, v >> 8 & 255) if v >> 16 else
             ("ring", "F" * (v & 1) + "Q" * (v >> 3 & 1) + "H" * (v >> 1 & 1), bool(v & 4), v >> 8) for v in f[:4]]
    return gemms, {0: None, 1: 4, 2: 8}[f[4]], f[5]


def st_decode_persist_plan(cfg, n_cu):
    """Host-only plan of the single-kernel decode step: dict(lds_bytes, handover_words, regions[7], parts[5])."""
    lds, words = C.c_size_t(), C.c_size_t()
    regions, parts = (C.c_int32 * 7)(), (C.c_int32 * 5)()
    _check(lib().st_decode_persist_plan(C.byref(make_config(cfg)), int(n_cu), C.byref(lds), C.byref(words), regions, parts))
    return dict(lds_bytes=lds.value, handover_words=words.value, regions=list(regions), parts=list(parts))


def _np_ptr(a):
    return a.ctypes.data_as(C.c_void_p)


class TriggerRule:
    """Device bitmaps of the keyword and delimiter token sets."""

    def __init__(self, vocab, kw_bitmap, delim_bitmap=None, window=1, device="cuda"):
        self.kw = torch.from_numpy(np.ascontiguousarray(kw_bitmap).view(np.int32)).to(device)
        self.delim = None if delim_bitmap is None else \
            torch.from_numpy(np.ascontiguousarray(delim_bitmap).view(np.int32)).to(device)
        self.c = st_trigger_rule(self.kw.data_ptr(), 0 if self.delim is None else self.delim.data_ptr(), window, vocab)


def st_trigger_scan(rule, tokens_dev, lo, hi, cap, stream=None):
    """tokens_dev: int32 CUDA tensor.  Returns (total_count, positions ndarray)."""
    scratch = torch.empty(cap + 1, dtype=torch.int32, device=tokens_dev.device)
    pos = np.empty(max(cap, 1), dtype=np.int32)
    n = C.c_int32()
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    _check(lib().st_trigger_scan(C.byref(rule.c), tokens_dev.data_ptr(), lo, hi, _np_ptr(pos), cap, C.byref(n),
                                 scratch.data_ptr(), s, 0))
    return n.value, pos[:min(n.value, cap)].copy()


ST_SCAN_STATIC_MAX_CAP = 4096


def st_trigger_scan_static(rule, tokens_dev, lo, hi, cap, stream=None):
    """st_trigger_scan without a caller-provided device scratch (the library's own staging: pinned host memory the first
    call on a GPU allocates, nothing on the device).  Returns (total_count, positions ndarray)."""
    pos = np.empty(max(cap, 1), dtype=np.int32)
    n = C.c_int32()
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    _check(lib().st_trigger_scan_static(C.byref(rule.c), tokens_dev.data_ptr(), lo, hi, _np_ptr(pos), cap, C.byref(n), s))
    return n.value, pos[:min(n.value, cap)].copy()


def _pass_flags(two_term, fast):
    return (ST_PREFILL_TWO_TERM if two_term else 0) | (ST_PREFILL_FAST if fast else 0)


class Model:
    """st_model over torch-owned device buffers.  `weights` is the dict made by synth.make_weights on the GPU."""

    def __init__(self, cfg, weights, stream=None):
        self.cfg = dict(cfg)
        self.weights = weights                      # keeps the tensors alive
        dev = weights["embed"].device
        if dev.type != "cuda":
            raise RuntimeError("weights must live on the GPU")
        kv_bytes, ws_bytes = st_query_sizes(cfg)
        self.kv = torch.empty(kv_bytes, dtype=torch.uint8, device=dev)
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        L = cfg["n_layers"]
        w = st_weights()
        w.embed = weights["embed"].data_ptr()
        w.lm_head = 0 if weights.get("lm_head") is None else weights["lm_head"].data_ptr()
        w.final_norm = weights["final_norm"].data_ptr()
        self._arrays = []
        for name in ("wqkv", "bqkv", "wo", "w_gate_up", "w_down", "norm_attn", "norm_mlp"):
            arr = (C.c_void_p * L)(*[lw[name].data_ptr() for lw in weights["layers"]])
            self._arrays.append(arr)
            setattr(w, name, C.cast(arr, _vpp))
        self.stream = torch.cuda.current_stream(dev).cuda_stream if stream is None else stream
        h = C.c_void_p()
        _check(lib().st_model_create(C.byref(make_config(cfg)), C.byref(w), self.kv.data_ptr(), kv_bytes,
                                     self.ws.data_ptr(), ws_bytes, self.stream, C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().st_model_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:       # interpreter shutdown: the library wrapper may already be gone
            pass

    @property
    def kv_len(self):
        n = C.c_int32()
        _check(lib().st_kv_len(self._h, C.byref(n)))
        return n.value

    def truncate(self, n):
        _check(lib().st_kv_truncate(self._h, n))

    def prefill(self, tokens, want_logits=True, two_term=False, fast=False):
        """tokens: host int array; two_term: passes of at most 256 rows (ST_PREFILL_TWO_TERM); fast: single-bf16 GEMM
        inputs in passes of more than 128 rows (ST_PREFILL_FAST).  Returns (logits ndarray or None, greedy token)."""
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        lg = np.empty(self.cfg["vocab"], dtype=np.float32) if want_logits else None
        nt = C.c_int32()
        _check(lib().st_prefill(self._h, _np_ptr(t), t.size, _np_ptr(lg) if want_logits else None,
                                C.addressof(nt), _pass_flags(two_term, fast)))
        return lg, nt.value

    def prefill_device(self, tokens_dev, two_term=False, fast=False):
        """tokens_dev: int32 CUDA tensor; enqueues only (no outputs, no synchronisation)."""
        _check(lib().st_prefill(self._h, tokens_dev.data_ptr(), tokens_dev.numel(), None, None,
                                ST_TOKENS_DEVICE | ST_OUT_DEVICE | _pass_flags(two_term, fast)))

    def decode_step(self, token, want_logits=True):
        lg = np.empty(self.cfg["vocab"], dtype=np.float32) if want_logits else None
        nt = C.c_int32()
        _check(lib().st_decode_step(self._h, int(token), _np_ptr(lg) if want_logits else None, C.addressof(nt), 0))
        return lg, nt.value

    def attach_f16(self, on=True):
        """Gives the model an fp16 copy of its projection weights (torch-owned buffer): long default-precision passes
        then run on the fp16 MFMA with single fp16 activations.  on=False detaches and frees the buffer."""
        if not on:
            _check(lib().st_model_attach_f16(self._h, None, 0))
            self.f16_buf = None
            return
        n = C.c_size_t()
        _check(lib().st_query_f16_bytes(C.byref(make_config(self.cfg)), C.byref(n)))
        self.f16_buf = torch.empty(n.value, dtype=torch.uint8, device=self.kv.device)
        _check(lib().st_model_attach_f16(self._h, self.f16_buf.data_ptr(), n.value))

    def graph_state(self):
        """(step graphs captured so far, mode): mode 0 = graphs replayed, 1 = off by ST_NO_GRAPH, 2 = capture failed."""
        n, mode = C.c_int32(), C.c_int32()
        _check(lib().st_decode_graph_state(self._h, C.byref(n), C.byref(mode)))
        return n.value, mode.value

    def step_kind(self):
        """1 = the decode step is one persistent kernel, 0 = one kernel per stage."""
        k = C.c_int32()
        _check(lib().st_decode_step_kind(self._h, C.byref(k)))
        return k.value

    def decode_step_timed(self):
        """One chained step with per-launch events; returns (mean gate/up kernel us, whole step us)."""
        a, b = C.c_double(), C.c_double()
        _check(lib().st_decode_step_timed(self._h, C.byref(a), C.byref(b)))
        return a.value, b.value

    def decode_greedy(self, first_token, n, chained=False, out_dev=None):
        """n chained greedy steps.  Returns the tokens (host) unless out_dev (int32 CUDA tensor) is given."""
        flags = ST_TOKEN_CHAINED if chained else 0
        if out_dev is not None:
            _check(lib().st_decode_greedy(self._h, int(first_token), n, out_dev.data_ptr(), flags | ST_OUT_DEVICE))
            return None
        out = np.empty(n, dtype=np.int32)
        _check(lib().st_decode_greedy(self._h, int(first_token), n, _np_ptr(out), flags))
        return out


def st_handoff(small, large, seq, T, n_large, budget, want_logits=False):
    """seq: host int32 ndarray with room for the segment.  Returns (new_T, small_next_tok, spans dict, logits)."""
    t = C.c_int32(T)
    nt = C.c_int32(-1)
    sp = st_spans()
    lg = np.empty(small.cfg["vocab"], dtype=np.float32) if want_logits else None
    _check(lib().st_handoff(small._h, large._h, _np_ptr(seq), C.byref(t), n_large, budget,
                            _np_ptr(lg) if want_logits else None, C.byref(nt), C.byref(sp), 0))
    return t.value, nt.value, sp.as_dict(), lg


def st_generate(small, large, rule, prompt, n_out, n_seg, forced_period=0, span_cap=4096):
    """Runs the whole loop.  Returns dict(seq, src, spans, stats)."""
    p = np.ascontiguousarray(prompt, dtype=np.int32)
    seq = np.zeros(p.size + n_out, dtype=np.int32)
    src = np.zeros(max(n_out, 1), dtype=np.uint8)
    spans = (st_spans * max(span_cap, 1))()
    stats = st_gen_stats()
    _check(lib().st_generate(small._h, large._h, C.byref(rule.c) if rule is not None else None, forced_period,
                             _np_ptr(p), p.size, n_out, n_seg, _np_ptr(seq), _np_ptr(src),
                             C.cast(spans, C.POINTER(st_spans)), span_cap, C.byref(stats)))
    return dict(seq=seq[:p.size + stats.n_out], src=src[:stats.n_out],
                spans=[spans[i].as_dict() for i in range(stats.n_spans)],
                stats={n: getattr(stats, n) for n, _ in st_gen_stats._fields_})


class st_policy(C.Structure):
    _fields_ = [("delim_bitmap", C.c_void_p), ("ar_bitmap", C.c_void_p), ("verify_bitmap", C.c_void_p),
                ("neg_bitmap", C.c_void_p), ("vocab", C.c_int32), ("sentence_len", C.c_int32), ("n1", C.c_int32),
                ("n2", C.c_int32), ("n3", C.c_int32), ("neg_threshold", C.c_int32), ("aux_tokens", C.c_void_p),
                ("n_aux", C.c_int32), ("replace", C.c_int32), ("unconditional", C.c_int32),
                ("initial_target", C.c_int32)]


class st_action(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "sentence_end", "dropped", "aux_lo", "aux_hi", "granted")]


def host_bitmap(vocab, ids):
    """Host bitmap of `vocab` bits with the given token ids set (uint32 words, bit t of word t // 32)."""
    bm = np.zeros((vocab + 31) // 32, dtype=np.uint32)
    ids = np.asarray(list(ids), dtype=np.int64)
    np.bitwise_or.at(bm, ids >> 5, (np.uint32(1) << (ids & 31).astype(np.uint32)))
    return bm


def st_generate_policy(small, large, prompt, n_out, vocab, delim, sentence_len=1, ar=None, n1=20, verify=None, n2=125,
                       neg=None, neg_threshold=15, aux=(), n3=125, replace=False, unconditional=False,
                       initial_target=0, action_cap=4096):
    """Runs the full takeover policy; delim / ar / verify / neg are host bitmaps (see host_bitmap) or None.
    Returns dict(seq, src, actions, stats)."""
    p = np.ascontiguousarray(prompt, dtype=np.int32)
    seq = np.zeros(p.size + n_out, dtype=np.int32)
    src = np.zeros(max(n_out, 1), dtype=np.uint8)
    keep = [np.ascontiguousarray(b, dtype=np.uint32) if b is not None else None for b in (delim, ar, verify, neg)]
    auxa = np.ascontiguousarray(list(aux), dtype=np.int32)
    ptr = lambda a: a.ctypes.data if a is not None and a.size else None
    pol = st_policy(ptr(keep[0]), ptr(keep[1]), ptr(keep[2]), ptr(keep[3]), vocab, sentence_len, n1, n2, n3,
                    neg_threshold, ptr(auxa), auxa.size, int(replace), int(unconditional), initial_target)
    acts = (st_action * max(action_cap, 1))()
    stats = st_gen_stats()
    _check(lib().st_generate_policy(small._h, large._h, C.byref(pol), _np_ptr(p), p.size, n_out, _np_ptr(seq),
                                    _np_ptr(src), C.cast(acts, C.POINTER(st_action)), action_cap, C.byref(stats)))
    return dict(seq=seq[:p.size + stats.n_out], src=src[:stats.n_out],
                actions=[tuple(getattr(acts[i], n) for n, _ in st_action._fields_) for i in range(stats.n_spans)],
                stats={n: getattr(stats, n) for n, _ in st_gen_stats._fields_})


def _weights_struct(cfg, weights):
    """st_weights over the tensors of synth.make_weights; returns (struct, objects to keep alive)."""
    L = cfg["n_layers"]
    w = st_weights()
    w.embed = weights["embed"].data_ptr()
    w.lm_head = 0 if weights.get("lm_head") is None else weights["lm_head"].data_ptr()
    w.final_norm = weights["final_norm"].data_ptr()
    keep = []
    for name in ("wqkv", "bqkv", "wo", "w_gate_up", "w_down", "norm_attn", "norm_mlp"):
        arr = (C.c_void_p * L)(*[lw[name].data_ptr() for lw in weights["layers"]])
        keep.append(arr)
        setattr(w, name, C.cast(arr, _vpp))
    return w, keep


class Batch:
    """st_batch: n_seq independent sequences over one set of weights, torch-owned device buffers."""

    def __init__(self, cfg, weights, n_seq, stream=None):
        self.cfg, self.weights, self.n_seq = dict(cfg), weights, n_seq
        dev = weights["embed"].device
        if dev.type != "cuda":
            raise RuntimeError("weights must live on the GPU")
        kv, ws = C.c_size_t(), C.c_size_t()
        _check(lib().st_batch_query_sizes(C.byref(make_config(cfg)), n_seq, C.byref(kv), C.byref(ws)))
        self.kv = torch.empty(kv.value, dtype=torch.uint8, device=dev)
        self.ws = torch.empty(ws.value, dtype=torch.uint8, device=dev)
        w, self._arrays = _weights_struct(cfg, weights)
        self.stream = torch.cuda.current_stream(dev).cuda_stream if stream is None else stream
        h = C.c_void_p()
        _check(lib().st_batch_create(C.byref(make_config(cfg)), C.byref(w), n_seq, self.kv.data_ptr(), kv.value,
                                     self.ws.data_ptr(), ws.value, self.stream, C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().st_batch_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def kv_len(self, seq):
        n = C.c_int32()
        _check(lib().st_batch_kv_len(self._h, seq, C.byref(n)))
        return n.value

    def truncate(self, seq, n):
        _check(lib().st_batch_truncate(self._h, seq, n))

    def attach_f16(self):
        """fp16 copy of the shared projection weights (see Model.attach_f16)."""
        n = C.c_size_t()
        _check(lib().st_query_f16_bytes(C.byref(make_config(self.cfg)), C.byref(n)))
        self.f16_buf = torch.empty(n.value, dtype=torch.uint8, device=self.kv.device)
        _check(lib().st_batch_attach_f16(self._h, self.f16_buf.data_ptr(), n.value))

    def prefill(self, seq, tokens, want_logits=True):
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        lg = np.empty(self.cfg["vocab"], dtype=np.float32) if want_logits else None
        tok = C.c_int32()
        _check(lib().st_batch_prefill(self._h, seq, _np_ptr(t), t.size, _np_ptr(lg) if want_logits else None,
                                      C.byref(tok)))
        return lg, tok.value

    def prefill_many(self, seqs, token_lists, want_logits=False):
        """One ragged catch-up pass: token_lists[j] goes to sequence seqs[j].  Returns (logits [n][V] or None, next)."""
        s = np.ascontiguousarray(seqs, dtype=np.int32)
        ts = [np.ascontiguousarray(t, dtype=np.int32) for t in token_lists]
        lens = np.array([t.size for t in ts], dtype=np.int32)
        ptrs = (C.c_void_p * len(ts))(*[t.ctypes.data for t in ts])
        lg = np.empty((s.size, self.cfg["vocab"]), dtype=np.float32) if want_logits else None
        nxt = np.empty(s.size, dtype=np.int32)
        _check(lib().st_batch_prefill_many(self._h, s.size, _np_ptr(s), ptrs, _np_ptr(lens),
                                           _np_ptr(lg) if want_logits else None, _np_ptr(nxt)))
        return lg, nxt

    def decode_step(self, seqs, tokens, want_logits=False):
        s = np.ascontiguousarray(seqs, dtype=np.int32)
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        assert s.size == t.size
        lg = np.empty((s.size, self.cfg["vocab"]), dtype=np.float32) if want_logits else None
        nxt = np.empty(s.size, dtype=np.int32)
        _check(lib().st_batch_decode_step(self._h, s.size, _np_ptr(s), _np_ptr(t),
                                          _np_ptr(lg) if want_logits else None, _np_ptr(nxt)))
        return lg, nxt


class st_host_rule(C.Structure):
    _fields_ = [("kw_bitmap", C.c_void_p), ("delim_bitmap", C.c_void_p), ("window", C.c_int32), ("vocab", C.c_int32)]


def st_generate_batch(small, large, prompts, n_out, n_seg, vocab, kw=None, delim=None, window=1, forced_period=0,
                      forced_phase=None, gather=0):
    """The st_generate loop for len(prompts) sequences at once on two Batch objects; kw / delim are host bitmaps,
    forced_phase the per-sequence start of the forced-period count, gather the number of waiting sequences the
    target's passes are held for.  Returns dict(seqs, srcs, stats)."""
    n = len(prompts)
    ps = [np.ascontiguousarray(p, dtype=np.int32) for p in prompts]
    lens = np.array([p.size for p in ps], dtype=np.int32)
    seqs = [np.zeros(p.size + n_out, dtype=np.int32) for p in ps]
    srcs = [np.zeros(max(n_out, 1), dtype=np.uint8) for _ in ps]
    arr = lambda xs: (C.c_void_p * n)(*[x.ctypes.data for x in xs])
    kwa = None if kw is None else np.ascontiguousarray(kw, dtype=np.uint32)
    dla = None if delim is None else np.ascontiguousarray(delim, dtype=np.uint32)
    rule = st_host_rule(None if kwa is None else kwa.ctypes.data, None if dla is None else dla.ctypes.data, window, vocab)
    stats = st_gen_stats()
    phase = None if forced_phase is None else np.ascontiguousarray(forced_phase, dtype=np.int32)
    _check(lib().st_generate_batch(small._h, large._h, C.byref(rule) if kwa is not None else None, forced_period,
                                   None if phase is None else _np_ptr(phase), gather, n,
                                   arr(ps), _np_ptr(lens), n_out, n_seg, arr(seqs), arr(srcs), C.byref(stats)))
    return dict(seqs=seqs, srcs=srcs, stats={k: getattr(stats, k) for k, _ in st_gen_stats._fields_})


def _fits32(what, *numbers):
    """ctypes cuts numbers down to 32 bits without a word."""
    if min(numbers) < -2 ** 31 or max(numbers) >= 2 ** 31:
        raise StError(ST_ERANGE, f"{what}: {numbers} does not fit 32 bits")


class Kv4Spans:
    """The spans of a call, (seq, len, pos, rows) each (see st_kv4_span); made once for all layers of a step."""

    def __init__(self, spans):
        self.spans = [tuple(int(x) for x in s) for s in spans]
        if self.spans:
            _fits32("spans", min(map(min, self.spans)), max(map(max, self.spans)))
        self.n, self.rows = len(self.spans), sum(s[3] for s in self.spans)
        self.c = (st_kv4_span * max(self.n, 1))(*self.spans)


class Kv4Ledger:
    """Accumulated attention weights (float32) and positions (int32), CUDA tensors [layer][sequence][kv head][max_seq]."""

    def __init__(self, weights, positions):
        if weights.dtype != torch.float32 or positions.dtype != torch.int32:
            raise StError(ST_EINVAL, f"weights are float32 and positions int32, got {weights.dtype} and {positions.dtype}")
        if weights.shape != positions.shape or not weights.is_contiguous() or not positions.is_contiguous():
            raise StError(ST_EINVAL, "weights and positions are contiguous and of one shape")
        if not weights.is_cuda or positions.device != weights.device:
            raise StError(ST_EINVAL, "weights and positions must live on one GPU")
        self.weights, self.positions = weights, positions
        self.shape, self.device = tuple(weights.shape), weights.device
        self.c = st_kv4_ledger(weights.data_ptr(), positions.data_ptr())
        self.ref = C.byref(self.c)


def rope_table(max_pos, head_dim, theta, device="cuda"):
    """(cos, sin) of every position and rotation pair, float32 [max_pos][head_dim / 2][2], computed in 64 bits."""
    i = torch.arange(head_dim // 2, dtype=torch.float64, device=device)
    a = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] * theta ** (-2 * i / head_dim)
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


class Kv4Cache:
    """st_kv4 over torch-owned device buffers: a key/value cache held in 4 bits, with append, attend, evict and read.

    cfg: dict of the fields of st_kv4_config.  Without `stream` the calls enqueue on the stream that was current when the cache was made, and are
    refused under another one.  With it (a raw handle) ordering other streams' work against the calls is the caller's part."""

    def __init__(self, cfg, rope, cache=None, stream=None):
        self.cfg = dict(cfg)
        _fits32("config", *(cfg[n] for n, t in st_kv4_config._fields_ if t is C.c_int32))
        c = st_kv4_config(*(cfg[n] for n, _ in st_kv4_config._fields_))
        cb, wb = C.c_size_t(), C.c_size_t()
        _check(lib().st_kv4_query_sizes(C.byref(c), C.byref(cb), C.byref(wb)))
        if not rope.is_cuda or rope.dtype != torch.float32 or not rope.is_contiguous() or \
                tuple(rope.shape) != (cfg["max_pos"], cfg["head_dim"] // 2, 2):
            raise StError(ST_EINVAL, f"rope is a contiguous float32 CUDA tensor [max_pos][head_dim / 2][2], got {rope.dtype} {tuple(rope.shape)}")
        dev = rope.device           # (with its index)
        self._own_stream = stream is not None
        self.stream = torch.cuda.current_stream(dev).cuda_stream if stream is None else stream
        # what is allocated here belongs to the stream that uses it: freed, it does not go to another one while calls are still running
        on = torch.cuda.ExternalStream(self.stream, device=dev) if self._own_stream else torch.cuda.current_stream(dev)
        with torch.cuda.stream(on):
            self._ws = torch.empty(wb.value, dtype=torch.uint8, device=dev)
            if cache is None:
                cache = torch.empty(cb.value, dtype=torch.uint8, device=dev)
        if cache.device != dev or cache.dtype != torch.uint8 or not cache.is_contiguous():
            raise StError(ST_EINVAL, "cache is a contiguous uint8 tensor on the device of rope")
        self.cache, self.rope, self._dev, self._index = cache, rope, dev, dev.index
        h = C.c_void_p()
        _check(lib().st_kv4_create(C.byref(c), rope.data_ptr(), cache.data_ptr(), cache.numel(), self._ws.data_ptr(),
                                   wb.value, self.stream, C.byref(h)))
        self._h = h
        self._slots = (cfg["n_layers"], cfg["n_seq"], cfg["n_kv_heads"], cfg["max_seq"])
        self._nq, self._nkv, self._d = cfg["n_q_heads"], cfg["n_kv_heads"], cfg["head_dim"]
        self._new = torch.empty(0, dtype=torch.bfloat16, device=dev).new_empty
        L = lib()
        self._append, self._attend, self._evict, self._read = L.st_kv4_append, L.st_kv4_attend, L.st_kv4_evict, L.st_kv4_read

    def close(self):
        if getattr(self, "_h", None):
            lib().st_kv4_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # A decode step makes these calls for every layer, so the checks below stay at a few attribute reads.
    def _alloc(self, *shape):
        if not self._own_stream:
            return self._new(*shape)
        with torch.cuda.stream(torch.cuda.ExternalStream(self.stream, device=self._dev)):
            return self._new(*shape)

    def _elsewhere(self):
        """Whether another GPU than the cache's is current: a launch would go there, whichever GPU its pointers are on."""
        if not self._own_stream and torch._C._cuda_getCurrentRawStream(self._index) != self.stream:
            raise StError(ST_EINVAL, "called under another stream than the cache was made on")
        return torch._C._cuda_getDevice() != self._index

    def _matrix(self, name, x, rows, heads):
        """(pointer, row stride) of bf16 [rows][heads][head_dim] or [rows][heads * head_dim]; rows may be strided."""
        d, shape = self._d, x.shape
        if x.dtype is not torch.bfloat16 or x.get_device() != self._index:
            raise StError(ST_EINVAL, f"{name} is bfloat16 on {self._dev}, got {x.dtype} on {x.device}")
        if x.is_contiguous() and (shape == (rows, heads, d) or shape == (rows, heads * d)):
            return x.data_ptr(), heads * d
        stride = x.stride()
        if not (shape == (rows, heads * d) and stride[1] == 1 or
                shape == (rows, heads, d) and stride[2] == 1 and (stride[1] == d or heads == 1)):
            raise StError(ST_EINVAL, f"{name} has shape {tuple(shape)} and strides {stride}, needs {rows} rows of {heads} x {d}")
        return x.data_ptr(), stride[0] if rows > 1 else max(stride[0], heads * d)

    def _ledger(self, ledger):
        if ledger is None:
            return None
        if ledger.shape != self._slots:
            raise StError(ST_EINVAL, f"the ledger has shape {ledger.shape}, needs {self._slots}")
        if ledger.device != self._dev:
            raise StError(ST_EINVAL, f"the ledger is on {ledger.device}, the cache on {self._dev}")
        return ledger.ref

    def append(self, layer, spans, qkv, q_norm=None, k_norm=None, ledger=None):
        """Norms (bf16 [head_dim], or None), rotation and the write of the spans' new rows; qkv: bf16, a row per new token, all query
        heads, then key heads, then value heads.  Returns the rotated queries, bf16 [rows][n_q_heads][head_dim]."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.append(layer, spans, qkv, q_norm, k_norm, ledger)
        p, stride = self._matrix("qkv", qkv, spans.rows, self._nq + 2 * self._nkv)
        qn = kn = None
        if q_norm is not None or k_norm is not None:
            qn, kn = self._norm("q_norm", q_norm), self._norm("k_norm", k_norm)
        out = self._alloc(spans.rows, self._nq, self._d)
        if spans.rows:
            if not 0 <= layer < self._slots[0]:
                raise StError(ST_ERANGE, f"layer {layer} outside [0, {self._slots[0]})")
            rc = self._append(self._h, layer, spans.c, spans.n, p, stride, qn, kn, out.data_ptr(), self._nq * self._d, self._ledger(ledger))
            if rc:
                _check(rc)
        return out

    def _norm(self, name, w):
        if w is None:
            return None
        if w.dtype is not torch.bfloat16 or w.shape != (self._d,) or not w.is_contiguous() or w.get_device() != self._index:
            raise StError(ST_EINVAL, f"{name} is bfloat16 [{self._d}] on {self._dev}, got {w.dtype} {tuple(w.shape)}")
        return w.data_ptr()

    def attend(self, layer, spans, q, ledger=None, out=None):
        """Attention of the spans' rows over their sequences' slots; q: bf16, n_q_heads * head_dim a row.  With a ledger its weights grow by what every
        slot received.  Returns bf16 [rows][n_q_heads][head_dim] (or `out`)."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.attend(layer, spans, q, ledger, out)
        p, stride = self._matrix("q", q, spans.rows, self._nq)
        if out is None:
            out = self._alloc(spans.rows, self._nq, self._d)
            po, so = out.data_ptr(), self._nq * self._d
        else:
            po, so = self._matrix("out", out, spans.rows, self._nq)
        if spans.rows:
            if not 0 <= layer < self._slots[0]:
                raise StError(ST_ERANGE, f"layer {layer} outside [0, {self._slots[0]})")
            rc = self._attend(self._h, layer, spans.c, spans.n, p, stride, po, so, self._ledger(ledger))
            if rc:
                _check(rc)
        return out

    def attend_plan(self, spans, with_ledger=False):
        """(columns of a block, blocks, key ranges of every span) of such an attend (see st_kv4_attend_plan)."""
        c = st_kv4_config(*(self.cfg[n] for n, _ in st_kv4_config._fields_))
        columns, blocks, ranges = C.c_int32(), C.c_int32(), (C.c_int32 * max(spans.n, 1))()
        _check(lib().st_kv4_attend_plan(C.byref(c), spans.c, spans.n, int(with_ledger), C.byref(columns), C.byref(blocks), ranges))
        return columns.value, blocks.value, list(ranges)[:spans.n]

    def evict(self, layer_lo, layer_hi, spans, keep, recent, ledger, into=None):
        """Brings the spans' sequences to `keep` slots in layers [layer_lo, layer_hi) (see st_kv4_evict); the ledger's entries move along, in place or to `into`."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.evict(layer_lo, layer_hi, spans, keep, recent, ledger, into)
        if (layer_lo | layer_hi | keep | recent) >> 31:     # one of them is negative, or large
            _fits32("evict", layer_lo, layer_hi, keep, recent)
        _check(self._evict(self._h, layer_lo, layer_hi, spans.c, spans.n, keep, recent, self._ledger(ledger), self._ledger(into)))

    def read(self, layer_lo, layer_hi, spans):
        """Slots [len, len + rows) of the spans as bf16 (k, v), each [layers][rows][n_kv_heads][head_dim]."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.read(layer_lo, layer_hi, spans)
        if (layer_lo | layer_hi) >> 31:
            _fits32("read", layer_lo, layer_hi)
        layers = max(layer_hi - layer_lo, 0)
        k = self._alloc(layers, spans.rows, self._nkv, self._d)
        v = self._alloc(layers, spans.rows, self._nkv, self._d)
        if layers and spans.rows:
            _check(self._read(self._h, layer_lo, layer_hi, spans.c, spans.n, k.data_ptr(), v.data_ptr()))
        return k, v


class DraftSpans(Kv4Spans):
    """Spans whose rows are the last decided token and drafts after it: parents[j][i] is the row of span j that its row i follows, before it
    (parents[j][0] is not read).  Made once for all layers of a step, and moved to the next one's places by at(); a branch's rows see each other and
    the context, and a row's position is the span's pos and the number of rows before it in its branch."""

    def __init__(self, spans, parents, device="cuda"):
        super().__init__(spans)
        if len(parents) != self.n or any(len(p) != s[3] for p, s in zip(parents, self.spans)):
            raise StError(ST_EINVAL, "parents holds a list for every span, with an entry for every row")
        most = max([s[3] for s in self.spans], default=0)
        if most > 1024:
            raise StError(ST_ERANGE, f"{most} rows of a span, trees have at most 1024")
        words = max(1, -(-most // 64))
        parent, depth, masks, width, deepest = [], [], [], 1, []
        for ps in parents:
            ps = [-1, *map(int, ps[1:])][:len(ps)]
            d, m, after = [0] * len(ps), [1] * len(ps), [0] * len(ps)
            for i, p in enumerate(ps):
                if i:
                    if not 0 <= p < i:
                        raise StError(ST_EINVAL, f"row {i} follows row {p}: not a row before it")
                    d[i], m[i] = d[p] + 1, m[p] | 1 << i
                    after[p] += 1
            parent += ps
            depth += d
            masks += m
            width = max(width, *after, 1)
            deepest.append(max(d, default=-1))
        if width > 64:
            raise StError(ST_ERANGE, f"{width} rows follow one row, at most 64 are supported")
        if words > 1:
            masks = [m >> 64 * w & 2 ** 64 - 1 for m in masks for w in range(words)]
        parent, depth, sees = np.array(parent, dtype=np.int32), np.array(depth, dtype=np.int32), np.array(masks, dtype=np.uint64)
        n = self.rows
        bits = torch.from_numpy(np.concatenate([sees.view(np.int32), parent, depth])).to(device)     # (one copy)
        self._take(bits[2 * n * words:2 * n * words + n], bits[2 * n * words + n:], bits[:2 * n * words].view(torch.int64).view(n, words) if n else bits.new_empty((0, words), dtype=torch.int64), width, deepest)

    def at(self, spans):
        """The same trees at other places: spans of as many rows each, as a step later."""
        other = DraftSpans.__new__(DraftSpans)
        Kv4Spans.__init__(other, spans)
        if [s[3] for s in other.spans] != [s[3] for s in self.spans]:
            raise StError(ST_EINVAL, "the spans have other numbers of rows than the trees")
        other._take(self.parent, self.depth, self.sees, self.width, self.deepest)
        return other

    @classmethod
    def of_tensors(cls, spans, parent=None, depth=None, sees=None, width=1):
        """From tensors on the GPU, for trees that are made there: parent and depth int32 [rows], sees int64 [rows][words] (see st_draft_tree); a call that
        reads one that is None is refused.  Depths past the rotation table are not seen here, and are cut to it (see st_paged_append)."""
        self = cls.__new__(cls)
        Kv4Spans.__init__(self, spans)
        for name, x, t, dims in (("parent", parent, torch.int32, 1), ("depth", depth, torch.int32, 1), ("sees", sees, torch.int64, 2)):
            if x is not None and (x.dtype != t or x.dim() != dims or x.shape[0] != self.rows or not x.is_contiguous() or not x.is_cuda):
                raise StError(ST_EINVAL, f"{name} is a contiguous {t} CUDA tensor of {self.rows} rows, got {x.dtype} {tuple(x.shape)} on {x.device}")
        self._take(parent, depth, sees, int(width))
        return self

    def _take(self, parent, depth, sees, width, deepest=None):
        self.parent, self.depth, self.sees, self.width, self.deepest = parent, depth, sees, width, deepest
        self.positions = 0 if deepest is None else max((s[2] + d + 1 for s, d in zip(self.spans, deepest)), default=0)  # that the rows need of a rotation table
        ptr = lambda x: None if x is None else x.data_ptr()  # noqa: E731
        self._tree = st_draft_tree(ptr(parent), ptr(depth), ptr(sees), 1 if sees is None else sees.shape[1], width)
        self.tree = C.byref(self._tree)
        self.devices = {x.device for x in (parent, depth, sees) if x is not None}


class _OnStream:
    """Calls that enqueue on one stream of one GPU: the stream that was current when the object was made (they are refused under another one), or a
    raw handle, where ordering other streams' work against them is the caller's part."""

    def _bind(self, dev, stream):
        self._own_stream = stream is not None
        self.stream = torch.cuda.current_stream(dev).cuda_stream if stream is None else stream
        self._dev, self._index = dev, dev.index
        with self._on():
            self._new = torch.empty(0, dtype=torch.uint8, device=dev).new_empty

    def _on(self):
        # what is allocated belongs to the stream that uses it: freed, it does not go to another one while calls are still running
        return torch.cuda.stream(torch.cuda.ExternalStream(self.stream, device=self._dev) if self._own_stream else torch.cuda.current_stream(self._dev))

    def _empty(self, shape, dtype):
        if not self._own_stream:
            return self._new(shape, dtype=dtype)
        with self._on():
            return self._new(shape, dtype=dtype)

    def _elsewhere(self):
        """Whether another GPU is current: a launch would go there, whichever GPU its pointers are on."""
        if not self._own_stream and torch._C._cuda_getCurrentRawStream(self._index) != self.stream:
            raise StError(ST_EINVAL, "called under another stream than it was made on")
        return torch._C._cuda_getDevice() != self._index

    def _tree_of(self, spans):
        if not isinstance(spans, DraftSpans):
            return None
        if not all(d == self._dev for d in spans.devices):
            raise StError(ST_EINVAL, f"the tree of the spans is on {spans.devices}, the call on {self._dev}")
        return spans.tree

    def close(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_TYPE_OF = {torch.bfloat16: ST_BF16, torch.float16: ST_F16, torch.float32: ST_F32}
_PAIRS_OF = {"halves": ST_PAIRS_HALVES, "neighbours": ST_PAIRS_NEIGHBOURS}


def _device_of(device):
    dev = torch.device(device)
    if dev.type != "cuda":
        raise StError(ST_EINVAL, f"needs a GPU, got {dev}")
    return dev if dev.index is not None else torch.device("cuda", torch.cuda.current_device())


class PagedCache(_OnStream):
    """st_paged over torch-owned device buffers: a key/value cache in pages, with append, attend and keep for chains, chunks and trees of drafts.

    cfg: dict of the fields of st_paged_config, dtype a torch type (bfloat16 or float16), rot_dim head_dim where it is not given, rot_pairs "halves" (the
    default) or "neighbours".  table: int32 [n_seq][max_pages], read when a call runs (its entries may change, the tensor is kept).  cache: [2][n_layers]
    [n_pages][n_kv_heads][page_size][head_dim]; allocated here if it is not given."""

    def __init__(self, cfg, rope, table, cache=None, stream=None):
        cfg = dict(dict(rot_dim=cfg["head_dim"], rot_pairs="halves", dtype=torch.bfloat16), **cfg)
        if cfg["dtype"] not in (torch.bfloat16, torch.float16):
            raise StError(ST_EINVAL, f"dtype is bfloat16 or float16, got {cfg['dtype']}")
        if cfg["rot_pairs"] not in _PAIRS_OF:
            raise StError(ST_EINVAL, f"rot_pairs is 'halves' or 'neighbours', got {cfg['rot_pairs']!r}")
        self.cfg, self.dtype = cfg, cfg["dtype"]
        numbers = dict(cfg, dtype=_TYPE_OF[cfg["dtype"]], rot_pairs=_PAIRS_OF[cfg["rot_pairs"]])
        _fits32("config", *(numbers[n] for n, t in st_paged_config._fields_ if t is C.c_int32))
        self._c = st_paged_config(*(numbers[n] for n, _ in st_paged_config._fields_))
        cb, wb = C.c_size_t(), C.c_size_t()
        _check(lib().st_paged_query_sizes(C.byref(self._c), C.byref(cb), C.byref(wb)))
        shape = (2, cfg["n_layers"], cfg["n_pages"], cfg["n_kv_heads"], cfg["page_size"], cfg["head_dim"])
        if not table.is_cuda or table.dtype != torch.int32 or not table.is_contiguous() or tuple(table.shape) != (cfg["n_seq"], cfg["max_pages"]):
            raise StError(ST_EINVAL, f"table is a contiguous int32 CUDA tensor [n_seq][max_pages], got {table.dtype} {tuple(table.shape)}")
        dev = table.device
        if cfg["rot_dim"] and (rope is None or rope.device != dev or rope.dtype != torch.float32 or not rope.is_contiguous() or
                               tuple(rope.shape) != (cfg["max_pos"], cfg["rot_dim"] // 2, 2)):
            raise StError(ST_EINVAL, "rope is a contiguous float32 tensor [max_pos][rot_dim / 2][2] on the device of table")
        self._bind(dev, stream)
        self._ws = self._empty((wb.value,), torch.uint8)
        if cache is None:
            cache = self._empty(shape, self.dtype)
        if cache.device != dev or cache.dtype != self.dtype or not cache.is_contiguous() or tuple(cache.shape) != shape:
            raise StError(ST_EINVAL, f"cache is a contiguous {self.dtype} tensor {shape} on the device of table, got {cache.dtype} {tuple(cache.shape)} on {cache.device}")
        self.cache, self.rope, self.table = cache, rope, table
        h = C.c_void_p()
        _check(lib().st_paged_create(C.byref(self._c), rope.data_ptr() if cfg["rot_dim"] else None, table.data_ptr(), cache.data_ptr(),
                                     cache.numel() * 2, self._ws.data_ptr(), wb.value, self.stream, C.byref(h)))
        L = lib()
        self._h, self._destroy = h, L.st_paged_destroy
        self._append, self._attend, self._keep = L.st_paged_append, L.st_paged_attend, L.st_paged_keep
        self._nq, self._nkv, self._d, self._layers = cfg["n_q_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["n_layers"]
        self._positions = cfg["max_pos"] if cfg["rot_dim"] else 2 ** 31      # of a tree's rows

    def _matrix(self, name, x, rows, heads):
        """(pointer, row stride) of [rows][heads][head_dim] or [rows][heads * head_dim]; rows may be strided."""
        d, shape = self._d, x.shape
        if x.dtype is not self.dtype or x.get_device() != self._index:
            raise StError(ST_EINVAL, f"{name} is {self.dtype} on {self._dev}, got {x.dtype} on {x.device}")
        if x.is_contiguous() and (shape == (rows, heads, d) or shape == (rows, heads * d)):
            return x.data_ptr(), heads * d
        stride = x.stride()
        if not (shape == (rows, heads * d) and stride[1] == 1 or
                shape == (rows, heads, d) and stride[2] == 1 and (stride[1] == d or heads == 1)):
            raise StError(ST_EINVAL, f"{name} has shape {tuple(shape)} and strides {stride}, needs {rows} rows of {heads} x {d}")
        return x.data_ptr(), stride[0] if rows > 1 else heads * d

    def _norm(self, name, w):
        if w is None:
            return None
        if w.dtype is not self.dtype or w.shape != (self._d,) or not w.is_contiguous() or w.get_device() != self._index:
            raise StError(ST_EINVAL, f"{name} is {self.dtype} [{self._d}] on {self._dev}, got {w.dtype} {tuple(w.shape)}")
        return w.data_ptr()

    def _layer(self, layer):
        if not 0 <= layer < self._layers:
            raise StError(ST_ERANGE, f"layer {layer} outside [0, {self._layers})")

    def append(self, layer, spans, qkv, q_norm=None, k_norm=None):
        """Norms ([head_dim], or None), rotation and the write of the spans' new rows; qkv: a row per new token, all query heads, then key heads, then
        value heads.  Returns the rotated queries, [rows][n_q_heads][head_dim]."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.append(layer, spans, qkv, q_norm, k_norm)
        p, stride = self._matrix("qkv", qkv, spans.rows, self._nq + 2 * self._nkv)
        qn, kn = self._norm("q_norm", q_norm), self._norm("k_norm", k_norm)
        out = self._empty((spans.rows, self._nq, self._d), self.dtype)
        if spans.rows:
            self._layer(layer)
            tree = self._tree_of(spans)
            if tree is not None and spans.positions > self._positions:
                raise StError(ST_ERANGE, f"the drafts need {spans.positions} positions, the rotation table has {self._positions}")
            rc = self._append(self._h, layer, spans.c, spans.n, tree, p, stride, qn, kn, out.data_ptr(), self._nq * self._d)
            if rc:
                _check(rc)
        return out

    def attend(self, layer, spans, q, out=None):
        """Attention of the spans' rows over their sequences' slots; q: n_q_heads * head_dim a row.  With DraftSpans a row sees the context and its
        branch, else what lies before it and itself.  Returns [rows][n_q_heads][head_dim] (or `out`)."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.attend(layer, spans, q, out)
        p, stride = self._matrix("q", q, spans.rows, self._nq)
        if out is None:
            out = self._empty((spans.rows, self._nq, self._d), self.dtype)
            po, so = out.data_ptr(), self._nq * self._d
        else:
            po, so = self._matrix("out", out, spans.rows, self._nq)
        if spans.rows:
            self._layer(layer)
            rc = self._attend(self._h, layer, spans.c, spans.n, self._tree_of(spans), p, stride, po, so)
            if rc:
                _check(rc)
        return out

    def attend_plan(self, spans, with_tree=False):
        """(columns of a block, blocks, key ranges of every span) of such an attend (see st_paged_attend_plan)."""
        columns, blocks, ranges = C.c_int32(), C.c_int32(), (C.c_int32 * max(spans.n, 1))()
        _check(lib().st_paged_attend_plan(C.byref(self._c), spans.c, spans.n, int(with_tree), C.byref(columns), C.byref(blocks), ranges))
        return columns.value, blocks.value, list(ranges)[:spans.n]

    def keep(self, layer_lo, layer_hi, spans, path, accepted):
        """Moves the rows that stay, path[j][:accepted[j]] of span j (int32 tensors on the GPU, as DraftVerifier.verify returns them), to the slots behind the
        span's row 0 in layers [layer_lo, layer_hi).  The sequence then has len + 1 + accepted[j] slots."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.keep(layer_lo, layer_hi, spans, path, accepted)
        if (layer_lo | layer_hi) >> 31:
            _fits32("keep", layer_lo, layer_hi)
        for name, x, shape in (("path", path, (spans.n, path.shape[-1])), ("accepted", accepted, (spans.n,))):
            if x.dtype is not torch.int32 or x.get_device() != self._index or x.shape != shape or not x.is_contiguous():
                raise StError(ST_EINVAL, f"{name} is contiguous int32 with a row for each of {spans.n} spans on {self._dev}, got {x.dtype} {tuple(x.shape)} on {x.device}")
        if spans.n:
            _check(self._keep(self._h, layer_lo, layer_hi, spans.c, spans.n, path.data_ptr(), path.shape[1], accepted.data_ptr()))


class DraftVerifier(_OnStream):
    """st_verify over a torch-owned workspace: the verdict over drafted tokens (see st_verify_drafts64)."""

    def __init__(self, vocab, max_rows, max_width=1, dtype=torch.float32, device="cuda", stream=None):
        if dtype not in _TYPE_OF:
            raise StError(ST_EINVAL, f"dtype is float32, bfloat16 or float16, got {dtype}")
        _fits32("config", vocab, max_rows, max_width)
        c = st_verify_config(vocab, _TYPE_OF[dtype], max_rows, max_width)
        wb = C.c_size_t()
        _check(lib().st_verify_query_sizes(C.byref(c), C.byref(wb)))
        self.vocab, self.dtype = vocab, dtype
        self._bind(_device_of(device), stream)
        self._ws = self._empty((wb.value,), torch.uint8)
        h = C.c_void_p()
        _check(lib().st_verify_create(C.byref(c), self._ws.data_ptr(), wb.value, self.stream, C.byref(h)))
        self._h, self._destroy, self._drafts = h, lib().st_verify_destroy, lib().st_verify_drafts64

    def _logits(self, name, x, rows):
        if x.dtype is not self.dtype or x.get_device() != self._index or x.shape != (rows, self.vocab) or (x.stride(1) != 1 and self.vocab > 1):
            raise StError(ST_EINVAL, f"{name} is {self.dtype} [{rows}][{self.vocab}] on {self._dev}, got {x.dtype} {tuple(x.shape)} {x.stride()} on {x.device}")
        return x.data_ptr(), x.stride(0) if rows > 1 else self.vocab

    def _numbers(self, name, x, n, dtype):
        if x.dtype is not dtype or x.get_device() != self._index or x.shape != (n,) or not x.is_contiguous():
            raise StError(ST_EINVAL, f"{name} is {dtype} [{n}] on {self._dev}, got {x.dtype} {tuple(x.shape)} on {x.device}")
        return x.data_ptr()

    def verify(self, spans, tokens, target, temperature, accept, sample, draft=None):
        """spans: the rows of every sequence, each a tree (DraftSpans) or a chain.  tokens int32 [rows]; target, draft: logits [rows][vocab] of what follows each
        row; temperature: a number, or one of each sequence; accept [rows] and sample [sequences]: float64 random numbers of [0, 1).
        Returns (path [sequences][most rows] with -1 behind the rows that stay, their numbers [sequences], next tokens [sequences]), int32."""
        if self._elsewhere():
            with torch.cuda.device(self._index):
                return self.verify(spans, tokens, target, temperature, accept, sample, draft)
        n, rows = spans.n, spans.rows
        counts = [s[3] for s in spans.spans]
        heat = [float(x) for x in temperature] if hasattr(temperature, "__len__") else [float(temperature)] * n
        if len(heat) != n:
            raise StError(ST_EINVAL, f"{len(heat)} temperatures for {n} sequences")
        pt, st = self._logits("target", target, rows)
        pd, sd = (None, 0) if draft is None else self._logits("draft", draft, rows)
        pk = self._numbers("tokens", tokens, rows, torch.int32)
        pa, ps = self._numbers("accept", accept, rows, torch.float64), self._numbers("sample", sample, n, torch.float64)
        most = max(counts, default=0)
        out = self._empty((n * (most + 2),), torch.int32)       # (one allocation)
        if n:
            at = out.data_ptr()
            _check(self._drafts(self._h, (C.c_int32 * n)(*counts), n, self._tree_of(spans), pk, pt, st, pd, sd, (C.c_double * n)(*heat), pa, ps,
                                at, most, at + 4 * n * most, at + 4 * n * (most + 1)))
        path, accepted, after = out.split_with_sizes((n * most, n, n))
        return path.view(n, most), accepted, after
