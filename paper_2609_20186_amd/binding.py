"""ctypes binding of libswitchsd.so (the C ABI in include/switchsd.h).

Argument marshalling only: every step runs in the HIP kernels of the library.
Tensors must be contiguous device tensors of the documented dtypes; bf16
arrays may be passed as torch.bfloat16 or as their 16-bit patterns
(int16/uint16).  Calls are asynchronous on the given (default: current) stream.
If the library is not built, importing raises instead of falling back to
anything else.
"""
import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libswitchsd.so")

MAX_NGRAM = 8
MAX_CAND = 16
MAX_BIAS = 511
MAX_HISTORY = 2 ** 21 - 1
MODE_AUTO, MODE_FUSED, MODE_SPLIT = 0, 1, 2
BF16, F16, F32, E4M3 = 0, 1, 2, 3
MAX_TOP = 64

STATUS = {0: "OK", -1: "EINVAL", -2: "ESHAPE", -3: "EHIP", -4: "EWORKSPACE", -5: "EDEVICE",
          -6: "ESCRATCH"}

EXPORTS = ("switchsd_ngram_match", "switchsd_probe_score", "switchsd_select_draft",
           "switchsd_verify_accept", "switchsd_verify_sample", "switchsd_tree_mask",
           "switchsd_commit", "switchsd_step", "switchsd_copy_labels",
           "switchsd_workspace_bytes", "switchsd_sample_workspace_bytes",
           "switchsd_label_workspace_bytes", "switchsd_workspace_status", "switchsd_step_noalloc",
           "switchsd_process_logits", "switchsd_verify_processed", "switchsd_page_plan",
           "switchsd_span_slots", "switchsd_compact_cache", "switchsd_store_cache",
           "switchsd_paged_attention", "switchsd_attention_workspace_bytes",
           "switchsd_token_logprobs", "switchsd_token_logprobs_grad",
           "switchsd_logprob_workspace_bytes",
           "switchsd_test_withhold_probe_flag", "switchsd_test_withhold_segment",
           "switchsd_status_string")


class SwitchsdError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__(f"{fn} returned {status} ({STATUS.get(status, '?')}): "
                         f"{status_string(status)}")


class Cfg(ctypes.Structure):
    _fields_ = [("n_ngram", ctypes.c_int32),
                ("ngram_lens", ctypes.c_int32 * MAX_NGRAM),
                ("kappa", ctypes.c_int32),
                ("k", ctypes.c_int32),
                ("theta", ctypes.c_float),
                ("n_cand", ctypes.c_int32)]


def make_cfg(ngram_lens=(3, 2, 1), kappa=1, k=7, theta=0.0, n_cand=1):
    c = Cfg()
    c.n_ngram = len(ngram_lens)
    for i, n in enumerate(ngram_lens):
        c.ngram_lens[i] = int(n)
    c.kappa = int(kappa)
    c.k = int(k)
    c.theta = float(theta)
    c.n_cand = int(n_cand)
    return c


_P = ctypes.c_void_p
_I = ctypes.c_int32


class StepArgs(ctypes.Structure):
    _fields_ = [("tokens", _P), ("lengths", _P), ("hidden", _P), ("w", _P), ("ntok", _P),
                ("npar", _P), ("nn", _P), ("logits", _P),
                ("B", _I), ("Lmax", _I), ("d", _I), ("R", _I), ("V", _I),
                ("bias", ctypes.c_float), ("cfg", Cfg), ("mode", _I),
                ("match_n", _P), ("match_end", _P), ("copy_len", _P), ("copy_tokens", _P),
                ("z", _P), ("use_copy", _P), ("dtok", _P), ("dpar", _P), ("dn", _P),
                ("amax", _P), ("accept_len", _P), ("accept_node", _P), ("bonus", _P),
                ("out_tokens", _P), ("temperature", ctypes.c_float), ("uniforms", _P),
                ("sample_workspace", _P), ("sample_workspace_bytes", ctypes.c_size_t),
                ("commit", _I), ("draft_pos", _P), ("lag", _P),
                ("draft_logits", _P), ("accept_uniforms", _P)]


class LogitsArgs(ctypes.Structure):
    _fields_ = [("logits", _P), ("logits_type", _I),
                ("B", _I), ("R", _I), ("V", _I), ("Lmax", _I), ("n_bias", _I),
                ("dtok", _P), ("dpar", _P), ("dn", _P),
                ("tokens", _P), ("lengths", _P), ("prompt_lens", _P),
                ("repetition", _P), ("frequency", _P), ("presence", _P),
                ("bias_ids", _P), ("bias_vals", _P), ("allowed", _P), ("allowed_on", _P)]


class PageArgs(ctypes.Structure):
    _fields_ = [("lengths", _P), ("dpar", _P), ("dn", _P),
                ("B", _I), ("R", _I), ("Lmax", _I), ("page_size", _I), ("max_pages", _I),
                ("ring_pages", _I), ("table", _P), ("held", _P), ("ring", _P),
                ("ring_state", _P), ("slots", _P), ("positions", _P), ("missing", _P)]


class AttentionArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("R", _I), ("rows", _I), ("Hq", _I), ("Hkv", _I), ("D", _I),
                ("Lmax", _I), ("page_size", _I), ("max_pages", _I), ("scale", ctypes.c_float),
                ("lengths", _P), ("dn", _P), ("begin", _P), ("cu", _P), ("mask", _P),
                ("table", _P), ("held", _P)]


class LogprobArgs(ctypes.Structure):
    _fields_ = [("logits", _P), ("logits_type", _I), ("B", _I), ("R", _I), ("V", _I),
                ("tokens", _P), ("dn", _P), ("dpar", _P), ("accept_node", _P),
                ("temperature", ctypes.c_float), ("workspace", _P),
                ("workspace_bytes", ctypes.c_size_t)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2609_20186_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    S = ctypes.c_size_t
    lib.switchsd_ngram_match.argtypes = [_P, _P, _I, _I, ctypes.POINTER(Cfg), _P, _P, _P, _P,
                                         _P, S, _P]
    lib.switchsd_probe_score.argtypes = [_P, _P, ctypes.c_float, _I, _I, _P, _P]
    lib.switchsd_select_draft.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I, _I,
                                          ctypes.POINTER(Cfg), _P, _P, _P, _P, _P]
    lib.switchsd_verify_accept.argtypes = [_P, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                           S, _P]
    lib.switchsd_tree_mask.argtypes = [_P, _P, _I, _I, _P, _P]
    lib.switchsd_verify_sample.argtypes = [_P, _I, _I, _I, ctypes.c_float, _P, _P, _P, _P, _P,
                                           _P, _P, _P, _P, _P, _P, _P, S, _P, S, _P]
    lib.switchsd_sample_workspace_bytes.argtypes = [_I, _I, _I]
    lib.switchsd_commit.argtypes = [_P, _P, _I, _I, _P, _I, _P, _P, _P, _P, _P]
    lib.switchsd_copy_labels.argtypes = [_P, _P, _I, _I, _I, _P, _P, S, _P]
    lib.switchsd_label_workspace_bytes.argtypes = [_I, _I]
    lib.switchsd_label_workspace_bytes.restype = S
    lib.switchsd_sample_workspace_bytes.restype = S
    lib.switchsd_step.argtypes = [ctypes.POINTER(StepArgs), _P, S, _P]
    lib.switchsd_step_noalloc.argtypes = [ctypes.POINTER(StepArgs), _P]
    lib.switchsd_workspace_bytes.argtypes = [_I, _I, _I, _I]
    lib.switchsd_workspace_bytes.restype = S
    lib.switchsd_workspace_status.argtypes = [_P, S, _I, _P, _P]
    lib.switchsd_process_logits.argtypes = [ctypes.POINTER(LogitsArgs), _P, _I, _P]
    lib.switchsd_verify_processed.argtypes = [ctypes.POINTER(LogitsArgs), _P, _P, _P, _P, _P, _P,
                                              S, _P]
    lib.switchsd_page_plan.argtypes = [ctypes.POINTER(PageArgs), _P, S, _P]
    lib.switchsd_span_slots.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, _I, _P, _P, _P, _P, _P,
                                        _I, _P]
    lib.switchsd_compact_cache.argtypes = [_P, _I, ctypes.c_int64, ctypes.c_int64, _I, _P, _P,
                                           _P, _P, _I, _I, _P]
    L = ctypes.c_int64
    lib.switchsd_store_cache.argtypes = [_P, L, _P, L, _I, _P, _I, _P, _I, _I, _P, _P, _I, L, _P,
                                         _P, _P]
    lib.switchsd_paged_attention.argtypes = [ctypes.POINTER(AttentionArgs), _P, L, _I, _P, _P, _I,
                                             L, _P, _P, _P, _P, _P, S, _P]
    lib.switchsd_attention_workspace_bytes.argtypes = [ctypes.POINTER(AttentionArgs)]
    lib.switchsd_attention_workspace_bytes.restype = S
    lib.switchsd_token_logprobs.argtypes = [ctypes.POINTER(LogprobArgs), _P, _P, _P, _P, _I, _P,
                                            _P, _P]
    lib.switchsd_logprob_workspace_bytes.argtypes = [ctypes.POINTER(LogprobArgs)]
    lib.switchsd_logprob_workspace_bytes.restype = S
    lib.switchsd_token_logprobs_grad.argtypes = [ctypes.POINTER(LogprobArgs), _P, _P, _P, _P, _P,
                                                 _P]
    for knob in ("switchsd_test_withhold_probe_flag", "switchsd_test_withhold_segment"):
        getattr(lib, knob).argtypes = [_I]
        getattr(lib, knob).restype = None
    lib.switchsd_status_string.argtypes = [ctypes.c_int]
    lib.switchsd_status_string.restype = ctypes.c_char_p
    for name in EXPORTS:
        if not name.startswith("switchsd_test_"):
            getattr(lib, name).restype = getattr(lib, name).restype or ctypes.c_int
    return lib


lib = _load()


def status_string(status):
    return lib.switchsd_status_string(int(status)).decode()


def workspace_bytes(B, R, Lmax=0, n_cand=0):
    return int(lib.switchsd_workspace_bytes(int(B), int(R), int(Lmax), int(n_cand)))


def sample_workspace_bytes(B, R, V):
    return int(lib.switchsd_sample_workspace_bytes(int(B), int(R), int(V)))


_DT = {"i32": (torch.int32,), "f32": (torch.float32,),
       "bf16": (torch.bfloat16, torch.int16, torch.uint16), "u8": (torch.uint8,),
       "u32": (torch.int32, torch.uint32), "u64": (torch.int64, torch.uint64)}


_Tensor = torch.Tensor


def _ptr(t, kind, name, optional=False):
    # the accepted case first: a stage call checks up to eleven tensors
    if isinstance(t, _Tensor) and t.is_cuda and t.dtype in _DT[kind] and t.is_contiguous():
        return t.data_ptr()
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in _DT[kind]:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {_DT[kind]}")
    raise ValueError(f"{name} must be contiguous")


# The current stream's handle without a Stream object around it, where torch
# offers that (six stage calls with both: 50 -> 37 us).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)
_initialized = torch.cuda.is_initialized


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device is None or not _initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _check(fn, rc):
    if rc != 0:
        raise SwitchsdError(fn, rc)


def switchsd_ngram_match(tokens, lengths, cfg, match_n, match_end, copy_len, copy_tokens,
                         workspace, stream=None):
    B, Lmax = tokens.shape
    _check("switchsd_ngram_match", lib.switchsd_ngram_match(
        _ptr(tokens, "i32", "tokens"), _ptr(lengths, "i32", "lengths"), B, Lmax,
        ctypes.byref(cfg), _ptr(match_n, "i32", "match_n"), _ptr(match_end, "i32", "match_end"),
        _ptr(copy_len, "i32", "copy_len"), _ptr(copy_tokens, "i32", "copy_tokens", True),
        _ptr(workspace, "u8", "workspace"), workspace.numel(), _stream(stream)))


def switchsd_probe_score(hidden, w, bias, z, stream=None):
    B, d = hidden.shape
    _check("switchsd_probe_score", lib.switchsd_probe_score(
        _ptr(hidden, "bf16", "hidden"), _ptr(w, "f32", "w"), float(bias), B, d,
        _ptr(z, "f32", "z"), _stream(stream)))


def switchsd_select_draft(match_n, copy_len, copy_tokens, z, ntok, npar, nn, cfg, use_copy,
                          dtok, dpar, dn, stream=None):
    B, R = ntok.shape
    _check("switchsd_select_draft", lib.switchsd_select_draft(
        _ptr(match_n, "i32", "match_n"), _ptr(copy_len, "i32", "copy_len"),
        _ptr(copy_tokens, "i32", "copy_tokens", True), _ptr(z, "f32", "z"),
        _ptr(ntok, "i32", "ntok"), _ptr(npar, "i32", "npar", True), _ptr(nn, "i32", "nn"),
        B, R, ctypes.byref(cfg), _ptr(use_copy, "i32", "use_copy"), _ptr(dtok, "i32", "dtok"),
        _ptr(dpar, "i32", "dpar"), _ptr(dn, "i32", "dn"), _stream(stream)))


def switchsd_verify_accept(logits, dtok, dpar, dn, accept_len, accept_node, bonus, out_tokens,
                           amax, workspace, stream=None):
    B, R, V = logits.shape
    _check("switchsd_verify_accept", lib.switchsd_verify_accept(
        _ptr(logits, "bf16", "logits"), B, R, V, _ptr(dtok, "i32", "dtok"),
        _ptr(dpar, "i32", "dpar", True), _ptr(dn, "i32", "dn"),
        _ptr(accept_len, "i32", "accept_len"), _ptr(accept_node, "i32", "accept_node"),
        _ptr(bonus, "i32", "bonus"), _ptr(out_tokens, "i32", "out_tokens"),
        _ptr(amax, "i32", "amax", True), _ptr(workspace, "u8", "workspace"),
        workspace.numel(), _stream(stream)))


def switchsd_verify_sample(logits, temperature, uniforms, dtok, dpar, dn, accept_len,
                           accept_node, bonus, out_tokens, amax, workspace, sample_workspace,
                           stream=None, draft_logits=None, accept_uniforms=None):
    """uniforms, accept_uniforms: uint64 (or int64 holding the same bits) [B, R];
    draft_logits (bf16 [B, R, V]) verifies chains by speculative sampling with
    the draft's distribution."""
    B, R, V = logits.shape
    _check("switchsd_verify_sample", lib.switchsd_verify_sample(
        _ptr(logits, "bf16", "logits"), B, R, V, float(temperature),
        _ptr(uniforms, "u64", "uniforms"), _ptr(draft_logits, "bf16", "draft_logits", True),
        _ptr(accept_uniforms, "u64", "accept_uniforms", True), _ptr(dtok, "i32", "dtok"),
        _ptr(dpar, "i32", "dpar", True), _ptr(dn, "i32", "dn"),
        _ptr(accept_len, "i32", "accept_len"), _ptr(accept_node, "i32", "accept_node"),
        _ptr(bonus, "i32", "bonus"), _ptr(out_tokens, "i32", "out_tokens"),
        _ptr(amax, "i32", "amax", True), _ptr(workspace, "u8", "workspace"),
        workspace.numel(), _ptr(sample_workspace, "u8", "sample_workspace"),
        sample_workspace.numel(), _stream(stream)))


def switchsd_commit(tokens, lengths, out_tokens, accept_len, use_copy, draft_pos, lag,
                    stream=None):
    B, Lmax = tokens.shape
    R = out_tokens.shape[1]
    _check("switchsd_commit", lib.switchsd_commit(
        _ptr(tokens, "i32", "tokens"), _ptr(lengths, "i32", "lengths"), B, Lmax,
        _ptr(out_tokens, "i32", "out_tokens"), R, _ptr(accept_len, "i32", "accept_len"),
        _ptr(use_copy, "i32", "use_copy"), _ptr(draft_pos, "i32", "draft_pos"),
        _ptr(lag, "i32", "lag"), _stream(stream)))


def label_workspace_bytes(B, Lmax):
    return int(lib.switchsd_label_workspace_bytes(int(B), int(Lmax)))


def switchsd_copy_labels(tokens, lengths, n, labels, workspace, stream=None):
    """labels: uint8 [B, Lmax]; workspace: zeroed uint8 of label_workspace_bytes."""
    B, Lmax = tokens.shape
    _check("switchsd_copy_labels", lib.switchsd_copy_labels(
        _ptr(tokens, "i32", "tokens"), _ptr(lengths, "i32", "lengths"), B, Lmax, int(n),
        _ptr(labels, "u8", "labels"), _ptr(workspace, "u8", "workspace"), workspace.numel(),
        _stream(stream)))


def switchsd_workspace_status(workspace, B, status, stream=None):
    """Writes OK (0) or EDEVICE (-5) to the device int32 ``status`` [1] and
    clears the workspace's error words of B sequences."""
    _check("switchsd_workspace_status", lib.switchsd_workspace_status(
        _ptr(workspace, "u8", "workspace"), workspace.numel(), int(B),
        _ptr(status, "i32", "status"), _stream(stream)))


def withhold_probe_flag_for_tests(on):
    """Test support: force the step's bounded wait for the probe flag to give up."""
    lib.switchsd_test_withhold_probe_flag(1 if on else 0)


def withhold_segment_for_tests(on):
    """Test support: force the fused step's poll of the segment results to give up."""
    lib.switchsd_test_withhold_segment(1 if on else 0)


def switchsd_tree_mask(dpar, dn, mask, stream=None):
    """mask: uint32 (or int32 holding the same bits) [B, R, (R + 31) // 32]."""
    B, R = mask.shape[0], mask.shape[1]
    if mask.shape[2] != (R + 31) // 32:
        raise ValueError("mask must be [B, R, (R + 31) // 32]")
    _check("switchsd_tree_mask", lib.switchsd_tree_mask(
        _ptr(dpar, "i32", "dpar", True), _ptr(dn, "i32", "dn"), B, R,
        _ptr(mask, "u32", "mask"), _stream(stream)))


OUTPUTS = ("match_n", "match_end", "copy_len", "copy_tokens", "z", "use_copy", "dtok", "dpar",
           "dn", "amax", "accept_len", "accept_node", "bonus", "out_tokens")


def alloc_outputs(B, R, k, n_cand=1, device="cuda"):
    """Output tensors of a step; with n_cand > 1 the candidate outputs carry a
    W axis (match_end, copy_len [B, W], copy_tokens [B, W, k])."""
    i32 = dict(dtype=torch.int32, device=device)
    wsh = (B,) if n_cand <= 1 else (B, n_cand)
    return {"match_n": torch.empty(B, **i32), "match_end": torch.empty(wsh, **i32),
            "copy_len": torch.empty(wsh, **i32), "copy_tokens": torch.empty(wsh + (k,), **i32),
            "z": torch.empty(B, dtype=torch.float32, device=device),
            "use_copy": torch.empty(B, **i32), "dtok": torch.empty((B, R), **i32),
            "dpar": torch.empty((B, R), **i32), "dn": torch.empty(B, **i32),
            "amax": torch.empty((B, R), **i32), "accept_len": torch.empty(B, **i32),
            "accept_node": torch.empty(B, **i32), "bonus": torch.empty(B, **i32),
            "out_tokens": torch.empty((B, R), **i32)}


def alloc_sample_workspace(B, R, V, device="cuda"):
    return torch.empty(max(sample_workspace_bytes(B, R, V), 256), dtype=torch.uint8,
                       device=device)


def alloc_workspace(B, R, Lmax=0, n_cand=0, device="cuda"):
    """Zeroed once here; the kernels keep it usable for every later call."""
    return torch.zeros(max(workspace_bytes(B, R, Lmax, n_cand), 256), dtype=torch.uint8,
                       device=device)


def build_step_args(inp, out, cfg, mode=MODE_AUTO, temperature=0.0, uniforms=None,
                    sample_workspace=None, draft_pos=None, lag=None, draft_logits=None,
                    accept_uniforms=None):
    """StepArgs for switchsd_step.  ``inp`` holds device tensors tokens [B,Lmax],
    lengths [B], hidden [B,d], w [d], ntok [B,R], npar [B,R] or None, nn [B],
    logits [B,R,V] and the float ``bias``; ``out`` is from alloc_outputs.
    temperature > 0 draws the rows' tokens with ``uniforms`` [B,R] (uint64
    bits) and ``sample_workspace`` (alloc_sample_workspace); with
    ``draft_logits`` [B,R,V] and ``accept_uniforms`` [B,R] a chosen neural draft
    is verified by speculative sampling with its distribution.  With ``draft_pos``
    and ``lag`` [B] the step also commits (decode loop): tokens and lengths are
    then updated in place."""
    tokens, logits, hidden = inp["tokens"], inp["logits"], inp["hidden"]
    B, Lmax = tokens.shape
    R, V = logits.shape[1], logits.shape[2]
    a = StepArgs()
    a.tokens = _ptr(tokens, "i32", "tokens")
    a.lengths = _ptr(inp["lengths"], "i32", "lengths")
    a.hidden = _ptr(hidden, "bf16", "hidden")
    a.w = _ptr(inp["w"], "f32", "w")
    a.ntok = _ptr(inp["ntok"], "i32", "ntok")
    a.npar = _ptr(inp.get("npar"), "i32", "npar", True)
    a.nn = _ptr(inp["nn"], "i32", "nn")
    a.logits = _ptr(logits, "bf16", "logits")
    a.B, a.Lmax, a.d, a.R, a.V = B, Lmax, hidden.shape[1], R, V
    a.bias = float(inp["bias"])
    a.cfg = cfg
    a.mode = int(mode)
    for name in OUTPUTS:
        setattr(a, name, _ptr(out[name], "f32" if name == "z" else "i32", name,
                              optional=(name == "amax" or name == "copy_tokens")))
    if draft_pos is not None:
        a.commit = 1
        a.draft_pos = _ptr(draft_pos, "i32", "draft_pos")
        a.lag = _ptr(lag, "i32", "lag")
    a.temperature = float(temperature)
    if temperature != 0.0:
        a.uniforms = _ptr(uniforms, "u64", "uniforms")
        a.sample_workspace = _ptr(sample_workspace, "u8", "sample_workspace")
        a.sample_workspace_bytes = sample_workspace.numel()
        a.draft_logits = _ptr(draft_logits, "bf16", "draft_logits", True)
        a.accept_uniforms = _ptr(accept_uniforms, "u64", "accept_uniforms",
                                 draft_logits is None)
    return a


def switchsd_step(args, workspace, stream=None):
    _check("switchsd_step", lib.switchsd_step(ctypes.byref(args), _ptr(workspace, "u8",
                                              "workspace"), workspace.numel(),
                                              _stream(stream)))


def switchsd_step_noalloc(args, stream=None):
    """switchsd_step with the library's own fixed device scratch (no workspace
    argument; args.sample_workspace is ignored)."""
    _check("switchsd_step_noalloc", lib.switchsd_step_noalloc(ctypes.byref(args),
                                                              _stream(stream)))


# ------------------------------------------------------------------ calls around the step

_TYPES = {torch.bfloat16: BF16, torch.int16: BF16, torch.uint16: BF16, torch.float16: F16,
          torch.float32: F32}
_DT["i64"] = (torch.int64,)
_DT["logits"] = tuple(_TYPES)


def _current_device():
    # -2 without a GPU: no tensor's number (-1 is the CPU's)
    if _device is None or not _initialized():
        return torch.cuda.current_device() if torch.cuda.is_available() else -2
    return _device()


def _arr(t, kind, name, shape, dev, optional=False):
    """Device pointer of a tensor of exactly this shape on device `dev`."""
    # the accepted case first: a call checks up to ten tensors; what has the
    # device's number is on a GPU
    if isinstance(t, _Tensor) and t.get_device() == dev and t.dtype in _DT[kind] and \
            t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    ptr = _ptr(t, kind, name, optional)
    if ptr is not None or t is not None:
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        _here(t, name, dev)
    return ptr


def _workspace(t, dev):
    """Device pointer of a workspace on device `dev`."""
    ptr = _ptr(t, "u8", "workspace")
    _here(t, "workspace", dev)
    return ptr


_INT_MAX = 2 ** 31 - 1


def _sizes(**sizes):
    """ctypes keeps the low 32 bits of an int32 argument: a size beyond them
    would be taken for another, valid one."""
    for name, n in sizes.items():
        if not -_INT_MAX - 1 <= n <= _INT_MAX:
            raise ValueError(f"{name} = {n} does not fit 32 bits")


def _here(t, name, dev):
    if t.get_device() != dev:
        raise ValueError(f"{name} is on device {t.get_device()}, the current device is {dev}")


def build_logits_args(logits, dtok, dpar, dn, tokens=None, lengths=None, prompt_lens=None,
                      repetition=None, frequency=None, presence=None, bias_ids=None,
                      bias_vals=None, allowed=None, allowed_on=None):
    """LogitsArgs for switchsd_process_logits and switchsd_verify_processed:
    logits [B, R, V] (bf16 or its bits, fp16 or fp32) of the drafted rows and the
    draft's dtok, dpar (None: chains) [B, R] and dn [B].  repetition, frequency,
    presence: float [B] each, with the context tokens [B, Lmax], lengths [B] and
    prompt_lens [B] (None: no prompt); bias_ids int32 and bias_vals float
    [B, n]; allowed: bits, uint32 (or int32) [B, R, (V + 31) // 32], for the
    sequences with allowed_on[b] != 0 (None: all).  The tensors are kept alive by
    the result."""
    if not isinstance(logits, _Tensor) or logits.dim() != 3:
        raise ValueError("logits must be a device tensor [B, R, V]")
    B, R, V = logits.shape
    _sizes(B=B, R=R, V=V)
    dev = _current_device()
    a = LogitsArgs()
    a.logits = _arr(logits, "logits", "logits", (B, R, V), dev)
    a.logits_type = _TYPES[logits.dtype]
    a.B, a.R, a.V = B, R, V
    a.dtok = _arr(dtok, "i32", "dtok", (B, R), dev)
    a.dpar = _arr(dpar, "i32", "dpar", (B, R), dev, True)
    a.dn = _arr(dn, "i32", "dn", (B,), dev)
    penal = any(t is not None for t in (repetition, frequency, presence))
    if tokens is not None:
        if not isinstance(tokens, _Tensor) or tokens.dim() != 2:
            raise ValueError("tokens must be a device tensor [B, Lmax]")
        _sizes(Lmax=tokens.shape[1])
        a.Lmax = tokens.shape[1]
        a.tokens = _arr(tokens, "i32", "tokens", (B, a.Lmax), dev)
    elif penal:
        raise ValueError("tokens is required")
    a.lengths = _arr(lengths, "i32", "lengths", (B,), dev, not penal)
    a.prompt_lens = _arr(prompt_lens, "i32", "prompt_lens", (B,), dev, True)
    for name, t in (("repetition", repetition), ("frequency", frequency),
                    ("presence", presence)):
        setattr(a, name, _arr(t, "f32", name, (B,), dev, True))
    if (bias_ids is None) != (bias_vals is None):
        raise ValueError("bias_ids and bias_vals come together")
    if bias_ids is not None:
        if not isinstance(bias_ids, _Tensor) or bias_ids.dim() != 2:
            raise ValueError("bias_ids must be a device tensor [B, n]")
        _sizes(n_bias=bias_ids.shape[1])
        a.n_bias = bias_ids.shape[1]
        a.bias_ids = _arr(bias_ids, "i32", "bias_ids", (B, a.n_bias), dev)
        a.bias_vals = _arr(bias_vals, "f32", "bias_vals", (B, a.n_bias), dev)
    a.allowed = _arr(allowed, "u32", "allowed", (B, R, (V + 31) // 32), dev, True)
    a.allowed_on = _arr(allowed_on, "i32", "allowed_on", (B,), dev, True)
    a.shape, a.device = (B, R, V), dev
    a.keep = (logits, dtok, dpar, dn, tokens, lengths, prompt_lens, repetition, frequency,
              presence, bias_ids, bias_vals, allowed, allowed_on)
    return a


def _args_here(args):
    dev = _current_device()
    if args.device != dev:
        raise ValueError(f"the arguments are on device {args.device}, the current device is "
                         f"{dev}")
    return dev


def switchsd_process_logits(args, out, stream=None):
    """out [B, R, V]: bf16 or the logits' type (the logits themselves: in place)."""
    dev = _args_here(args)
    _check("switchsd_process_logits", lib.switchsd_process_logits(
        ctypes.byref(args), _arr(out, "logits", "out", args.shape, dev), _TYPES[out.dtype],
        _stream(stream)))


def switchsd_verify_processed(args, accept_len, accept_node, bonus, out_tokens, amax, workspace,
                              stream=None):
    dev = _args_here(args)
    B, R, _ = args.shape
    p_workspace = _workspace(workspace, dev)
    _check("switchsd_verify_processed", lib.switchsd_verify_processed(
        ctypes.byref(args), _arr(accept_len, "i32", "accept_len", (B,), dev),
        _arr(accept_node, "i32", "accept_node", (B,), dev),
        _arr(bonus, "i32", "bonus", (B,), dev),
        _arr(out_tokens, "i32", "out_tokens", (B, R), dev),
        _arr(amax, "i32", "amax", (B, R), dev, True),
        p_workspace, workspace.numel(), _stream(stream)))


def build_page_args(lengths, dpar, dn, Lmax, page_size, table, held, ring, ring_state, slots,
                    positions, missing, R=None):
    """PageArgs for switchsd_page_plan: lengths, dn, held, missing [B], dpar
    [B, R] (None: chains), table [B, max_pages], ring [ring_pages], ring_state [2]
    int32; slots int64 and positions int32 [B, R] (None: not wanted; R then comes
    from dpar or R).  The tensors are kept alive by the result."""
    if not isinstance(table, _Tensor) or table.dim() != 2:
        raise ValueError("table must be a device tensor [B, max_pages]")
    for t in (slots, positions, dpar):
        if R is None and isinstance(t, _Tensor) and t.dim() == 2:
            R = t.shape[1]
    if R is None:
        raise ValueError("R is required")
    B, most = table.shape
    Lmax, page_size = int(Lmax), int(page_size)
    _sizes(B=B, R=R, Lmax=Lmax, page_size=page_size, max_pages=most)
    dev = _current_device()
    a = PageArgs()
    a.B, a.R, a.Lmax, a.page_size, a.max_pages = B, R, Lmax, page_size, most
    a.table = _arr(table, "i32", "table", (B, most), dev)
    for name, t in (("lengths", lengths), ("dn", dn), ("held", held), ("missing", missing)):
        setattr(a, name, _arr(t, "i32", name, (B,), dev))
    a.dpar = _arr(dpar, "i32", "dpar", (B, R), dev, True)
    if not isinstance(ring, _Tensor) or ring.dim() != 1:
        raise ValueError("ring must be a device tensor [ring_pages]")
    _sizes(ring_pages=ring.shape[0])
    a.ring_pages = ring.shape[0]
    a.ring = _arr(ring, "i32", "ring", (a.ring_pages,), dev)
    a.ring_state = _arr(ring_state, "i32", "ring_state", (2,), dev)
    a.slots = _arr(slots, "i64", "slots", (B, R), dev, True)
    a.positions = _arr(positions, "i32", "positions", (B, R), dev, True)
    a.device = dev
    a.keep = (lengths, dpar, dn, table, held, ring, ring_state, slots, positions, missing)
    return a


def switchsd_page_plan(args, workspace, stream=None):
    p_workspace = _workspace(workspace, _args_here(args))
    _check("switchsd_page_plan", lib.switchsd_page_plan(
        ctypes.byref(args), p_workspace, workspace.numel(), _stream(stream)))


def switchsd_span_slots(begin, end, tokens, table, held, page_size, cu, slots, positions, packed,
                        seq, stream=None, Lmax=None):
    """begin, end, held [B], tokens [B, Lmax], table [B, max_pages] int32; cu
    [B + 1] int32, slots int64 and positions, packed, seq int32 [capacity] (each
    None if not wanted).  Without packed, tokens may be None; the limit of the
    positions is then given as Lmax."""
    if tokens is None:
        if packed is not None or Lmax is None:
            raise ValueError("tokens is required (without packed: tokens or Lmax)")
        if not isinstance(begin, _Tensor) or begin.dim() != 1:
            raise ValueError("begin must be a device tensor [B]")
        B, Lmax = begin.shape[0], int(Lmax)
    else:
        try:
            B, cols = tokens.shape
        except (AttributeError, ValueError):
            raise ValueError("tokens must be a device tensor [B, Lmax]") from None
        if Lmax is not None and Lmax != cols:
            raise ValueError(f"tokens has {cols} columns, Lmax is {Lmax}")
        Lmax = cols
    one = slots if slots is not None else positions if positions is not None else \
        packed if packed is not None else seq
    cap, room = (0,), 0
    if one is not None:
        # the library is told one capacity: of an output of several axes it would
        # fill no more than the first axis' length
        try:
            cap = one.shape
            room, = cap
        except (AttributeError, ValueError):
            raise ValueError("slots, positions, packed and seq must be device tensors "
                             "[capacity]") from None
    dev = _current_device()
    most, p_table, p_held = 0, None, None
    if slots is not None:
        if not isinstance(table, _Tensor) or table.dim() != 2 or held is None:
            raise ValueError("slots need table [B, max_pages] and held [B]")
        most = table.shape[1]
        p_table = _arr(table, "i32", "table", (B, most), dev)
        p_held = _arr(held, "i32", "held", (B,), dev)
    page_size = int(page_size)
    if (B | Lmax | most | page_size | room) >> 31:
        _sizes(B=B, Lmax=Lmax, max_pages=most, page_size=page_size)
        room = min(room, _INT_MAX)  # no total is larger
    _check("switchsd_span_slots", lib.switchsd_span_slots(
        _arr(begin, "i32", "begin", (B,), dev), _arr(end, "i32", "end", (B,), dev),
        None if tokens is None else _arr(tokens, "i32", "tokens", (B, Lmax), dev), p_table, p_held,
        B, Lmax, most, page_size, _arr(cu, "i32", "cu", (B + 1,), dev),
        None if slots is None else _arr(slots, "i64", "slots", cap, dev),
        None if positions is None else _arr(positions, "i32", "positions", cap, dev),
        None if packed is None else _arr(packed, "i32", "packed", cap, dev),
        None if seq is None else _arr(seq, "i32", "seq", cap, dev), room, _stream(stream)))


def switchsd_compact_cache(cache, slots, dpar, dn, accept_node, stream=None):
    """cache [planes, n_slots, ...] of any type, each plane contiguous; slots
    [B, R] int64, dpar [B, R] (None: chains), dn, accept_node [B] int32."""
    if not isinstance(cache, _Tensor) or not cache.is_cuda or cache.dim() < 2:
        raise ValueError("cache must be a device tensor [planes, n_slots, ...]")
    planes, n_slots = cache.shape[:2]
    if not cache.is_contiguous() and not cache[0].is_contiguous():
        raise ValueError("cache planes must be contiguous")
    try:
        B, R = slots.shape
    except (AttributeError, ValueError):
        raise ValueError("slots must be a device tensor [B, R]") from None
    dev = _current_device()
    _here(cache, "cache", dev)
    size, numel = cache.element_size(), cache.numel()
    row = size * (numel // (planes * n_slots) if numel else 0)
    if (planes | B | R | row) >> 31:
        _sizes(planes=planes, B=B, R=R, row_bytes=row)
    _check("switchsd_compact_cache", lib.switchsd_compact_cache(
        cache.data_ptr(), planes, cache.stride(0) * size, n_slots, row,
        _arr(slots, "i64", "slots", (B, R), dev), _arr(dpar, "i32", "dpar", (B, R), dev, True),
        _arr(dn, "i32", "dn", (B,), dev), _arr(accept_node, "i32", "accept_node", (B,), dev), B, R,
        _stream(stream)))


# ------------------------------------------------------------------ attention over the paged cache

_HALF = {torch.bfloat16: BF16, torch.float16: F16}
_CACHES = dict(_HALF)
_CACHES[torch.float8_e4m3fn] = E4M3
_DT["cache"] = tuple(_CACHES)
_DT["half"] = tuple(_HALF)


def _rows(t, name, dev, heads=None):
    """Shape, row stride and device pointer of [rows, heads, D] elements whose rows
    may lie apart (parts of one projection's output)."""
    # the accepted case first, as in _arr
    if not isinstance(t, _Tensor) or t.get_device() != dev or t.dtype not in _HALF or \
            t.dim() != 3:
        if not isinstance(t, _Tensor) or not t.is_cuda or t.dim() != 3:
            raise ValueError(f"{name} must be a device tensor [rows, heads, D]")
        if t.dtype not in _HALF:
            raise ValueError(f"{name} has dtype {t.dtype}, expected one of {_DT['half']}")
        _here(t, name, dev)
    shape = t.shape
    if heads is not None and shape != heads:
        raise ValueError(f"{name} has shape {tuple(shape)}, expected {tuple(heads)}")
    row, head, one = t.stride()
    n, H, D = shape
    if (one != 1 and D > 1) or (head != D and H > 1):
        raise ValueError(f"the heads of {name} must be contiguous")
    return shape, row if n > 1 else max(row, H * D), t.data_ptr()


def _caches(k_cache, v_cache, dtype, Hkv, D, k_scale, v_scale, dev):
    """Type, slots and pointers of a pair of cache planes."""
    if not isinstance(k_cache, _Tensor) or k_cache.dim() != 3:
        raise ValueError("k_cache must be a device tensor [n_slots, Hkv, D]")
    n = k_cache.shape[0]
    kind = k_cache.dtype
    ptrs = (_arr(k_cache, "cache", "k_cache", (n, Hkv, D), dev),
            _arr(v_cache, "cache", "v_cache", (n, Hkv, D), dev))
    if v_cache.dtype != kind or (kind != dtype and _CACHES[kind] != E4M3):
        raise ValueError(f"caches of {kind} and {v_cache.dtype} for rows of {dtype}")
    if k_scale is None and v_scale is None:
        return _CACHES[kind], n, ptrs, (None, None)
    return _CACHES[kind], n, ptrs, (
        None if k_scale is None else _arr(k_scale, "f32", "k_scale", (Hkv,), dev),
        None if v_scale is None else _arr(v_scale, "f32", "v_scale", (Hkv,), dev))


def switchsd_store_cache(keys, values, slots, k_cache, v_cache, count=None, k_scale=None,
                         v_scale=None, stream=None):
    """keys, values [n, Hkv, D] (bf16 or fp16; rows may lie apart) into the slots
    [n] int64 (any shape of n elements) of k_cache, v_cache [n_slots, Hkv, D] (the same
    type, or float8_e4m3fn with k_scale, v_scale [Hkv] float or None); count: how many
    of the rows there are, [1] int32 on the device (None: all)."""
    dev = _current_device()
    shape, k_stride, p_k = _rows(keys, "keys", dev)
    n, Hkv, D = shape
    _, v_stride, p_v = _rows(values, "values", dev, shape)
    if values.dtype != keys.dtype:
        raise ValueError(f"keys have dtype {keys.dtype}, values {values.dtype}")
    if not isinstance(slots, _Tensor) or slots.numel() != n:
        raise ValueError(f"slots must be a device tensor of {n} elements")
    if n > _INT_MAX or Hkv > _INT_MAX or D > _INT_MAX:
        _sizes(n=n, Hkv=Hkv, D=D)
    kind, n_slots, (p_kc, p_vc), (p_ks, p_vs) = _caches(k_cache, v_cache, keys.dtype, Hkv, D,
                                                        k_scale, v_scale, dev)
    _check("switchsd_store_cache", lib.switchsd_store_cache(
        p_k, k_stride, p_v, v_stride, _HALF[keys.dtype],
        _arr(slots, "i64", "slots", slots.shape, dev), n,
        None if count is None else _arr(count, "i32", "count", (1,), dev), Hkv, D, p_kc, p_vc,
        kind, n_slots, p_ks, p_vs, _stream(stream)))


def build_attention_args(rows, R, Hq, Hkv, D, page_size, table, held, Lmax, lengths=None, dn=None,
                         begin=None, cu=None, mask=None, scale=None):
    """AttentionArgs for switchsd_paged_attention, the same for all layers of a
    step: table [B, max_pages] and held [B] int32, and either the drafted rows'
    lengths and dn [B] (rows = B * R) or the packed rows' begin [B] and cu [B + 1]
    (R: the most rows of a sequence).  mask: uint32 (or int32) [rows, (R + 31) // 32]
    (or [B, R, ...]) of the new positions each row sees, None: its own and earlier
    ones.  scale: default 1 / sqrt(D).  The tensors are kept alive by the result."""
    if not isinstance(table, _Tensor) or table.dim() != 2:
        raise ValueError("table must be a device tensor [B, max_pages]")
    B, most = table.shape
    rows, R, Hq, Hkv, D = int(rows), int(R), int(Hq), int(Hkv), int(D)
    page_size, Lmax = int(page_size), int(Lmax)
    _sizes(B=B, rows=rows, R=R, Hq=Hq, Hkv=Hkv, D=D, Lmax=Lmax, page_size=page_size,
           max_pages=most)
    dev = _current_device()
    a = AttentionArgs()
    a.B, a.R, a.rows, a.Hq, a.Hkv, a.D = B, R, rows, Hq, Hkv, D
    a.Lmax, a.page_size, a.max_pages = Lmax, page_size, most
    a.scale = D ** -0.5 if scale is None else float(scale)
    a.table = _arr(table, "i32", "table", (B, most), dev)
    a.held = _arr(held, "i32", "held", (B,), dev)
    if (cu is None) != (begin is None) or (cu is None) == (lengths is None) or \
            (lengths is None) != (dn is None):
        raise ValueError("either lengths and dn, or begin and cu")
    if cu is None:
        a.lengths = _arr(lengths, "i32", "lengths", (B,), dev)
        a.dn = _arr(dn, "i32", "dn", (B,), dev)
    else:
        a.begin = _arr(begin, "i32", "begin", (B,), dev)
        a.cu = _arr(cu, "i32", "cu", (B + 1,), dev)
    if mask is not None:
        words = (R + 31) // 32
        a.mask = _arr(mask, "u32", "mask", (B, R, words) if isinstance(mask, _Tensor) and
                      mask.dim() == 3 and rows == B * R else (rows, words), dev)
    a.shape, a.device = (rows, Hq, D), dev
    a.keep = (table, held, lengths, dn, begin, cu, mask)
    return a


def attention_workspace_bytes(args):
    return int(lib.switchsd_attention_workspace_bytes(ctypes.byref(args)))


def alloc_attention_workspace(args, device="cuda"):
    return torch.empty(max(attention_workspace_bytes(args), 256), dtype=torch.uint8,
                       device=device)


def switchsd_paged_attention(args, q, k_cache, v_cache, out, workspace, lse=None, k_scale=None,
                             v_scale=None, stream=None):
    """q [rows, Hq, D] (bf16 or fp16; rows may lie apart) over k_cache, v_cache
    [n_slots, Hkv, D] (the same type, or float8_e4m3fn with k_scale, v_scale [Hkv] float
    or None) into out [rows, Hq, D] and lse [rows, Hq] float (None: not wanted)."""
    dev = _args_here(args)
    shape, q_stride, p_q = _rows(q, "q", dev, args.shape)
    kind, n_slots, (p_kc, p_vc), (p_ks, p_vs) = _caches(k_cache, v_cache, q.dtype, args.Hkv,
                                                        args.D, k_scale, v_scale, dev)
    p_out = _arr(out, "half", "out", shape, dev)
    if out.dtype != q.dtype:
        raise ValueError(f"out has dtype {out.dtype}, q {q.dtype}")
    p_workspace = _workspace(workspace, dev)
    _check("switchsd_paged_attention", lib.switchsd_paged_attention(
        ctypes.byref(args), p_q, q_stride, _HALF[q.dtype], p_kc, p_vc, kind, n_slots, p_ks, p_vs,
        p_out, None if lse is None else _arr(lse, "f32", "lse", shape[:2], dev), p_workspace,
        workspace.numel(), _stream(stream)))


# ------------------------------------------------------------------ log probabilities

def build_logprob_args(logits, tokens=None, dn=None, dpar=None, accept_node=None,
                       temperature=1.0, workspace=None):
    """LogprobArgs for switchsd_token_logprobs and its gradient: logits [B, R, V]
    (bf16 or its bits, fp16 or fp32), tokens [B, R] int32 (None where neither logprob
    nor rank is wanted), dn [B] (None: all rows); with accept_node [B], and dpar [B, R]
    (None: chains), the rows along each accepted path, tokens being the step's
    out_tokens.  workspace: zeroed, of logprob_workspace_bytes, None: one of its own, zeroed
    on the current stream: the first call waits for that whatever its stream, but for a
    captured one, which needs it done before the capture begins (torch.cuda.graph
    waits for the device); what is built in a capture is for that capture.
    switchsd_token_logprobs calls that share a workspace (the result too) must be ordered.
    The tensors are kept alive by the result."""
    if not isinstance(logits, _Tensor) or logits.dim() != 3:
        raise ValueError("logits must be a device tensor [B, R, V]")
    B, R, V = logits.shape
    _sizes(B=B, R=R, V=V)
    if dpar is not None and accept_node is None:
        raise ValueError("dpar comes with accept_node")
    dev = _current_device()
    a = LogprobArgs()
    a.logits = _arr(logits, "logits", "logits", (B, R, V), dev)
    a.logits_type = _TYPES[logits.dtype]
    a.B, a.R, a.V = B, R, V
    a.tokens = _arr(tokens, "i32", "tokens", (B, R), dev, True)
    a.dn = _arr(dn, "i32", "dn", (B,), dev, True)
    a.dpar = _arr(dpar, "i32", "dpar", (B, R), dev, True)
    a.accept_node = _arr(accept_node, "i32", "accept_node", (B,), dev, True)
    a.temperature = float(temperature)
    need = logprob_workspace_bytes(a)
    a.zeroed = None
    if workspace is None and need:
        workspace = torch.zeros(need, dtype=torch.uint8, device=logits.device)
        if not torch.cuda.is_current_stream_capturing():
            a.zeroed = torch.cuda.current_stream().record_event()
    if workspace is not None:
        a.workspace, a.workspace_bytes = _workspace(workspace, dev), workspace.numel()
    a.shape, a.device = (B, R, V), dev
    a.keep = (logits, tokens, dn, dpar, accept_node, workspace)
    return a


def logprob_workspace_bytes(args):
    return int(lib.switchsd_logprob_workspace_bytes(ctypes.byref(args)))


def alloc_logprob_workspace(args, device="cuda"):
    """Zeroed once here, on the current stream; the kernels keep it usable for every later
    call."""
    return torch.zeros(max(logprob_workspace_bytes(args), 256), dtype=torch.uint8, device=device)


def _after_zeroing(args, stream):
    """The first call's stream waits for the workspace that build_logprob_args zeroed;
    later calls are ordered behind that call."""
    if stream is None:
        stream = torch.cuda.current_stream()
    elif not isinstance(stream, torch.cuda.Stream):  # what has a handle, as for all calls
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    with torch.cuda.stream(stream):
        if torch.cuda.is_current_stream_capturing():
            return  # a capture cannot wait for what lies outside of it
    stream.wait_event(args.zeroed)
    args.zeroed = None


def switchsd_token_logprobs(args, logprob=None, lse=None, entropy=None, rank=None, top_ids=None,
                            top_logprobs=None, stream=None):
    """logprob, lse, entropy [B, R] float, rank [B, R] int32, top_ids int32 and
    top_logprobs float [B, R, n_top], each None if not wanted."""
    dev = _args_here(args)
    shape = args.shape[:2]
    n_top = 0
    one = top_ids if top_ids is not None else top_logprobs
    if one is not None:
        if not isinstance(one, _Tensor) or one.dim() != 3:
            raise ValueError("top_ids and top_logprobs must be device tensors [B, R, n_top]")
        n_top = one.shape[2]
        _sizes(n_top=n_top)
    top = (*shape, n_top)
    if args.zeroed is not None:
        _after_zeroing(args, stream)
    _check("switchsd_token_logprobs", lib.switchsd_token_logprobs(
        ctypes.byref(args), _arr(logprob, "f32", "logprob", shape, dev, True),
        _arr(lse, "f32", "lse", shape, dev, True),
        _arr(entropy, "f32", "entropy", shape, dev, True),
        _arr(rank, "i32", "rank", shape, dev, True), n_top,
        _arr(top_ids, "i32", "top_ids", top, dev, True),
        _arr(top_logprobs, "f32", "top_logprobs", top, dev, True), _stream(stream)))


def switchsd_token_logprobs_grad(args, lse, entropy, g_logprob, g_entropy, grad, stream=None):
    """grad [B, R, V] of the logits' type (the logits themselves: in place) from lse
    and entropy [B, R] of switchsd_token_logprobs and the loss's gradients g_logprob,
    g_entropy [B, R] float (one of the two may be None; entropy is needed with
    g_entropy)."""
    dev = _args_here(args)
    shape = args.shape[:2]
    p_grad = _arr(grad, "logits", "grad", args.shape, dev)
    if _TYPES[grad.dtype] != args.logits_type:
        raise ValueError(f"grad has dtype {grad.dtype}, the logits another")
    _check("switchsd_token_logprobs_grad", lib.switchsd_token_logprobs_grad(
        ctypes.byref(args), _arr(lse, "f32", "lse", shape, dev),
        _arr(entropy, "f32", "entropy", shape, dev, True),
        _arr(g_logprob, "f32", "g_logprob", shape, dev, True),
        _arr(g_entropy, "f32", "g_entropy", shape, dev, True), p_grad, _stream(stream)))
