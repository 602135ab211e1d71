"""ctypes binding of libpsd_b200.so: the same entry points as include/psd.h, argument marshalling only.

Tensor arguments are torch tensors (device tensors for the device entry points, pinned or plain
host tensors for ``psd_step_host``); every step of the path runs inside the library's CUDA
kernels.  There is no fallback: if the shared library cannot be loaded the import of this module
raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass

import torch

from . import build as _build

_i32, _i64, _f32, _f64, _vp, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_void_p, ctypes.c_size_t

PSD_OK = 0
PSD_ERR_NULL, PSD_ERR_SHAPE, PSD_ERR_ALIGN, PSD_ERR_WORKSPACE = -1, -2, -3, -4
PSD_ERR_POLICY, PSD_ERR_CUDA, PSD_ERR_UNSUPPORTED, PSD_ERR_TIMEOUT, PSD_ERR_INTERNAL = -5, -6, -7, -8, -9
PSD_MAX_M, PSD_MAX_DEPTH = 1024, 64
ACCEPT_AGREE_AND_CONF, ACCEPT_AGREE_ONLY, ACCEPT_AGREE_AND_POLICY = 0, 1, 2


class PsdPolicy(ctypes.Structure):
    """psd_policy_t"""
    _fields_ = [("tau", _f32), ("k_min", _i32), ("k_max", _i32), ("depth", _i32), ("stride", _i32),
                ("accept_mode", _i32), ("mask_id", _i32)]


class PsdStepIO(ctypes.Structure):
    """psd_step_io_t"""
    _fields_ = [(n, _vp) for n in ("hidden_bf16", "w_lm_bf16", "sigma", "n_fill", "draft_tokens", "draft_mask",
                                   "tokV", "confV", "tokens", "mask", "k_star", "n_spec_accepted",
                                   "n_committed", "sel", "n_sel", "sel_pos")]


class PsdDag(ctypes.Structure):
    """psd_dag_t"""
    _fields_ = [("n_nodes", _i32), ("reserved", _i32), ("ranks", ctypes.c_uint64 * 64),
                ("parents", ctypes.c_uint64 * 64)]


class PsdDecodeStats(ctypes.Structure):
    """psd_decode_stats_t"""
    _fields_ = [("iterations", _i32), ("forward_passes", _i32), ("masked_left", _i32)]


class PsdTableBody(ctypes.Structure):
    """psd_table_body_t"""
    _fields_ = [("table_bf16", _vp), ("B", _i32), ("H", _i32)]


class PsdKvStrides(ctypes.Structure):
    """psd_kv_strides_t"""
    _fields_ = [("outer", _i64), ("token", _i64), ("head", _i64)]


class PsdAttention(ctypes.Structure):
    """psd_attention_t"""
    _fields_ = [*[(n, _i32) for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P", "S", "dtype", "causal")],
                ("scale", _f32), ("reserved", _i32),
                *[(n, _i64) for n in ("q_token", "q_head", "out_token", "out_head")],
                *[(n, PsdKvStrides) for n in ("kp", "vp", "ko", "vo")]]


class PsdEvict(ctypes.Structure):
    """psd_evict_t"""
    _fields_ = [*[(n, _i32) for n in ("B", "Hkv", "Dh", "P", "keep", "n_sink", "n_recent", "dtype")],
                *[(n, PsdKvStrides) for n in ("k", "v", "k_out", "v_out")]]


class PsdLogitsEdit(ctypes.Structure):
    """psd_logits_edit_t"""
    _fields_ = [*[(n, _vp) for n in ("history", "history_len", "draft_tokens", "draft_mask", "bias", "allow")],
                *[(n, _i32) for n in ("history_cap", "bias_rows", "allow_rows")],
                *[(n, _f32) for n in ("repetition", "presence", "frequency")], ("reserved", _i32)]


class PsdRotate(ctypes.Structure):
    """psd_rotate_t"""
    _fields_ = [*[(n, _i32) for n in ("n_tokens", "Hq", "Hkv", "Dh", "dtype", "rotary", "interleaved", "n_slots")],
                ("eps", _f32), ("gain", _f32),
                *[(f"{n}_{d}", _i64) for n in ("q", "k", "v", "q_out", "k_out", "v_out") for d in ("token", "head")]]


class PsdQuantize(ctypes.Structure):
    """psd_quantize_t"""
    _fields_ = [*[(n, _i32) for n in ("B", "Hkv", "Dh", "P", "block", "dtype", "span", "reserved")],
                *[(n, PsdKvStrides) for n in ("k", "v", "k_codes", "v_codes")]]


# psd_body_fn
BODY_FN = ctypes.CFUNCTYPE(ctypes.c_int, _vp, _vp, _vp, _i32, _i32, _vp, _vp)
ORDER_TWO_PASSES, ORDER_ONE_PASS = 0, 1


class PsdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


def _load() -> ctypes.CDLL:
    # build() compares the library's time stamp with the sources' and recompiles when a source is newer,
    # so a stale library is never loaded silently
    # PSD_B200_DEBUG=1 in the environment selects the debug build of the library (device-side bounds and
    # ring-order checks that report PSD_ERR_INTERNAL through the status word); same entry points
    lib = ctypes.CDLL(_build.build(debug=DEBUG_BUILD))
    pol = PsdPolicy
    lib.psd_status_string.restype = ctypes.c_char_p
    lib.psd_status_string.argtypes = [ctypes.c_int]
    lib.psd_workspace_bytes.restype = _sz
    lib.psd_workspace_bytes.argtypes = [_i32, _i32, _i32]
    lib.psd_compact_workspace_bytes.restype = _sz
    lib.psd_compact_workspace_bytes.argtypes = [_i32, _i32, _i32]
    lib.psd_confidence.restype = ctypes.c_int
    lib.psd_confidence.argtypes = [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
    lib.psd_confidence_masked.restype = ctypes.c_int
    lib.psd_confidence_masked.argtypes = [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
    lib.psd_compact_rows_enabled.restype = ctypes.c_int
    lib.psd_compact_rows_enabled.argtypes = [_i32]
    lib.psd_confidence_partial.restype = ctypes.c_int
    lib.psd_confidence_partial.argtypes = [_vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
    lib.psd_merge_partials.restype = ctypes.c_int
    lib.psd_merge_partials.argtypes = [_vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp]
    lib.psd_confidence_static.restype = ctypes.c_int
    lib.psd_confidence_static.argtypes = [_vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp]
    lib.psd_select_unmask.restype = ctypes.c_int
    lib.psd_select_unmask.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _i32, pol, _vp, _vp, _vp, _vp]
    lib.psd_build_drafts.restype = ctypes.c_int
    lib.psd_build_drafts.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _i32, pol, _vp, _vp, _vp, _vp, _vp]
    lib.psd_verify_accept.restype = ctypes.c_int
    lib.psd_verify_accept.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, pol, _vp, _vp, _vp, _vp, _vp,
                                      _vp, _vp]
    lib.psd_step.restype = ctypes.c_int
    lib.psd_step.argtypes = [ctypes.POINTER(PsdStepIO), _i32, _i32, _i32, _i32, pol, _vp, _sz, _vp, _vp]
    lib.psd_step_host_bytes.restype = _sz
    lib.psd_step_host_bytes.argtypes = [_i32, _i32, _i32, _i32, _i32]
    lib.psd_step_host_block.restype = _sz
    lib.psd_step_host_block.argtypes = [_i32, _i32, _i32, ctypes.POINTER(_sz)]
    lib.psd_step_host.restype = ctypes.c_int
    lib.psd_step_host.argtypes = [ctypes.POINTER(PsdStepIO), _i32, _i32, _i32, _i32, pol, _vp, _sz, _vp, _vp]
    lib.psd_dag_init.restype = ctypes.c_int
    lib.psd_dag_init.argtypes = [ctypes.POINTER(PsdDag), _i32, _vp, _vp]
    lib.psd_build_drafts_dag.restype = ctypes.c_int
    lib.psd_build_drafts_dag.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _i32, pol, ctypes.POINTER(PsdDag), _vp,
                                         _vp, _vp, _vp, _vp]
    lib.psd_verify_accept_dag.restype = ctypes.c_int
    lib.psd_verify_accept_dag.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _i32, pol, ctypes.POINTER(PsdDag), _vp, _vp,
                                          _vp, _vp, _vp, _vp, _vp]
    lib.psd_decode_scratch_bytes.restype = _sz
    lib.psd_decode_scratch_bytes.argtypes = [_i32, _i32]
    lib.psd_decode_blocks.restype = ctypes.c_int
    lib.psd_step_dag.restype = ctypes.c_int
    lib.psd_step_dag.argtypes = [ctypes.POINTER(PsdStepIO), _i32, _i32, _i32, _i32, pol, ctypes.POINTER(PsdDag), _vp,
                                 _sz, _vp, _vp]
    lib.psd_decode_blocks.argtypes = [_vp, _vp, ctypes.POINTER(PsdStepIO), _i32, _i32, _i32, _i32, pol,
                                      ctypes.POINTER(PsdDag), _i32, _i32,
                                      _vp, _sz, _vp, _sz, _vp, _vp, _vp, _vp, ctypes.POINTER(PsdDecodeStats), _vp]
    lib.psd_table_body.restype = ctypes.c_int
    lib.psd_table_body.argtypes = [_vp, _vp, _vp, _i32, _i32, _vp, _vp]
    lib.psd_attention_workspace_bytes.restype = _sz
    lib.psd_attention_workspace_bytes.argtypes = [_i32] * 8
    lib.psd_attention_kernel_names.restype = ctypes.c_char_p
    lib.psd_attention_kernel_names.argtypes = [_i32] * 8 + [_vp]
    lib.psd_draft_attention.restype = ctypes.c_int
    lib.psd_draft_attention.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                        _sz, _vp, _vp]
    lib.psd_weights_workspace_bytes.restype = _sz
    lib.psd_weights_workspace_bytes.argtypes = [_i32] * 7
    lib.psd_prefix_weights.restype = ctypes.c_int
    lib.psd_prefix_weights.argtypes = [_vp, _vp, _vp, _vp, _vp, _f32, _vp, _vp, _vp, _sz, _vp,
                                       _vp]
    lib.psd_prefix_evict.restype = ctypes.c_int
    lib.psd_prefix_evict.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.psd_logits_workspace_bytes.restype = _sz
    lib.psd_logits_workspace_bytes.argtypes = [_i32, _i32]
    lib.psd_confidence_logits.restype = ctypes.c_int
    lib.psd_confidence_logits.argtypes = [_vp, _i32, _i64, _i32, _i32, _i32, _i32, _vp, _vp,
                                          _vp, _vp, _vp, _sz, _vp, _vp]
    lib.psd_rope_frequencies.restype = ctypes.c_int
    lib.psd_rope_frequencies.argtypes = [_i32, _f64, _i32, _f64, _f64, _f64, _f64, _vp, _vp]
    lib.psd_rotate_qk.restype = ctypes.c_int
    lib.psd_rotate_qk.argtypes = [_vp] * 13
    lib.psd_quantize_rows.restype = ctypes.c_int
    lib.psd_quantize_rows.argtypes = [_vp, _i32, _i64, _i64, _i32, _vp, _i64, _vp, _vp]
    lib.psd_prefix_quantize.restype = ctypes.c_int
    lib.psd_prefix_quantize.argtypes = [_vp] * 10
    lib.psd_attention_q8_workspace_bytes.restype = _sz
    lib.psd_attention_q8_workspace_bytes.argtypes = [_i32] * 8
    lib.psd_attention_q8_kernel_names.restype = ctypes.c_char_p
    lib.psd_attention_q8_kernel_names.argtypes = [_i32] * 8 + [_vp]
    lib.psd_draft_attention_q8.restype = ctypes.c_int
    lib.psd_draft_attention_q8.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
    lib.psd_confidence_q8_workspace_bytes.restype = _sz
    lib.psd_confidence_q8_workspace_bytes.argtypes = [_i32] * 3
    lib.psd_confidence_q8.restype = ctypes.c_int
    lib.psd_confidence_q8.argtypes = [_vp, _i32, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
    lib.psd_set_confidence_impl.restype = ctypes.c_int
    lib.psd_set_confidence_impl.argtypes = [ctypes.c_int]
    lib.psd_set_tuning.restype = ctypes.c_int
    lib.psd_set_tuning.argtypes = [ctypes.c_int, ctypes.c_int]
    lib.psd_set_kernel_events.restype = ctypes.c_int
    lib.psd_set_kernel_events.argtypes = [_vp, _vp]
    lib.psd_confidence_kernel_name.restype = ctypes.c_char_p
    lib.psd_confidence_kernel_name.argtypes = [_i32]
    lib.psd_launch_count.restype = _i64
    lib.psd_launch_count.argtypes = []
    return lib


DEBUG_BUILD = os.environ.get("PSD_B200_DEBUG", "0") not in ("", "0")
LIB = _load()
LIB_PATH = _build.LIB_DEBUG if DEBUG_BUILD else _build.LIB


def status_string(code: int) -> str:
    return LIB.psd_status_string(int(code)).decode()


def _check(code: int, where: str):
    if code != PSD_OK:
        raise PsdError(code, where)


def _ptr(t):
    """Address of a tensor's first element, or None."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("psd binding: tensors must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def policy(tau=0.9, k_min=1, k_max=0, depth=1, stride=0, accept_mode=0, mask_id=0) -> PsdPolicy:
    return PsdPolicy(float(tau), int(k_min), int(k_max), int(depth), int(stride), int(accept_mode), int(mask_id))


def psd_workspace_bytes(n_rows: int, H: int, V: int) -> int:
    return int(LIB.psd_workspace_bytes(n_rows, H, V))


def psd_compact_workspace_bytes(n_rows: int, H: int, V: int) -> int:
    return int(LIB.psd_compact_workspace_bytes(n_rows, H, V))


def psd_set_confidence_impl(impl: int) -> int:
    return int(LIB.psd_set_confidence_impl(int(impl)))


PSD_TUNE_BAND_BYTES = 1
PSD_TUNE_PDL = 2
PSD_TUNE_TILE_ORDER = 3
PSD_TUNE_COMPACT_ROWS = 4
PSD_TUNE_WAIT_LIMIT = 5
PSD_TUNE_SELFTEST_STALL = 6


def psd_set_tuning(knob: int, value: int) -> int:
    return int(LIB.psd_set_tuning(int(knob), int(value)))


def psd_set_kernel_events(start_event, stop_event) -> int:
    """torch.cuda.Event objects (already recorded once or created with enable_timing=True), or None."""
    def h(e):
        if e is None:
            return None
        return e.cuda_event if hasattr(e, "cuda_event") else int(e)
    return int(LIB.psd_set_kernel_events(h(start_event), h(stop_event)))


def psd_confidence_kernel_name(n_rows: int) -> str:
    """Name of the kernel the confidence pass launches for ``n_rows`` rows under the current setting."""
    return LIB.psd_confidence_kernel_name(int(n_rows)).decode()


def psd_launch_count() -> int:
    return int(LIB.psd_launch_count())


def psd_confidence(hidden, w_lm, out_token, out_conf, out_lse=None, workspace=None, status=None, stream=None,
                   row_ids=None):
    """hidden [n_rows, H] bf16, w_lm [V, H] bf16 -> out_token int32, out_conf fp32 (and out_lse) [n_rows]."""
    n_rows, H = hidden.shape
    if row_ids is not None:
        n_rows = row_ids.numel()
    V = w_lm.shape[0]
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(LIB.psd_confidence(_ptr(hidden), _ptr(w_lm), _ptr(row_ids), n_rows, H, V, _ptr(out_token),
                              _ptr(out_conf), _ptr(out_lse), _ptr(workspace), ws_bytes, _ptr(status),
                              _stream(stream)), "psd_confidence")


def psd_confidence_masked(hidden, w_lm, row_mask, out_token, out_conf, out_lse=None, workspace=None, status=None,
                          stream=None):
    """psd_confidence on the rows whose ``row_mask`` (int32, device, one entry per row of ``hidden``) is
    non-zero; the other rows' outputs are left untouched.  No host synchronisation."""
    n_rows, H = hidden.shape
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(LIB.psd_confidence_masked(_ptr(hidden), _ptr(w_lm), _ptr(row_mask), n_rows, H, w_lm.shape[0],
                                     _ptr(out_token), _ptr(out_conf), _ptr(out_lse), _ptr(workspace), ws_bytes,
                                     _ptr(status), _stream(stream)), "psd_confidence_masked")


def psd_compact_rows_enabled(n_rows: int) -> int:
    return int(LIB.psd_compact_rows_enabled(int(n_rows)))


def psd_confidence_partial(hidden, w_shard, v_offset, out_max, out_sumexp, out_arg, workspace, status=None,
                           stream=None):
    """Per-row (max, sum-exp, global argmax) over the vocabulary rows held in ``w_shard`` [V_shard, H]."""
    n_rows, H = hidden.shape
    _check(LIB.psd_confidence_partial(_ptr(hidden), _ptr(w_shard), n_rows, H, w_shard.shape[0], int(v_offset),
                                      _ptr(out_max), _ptr(out_sumexp), _ptr(out_arg), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _ptr(status), _stream(stream)),
           "psd_confidence_partial")


def psd_merge_partials(max_, sumexp, arg, out_token, out_conf, out_lse=None, stream=None):
    """Merge [n_shards, n_rows] triples into token / confidence / lse per row."""
    n_shards, n_rows = max_.shape
    _check(LIB.psd_merge_partials(_ptr(max_), _ptr(sumexp), _ptr(arg), n_shards, n_rows, _ptr(out_token),
                                  _ptr(out_conf), _ptr(out_lse), _stream(stream)), "psd_merge_partials")


PSD_STATIC_SCRATCH_BYTES = 4 << 20


def psd_confidence_static(hidden, w_lm, out_token, out_conf, out_lse=None, status=None, stream=None):
    """psd_confidence for callers that cannot allocate: the scratch is a fixed array inside the
    library (PSD_STATIC_SCRATCH_BYTES); larger problems raise PSD_ERR_WORKSPACE.  Calls on one device
    must not overlap."""
    n_rows, H = hidden.shape
    _check(LIB.psd_confidence_static(_ptr(hidden), _ptr(w_lm), n_rows, H, w_lm.shape[0], _ptr(out_token),
                                     _ptr(out_conf), _ptr(out_lse), _ptr(status), _stream(stream)),
           "psd_confidence_static")


def psd_select_unmask(conf, tok, tokens, mask, p: PsdPolicy, sel, n_sel, sel_pos, node=None, n_nodes=1,
                      stream=None):
    B, M = mask.shape
    _check(LIB.psd_select_unmask(_ptr(conf), _ptr(tok), _ptr(node), n_nodes, _ptr(tokens), _ptr(mask), B, M, p,
                                 _ptr(sel), _ptr(n_sel), _ptr(sel_pos), _stream(stream)), "psd_select_unmask")


def psd_build_drafts(conf, tok, tokens, mask, p: PsdPolicy, sigma, n_fill, draft_tokens, draft_mask, node=None,
                     n_nodes=1, stream=None):
    B, M = mask.shape
    _check(LIB.psd_build_drafts(_ptr(conf), _ptr(tok), _ptr(node), n_nodes, _ptr(tokens), _ptr(mask), B, M, p,
                                _ptr(sigma), _ptr(n_fill), _ptr(draft_tokens), _ptr(draft_mask), _stream(stream)),
           "psd_build_drafts")


def psd_verify_accept(tokV, confV, sigma, n_fill, draft_tokens, draft_mask, p: PsdPolicy, tokens, mask, k_star,
                      n_spec_accepted, n_committed, accepted=None, stream=None):
    B, M = tokens.shape
    _check(LIB.psd_verify_accept(_ptr(tokV), _ptr(confV), _ptr(sigma), _ptr(n_fill), _ptr(draft_tokens),
                                 _ptr(draft_mask), B, M, p, _ptr(tokens), _ptr(mask), _ptr(k_star),
                                 _ptr(n_spec_accepted), _ptr(n_committed), _ptr(accepted), _stream(stream)),
           "psd_verify_accept")


_STEP_FIELDS = [n for n, _ in PsdStepIO._fields_]


@dataclass
class StepBuffers:
    """The tensors of one decoding step (psd_step_io_t), all on one device or all on the host
    (``w_lm`` always on the device)."""
    hidden: torch.Tensor
    w_lm: torch.Tensor
    sigma: torch.Tensor
    n_fill: torch.Tensor
    draft_tokens: torch.Tensor
    draft_mask: torch.Tensor
    tokV: torch.Tensor
    confV: torch.Tensor
    tokens: torch.Tensor
    mask: torch.Tensor
    k_star: torch.Tensor
    n_spec_accepted: torch.Tensor
    n_committed: torch.Tensor
    sel: torch.Tensor
    n_sel: torch.Tensor
    sel_pos: torch.Tensor

    def io(self) -> PsdStepIO:
        vals = [self.hidden, self.w_lm, self.sigma, self.n_fill, self.draft_tokens, self.draft_mask, self.tokV,
                self.confV, self.tokens, self.mask, self.k_star, self.n_spec_accepted, self.n_committed, self.sel,
                self.n_sel, self.sel_pos]
        return PsdStepIO(*[_ptr(v) for v in vals])

    @staticmethod
    def allocate(B, M, D, H, hidden, w_lm, device, pin=False):
        kw = dict(device=device)
        if pin:
            kw["pin_memory"] = True
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, **kw)
        return StepBuffers(hidden=hidden, w_lm=w_lm, sigma=i32(B, M), n_fill=i32(B, D), draft_tokens=i32(B, D, M),
                           draft_mask=i32(B, D, M), tokV=i32(B, D, M),
                           confV=torch.zeros(B, D, M, dtype=torch.float32, **kw), tokens=i32(B, M), mask=i32(B, M),
                           k_star=i32(B), n_spec_accepted=i32(B), n_committed=i32(B), sel=i32(B, M), n_sel=i32(B),
                           sel_pos=i32(B, M))


def psd_step_host_block(B, M, D):
    """(bytes, offsets[15]) of the one-block host layout that psd_step_host moves with single copies."""
    off = (_sz * 15)()
    n = int(LIB.psd_step_host_block(B, M, D, off))
    return n, [int(x) for x in off]


def host_step_buffers(B, M, D, hidden, w_lm) -> StepBuffers:
    """StepBuffers whose arrays are views of ONE pinned host block laid out as psd_step_host_block says
    (``hidden``: a host tensor, ``w_lm``: a device tensor).  The block is kept alive by the views."""
    n, off = psd_step_host_block(B, M, D)
    block = torch.zeros(n, dtype=torch.uint8).pin_memory()

    def view(o, shape, dtype=torch.int32):
        count = 1
        for d in shape:
            count *= d
        return block[o:o + 4 * count].view(dtype).view(*shape)

    return StepBuffers(hidden=hidden, w_lm=w_lm, sigma=view(off[0], (B, M)), n_fill=view(off[1], (B, D)),
                       draft_tokens=view(off[2], (B, D, M)), draft_mask=view(off[3], (B, D, M)),
                       tokV=view(off[4], (B, D, M)), confV=view(off[5], (B, D, M), torch.float32),
                       tokens=view(off[6], (B, M)), mask=view(off[7], (B, M)), k_star=view(off[8], (B,)),
                       n_spec_accepted=view(off[9], (B,)), n_committed=view(off[10], (B,)), sel=view(off[11], (B, M)),
                       n_sel=view(off[12], (B,)), sel_pos=view(off[13], (B, M)))


def psd_step(buf: StepBuffers, p: PsdPolicy, workspace, status=None, stream=None):
    B, M = buf.tokens.shape
    H = buf.hidden.shape[1]
    V = buf.w_lm.shape[0]
    io = buf.io()
    _check(LIB.psd_step(ctypes.byref(io), B, M, H, V, p, _ptr(workspace),
                        workspace.numel() * workspace.element_size(), _ptr(status), _stream(stream)), "psd_step")


def psd_step_host_bytes(B, M, H, V, D) -> int:
    return int(LIB.psd_step_host_bytes(B, M, H, V, D))


def psd_step_host(buf: StepBuffers, p: PsdPolicy, staging, stream=None) -> int:
    """``buf`` holds host tensors (w_lm on the device).  Returns the device status word."""
    B, M = buf.tokens.shape
    H = buf.hidden.shape[1]
    V = buf.w_lm.shape[0]
    io = buf.io()
    st = _i32(0)
    _check(LIB.psd_step_host(ctypes.byref(io), B, M, H, V, p, _ptr(staging),
                             staging.numel() * staging.element_size(), ctypes.byref(st), _stream(stream)),
           "psd_step_host")
    return int(st.value)


def psd_decode_scratch_bytes(B: int, M: int) -> int:
    return int(LIB.psd_decode_scratch_bytes(B, M))


def psd_step_dag(buf: StepBuffers, p: PsdPolicy, g: PsdDag, workspace, status=None, stream=None):
    B, M = buf.tokens.shape
    io = buf.io()
    _check(LIB.psd_step_dag(ctypes.byref(io), B, M, buf.hidden.shape[1], buf.w_lm.shape[0], p, ctypes.byref(g),
                            _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(status),
                            _stream(stream)), "psd_step_dag")


def psd_decode_blocks(body, user, buf: StepBuffers, p: PsdPolicy, order: int, max_iterations: int, scratch,
                      workspace, status=None, passes=None, done_iteration=None, trace=None, stream=None, dag=None):
    """Algorithm 1 over the blocks of ``buf`` (device tensors; ``buf.hidden`` is scratch the body fills).

    ``body`` is either the address of a native ``psd_body_fn`` (an int, e.g. ``table_body_address()``)
    with ``user`` the address of its argument, or a Python callable
    ``body(tokens_ptr, mask_ptr, n_seq, M, hidden_ptr, stream_ptr) -> int``.  Returns PsdDecodeStats."""
    B, M = buf.tokens.shape
    H = buf.hidden.shape[1]
    V = buf.w_lm.shape[0]
    if callable(body):
        fn = body
        cb = BODY_FN(lambda u, t, m, n, mm, h, s: int(fn(t, m, n, mm, h, s)))
        body_ptr = ctypes.cast(cb, _vp)
    else:
        cb, body_ptr = None, _vp(int(body))
    io = buf.io()
    stats = PsdDecodeStats()
    code = LIB.psd_decode_blocks(body_ptr, user, ctypes.byref(io), B, M, H, V, p,
                                 ctypes.byref(dag) if dag is not None else None, int(order), int(max_iterations),
                                 _ptr(scratch), scratch.numel() * scratch.element_size(), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _ptr(status), _ptr(passes),
                                 _ptr(done_iteration), _ptr(trace), ctypes.byref(stats), _stream(stream))
    del cb
    _check(code, "psd_decode_blocks")
    return stats


def table_body_address() -> int:
    """Address of the native stand-in body psd_table_body, to pass as ``body``."""
    return ctypes.cast(LIB.psd_table_body, _vp).value


def table_body_user(table, B: int) -> PsdTableBody:
    """psd_table_body_t for a device table [B, M, 3, H] bf16; keep the object alive during the call and
    pass ``ctypes.addressof(obj)`` as ``user``."""
    return PsdTableBody(_ptr(table), int(B), int(table.shape[-1]))


def psd_table_body(user: PsdTableBody, mask, hidden, stream=None):
    """One call of the stand-in body: ``mask`` [n_seq, M] int32 -> ``hidden`` [n_seq*M, H] bf16 (device)."""
    n_seq, M = mask.shape
    _check(LIB.psd_table_body(ctypes.addressof(user), None, _ptr(mask), n_seq, M, _ptr(hidden), _stream(stream)),
           "psd_table_body")


def psd_dag_init(node_ranks, edges=None) -> PsdDag:
    """A draft graph from node rank sets (node 0 = the root, empty) and, optionally, an edge list
    [(p, k), ...]; without one every strict-subset pair is an edge."""
    K = len(node_ranks)
    ranks = (ctypes.c_uint64 * max(K, 1))(*[sum(1 << int(j) for j in s) for s in node_ranks])
    par = None
    if edges is not None:
        words = [0] * K
        for q, k in edges:
            words[k] |= 1 << q
        par = (ctypes.c_uint64 * max(K, 1))(*words)
    g = PsdDag()
    _check(LIB.psd_dag_init(ctypes.byref(g), K, ctypes.cast(ranks, _vp), ctypes.cast(par, _vp) if par else None),
           "psd_dag_init")
    return g


def psd_build_drafts_dag(conf, tok, tokens, mask, p: PsdPolicy, g: PsdDag, sigma, n_fill, draft_tokens, draft_mask,
                         node=None, n_nodes=1, stream=None):
    B, M = mask.shape
    _check(LIB.psd_build_drafts_dag(_ptr(conf), _ptr(tok), _ptr(node), n_nodes, _ptr(tokens), _ptr(mask), B, M, p,
                                    ctypes.byref(g), _ptr(sigma), _ptr(n_fill), _ptr(draft_tokens), _ptr(draft_mask),
                                    _stream(stream)), "psd_build_drafts_dag")


def psd_verify_accept_dag(tokV, confV, sigma, draft_tokens, draft_mask, p: PsdPolicy, g: PsdDag, tokens, mask, k_star,
                          n_spec_accepted, n_committed, accepted=None, stream=None):
    B, M = tokens.shape
    _check(LIB.psd_verify_accept_dag(_ptr(tokV), _ptr(confV), _ptr(sigma), _ptr(draft_tokens), _ptr(draft_mask), B, M,
                                     p, ctypes.byref(g), _ptr(tokens), _ptr(mask), _ptr(k_star), _ptr(n_spec_accepted),
                                     _ptr(n_committed), _ptr(accepted), _stream(stream)), "psd_verify_accept_dag")


# ---- around the step: attention of the drafts, the prefix's cache, confidences from logits -------------------------
#
# These calls are made many times per forward pass (once per layer), on work that can be a few microseconds long, so their
# marshalling is kept short: descriptors are packed into bytes in the layout of the C structs (PsdAttention, PsdEvict and
# PsdLogitsEdit describe the same layouts), and the current stream's handle is asked for without building a Stream object.

PSD_BF16, PSD_FP16, PSD_FP32 = 0, 1, 2
_DTYPES = {torch.bfloat16: PSD_BF16, torch.float16: PSD_FP16, torch.float32: PSD_FP32}
_I32, _F32 = torch.int32, torch.float32
_pack_attention = struct.Struct("=10ifi4q12q").pack
_pack_evict = struct.Struct("=8i12q").pack
_pack_edit = struct.Struct("=6Q3i3fi4x").pack


def _here(stream, *tensors):
    """The handle of the stream to launch on.  All tensors (None: not given) have to be on the current CUDA device, since the
    kernels would follow any other address as well: a list of lengths left on the host would fault the GPU."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"psd binding: tensors of one call are on one CUDA device, got {tensors[0].device} and {t.device}")
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise ValueError(f"psd binding: tensors have to be on the current CUDA device, got {tensors[0].device}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _want(t, shape, dtype, name):
    """Address of a dense tensor of this shape and type, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"psd binding: {name} must be dense {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _want_n(t, n, dtype, name):
    """Address of a dense tensor of n elements of this type, whatever its shape, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"psd binding: {name} must be dense {dtype} with {n} elements, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _space(t):
    """(address, bytes) of a workspace."""
    return (None, 0) if t is None else (_ptr(t), t.nbytes)


def _tokens_strides(t, N, M, H, Dh, name):
    """(token, head) strides of [N, M, H, Dh] whose first two dimensions are one run of tokens."""
    sn, sm, sh, sd = t.stride()
    if (sd != 1 and Dh > 1) or (N > 1 and M > 1 and sn != M * sm):
        raise ValueError(f"psd binding: {name} needs a dense last dimension and nodes M tokens apart")
    return (sm if M > 1 else sn if N > 1 else H * Dh), (sh if H > 1 else Dh)


_NO_CACHE = (0, 8, 0, 0, 8, 0)


def _kv_strides(strides, no, nt, nh, nd, name):
    """(outer, token, head) strides of a cache; that of a dimension of one is never walked: 0 (shared), or the smallest the
    library takes."""
    so, st, sh, sd = strides
    if sd != 1 and nd > 1:
        raise ValueError(f"psd binding: {name} needs a dense last dimension")
    return so if no > 1 else 0, st if nt > 1 else 8, sh if nh > 1 else 0


def _pair_strides(k, v, no, nt, nh, nd, name):
    """Strides of a cache's keys and of its values (one shape, and mostly one layout)."""
    of_k, of_v = k.stride(), v.stride()
    s = _kv_strides(of_k, no, nt, nh, nd, name)
    return s + s if of_v == of_k else s + _kv_strides(of_v, no, nt, nh, nd, name)


def _one_type(dt, *tensors):
    for t in tensors:
        if t is not None and t.dtype is not dt:
            raise ValueError(f"psd binding: tensors of one call differ in type ({dt} and {t.dtype})")
    return _DTYPES.get(dt, -1)      # a type the library does not know is refused by the call


def psd_attention_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S) -> int:
    return int(LIB.psd_attention_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S))


def psd_attention_kernel_names(B, D, M, Hq, Hkv, Dh, P, S):
    """(names of the kernels that psd_draft_attention launches at these sizes, partial results per row), or None."""
    splits = _i32(0)
    names = LIB.psd_attention_kernel_names(B, D, M, Hq, Hkv, Dh, P, S, ctypes.byref(splits))
    return None if names is None else (names.decode(), splits.value)


def psd_draft_attention(q, k_prefix, v_prefix, out, lse=None, k_own=None, v_own=None, prefix_len=None, own_len=None,
                        scale=None, causal=False, workspace=None, status=None, stream=None):
    """q [B*D, M, Hq, Dh] over the prefix caches [B, P, Hkv, Dh] and each node's own keys [B*D, S, Hkv, Dh] -> out
    (like q) and lse [B*D, M, Hq].  Strided tensors are taken as they are; ``scale`` defaults to 1/sqrt(Dh)."""
    rows, cache = q.shape, k_prefix.shape
    N, M, Hq, Dh = rows
    B, P, Hkv, dk = cache
    if B < 1 or N % B or dk != Dh:
        raise ValueError("psd binding: q [B*D, M, Hq, Dh] and k_prefix [B, P, Hkv, Dh] do not belong together")
    if v_prefix.shape != cache or out.shape != rows or (k_own is None) != (v_own is None):
        raise ValueError("psd binding: keys and values, and out and q, have one shape; k_own and v_own come together")
    S, ko, vo, own = 0, None, None, _NO_CACHE
    if k_own is not None:
        shape = k_own.shape
        S = shape[1]
        if shape != (N, S, Hkv, Dh) or v_own.shape != shape:
            raise ValueError("psd binding: k_own and v_own are [B*D, S, Hkv, Dh]")
        own = _pair_strides(k_own, v_own, N, S, Hkv, Dh, "k_own, v_own")
        ko, vo = k_own.data_ptr() or None, v_own.data_ptr() or None
    a = _pack_attention(B, N // B, M, Hq, Hkv, Dh, P, S, _one_type(q.dtype, k_prefix, v_prefix, k_own, v_own, out),
                        1 if causal else 0, Dh ** -0.5 if scale is None else scale, 0,
                        *_tokens_strides(q, N, M, Hq, Dh, "q"), *_tokens_strides(out, N, M, Hq, Dh, "out"),
                        *_pair_strides(k_prefix, v_prefix, B, P, Hkv, Dh, "k_prefix, v_prefix"), *own)
    stream = _here(stream, q, k_prefix, v_prefix, out, lse, k_own, v_own, prefix_len, own_len, workspace, status)
    ws, ws_bytes = _space(workspace)
    _check(LIB.psd_draft_attention(q.data_ptr(), k_prefix.data_ptr() or None, v_prefix.data_ptr() or None,
                                   _want(prefix_len, (B,), _I32, "prefix_len"), ko, vo,
                                   _want(own_len, (N,), _I32, "own_len"), a, out.data_ptr(),
                                   _want(lse, (N, M, Hq), _F32, "lse"), ws, ws_bytes, _ptr(status), stream),
           "psd_draft_attention")


def psd_weights_workspace_bytes(B, D, M, Hq, Hkv, Dh, P) -> int:
    return int(LIB.psd_weights_workspace_bytes(B, D, M, Hq, Hkv, Dh, P))


def psd_prefix_weights(q, k_prefix, lse, acc_out, acc_in=None, beta=1.0, prefix_len=None, scale=None, workspace=None,
                       status=None, stream=None):
    """acc_out [B, Hkv, P] = beta * acc_in + the attention weight each prefix key draws from the rows of ``q`` (``lse``
    [B*D, M, Hq] as psd_draft_attention wrote it).  acc_in may be acc_out."""
    N, M, Hq, Dh = q.shape
    B, P, Hkv, dk = k_prefix.shape
    if B < 1 or N % B or dk != Dh:
        raise ValueError("psd binding: q [B*D, M, Hq, Dh] and k_prefix [B, P, Hkv, Dh] do not belong together")
    a = _pack_attention(B, N // B, M, Hq, Hkv, Dh, P, 0, _one_type(q.dtype, k_prefix), 0,
                        Dh ** -0.5 if scale is None else scale, 0,
                        *_tokens_strides(q, N, M, Hq, Dh, "q"), 0, 0,
                        *_kv_strides(k_prefix.stride(), B, P, Hkv, Dh, "k_prefix"), 0, 0, 0, 0, 0, 0, 0, 0, 0)
    sums = (B, Hkv, P)
    stream = _here(stream, q, k_prefix, lse, acc_out, acc_in, prefix_len, workspace, status)
    ws, ws_bytes = _space(workspace)
    _check(LIB.psd_prefix_weights(q.data_ptr(), k_prefix.data_ptr() or None, _want(prefix_len, (B,), _I32, "prefix_len"),
                                  _want(lse, (N, M, Hq), _F32, "lse"), a, beta, _want(acc_in, sums, _F32, "acc_in"),
                                  _want(acc_out, sums, _F32, "acc_out"), ws, ws_bytes, _ptr(status), stream),
           "psd_prefix_weights")


def psd_prefix_evict(scores, k, v, k_out, v_out, index, scores_out=None, len_out=None, prefix_len=None, n_sink=0,
                     n_recent=0, stream=None):
    """Keep index.shape[2] keys per sequence and key head of the caches k, v [B, P, Hkv, Dh]: packed into k_out, v_out
    [B, keep, Hkv, Dh], their positions into index [B, Hkv, keep]."""
    cache, kept_rows = k.shape, k_out.shape
    B, P, Hkv, Dh = cache
    keep = index.shape[-1]
    if v.shape != cache or kept_rows != (B, keep, Hkv, Dh) or v_out.shape != kept_rows:
        raise ValueError("psd binding: k, v are [B, P, Hkv, Dh], k_out, v_out [B, keep, Hkv, Dh]")
    e = _pack_evict(B, Hkv, Dh, P, keep, n_sink, n_recent, _one_type(k.dtype, v, k_out, v_out),
                    *_pair_strides(k, v, B, P, Hkv, Dh, "k, v"), *_pair_strides(k_out, v_out, B, keep, Hkv, Dh, "k_out, v_out"))
    stream = _here(stream, k, v, scores, k_out, v_out, index, scores_out, len_out, prefix_len)
    kept = (B, Hkv, keep)
    _check(LIB.psd_prefix_evict(_want(scores, (B, Hkv, P), _F32, "scores"), k.data_ptr(), v.data_ptr(),
                                _want(prefix_len, (B,), _I32, "prefix_len"), e, k_out.data_ptr(), v_out.data_ptr(),
                                _want(index, kept, _I32, "index"), _want(scores_out, kept, _F32, "scores_out"),
                                _want(len_out, (B,), _I32, "len_out"), stream), "psd_prefix_evict")


def psd_logits_workspace_bytes(n_rows: int, V: int) -> int:
    return int(LIB.psd_logits_workspace_bytes(n_rows, V))


def psd_confidence_logits(logits, out_token, out_conf, out_lse=None, B=None, D=1, M=1, history=None, history_len=None,
                          draft_tokens=None, draft_mask=None, repetition=1.0, presence=0.0, frequency=0.0, bias=None,
                          allow=None, workspace=None, status=None, stream=None):
    """Token, confidence and lse of every row of ``logits`` [B*D*M, V] after the edits: penalties for tokens of
    ``history`` [B, T] (the first history_len[b]) and of a draft's filled slots, ``bias`` [V] or [rows, V], ``allow``
    [rows, ceil(V/32)] int32 bit masks (a row of bias or allow serves R / rows consecutive rows)."""
    R, V = logits.shape
    if B is None:
        B = R // (D * M)
    row, one = logits.stride()
    if B * D * M != R or (one != 1 and V > 1):
        raise ValueError("psd binding: logits [B*D*M, V] needs a dense last dimension")
    stream = _here(stream, logits, out_token, out_conf, out_lse, history, history_len, draft_tokens, draft_mask, bias, allow,
                   workspace, status)
    T = bias_rows = allow_rows = 0
    h = hl = dt = dm = bi = al = 0
    if history is not None:
        shape = history.shape
        T = shape[1]
        if shape[0] != B:
            raise ValueError(f"psd binding: history must have {B} rows, got {tuple(shape)}")
        h = _want_n(history, B * T, _I32, "history")
        hl = _want(history_len, (B,), _I32, "history_len") or 0
    if draft_tokens is not None:
        dt = _want_n(draft_tokens, R, _I32, "draft_tokens")
    if draft_mask is not None:
        dm = _want_n(draft_mask, R, _I32, "draft_mask")
    if bias is not None:
        bias_rows = 1 if bias.dim() == 1 else bias.shape[0]
        bi = _want_n(bias, bias_rows * V, _F32, "bias")
    if allow is not None:
        allow_rows = allow.shape[0]
        al = _want(allow, (allow_rows, (V + 31) // 32), _I32, "allow")
    e = _pack_edit(h, hl, dt, dm, bi, al, T, bias_rows, allow_rows, repetition, presence, frequency, 0)
    ws, ws_bytes = _space(workspace)
    _check(LIB.psd_confidence_logits(logits.data_ptr(), _DTYPES.get(logits.dtype, -1), row if R > 1 else V, B, D, M, V, e,
                                     _want_n(out_token, R, _I32, "out_token"), _want_n(out_conf, R, _F32, "out_conf"),
                                     _want_n(out_lse, R, _F32, "out_lse"), ws, ws_bytes, _ptr(status), stream),
           "psd_confidence_logits")


# ---- a step in 8 bits: rotation, the prefix's cache and the LM head in codes -----------------------------------------------

PSD_ROPE_PLAIN, PSD_ROPE_LINEAR, PSD_ROPE_STRETCHED, PSD_ROPE_BY_PARTS = 0, 1, 2, 3
_F64, _I8 = torch.float64, torch.int8
_pack_rotate = struct.Struct("=8i2f12q").pack
_pack_quantize = struct.Struct("=8i12q").pack


def _fits(*sizes):
    """Sizes that go to the library as 32-bit arguments: ctypes would pass on their low bits."""
    for n in sizes:
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"psd binding: {n} does not fit into 32 bits")


def psd_rope_frequencies(rotary, base=10000.0, kind=PSD_ROPE_PLAIN, factor=1.0, original=0.0, low=1.0, high=32.0):
    """(frequencies [rotary/2] float64 on the CPU, the gain that goes with them) for psd_rotate_qk."""
    _fits(int(rotary), int(kind))
    table, gain = torch.empty(max(int(rotary) // 2, 1), dtype=_F64), _f32(1.0)
    _check(LIB.psd_rope_frequencies(int(rotary), float(base), int(kind), float(factor), float(original), float(low), float(high),
                                    table.data_ptr(), ctypes.byref(gain)), "psd_rope_frequencies")
    return table, gain.value


def _heads_strides(t, name):
    """(tokens, heads, head size, token stride, head stride) of [T, H, Dh], or of [N, M, H, Dh] whose first two dimensions are
    one run."""
    shape = t.shape
    if len(shape) == 3:
        T, H, Dh = shape
        st, sh, sd = t.stride()
        if sd != 1 and Dh > 1:
            raise ValueError(f"psd binding: {name} needs a dense last dimension")
        return T, H, Dh, st if T > 1 else H * Dh, sh if H > 1 else Dh
    N, M, H, Dh = shape
    return N * M, H, Dh, *_tokens_strides(t, N, M, H, Dh, name)


def psd_rotate_qk(q, k, q_out, k_out, position, frequency, v=None, v_out=None, slot=None, q_norm=None, k_norm=None, eps=1e-6,
                  interleaved=False, gain=1.0, stream=None):
    """Norms and position rotation of q [T, Hq, Dh] and k [T, Hkv, Dh] (or [N, M, H, Dh]; either may be None with its output)
    into q_out and k_out, v into v_out; with ``slot`` [T] int32, token t of k and v goes to row slot[t].  ``frequency``
    [rotary/2] float64 says how much of a head is rotated (None: nothing)."""
    some = q if q is not None else k
    if some is None or (q is None) != (q_out is None) or (k is None) != (k_out is None) or (v is None) != (v_out is None) or \
            (v is not None and k is None):
        raise ValueError("psd binding: q, k and v come with their outputs, v with k")
    T = Hq = Hkv = n_slots = 0
    qa = qb = qc = qd = ka = kb = kc = kd = va = vb = vc = vd = 8
    pq = pk = pv = oq = ok = ov = None
    if q is not None:
        T, Hq, Dh, qa, qb = _heads_strides(q, "q")
        To, Ho, Do, qc, qd = _heads_strides(q_out, "q_out")
        if To != T or Ho != Hq or Do != Dh:
            raise ValueError("psd binding: q_out has q's tokens, heads and head size")
        pq, oq = q.data_ptr(), q_out.data_ptr()
    if k is not None:
        Tk, Hkv, Dk, ka, kb = _heads_strides(k, "k")
        n_slots, Ho, Do, kc, kd = _heads_strides(k_out, "k_out")
        if q is None:
            T, Dh = Tk, Dk
        if Tk != T or Dk != Dh or Ho != Hkv or Do != Dh or (slot is None and n_slots != T):
            raise ValueError("psd binding: k has q's tokens and head size, k_out k's heads (and, without slots, its tokens)")
        pk, ok = k.data_ptr(), k_out.data_ptr()
        if v is not None:
            Tv, Hv, Dv, va, vb = _heads_strides(v, "v")
            To, Ho, Do, vc, vd = _heads_strides(v_out, "v_out")
            if Tv != T or Hv != Hkv or Dv != Dh or To != n_slots or Ho != Hkv or Do != Dh:
                raise ValueError("psd binding: v has k's shape, v_out k_out's")
            pv, ov = v.data_ptr(), v_out.data_ptr()
    pairs = 0 if frequency is None else frequency.numel()
    r = _pack_rotate(T, Hq, Hkv, Dh, _one_type(some.dtype, q, k, v, q_out, k_out, v_out), 2 * pairs, 1 if interleaved else 0, n_slots, eps,
                     gain, qa, qb, ka, kb, va, vb, qc, qd, kc, kd, vc, vd)
    stream = _here(stream, some, k, v, q_out, k_out, v_out, position, frequency, slot, q_norm, k_norm)
    _check(LIB.psd_rotate_qk(pq, pk, pv, _want_n(position, T, _I32, "position"), _want_n(frequency, pairs, _F64, "frequency"),
                             _want(q_norm, (Dh,), some.dtype, "q_norm"), _want(k_norm, (Dh,), some.dtype, "k_norm"),
                             _want_n(slot, T, _I32, "slot"), r, oq, ok, ov, stream), "psd_rotate_qk")


def psd_quantize_rows(x, codes, scale, stream=None):
    """Codes [R, H] int8 and scale [R] of the rows of x [R, H] (bf16 or fp16); rows may be strided."""
    R, H = x.shape
    if codes.shape != x.shape or codes.dtype is not _I8 or (x.stride(1) != 1 or codes.stride(1) != 1) and H > 1:
        raise ValueError("psd binding: x [R, H] and codes [R, H] int8 need a dense last dimension")
    _fits(H)
    stream = _here(stream, x, codes, scale)
    _check(LIB.psd_quantize_rows(x.data_ptr(), _DTYPES.get(x.dtype, -1), x.stride(0) if R > 1 else H, R, H, codes.data_ptr(),
                                 codes.stride(0) if R > 1 else H, _want(scale, (R,), _F32, "scale"), stream), "psd_quantize_rows")


def psd_prefix_quantize(k, v, k_codes, v_codes, k_scale, v_scale, block=32, begin=None, end=None, span=0, stream=None):
    """Tokens [begin[b], end[b]) of the caches k, v [B, P, Hkv, Dh] into codes [B, P, Hkv, Dh] int8 with scales
    [B, Hkv, ceil(P / block)].  ``span``: the most tokens of any range, where the host knows (0: P)."""
    cache = k.shape
    B, P, Hkv, Dh = cache
    if v.shape != cache or k_codes.shape != cache or v_codes.shape != cache or k_codes.dtype is not _I8 or v_codes.dtype is not _I8:
        raise ValueError("psd binding: k, v and their codes (int8) are [B, P, Hkv, Dh]")
    if block < 1:
        raise ValueError("psd binding: block must be positive")
    q = _pack_quantize(B, Hkv, Dh, P, block, _one_type(k.dtype, v), span, 0, *_pair_strides(k, v, B, P, Hkv, Dh, "k, v"),
                       *_pair_strides(k_codes, v_codes, B, P, Hkv, Dh, "k_codes, v_codes"))
    stream = _here(stream, k, v, k_codes, v_codes, k_scale, v_scale, begin, end)
    sc = (B, Hkv, -(-P // block))
    _check(LIB.psd_prefix_quantize(k.data_ptr(), v.data_ptr(), _want(begin, (B,), _I32, "begin"), _want(end, (B,), _I32, "end"), q,
                                   k_codes.data_ptr(), v_codes.data_ptr(), _want(k_scale, sc, _F32, "k_scale"),
                                   _want(v_scale, sc, _F32, "v_scale"), stream), "psd_prefix_quantize")


def psd_attention_q8_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S) -> int:
    _fits(B, D, M, Hq, Hkv, Dh, P, S)
    return int(LIB.psd_attention_q8_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S))


def psd_attention_q8_kernel_names(B, D, M, Hq, Hkv, Dh, P, S):
    """(names of the kernels that psd_draft_attention_q8 launches at these sizes, partial results per row), or None."""
    _fits(B, D, M, Hq, Hkv, Dh, P, S)
    splits = _i32(0)
    names = LIB.psd_attention_q8_kernel_names(B, D, M, Hq, Hkv, Dh, P, S, ctypes.byref(splits))
    return None if names is None else (names.decode(), splits.value)


def _codes_strides(strides, no, nt, nh, nd, name):
    """As _kv_strides, for codes: the smallest stride the library takes is 16."""
    so, st, sh, sd = strides
    if sd != 1 and nd > 1:
        raise ValueError(f"psd binding: {name} needs a dense last dimension")
    return so if no > 1 else 0, st if nt > 1 else 16, sh if nh > 1 else 0


def psd_draft_attention_q8(q, k_codes, v_codes, k_scale, v_scale, out, lse=None, k_own=None, v_own=None, block=32, prefix_len=None,
                           own_len=None, scale=None, causal=False, workspace=None, status=None, stream=None):
    """psd_draft_attention over prefix caches in codes [B, P, Hkv, Dh] int8 with scales [B, Hkv, ceil(P / block)]."""
    rows, cache = q.shape, k_codes.shape
    N, M, Hq, Dh = rows
    B, P, Hkv, dk = cache
    if B < 1 or N % B or dk != Dh:
        raise ValueError("psd binding: q [B*D, M, Hq, Dh] and k_codes [B, P, Hkv, Dh] do not belong together")
    if v_codes.shape != cache or k_codes.dtype is not _I8 or v_codes.dtype is not _I8:
        raise ValueError("psd binding: k_codes and v_codes are int8 of one shape")
    if out.shape != rows or (k_own is None) != (v_own is None) or block < 1:
        raise ValueError("psd binding: out and q have one shape, k_own and v_own come together, block is positive")
    _fits(block)
    S, ko, vo, own = 0, None, None, _NO_CACHE
    if k_own is not None:
        shape = k_own.shape
        S = shape[1]
        if shape != (N, S, Hkv, Dh) or v_own.shape != shape:
            raise ValueError("psd binding: k_own and v_own are [B*D, S, Hkv, Dh]")
        own = _pair_strides(k_own, v_own, N, S, Hkv, Dh, "k_own, v_own")
        ko, vo = k_own.data_ptr() or None, v_own.data_ptr() or None
    a = _pack_attention(B, N // B, M, Hq, Hkv, Dh, P, S, _one_type(q.dtype, k_own, v_own, out), 1 if causal else 0,
                        Dh ** -0.5 if scale is None else scale, 0, *_tokens_strides(q, N, M, Hq, Dh, "q"),
                        *_tokens_strides(out, N, M, Hq, Dh, "out"), *_codes_strides(k_codes.stride(), B, P, Hkv, Dh, "k_codes"),
                        *_codes_strides(v_codes.stride(), B, P, Hkv, Dh, "v_codes"), *own)
    stream = _here(stream, q, k_codes, v_codes, k_scale, v_scale, out, lse, k_own, v_own, prefix_len, own_len, workspace, status)
    sc = (B, Hkv, -(-P // block))
    ws, ws_bytes = _space(workspace)
    _check(LIB.psd_draft_attention_q8(q.data_ptr(), k_codes.data_ptr() or None, v_codes.data_ptr() or None,
                                      _want(k_scale, sc, _F32, "k_scale") or None, _want(v_scale, sc, _F32, "v_scale") or None, block,
                                      _want(prefix_len, (B,), _I32, "prefix_len"), ko, vo, _want(own_len, (N,), _I32, "own_len"), a,
                                      out.data_ptr(), _want(lse, (N, M, Hq), _F32, "lse"), ws, ws_bytes, _ptr(status), stream),
           "psd_draft_attention_q8")


def psd_confidence_q8_workspace_bytes(n_rows: int, H: int, V: int) -> int:
    _fits(n_rows, H, V)
    return int(LIB.psd_confidence_q8_workspace_bytes(n_rows, H, V))


def psd_confidence_q8(hidden, w_codes, w_scale, out_token, out_conf, out_lse=None, workspace=None, status=None, stream=None):
    """Token, confidence and lse of every row of ``hidden`` [R, H] (bf16 or fp16) over an LM head in codes [V, H] int8 with a
    scale [V] per vocabulary row."""
    R, H = hidden.shape
    V = w_codes.shape[0]
    if not hidden.is_contiguous():
        raise ValueError("psd binding: hidden must be contiguous")
    _fits(R, H, V)
    stream = _here(stream, hidden, w_codes, w_scale, out_token, out_conf, out_lse, workspace, status)
    ws, ws_bytes = _space(workspace)
    _check(LIB.psd_confidence_q8(hidden.data_ptr(), _DTYPES.get(hidden.dtype, -1), _want(w_codes, (V, H), _I8, "w_codes"),
                                 _want(w_scale, (V,), _F32, "w_scale"), R, H, V, _want_n(out_token, R, _I32, "out_token"),
                                 _want_n(out_conf, R, _F32, "out_conf"), _want_n(out_lse, R, _F32, "out_lse"), ws, ws_bytes, _ptr(status),
                                 stream), "psd_confidence_q8")
