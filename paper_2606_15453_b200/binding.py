"""ctypes binding of include/stmoe.h: same names, argument marshalling only.

torch is used for device memory and stream handles; every tensor handed to a
call must live on the CUDA device (or be a host tensor where the header says
"host").  The library is loaded from the package directory and must have been
built (paper_2606_15453_b200.build.build()); there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import torch
from torch.autograd import forward_ad as _forward_ad

from . import build as _build

DTYPE = {"f32": 0, "bf16": 1, "fp8": 2}
WEIGHT_DTYPE = {**DTYPE, "mx4": 3}      # expert weights of the FFN entry points and of a stack
MODE = {"off": 0, "temporal": 1, "spatial": 2, "st": 3}
FLAG_RENORM_TOPK = 1
FLAG_NO_PERSISTENT = 2
FLAG_NO_DENSE = 4
FLAG_NO_FUSED = 8
HOOK_DROP_PREFETCH, HOOK_FAIL_COPY, HOOK_DELAY_COPY_US, HOOK_CORRUPT_TAG, HOOK_HOST_WAIT_MS, HOOK_POLL_LIMIT = 1, 2, 3, 4, 5, 6
HOOK_MX4_POLL_LIMIT = 7


class StmoeError(RuntimeError):
    pass


class Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_experts", C.c_int32), ("top_k", C.c_int32),
                ("n_shared", C.c_int32), ("hidden", C.c_int32), ("inter", C.c_int32),
                ("max_batch", C.c_int32), ("weight_dtype", C.c_int32), ("cache_slots", C.c_int64),
                ("profile_tokens", C.c_int32), ("predictor_mode", C.c_int32), ("flags", C.c_int32),
                ("prefetch_limit", C.c_int32), ("rms_eps", C.c_float), ("residual_scale", C.c_float)]


class Stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in (
        "decode_steps", "runtime_steps", "routed", "predicted", "hits", "near_ties", "cache_hits",
        "cache_misses", "prefetch_issued", "prefetch_useful", "prefetch_wasted", "prefetch_dropped",
        "prefetch_resident", "h2d_bytes_demand", "h2d_bytes_prefetch")] + \
        [("transfer_ms", C.c_double), ("exposed_ms", C.c_double), ("kernel_launches", C.c_int64),
         ("timed_ffn_launches", C.c_int64), ("gate_up_ms", C.c_double), ("down_ms", C.c_double),
         ("router_ms", C.c_double), ("recovered_faults", C.c_int64)]


_lib = None


def lib():
    """Load libstmoe.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            raise StmoeError(f"{_build.LIB} is missing: run paper_2606_15453_b200.build.build()")
        L = C.CDLL(_build.LIB)
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_size_t
        L.stmoe_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
        L.stmoe_destroy.argtypes = [vp]
        L.stmoe_strerror.restype = C.c_char_p
        L.stmoe_strerror.argtypes = [i32]
        L.stmoe_load_router.argtypes = [vp, i32, vp]
        L.stmoe_load_experts.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, i32]
        L.stmoe_decode_step.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.stmoe_decode_token.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.stmoe_decode_token_host.argtypes = [vp, i32, vp, vp, vp, vp]
        L.stmoe_max_predicted.argtypes = [vp]
        L.stmoe_set_kernel_timing.argtypes = [vp, i32]
        L.stmoe_set_dense_min_batch.argtypes = [vp, i32]
        L.stmoe_set_prefetch_min_score.argtypes = [vp, i32]
        L.stmoe_set_onchip_staging.argtypes = [vp, i64, i64]
        L.stmoe_set_cache_policy.argtypes = [vp, i32, i32, i32]
        L.stmoe_set_predict_threshold.argtypes = [vp, i32]
        L.stmoe_set_replacement_rule.argtypes = [vp, i32]
        L.stmoe_set_copy_throttle.argtypes = [vp, i64, i32]
        L.stmoe_test_hook.argtypes = [vp, i32, i64]
        L.stmoe_selftest_bounded_wait.argtypes = [vp, i32, i32, vp]
        L.stmoe_stats.argtypes = [vp, C.POINTER(Stats)]
        L.stmoe_export_state.argtypes = [vp, vp, C.POINTER(sz)]
        L.stmoe_import_state.argtypes = [vp, vp, sz]
        L.stmoe_export_cache_tags.argtypes = [vp, vp, i64]
        L.stmoe_router_topk.argtypes = [vp, vp, i32, i32, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp]
        L.stmoe_predictor_step.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.stmoe_expert_image_bytes.restype = sz
        L.stmoe_expert_image_bytes.argtypes = [i32, i32, i32]
        L.stmoe_moe_ffn_scratch_bytes.restype = sz
        L.stmoe_moe_ffn_scratch_bytes.argtypes = [i32, i32, i32, i32]
        L.stmoe_mx4_ffn_scratch_bytes.restype = sz
        L.stmoe_mx4_ffn_scratch_bytes.argtypes = [i32, i32, i32, i32]
        L.stmoe_moe_ffn.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, f32, vp, vp, sz, vp]
        L.stmoe_moe_ffn_static.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, f32, vp, vp]
        L.stmoe_expert_ffn_dense_scratch_bytes.restype = sz
        L.stmoe_expert_ffn_dense_scratch_bytes.argtypes = [i32, i32, i32]
        L.stmoe_expert_ffn_dense.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        L.stmoe_mx4_quantize.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, i64, vp]
        L.stmoe_mx4_dequantize.argtypes = [vp, i64, vp, i64, i64, i64, vp, i32, i64, vp]
        L.stmoe_mx4_matmul.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, i64, i32, i32, i32, vp, vp, i32, i64, vp, vp]
        L.stmoe_router_balance_scratch_bytes.restype = sz
        L.stmoe_router_balance_scratch_bytes.argtypes = [i64, i32]
        L.stmoe_router_balance.argtypes = [vp, i32, i64, vp, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp]
        L.stmoe_router_balance_backward.argtypes = [vp, i32, i64, vp, i64, i32, i32, vp, vp, vp, vp, i64, vp]
        L.stmoe_router_select.argtypes = [vp, i32, i64, vp, vp, i64, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp]
        L.stmoe_router_select_backward.argtypes = [vp, i32, i64, i64, i32, i32, i32, f32, vp, vp, vp, vp, i64, vp]
        L.stmoe_group_rows_scratch_bytes.restype = sz
        L.stmoe_group_rows_scratch_bytes.argtypes = [i64, i32, i32]
        L.stmoe_group_rows.argtypes = [vp, i64, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.stmoe_dispatch_rows.argtypes = [vp, i64, i64, i64, i32, vp, vp, vp, i64, i64, vp]
        L.stmoe_combine_rows.argtypes = [vp, i32, i64, i64, vp, vp, vp, i64, f32, i64, i32, i64, vp, i32, i64, vp]
        L.stmoe_combine_rows_backward.argtypes = [vp, i32, i64, vp, i32, i64, i64, vp, vp, f32, i64, i32, i64, vp, vp, i64, vp, vp]
        L.stmoe_lora_scratch_bytes.restype = L.stmoe_lora_backward_scratch_bytes.restype = sz
        L.stmoe_lora_scratch_bytes.argtypes = L.stmoe_lora_backward_scratch_bytes.argtypes = [i64, i32, i32, i32, i32]
        L.stmoe_lora.argtypes = [vp, i32, i64, i64, vp, i64, i64, vp, i64, i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, f32, vp, i64, vp, i32,
                                 i64, vp, vp, sz, vp]
        L.stmoe_lora_backward.argtypes = [vp, i32, i64, vp, i64, i64, vp, i64, i64, vp, i64, i64, i32, i32, i32, i32, vp, vp, vp, vp, vp,
                                          f32, vp, vp, i64, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise StmoeError(f"{what}: {lib().stmoe_strerror(rc).decode()} ({rc})")


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous()
    return t.data_ptr()


def _dev(t, dtype=None):
    assert t.is_cuda and t.is_contiguous(), "expected a contiguous CUDA tensor"
    if dtype is not None:
        assert t.dtype == dtype, f"expected {dtype}, got {t.dtype}"
    return t.data_ptr()


# torch's current stream of a device as a bare handle; the Stream object costs microseconds to make
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda i: torch.cuda.current_stream(i).cuda_stream)


def _stream(stream):
    return stream.cuda_stream if stream is not None else _raw_stream(torch.cuda.current_device())


class Stack:
    """Owns one stmoe_t.  Methods mirror the C entry points one to one."""

    def __init__(self, n_layers, n_experts, top_k, hidden, inter, n_shared=0, max_batch=1,
                 dtype="bf16", cache_slots=0, profile_tokens=0, mode="st", flags=0,
                 prefetch_limit=0, rms_eps=1e-6, residual_scale=0.1):
        self.cfg = Config(n_layers, n_experts, top_k, n_shared, hidden, inter, max_batch,
                          WEIGHT_DTYPE[dtype], cache_slots, profile_tokens, MODE[mode], flags,
                          prefetch_limit, rms_eps, residual_scale)
        self._h = C.c_void_p()
        _check(lib().stmoe_create(C.byref(self.cfg), C.byref(self._h)), "stmoe_create")
        self.max_pred = lib().stmoe_max_predicted(self._h)
        self.dtype = dtype

    @classmethod
    def from_config(cls, cfg, max_batch=1, **kw):
        """cfg: an object with the fields of datagen.StackConfig."""
        args = dict(n_layers=cfg.n_layers, n_experts=cfg.n_experts, top_k=cfg.top_k,
                    hidden=cfg.hidden, inter=cfg.inter, n_shared=cfg.n_shared,
                    max_batch=max_batch, dtype=cfg.dtype, cache_slots=cfg.cache_slots,
                    profile_tokens=cfg.profile_tokens, rms_eps=cfg.rms_eps,
                    residual_scale=cfg.residual_scale)
        args.update(kw)
        return cls(**args)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().stmoe_destroy(self._h)
            self._h = C.c_void_p()

    __del__ = close

    def load_router(self, layer: int, w: torch.Tensor) -> None:
        _check(lib().stmoe_load_router(self._h, layer, _ptr(w)), "stmoe_load_router")

    def load_experts(self, layer, first_expert, gate, up, down, scales=None, shared=False) -> None:
        """gate/up [n][I][H], down [n][H][I] (or 2-D for one expert), host or device; dtype "mx4": uint8
        codes [n][I][H/2], [n][H][I/2] and scales (mx4_expert).  The call copies
        at once and does not know torch's streams: synchronise the stream that produced a device
        source before calling."""
        count = 1 if gate.dim() == 2 else gate.shape[0]
        _check(lib().stmoe_load_experts(self._h, layer, first_expert, count, _ptr(gate), _ptr(up),
                                        _ptr(down), _ptr(scales), int(shared)), "stmoe_load_experts")

    def decode_step(self, layer, h_in, h_out, routed_ids=None, routed_w=None, predicted_ids=None,
                    n_predicted=None, flags=None, stream=None) -> None:
        b = h_in.shape[0]
        _check(lib().stmoe_decode_step(self._h, layer, b, _dev(h_in, torch.float32),
                                       _dev(h_out, torch.float32), _ptr(routed_ids), _ptr(routed_w),
                                       _ptr(predicted_ids), _ptr(n_predicted), _ptr(flags),
                                       _stream(stream)), "stmoe_decode_step")

    def decode_token(self, h_in, h_out, routed_ids=None, routed_w=None, predicted_ids=None,
                     n_predicted=None, flags=None, stream=None) -> None:
        b = h_in.shape[0]
        _check(lib().stmoe_decode_token(self._h, b, _dev(h_in, torch.float32),
                                        _dev(h_out, torch.float32), _ptr(routed_ids), _ptr(routed_w),
                                        _ptr(predicted_ids), _ptr(n_predicted), _ptr(flags),
                                        _stream(stream)), "stmoe_decode_token")

    def decode_token_host(self, h_in, h_out, routed_ids=None, stream=None) -> None:
        """h_in / h_out / routed_ids: CPU tensors (pinned for full copy speed); returns when done."""
        assert not h_in.is_cuda and not h_out.is_cuda and h_in.is_contiguous() and h_out.is_contiguous()
        assert h_in.dtype == torch.float32 and h_out.dtype == torch.float32
        assert routed_ids is None or (not routed_ids.is_cuda and routed_ids.dtype == torch.int32)
        _check(lib().stmoe_decode_token_host(self._h, h_in.shape[0], h_in.data_ptr(), h_out.data_ptr(),
                                             _ptr(routed_ids), _stream(stream)), "stmoe_decode_token_host")

    def predictor_step(self, layer, routed_ids, predicted_ids=None, n_predicted=None,
                       stream=None) -> None:
        _check(lib().stmoe_predictor_step(self._h, layer, routed_ids.shape[0],
                                          _dev(routed_ids, torch.int32), _ptr(predicted_ids),
                                          _ptr(n_predicted), _stream(stream)), "stmoe_predictor_step")

    def set_kernel_timing(self, on: bool) -> None:
        _check(lib().stmoe_set_kernel_timing(self._h, int(on)), "stmoe_set_kernel_timing")

    def set_prefetch_min_score(self, min_score: int) -> None:
        _check(lib().stmoe_set_prefetch_min_score(self._h, int(min_score)), "stmoe_set_prefetch_min_score")

    def set_onchip_staging(self, known_bytes: int, predicted_bytes: int) -> None:
        _check(lib().stmoe_set_onchip_staging(self._h, int(known_bytes), int(predicted_bytes)),
               "stmoe_set_onchip_staging")

    def set_predict_threshold(self, threshold: int) -> None:
        _check(lib().stmoe_set_predict_threshold(self._h, int(threshold)), "stmoe_set_predict_threshold")

    def set_replacement_rule(self, live_counts: bool) -> None:
        _check(lib().stmoe_set_replacement_rule(self._h, int(bool(live_counts))), "stmoe_set_replacement_rule")

    def set_cache_policy(self, history_window: int, by_turn: bool, prefetch_floor: int = -1) -> None:
        _check(lib().stmoe_set_cache_policy(self._h, int(history_window), int(by_turn), int(prefetch_floor)),
               "stmoe_set_cache_policy")

    def set_copy_throttle(self, chunk_bytes: int, gap_us: int) -> None:
        _check(lib().stmoe_set_copy_throttle(self._h, int(chunk_bytes), int(gap_us)), "stmoe_set_copy_throttle")

    def test_hook(self, what: int, value: int) -> None:
        _check(lib().stmoe_test_hook(self._h, int(what), int(value)), "stmoe_test_hook")

    def selftest_bounded_wait(self, which: int, poll_limit: int = 4096, stream=None) -> None:
        _check(lib().stmoe_selftest_bounded_wait(self._h, int(which), int(poll_limit), _stream(stream)),
               "stmoe_selftest_bounded_wait")

    def set_dense_min_batch(self, min_batch: int) -> None:
        _check(lib().stmoe_set_dense_min_batch(self._h, int(min_batch)), "stmoe_set_dense_min_batch")

    def stats(self) -> dict:
        st = Stats()
        _check(lib().stmoe_stats(self._h, C.byref(st)), "stmoe_stats")
        return {n: getattr(st, n) for n, _ in Stats._fields_}

    def export_state(self) -> bytes:
        n = C.c_size_t(0)
        _check(lib().stmoe_export_state(self._h, None, C.byref(n)), "stmoe_export_state")
        buf = C.create_string_buffer(n.value)
        _check(lib().stmoe_export_state(self._h, buf, C.byref(n)), "stmoe_export_state")
        return buf.raw[:n.value]

    def import_state(self, blob: bytes) -> None:
        _check(lib().stmoe_import_state(self._h, blob, len(blob)), "stmoe_import_state")

    def export_cache_tags(self) -> torch.Tensor:
        t = torch.empty(self.cfg.cache_slots, dtype=torch.int32)
        _check(lib().stmoe_export_cache_tags(self._h, t.data_ptr(), t.numel()), "stmoe_export_cache_tags")
        return t


def router_topk(h, w_router, top_k, rms_eps=1e-6, renorm=False, stream=None):
    """Gating network for h [B][H] (fp32) and w_router [E][H] (fp32 or bf16), on the GPU.
    Returns dict(logits [B][E], inv_rms [B], ids [B][K], w [B][K], flags [B])."""
    B, H = h.shape
    E = w_router.shape[0]
    wdt = 0 if w_router.dtype == torch.float32 else 1
    buf = torch.empty(B * E + B, dtype=torch.float32, device=h.device)
    ids = torch.empty(B, top_k, dtype=torch.int32, device=h.device)
    w = torch.empty(B, top_k, dtype=torch.float32, device=h.device)
    flags = torch.empty(B, dtype=torch.int32, device=h.device)
    _check(lib().stmoe_router_topk(_dev(h, torch.float32), _dev(w_router), wdt, B, E, H, top_k,
                                   rms_eps, int(renorm), _dev(buf), _dev(ids), _dev(w), _dev(flags),
                                   _stream(stream)), "stmoe_router_topk")
    return dict(logits=buf[:B * E].view(B, E), inv_rms=buf[B * E:], ids=ids, w=w, flags=flags)


def expert_image_bytes(hidden, inter, dtype) -> int:
    return lib().stmoe_expert_image_bytes(hidden, inter, WEIGHT_DTYPE[dtype])


def moe_ffn_scratch_bytes(batch, top_k, hidden, inter, dtype="bf16") -> int:
    if dtype == "mx4":
        return lib().stmoe_mx4_ffn_scratch_bytes(batch, top_k, hidden, inter)
    return lib().stmoe_moe_ffn_scratch_bytes(batch, top_k, hidden, inter)


def moe_ffn(h, inv_rms, ids, w, experts, dtype, n_experts, hidden, inter, residual_scale, h_out,
            scratch, stream=None, entry="stmoe_moe_ffn"):
    """Routed SwiGLU FFN + weighted sum + residual for given routing (all tensors on the GPU).
    experts: uint8 tensor of n_experts expert images."""
    B, K = ids.shape
    fn = getattr(lib(), entry)
    _check(fn(_dev(h, torch.float32), _ptr(inv_rms), _dev(ids, torch.int32), _dev(w, torch.float32),
              _dev(experts), WEIGHT_DTYPE[dtype], B, n_experts, K, hidden, inter, residual_scale,
              _dev(h_out, torch.float32), _dev(scratch), scratch.numel() * scratch.element_size(),
              _stream(stream)), entry)
    return h_out


def moe_ffn_static(h, inv_rms, ids, w, experts, dtype, n_experts, hidden, inter, residual_scale, h_out,
                   stream=None):
    """stmoe_moe_ffn_static: the same computation as moe_ffn for callers that must not allocate
    device memory; scratch is an 8 MiB area inside the library, shared by every call on the
    device (order calls that could overlap).  Raises StmoeError when the problem needs more."""
    B, K = ids.shape
    _check(lib().stmoe_moe_ffn_static(_dev(h, torch.float32), _ptr(inv_rms), _dev(ids, torch.int32),
                                      _dev(w, torch.float32), _dev(experts), WEIGHT_DTYPE[dtype], B, n_experts, K,
                                      hidden, inter, residual_scale, _dev(h_out, torch.float32),
                                      _stream(stream)), "stmoe_moe_ffn_static")
    return h_out


def expert_ffn_dense(h, inv_rms, image, hidden, inter, stream=None):
    """stmoe_expert_ffn_dense: one bf16 expert's SwiGLU FFN for the m <= 64 tokens in h [m][hidden]
    on the tensor cores.  Returns (y [m][hidden] fp32, flags uint32 tensor; non-zero = a bounded
    wait inside a kernel ran out)."""
    m = h.shape[0]
    n = lib().stmoe_expert_ffn_dense_scratch_bytes(m, hidden, inter)
    scratch = torch.empty(max(n, 256), dtype=torch.uint8, device=h.device)
    y = torch.empty(m, hidden, dtype=torch.float32, device=h.device)
    flags = torch.zeros(1, dtype=torch.int32, device=h.device)
    _check(lib().stmoe_expert_ffn_dense(_dev(h, torch.float32), _ptr(inv_rms), _dev(image), m, hidden, inter,
                                        _dev(y), _dev(flags), _dev(scratch), scratch.numel(), _stream(stream)),
           "stmoe_expert_ffn_dense")
    return y, flags


# ---- microscaled 4-bit floating point and router statistics --------------------------------------
# These calls take microseconds on the device, so the host side is kept short: one condition in front
# of each call, messages made only when it fails.

_ELEM = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 4}
_U8, _I32, _F32 = torch.uint8, torch.int32, torch.float32


def _refuse(what: str):
    raise StmoeError(what)


def _is_rows(t, dtype=None) -> bool:
    """A CUDA matrix with contiguous rows, any row stride."""
    return t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] <= 1) and (dtype is None or t.dtype == dtype)


def _no_tangents(*tensors) -> None:
    """Refuses forward-mode derivatives, which the kernels would lose without a word."""
    if _forward_ad._current_level >= 0:
        for t in tensors:
            if t is not None and _forward_ad.unpack_dual(t).tangent is not None:
                _refuse("forward-mode derivatives are not provided")


def _stream_of(ref, stream):
    """Handle of the stream a call goes to: torch's current one, if ref lives on the current device and no
    stream was given; else None (see _there)."""
    i = ref.get_device()
    return _raw_stream(i) if stream is None and i == torch.cuda.current_device() else None


def _there(ref, stream, fn, *args, **kw):
    """fn again with ref's device current, on the given stream or that device's current one; tensors it
    allocates belong to that stream."""
    with torch.cuda.device(ref.device):
        s = stream if stream is not None else torch.cuda.current_stream()
        if s.device != ref.device:
            _refuse("the stream belongs to another device than the tensors")
        with torch.cuda.stream(s):
            return fn(*args, **kw)


def mx4_quantize(x, codes=None, scales=None, stream=None):
    """stmoe_mx4_quantize: x [rows][cols] (fp32, bf16 or fp16, any row stride) -> (codes uint8
    [rows][ceil(cols/32)*16], scales uint8 [rows][ceil(cols/32)]), into given tensors or new ones."""
    elem = _ELEM.get(x.dtype)
    if elem is None or not _is_rows(x) or x.shape[1] < 1:
        _refuse("x: expected a 2-D CUDA tensor of fp32, bf16 or fp16 with contiguous rows")
    rows, cols = x.shape
    nb = (cols + 31) // 32
    if codes is not None or scales is not None:
        if not all(t is None or (_is_rows(t, _U8) and t.shape[0] == rows and t.shape[1] == n and t.device == x.device)
                   for t, n in ((codes, nb * 16), (scales, nb))):
            _refuse(f"codes and scales: expected uint8 {(rows, nb * 16)} and {(rows, nb)} on x's device")
    st = _stream_of(x, stream)
    if st is None:
        return _there(x, stream, mx4_quantize, x, codes, scales)
    if codes is None:
        codes = torch.empty(rows, nb * 16, dtype=_U8, device=x.device)
    if scales is None:
        scales = torch.empty(rows, nb, dtype=_U8, device=x.device)
    if rows:
        rc = lib().stmoe_mx4_quantize(x.data_ptr(), elem, rows, cols, x.stride(0), codes.data_ptr(), codes.stride(0),
                                      scales.data_ptr(), scales.stride(0), st)
        if rc:
            _check(rc, "stmoe_mx4_quantize")
    return codes, scales


def mx4_dequantize(codes, scales, cols, dtype=torch.float32, out=None, stream=None):
    """stmoe_mx4_dequantize: the first `cols` values of every row, in dtype (or in out's)."""
    if out is not None:
        dtype = out.dtype
    elem = _ELEM.get(dtype)
    if elem is None or not (_is_rows(codes, _U8) and _is_rows(scales, _U8)):
        _refuse("expected 2-D uint8 CUDA tensors with contiguous rows, and fp32, bf16 or fp16 values")
    rows, nb = scales.shape
    if codes.shape[0] != rows or codes.shape[1] != nb * 16 or cols < 1 or (cols + 31) // 32 != nb or codes.device != scales.device:
        _refuse("codes, scales and cols do not belong together")
    if out is not None and not (_is_rows(out) and out.shape[0] == rows and out.shape[1] == cols and out.device == codes.device):
        _refuse(f"out: expected {(rows, cols)} with contiguous rows on the codes' device")
    st = _stream_of(codes, stream)
    if st is None:
        return _there(codes, stream, mx4_dequantize, codes, scales, cols, dtype, out)
    if out is None:
        out = torch.empty(rows, cols, dtype=dtype, device=codes.device)
    if rows:
        rc = lib().stmoe_mx4_dequantize(codes.data_ptr(), codes.stride(0), scales.data_ptr(), scales.stride(0), rows, cols,
                                        out.data_ptr(), elem, out.stride(0), st)
        if rc:
            _check(rc, "stmoe_mx4_dequantize")
    return out


def mx4_expert(gate, up, down, stream=None):
    """One expert's matrices (gate, up [I][H], down [H][I]; fp32, bf16 or fp16; H and I multiples of 32)
    quantised: dict(gate, up, down: codes; scales: those of the three, one after the other) for
    Stack.load_experts, and image: the same as one expert image for moe_ffn (the others are views
    into it)."""
    if not (_is_rows(gate) and _is_rows(up) and _is_rows(down)):
        _refuse("expected 2-D CUDA tensors with contiguous rows")
    I, H = gate.shape
    if H % 32 or I % 32 or H < 32 or I < 32 or up.shape != gate.shape or tuple(down.shape) != (H, I):
        _refuse("gate and up are [I][H], down is [H][I]; hidden and inter multiples of 32")
    if _stream_of(gate, stream) is None:
        return _there(gate, stream, mx4_expert, gate, up, down)
    n, nc, ns = expert_image_bytes(H, I, "mx4"), H * I // 2, H * I // 32
    image = torch.empty(n, dtype=_U8, device=gate.device)
    image[3 * (nc + ns):].zero_()
    parts = {"image": image, "scales": image[3 * nc:3 * (nc + ns)]}
    for i, (name, w) in enumerate((("gate", gate), ("up", up), ("down", down))):
        r, c = w.shape
        parts[name] = image[i * nc:(i + 1) * nc].view(r, c // 2)
        mx4_quantize(w, parts[name], image[3 * nc + i * ns:3 * nc + (i + 1) * ns].view(r, c // 32))
    return parts


def mx4_poll_limit(polls: int) -> None:
    """For tests: polls after which a wait inside the MX4 kernels gives up (STMOE_HOOK_MX4_POLL_LIMIT)."""
    _check(lib().stmoe_test_hook(None, HOOK_MX4_POLL_LIMIT, int(polls)), "stmoe_test_hook")


def mx4_matmul(a, b, counts=None, dtype=torch.bfloat16, out=None, flags=None, stream=None):
    """stmoe_mx4_matmul: out[t] = a[t] b_g(t)^T for MX4 operands (codes, scales) as mx4_quantize
    returns them.  a: [m] rows; b: [n] rows, or [groups][n] rows with counts (int32 [groups], on the
    device: how many rows of a belong to each group, in order; rows behind their sum are not written).
    flags: optional int32 [1], caller-zeroed; non-zero = a bounded wait inside the kernel ran out."""
    (a_codes, a_scales), (b_codes, b_scales) = a, b
    groups, dims = 1, b_codes.dim()
    if dims not in (2, 3) or b_scales.dim() != dims:
        _refuse("b: codes and scales of [n] or [groups][n] rows")
    if dims == 3:
        groups, n = b_codes.shape[:2]
        if groups < 1 or n < 1 or b_scales.shape[:2] != b_codes.shape[:2]:
            _refuse("b: codes and scales do not belong together")
        if groups > 1 and not (b_codes.stride(0) == n * b_codes.stride(1) and b_scales.stride(0) == n * b_scales.stride(1)):
            _refuse("b: the groups' rows have to follow one another")
        b_codes, b_scales = b_codes[0], b_scales[0]
    if not (_is_rows(a_codes, _U8) and _is_rows(a_scales, _U8) and _is_rows(b_codes, _U8) and _is_rows(b_scales, _U8)):
        _refuse("codes and scales: expected uint8 CUDA tensors with contiguous rows")
    m, nb = a_scales.shape
    n = b_scales.shape[0]
    if not (n and nb and a_codes.shape[0] == m and a_codes.shape[1] == nb * 16 and b_codes.shape[0] == n
            and b_codes.shape[1] == nb * 16 and b_scales.shape[1] == nb):
        _refuse("the operands' shapes do not belong together")
    dev = a_codes.device
    for t in (a_scales, b_codes, b_scales, counts, out, flags):
        if t is not None and t.device != dev:
            _refuse("all tensors have to be on one CUDA device")
    if counts is None:
        if groups != 1:
            _refuse("several groups need counts")
    elif counts.dtype != _I32 or counts.numel() != groups or not counts.is_contiguous():
        _refuse("counts: contiguous int32 [groups]")
    if out is not None:
        if not (_is_rows(out) and out.shape[0] == m and out.shape[1] == n):
            _refuse(f"out: expected {(m, n)} with contiguous rows")
        dtype = out.dtype
    elem = _ELEM.get(dtype)
    if elem is None or (flags is not None and (flags.dtype != _I32 or flags.numel() < 1)):
        _refuse("out is fp32, bf16 or fp16; flags is int32")
    st = _stream_of(a_codes, stream)
    if st is None:
        return _there(a_codes, stream, mx4_matmul, a, b, counts, dtype, out, flags)
    if out is None:
        out = torch.empty(m, n, dtype=dtype, device=dev)
    if m:
        rc = lib().stmoe_mx4_matmul(a_codes.data_ptr(), a_codes.stride(0), a_scales.data_ptr(), a_scales.stride(0), m,
                                    b_codes.data_ptr(), b_codes.stride(0), b_scales.data_ptr(), b_scales.stride(0),
                                    groups, n, nb, None if counts is None else counts.data_ptr(), out.data_ptr(),
                                    elem, out.stride(0), None if flags is None else flags.data_ptr(), st)
        if rc:
            _check(rc, "stmoe_mx4_matmul")
    return out


def _balance_elem(logits, mask):
    elem = _ELEM.get(logits.dtype)
    if elem is None or not _is_rows(logits):
        _refuse("logits: expected a 2-D CUDA tensor of fp32, bf16 or fp16 with contiguous rows")
    if mask is not None and not (mask.dtype in (torch.bool, _U8) and mask.is_contiguous() and mask.numel() == logits.shape[0]
                                 and mask.device == logits.device):
        _refuse("mask: contiguous bool [tokens] on the logits' device")
    _no_tangents(logits)
    return elem


class _RouterBalance(torch.autograd.Function):
    """router_balance as a step of torch's graph; the gradient is router_balance_backward's."""

    @staticmethod
    def forward(ctx, logits, ids, mask):
        f = router_balance(logits, ids, mask)
        ctx.save_for_backward(logits, mask, f["counts"], f["rows"])
        ctx.top_k = f["top_k"]
        ctx.mark_non_differentiable(f["counts"], f["rows"])
        ctx.set_materialize_grads(False)
        return f["loss"], f["counts"], f["rows"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss, *_):
        if grad_loss is None:
            return None, None, None
        logits, mask, counts, rows = ctx.saved_tensors
        f = {"counts": counts, "rows": rows, "top_k": ctx.top_k}
        return router_balance_backward(logits, f, grad_loss.to(_F32).contiguous(), mask), None, None


def router_balance(logits, ids, mask=None, stream=None):
    """stmoe_router_balance: losses and per-expert counts for logits [tokens][n_experts] and the
    chosen experts ids int32 [tokens][top_k] (-1: dropped); mask [tokens]: rows that count.
    Returns dict(loss fp32 [2] = balance, z; counts int32 [n_experts]; rows int32 [1]; top_k).
    Where logits require a gradient (and torch records one) the loss carries it, once differentiable."""
    elem = _balance_elem(logits, mask)
    T, E = logits.shape
    if not (ids.dtype == _I32 and ids.dim() == 2 and ids.is_contiguous() and ids.shape[0] == T and ids.device == logits.device):
        _refuse("ids: contiguous int32 [tokens][top_k] on the logits' device")
    K = ids.shape[1]
    st = _stream_of(logits, stream)
    if st is None:
        return _there(logits, stream, router_balance, logits, ids, mask)
    if logits.requires_grad and torch.is_grad_enabled():
        loss, counts, rows = _RouterBalance.apply(logits, ids, mask)
        return {"loss": loss, "counts": counts, "rows": rows, "top_k": K}
    L = lib()
    n = L.stmoe_router_balance_scratch_bytes(T, E)
    dev = logits.device
    loss, counts, rows = (torch.empty(k, dtype=t, device=dev) for k, t in ((2, _F32), (E, _I32), (1, _I32)))
    scratch = torch.empty(n, dtype=_U8, device=dev) if n else None
    # an empty tensor has no address; nothing of it is read
    src, idp = (logits.data_ptr(), ids.data_ptr()) if T else (loss.data_ptr(), loss.data_ptr())
    rc = L.stmoe_router_balance(src, elem, logits.stride(0), idp, None if mask is None else mask.data_ptr(), T, E, K, loss.data_ptr(),
                                counts.data_ptr(), rows.data_ptr(), None if scratch is None else scratch.data_ptr(), n, st)
    if rc:
        _check(rc, "stmoe_router_balance")
    return {"loss": loss, "counts": counts, "rows": rows, "top_k": K}


def router_balance_backward(logits, forward, grad_loss, mask=None, out=None, stream=None):
    """stmoe_router_balance_backward: gradient of grad_loss . loss with respect to the logits, from
    the dict that router_balance returned for the same logits and mask; grad_loss: fp32 [2]."""
    elem = _balance_elem(logits, mask)
    T, E = logits.shape
    counts, rows, dev = forward["counts"], forward["rows"], logits.device
    if not (counts.dtype == _I32 and counts.numel() == E and counts.is_contiguous() and rows.dtype == _I32 and counts.device == dev and rows.device == dev):
        _refuse("forward does not belong to these logits")
    if not (grad_loss.dtype == _F32 and grad_loss.numel() == 2 and grad_loss.is_contiguous() and grad_loss.device == dev):
        _refuse("grad_loss: fp32 [2] on the logits' device")
    _no_tangents(grad_loss)
    if out is not None and not (_is_rows(out, logits.dtype) and out.shape == logits.shape and out.device == dev):
        _refuse("out: expected the logits' shape and type")
    st = _stream_of(logits, stream)
    if st is None:
        return _there(logits, stream, router_balance_backward, logits, forward, grad_loss, mask, out)
    if out is None:
        out = torch.empty(T, E, dtype=logits.dtype, device=dev)
    if T:
        rc = lib().stmoe_router_balance_backward(logits.data_ptr(), elem, logits.stride(0), None if mask is None else mask.data_ptr(),
                                                 T, E, forward["top_k"], counts.data_ptr(), rows.data_ptr(), grad_loss.data_ptr(),
                                                 out.data_ptr(), out.stride(0), st)
        if rc:
            _check(rc, "stmoe_router_balance_backward")
    return out


# ---- around the experts' products: choice of experts, rows in their order and back, adapters ------------

SELECT_SIGMOID, SELECT_RENORM = 1, 2


def _addr(t):
    return None if t is None else t.data_ptr()


def _wants_grad(*tensors) -> bool:
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _is_vector(t, n, dtype, dev) -> bool:
    """n contiguous elements of dtype on the CUDA device of ordinal dev."""
    return t.dtype is dtype and t.numel() == n and t.is_contiguous() and t.get_device() == dev


class _RouterSelect(torch.autograd.Function):
    """router_select as a step of torch's graph; the gradient is router_select_backward's."""

    @staticmethod
    def forward(ctx, logits, *how):
        f = router_select(logits, *how)
        ctx.save_for_backward(logits, f["ids"], f["w"])
        ctx.how = f["flags"], f["scale"]
        ctx.mark_non_differentiable(f["ids"])
        ctx.set_materialize_grads(False)
        return f["ids"], f["w"], f["flags"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, _, grad_w, __):
        if grad_w is None:
            return (None,) * 10
        logits, ids, w = ctx.saved_tensors
        f = {"ids": ids, "w": w, "flags": ctx.how[0], "scale": ctx.how[1]}
        return (router_select_backward(logits, f, grad_w.to(_F32).contiguous()),) + (None,) * 9


def router_select(logits, top_k, scores="softmax", bias=None, groups=1, top_groups=None, group_best=1, renorm=False, scale=1.0, mask=None,
                  stream=None):
    """stmoe_router_select: the experts of every row of logits [tokens][n_experts] (fp32, bf16 or fp16) and their weights.
    scores: "softmax" or "sigmoid"; bias fp32 [n_experts]: added to the scores for the choice only (without one the order is that of the
    logits, also where scores are equal in 64 bits; with one, be it zeros, the lower index of such is chosen); groups, top_groups, group_best: the
    choice is made among the best top_groups groups, ranked by their group_best best members; renorm: weights of a row sum to scale;
    mask bool [tokens]: rows to choose for.  Returns dict(ids int32 [tokens][top_k], ascending, -1 behind the last; w fp32
    [tokens][top_k]; flags, scale: what the gradient has to know).  Where logits require a gradient w carries it, once differentiable."""
    elem = _balance_elem(logits, mask)
    T, E = logits.shape
    if scores not in ("softmax", "sigmoid"):
        _refuse("scores: softmax or sigmoid")
    if bias is not None and not _is_vector(bias, E, _F32, logits.get_device()):
        _refuse("bias: contiguous fp32 [n_experts] on the logits' device")
    if not 1 <= top_k <= E:
        _refuse("top_k: 1 to the number of experts")
    st = _stream_of(logits, stream)
    if st is None:
        return _there(logits, stream, router_select, logits, top_k, scores, bias, groups, top_groups, group_best, renorm, scale, mask)
    if _wants_grad(logits):
        ids, w, flags = _RouterSelect.apply(logits, top_k, scores, bias, groups, top_groups, group_best, renorm, scale, mask)
        return {"ids": ids, "w": w, "flags": flags, "scale": scale}
    flags = (SELECT_SIGMOID if scores == "sigmoid" else 0) | (SELECT_RENORM if renorm else 0)
    dev = logits.device
    ids = torch.empty(T, top_k, dtype=_I32, device=dev)
    w = torch.empty(T, top_k, dtype=_F32, device=dev)
    # an empty tensor has no address; nothing of it is read
    src, idp, wp = (logits.data_ptr(), ids.data_ptr(), w.data_ptr()) if T else (256, 256, 256)
    rc = lib().stmoe_router_select(src, elem, logits.stride(0), _addr(bias), _addr(mask), T, E, top_k, groups,
                                   groups if top_groups is None else top_groups, group_best, flags, scale, idp, wp, st)
    if rc:
        _check(rc, "stmoe_router_select")
    return {"ids": ids, "w": w, "flags": flags, "scale": scale}


def router_select_backward(logits, forward, grad_w, out=None, stream=None):
    """stmoe_router_select_backward: gradient of sum(grad_w * w) with respect to the logits, from the dict that
    router_select returned for them; grad_w: fp32 [tokens][top_k]."""
    elem = _balance_elem(logits, None)
    T, E = logits.shape
    ids, w, dev = forward["ids"], forward["w"], logits.get_device()
    K = ids.shape[1]
    if not (ids.shape[0] == T and _is_vector(ids, T * K, _I32, dev) and _is_vector(w, T * K, _F32, dev)):
        _refuse("forward does not belong to these logits")
    if not _is_vector(grad_w, T * K, _F32, dev):
        _refuse("grad_w: contiguous fp32 [tokens][top_k] on the logits' device")
    _no_tangents(grad_w)
    if out is not None and not (_is_rows(out, logits.dtype) and out.shape == logits.shape and out.get_device() == dev):
        _refuse("out: expected the logits' shape and type")
    st = _stream_of(logits, stream)
    if st is None:
        return _there(logits, stream, router_select_backward, logits, forward, grad_w, out)
    if out is None:
        out = torch.empty(T, E, dtype=logits.dtype, device=logits.device)
    if T:
        rc = lib().stmoe_router_select_backward(logits.data_ptr(), elem, logits.stride(0), T, E, K, forward["flags"], forward["scale"],
                                                ids.data_ptr(), w.data_ptr(), grad_w.data_ptr(), out.data_ptr(), out.stride(0), st)
        if rc:
            _check(rc, "stmoe_router_select_backward")
    return out


def group_rows(ids, n_groups, stream=None):
    """stmoe_group_rows: the grouping of ids int32 [rows][top_k] (or [rows]) by id; ids outside [0, n_groups) have no group.
    Returns the plan that dispatch_rows, combine_rows and (for ids [rows]) lora take: dict(counts int32 [n_groups], for mx4_matmul;
    starts [n_groups + 1]; order [rows * top_k]; slots, shaped as ids; ids, groups).  ids are kept, not copied: leave them as they are while
    the plan is in use (a gradient that reads the plan refuses one that torch saw written since the call)."""
    if not (ids.is_cuda and ids.dtype == _I32 and ids.dim() in (1, 2) and ids.is_contiguous()):
        _refuse("ids: contiguous int32 [rows][top_k] or [rows] on a CUDA device")
    T, K = (ids.shape[0], 1) if ids.dim() == 1 else ids.shape
    if K < 1 or not 1 <= n_groups <= 1024:
        _refuse("top_k at least 1, 1 to 1024 groups")
    st = _stream_of(ids, stream)
    if st is None:
        return _there(ids, stream, group_rows, ids, n_groups)
    L = lib()
    P, n = T * K, L.stmoe_group_rows_scratch_bytes(T, K, n_groups)
    counts, starts, order, slots, scratch = torch.empty(2 * n_groups + 1 + 2 * P + n // 4, dtype=_I32, device=ids.device).split(
        [n_groups, n_groups + 1, P, P, n // 4])
    idp = ids.data_ptr() if T else counts.data_ptr()
    c = counts.data_ptr()
    at = c + 4 * (2 * n_groups + 1)
    rc = L.stmoe_group_rows(idp, T, K, n_groups, c, c + 4 * n_groups, at, at + 4 * P, at + 8 * P, n, st)
    if rc:
        _check(rc, "stmoe_group_rows")
    return {"counts": counts, "starts": starts, "order": order, "slots": slots if ids.dim() == 1 else slots.view(T, K), "ids": ids, "groups": n_groups}


def _plan_of(plan, T, dev):
    """top_k of a plan for T rows."""
    slots = plan["slots"]
    if slots.shape[0] != T or slots.get_device() != dev:
        _refuse("the plan belongs to other rows")
    return 1 if slots.dim() == 1 else slots.shape[1]


class _KeptPlan:
    """A plan for a gradient that reads these of its tensors: refused there if they were written in between."""

    def __init__(self, plan, *names):
        self.plan, self.names = dict(plan), names
        self.versions = self._versions()

    def _versions(self):
        return [None if t.is_inference() else t._version for t in map(self.plan.get, self.names)]     # inference tensors have none

    def get(self):
        if self._versions() != self.versions:
            _refuse(f"the plan's {', '.join(self.names)} (or what shares their memory) were written between the call and its gradient")
        return self.plan


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, plan):
        ctx.plan = _KeptPlan(plan, "slots")
        return dispatch_rows(x, plan)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        return combine_rows(grad.contiguous(), ctx.plan.get()), None


def dispatch_rows(x, plan, out=None, stream=None):
    """stmoe_dispatch_rows: rows of x [rows][cols] (any type) in the order of group_rows' plan, [rows * top_k][cols].  Rows
    behind the last group are 0; in a given out they stay as they were.  Takes part in autograd (without out)."""
    if not _is_rows(x) or x.shape[1] < 1:
        _refuse("x: expected a 2-D CUDA tensor with contiguous rows")
    T, C = x.shape
    K = _plan_of(plan, T, x.get_device())
    if out is not None and not (_is_rows(out, x.dtype) and out.shape[0] == T * K and out.shape[1] == C and out.get_device() == x.get_device()):
        _refuse(f"out: expected {(T * K, C)} of x's type with contiguous rows on x's device")
    if out is not None and _wants_grad(x, out):
        _refuse("out is not part of torch's graph: leave it away where x requires a gradient")
    _no_tangents(x, out)
    st = _stream_of(x, stream)
    if st is None:
        return _there(x, stream, dispatch_rows, x, plan, out)
    if _wants_grad(x):
        if x.dtype not in _ELEM:
            _refuse("x: gradients are of fp32, bf16 or fp16 rows")
        return _Dispatch.apply(x, plan)
    fresh = out is None
    if fresh:
        out = torch.empty(T * K, C, dtype=x.dtype, device=x.device)
    if T:
        b = x.element_size()
        rc = lib().stmoe_dispatch_rows(x.data_ptr(), C * b, x.stride(0) * b, T, K, plan["slots"].data_ptr(),
                                       plan["starts"].data_ptr() + 4 * plan["groups"] if fresh else None, out.data_ptr(), T * K,
                                       out.stride(0) * b, st)
        if rc:
            _check(rc, "stmoe_dispatch_rows")
    return out


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, w, residual, plan, scale):
        ctx.save_for_backward(y, w)
        ctx.plan, ctx.scale, ctx.wants = _KeptPlan(plan, "slots", "starts"), scale, (y.requires_grad, w is not None and w.requires_grad)
        return combine_rows(y, plan, w, residual, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        y, w = ctx.saved_tensors
        dy = dw = None
        if any(ctx.wants):
            dy, dw = combine_rows_backward(grad.contiguous(), y, ctx.plan.get(), w, ctx.scale)
        return dy, dw, grad if ctx.needs_input_grad[2] else None, None, None


def _combine_args(y, plan, w, other, what):
    T = plan["slots"].shape[0]
    elem = _ELEM.get(y.dtype)
    if elem is None or not _is_rows(y) or y.shape[1] < 1:
        _refuse("y: expected a 2-D CUDA tensor of fp32, bf16 or fp16 with contiguous rows")
    dev = y.get_device()
    K = _plan_of(plan, T, dev)
    if y.shape[0] != T * K:
        _refuse("y has other rows than the plan")
    if w is not None and not _is_vector(w, T * K, _F32, dev):
        _refuse("w: contiguous fp32 [rows][top_k] on y's device")
    for t in other:
        if t is not None and not (_is_rows(t) and t.dtype in (y.dtype, _F32) and t.shape[0] == T and t.shape[1] == y.shape[1] and t.get_device() == dev):
            _refuse(f"{what}: expected [rows][cols] of y's type or fp32 with contiguous rows on y's device")
    _no_tangents(y, w, *other)
    return T, K, elem


def combine_rows(y, plan, w=None, residual=None, scale=1.0, out=None, stream=None):
    """stmoe_combine_rows: residual + scale * sum_k w[:, k] y[slot of (row, k)] for y [rows * top_k][cols] in the plan's order; the result
    has the residual's type (y's or fp32; without a residual out's or y's); out may be the residual.  Takes part in autograd (without out)."""
    T, K, elem = _combine_args(y, plan, w, (residual, out), "residual, out")
    if residual is not None and out is not None and residual.dtype != out.dtype:
        _refuse("residual and out have to be of one type")
    if out is not None and _wants_grad(y, w, residual, out):
        _refuse("out is not part of torch's graph: leave it away where an input requires a gradient")
    st = _stream_of(y, stream)
    if st is None:
        return _there(y, stream, combine_rows, y, plan, w, residual, scale, out)
    if _wants_grad(y, w, residual):
        return _Combine.apply(y, w, residual, plan, scale)
    C = y.shape[1]
    if out is None:
        out = torch.empty(T, C, dtype=y.dtype if residual is None else residual.dtype, device=y.device)
    if T:
        rc = lib().stmoe_combine_rows(y.data_ptr(), elem, y.stride(0), T * K, plan["slots"].data_ptr(), _addr(w), _addr(residual),
                                      0 if residual is None else residual.stride(0), scale, T, K, C, out.data_ptr(), _ELEM[out.dtype],
                                      out.stride(0), st)
        if rc:
            _check(rc, "stmoe_combine_rows")
    return out


def combine_rows_backward(grad, y, plan, w=None, scale=1.0, stream=None):
    """stmoe_combine_rows_backward: (gradient of y, of w) for grad [rows][cols]; rows of the first behind the last group
    are 0.  The second is None where w is."""
    T, K, elem = _combine_args(y, plan, w, (grad,), "grad")
    st = _stream_of(y, stream)
    if st is None:
        return _there(y, stream, combine_rows_backward, grad, y, plan, w, scale)
    C = y.shape[1]
    dy = torch.empty(T * K, C, dtype=y.dtype, device=y.device)
    dw = None if w is None else torch.empty_like(w)
    if T:
        rc = lib().stmoe_combine_rows_backward(grad.data_ptr(), _ELEM[grad.dtype], grad.stride(0), y.data_ptr(), elem, y.stride(0), T * K,
                                               plan["slots"].data_ptr(), _addr(w), scale, T, K, C,
                                               plan["starts"].data_ptr() + 4 * plan["groups"], dy.data_ptr(), C, _addr(dw), st)
        if rc:
            _check(rc, "stmoe_combine_rows_backward")
    return dy, dw


class _Lora(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, a, b, base, plan, scale, alpha):
        hidden = torch.empty(x.shape[0], a.shape[1], dtype=_F32, device=x.device)
        out = lora(x, a, b, plan, scale, alpha, base, hidden=hidden)
        ctx.save_for_backward(x, a, b, scale, hidden)
        ctx.plan, ctx.alpha = _KeptPlan(plan, "ids", "order", "counts", "starts"), alpha
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, a, b, scale, hidden = ctx.saved_tensors
        dx = da = db = None
        if any(ctx.needs_input_grad[:3]):
            dx, da, db = lora_backward(grad.to(x.dtype).contiguous(), x, a, b, ctx.plan.get(), hidden, scale, ctx.alpha)
        return dx, da, db, grad if ctx.needs_input_grad[3] else None, None, None, None


def _lora_args(x, a, b, plan, scale, hidden):
    elem = _ELEM.get(x.dtype)
    if not elem or not _is_rows(x) or x.shape[1] < 1:
        _refuse("x: expected a 2-D CUDA tensor of bf16 or fp16 with contiguous rows")
    T, I = x.shape
    dev, dtype = x.get_device(), x.dtype
    if a.dim() != 3 or b.dim() != 3 or a.dtype is not dtype or b.dtype is not dtype or a.get_device() != dev or b.get_device() != dev:
        _refuse("a [n][rank][inner] and b [n][outer][rank]: expected x's type and device")
    (n, r, inner), (nb, O, rb) = a.shape, b.shape
    if inner != I or nb != n or rb != r or n < 1 or O < 1 or not 1 <= r <= 256:
        _refuse("the adapters' shapes do not belong together, or rank is not in 1..256")
    if (a.stride(2) != 1 and I > 1) or (b.stride(2) != 1 and r > 1):
        _refuse("a and b: expected contiguous rows")
    if _plan_of(plan, T, dev) != 1 or plan["groups"] != n:
        _refuse("plan: group_rows of ids [rows], one group an adapter")
    if scale is not None and not _is_vector(scale, n, _F32, dev):
        _refuse("scale: contiguous fp32 [n] on x's device")
    if hidden is not None and not _is_vector(hidden, T * r, _F32, dev):
        _refuse("hidden: contiguous fp32 [rows][rank] on x's device")
    _no_tangents(x, a, b, scale, hidden)
    return elem, T, I, n, r, O


def lora(x, a, b, plan, scale=None, alpha=1.0, base=None, out=None, hidden=None, stream=None):
    """stmoe_lora: base + alpha * scale[g] * (x A_g^T) B_g^T, g the adapter of each row of x [rows][inner] (bf16 or fp16), a [n][rank][inner],
    b [n][outer][rank], plan = group_rows(ids [rows], n) (one plan serves all projections of a step; rows without a group keep the base).
    base [rows][outer]: the shared projection's result, in x's type or fp32, which is the result's type (without a base out's or
    x's); None: 0.  out may be the base.  hidden fp32 [rows][rank]: receives x A_g^T, for lora_backward.  Takes part in autograd (without out);
    the gradient of an fp32 result is rounded to x's type for those of x, a and b."""
    elem, T, I, n, r, O = _lora_args(x, a, b, plan, scale, hidden)
    for t in (base, out):
        if t is not None and not (_is_rows(t) and t.dtype in (x.dtype, _F32) and t.shape[0] == T and t.shape[1] == O and t.get_device() == x.get_device()):
            _refuse(f"base, out: expected {(T, O)} of x's type or fp32 with contiguous rows on x's device")
    if base is not None and out is not None and base.dtype != out.dtype:
        _refuse("base and out have to be of one type")
    _no_tangents(base, out)
    graph = _wants_grad(x, a, b, base, out, scale)
    if graph and (out is not None or hidden is not None):
        _refuse("out and hidden are not part of torch's graph: leave them away where an input requires a gradient")
    if graph and scale is not None and scale.requires_grad:
        _refuse("scale is held constant")
    st = _stream_of(x, stream)
    if st is None:
        return _there(x, stream, lora, x, a, b, plan, scale, alpha, base, out, hidden)
    if graph:
        return _Lora.apply(x, a, b, base, plan, scale, alpha)
    if out is None:
        out = torch.empty(T, O, dtype=x.dtype if base is None else base.dtype, device=x.device)
    if T:
        L = lib()
        size = L.stmoe_lora_scratch_bytes(T, n, r, I, O)
        scratch = torch.empty(size, dtype=_U8, device=x.device)
        rc = L.stmoe_lora(x.data_ptr(), elem, x.stride(0), T, a.data_ptr(), a.stride(0), a.stride(1), b.data_ptr(), b.stride(0), b.stride(1), n, r, I, O,
                          plan["ids"].data_ptr(), plan["order"].data_ptr(), plan["counts"].data_ptr(), plan["starts"].data_ptr(), _addr(scale), alpha,
                          _addr(base), 0 if base is None else base.stride(0), out.data_ptr(), _ELEM[out.dtype], out.stride(0), _addr(hidden),
                          scratch.data_ptr(), size, st)
        if rc:
            _check(rc, "stmoe_lora")
    return out


def lora_backward(grad, x, a, b, plan, hidden, scale=None, alpha=1.0, stream=None):
    """stmoe_lora_backward: gradients (of x, a, b) for grad [rows][outer] in x's type, from the hidden that lora wrote."""
    elem, T, I, n, r, O = _lora_args(x, a, b, plan, scale, hidden)
    if not (_is_rows(grad, x.dtype) and grad.shape[0] == T and grad.shape[1] == O and grad.get_device() == x.get_device()):
        _refuse(f"grad: expected {(T, O)} of x's type with contiguous rows on x's device")
    if hidden is None:
        _refuse("hidden: what lora wrote is needed")
    _no_tangents(grad)
    st = _stream_of(x, stream)
    if st is None:
        return _there(x, stream, lora_backward, grad, x, a, b, plan, hidden, scale, alpha)
    dx = torch.empty(T, I, dtype=x.dtype, device=x.device)
    da, db = torch.empty(n, r, I, dtype=x.dtype, device=x.device), torch.empty(n, O, r, dtype=x.dtype, device=x.device)
    L = lib()
    size = L.stmoe_lora_backward_scratch_bytes(T, n, r, I, O)
    scratch = torch.empty(size, dtype=_U8, device=x.device)
    if T:
        rc = L.stmoe_lora_backward(grad.data_ptr(), elem, grad.stride(0), x.data_ptr(), x.stride(0), T, a.data_ptr(), a.stride(0), a.stride(1),
                                   b.data_ptr(), b.stride(0), b.stride(1), n, r, I, O, plan["ids"].data_ptr(), plan["order"].data_ptr(),
                                   plan["counts"].data_ptr(), plan["starts"].data_ptr(), _addr(scale), alpha, hidden.data_ptr(), dx.data_ptr(),
                                   I, da.data_ptr(), db.data_ptr(), scratch.data_ptr(), size, st)
        if rc:
            _check(rc, "stmoe_lora_backward")
    else:
        da.zero_(), db.zero_()
    return dx, da, db
