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
