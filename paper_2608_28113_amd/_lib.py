"""ctypes binding of libhscale.so (include/hscale.h), same names as the C ABI.

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

LIB_PATH = Path(__file__).resolve().parent / "libhscale.so"

HSCALE_OK = 0
STATUS = {
    0: "HSCALE_OK", -1: "HSCALE_ERR_NULL", -2: "HSCALE_ERR_SHAPE", -3: "HSCALE_ERR_ALIGN",
    -4: "HSCALE_ERR_WINDOW", -5: "HSCALE_ERR_SCALE", -6: "HSCALE_ERR_WORKSPACE",
    -7: "HSCALE_ERR_HIP", -8: "HSCALE_ERR_OVERLAP", -9: "HSCALE_ERR_SCRATCH", -10: "HSCALE_ERR_DEVICE",
}

# Every symbol include/hscale.h declares.
EXPORTS = (
    "hscale_status_string",
    "hscale_hdiag_workspace_bytes",
    "hscale_hdiag",
    "hscale_hdiag_noalloc",
    "hscale_hdiag_accumulate",
    "hscale_hdiag_finalize",
    "hscale_search",
    "hscale_search_du",
    "hscale_search_4over6",
    "hscale_search_from",
    "hscale_search_block",
    "hscale_search_layers",
    "hscale_search_stats",
    "hscale_shift_summary_workspace_bytes",
    "hscale_shift_summary",
    "hscale_output_error_workspace_bytes",
    "hscale_output_error_least_workspace_bytes",
    "hscale_output_error",
    "hscale_quantize",
    "hscale_adapted_linear_workspace_bytes",
    "hscale_adapted_linear",
    "hscale_pack_activations",
    "hscale_unpack_activations",
    "hscale_adapted_linear_grad_workspace_bytes",
    "hscale_adapted_linear_grad",
    "hscale_token_loss_workspace_bytes",
    "hscale_token_loss",
    "hscale_token_loss_grad_workspace_bytes",
    "hscale_token_loss_grad",
    "hscale_route_tokens",
    "hscale_expert_layer_workspace_bytes",
    "hscale_expert_layer",
    "hscale_adjust_logits",
)

HSCALE_INIT_MAXABS, HSCALE_INIT_4OVER6, HSCALE_INIT_GIVEN = 0, 1, 2
HSCALE_BF16, HSCALE_F32 = 0, 1


class HScaleLayer(ctypes.Structure):
    """struct hscale_layer of include/hscale.h (natural C layout)."""
    _fields_ = [("W", ctypes.c_void_p), ("out", ctypes.c_int64), ("in_", ctypes.c_int64),
                ("h", ctypes.c_void_p), ("global_scale", ctypes.c_float), ("init_codes", ctypes.c_void_p),
                ("scale_codes", ctypes.c_void_p), ("packed_e2m1", ctypes.c_void_p)]



class HScaleAdapters(ctypes.Structure):
    """struct hscale_adapters of include/hscale.h (natural C layout)."""
    _fields_ = [("count", ctypes.c_int32), ("rank", ctypes.c_int32), ("A", ctypes.c_void_p), ("B", ctypes.c_void_p),
                ("alpha", ctypes.c_void_p), ("adapter", ctypes.c_void_p)]


class HScaleExperts(ctypes.Structure):
    """struct hscale_experts of include/hscale.h (natural C layout)."""
    _fields_ = [("global_scale", ctypes.c_void_p), ("scale_codes", ctypes.c_void_p), ("packed_e2m1", ctypes.c_void_p)]


class HScaleLogitRules(ctypes.Structure):
    """struct hscale_logit_rules of include/hscale.h (natural C layout)."""
    _fields_ = [("history", ctypes.c_void_p), ("history_length", ctypes.c_int64), ("history_ld", ctypes.c_int64),
                ("length", ctypes.c_void_p), ("prompt", ctypes.c_void_p), ("repetition", ctypes.c_void_p),
                ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("biases", ctypes.c_int32), ("bias_row", ctypes.c_void_p), ("mask", ctypes.c_void_p),
                ("masks", ctypes.c_int32), ("mask_row", ctypes.c_void_p)]


_lib = None


class HScaleError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def load() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not LIB_PATH.exists():
        raise ImportError(
            f"{LIB_PATH} is not built; run paper_2608_28113_amd/build.py "
            "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(str(LIB_PATH))
    P, i64, i32, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    lib.hscale_status_string.argtypes = [ctypes.c_int]
    lib.hscale_status_string.restype = ctypes.c_char_p
    lib.hscale_hdiag_workspace_bytes.argtypes = [i64, i64]
    lib.hscale_hdiag_workspace_bytes.restype = sz
    lib.hscale_hdiag.argtypes = [P, i64, i64, P, P, sz, P]
    lib.hscale_hdiag.restype = ctypes.c_int
    lib.hscale_hdiag_noalloc.argtypes = [P, i64, i64, P, P]
    lib.hscale_hdiag_noalloc.restype = ctypes.c_int
    lib.hscale_search.argtypes = [P, i64, i64, P, i32, f32, P, P, P]
    lib.hscale_search.restype = ctypes.c_int
    lib.hscale_search_du.argtypes = [P, i64, i64, P, i32, i32, f32, P, P, P]
    lib.hscale_search_du.restype = ctypes.c_int
    lib.hscale_quantize.argtypes = [P, i64, i64, f32, P, P, P]
    lib.hscale_quantize.restype = ctypes.c_int
    lib.hscale_hdiag_accumulate.argtypes = [P, i64, i64, P, P, sz, P]
    lib.hscale_hdiag_accumulate.restype = ctypes.c_int
    lib.hscale_hdiag_finalize.argtypes = [P, i64, P, P]
    lib.hscale_hdiag_finalize.restype = ctypes.c_int
    lib.hscale_search_4over6.argtypes = [P, i64, i64, P, i32, i32, f32, P, P, P]
    lib.hscale_search_4over6.restype = ctypes.c_int
    lib.hscale_search_from.argtypes = [P, i64, i64, P, i32, i32, f32, P, P, P, P]
    lib.hscale_search_from.restype = ctypes.c_int
    lib.hscale_search_block.argtypes = [P, i64, i64, i64, P, i32, i32, f32, i32, P, i64, P, i64, P, i64, P]
    lib.hscale_search_block.restype = ctypes.c_int
    lib.hscale_search_layers.argtypes = [ctypes.POINTER(HScaleLayer), i32, i32, i32, i32, P]
    lib.hscale_search_layers.restype = ctypes.c_int
    lib.hscale_search_stats.argtypes = [P, i64, i64, P, i32, i32, f32, i32, P, P, P, P, P, P, P]
    lib.hscale_search_stats.restype = ctypes.c_int
    lib.hscale_shift_summary_workspace_bytes.argtypes = [i64, i32, i32]
    lib.hscale_shift_summary_workspace_bytes.restype = sz
    lib.hscale_shift_summary.argtypes = [P, P, P, i64, i32, i32, P, P, P, P, P, sz, P]
    lib.hscale_shift_summary.restype = ctypes.c_int
    lib.hscale_output_error_workspace_bytes.argtypes = [i64, i64, i64]
    lib.hscale_output_error_workspace_bytes.restype = sz
    lib.hscale_output_error_least_workspace_bytes.argtypes = [i64, i64, i64]
    lib.hscale_output_error_least_workspace_bytes.restype = sz
    lib.hscale_output_error.argtypes = [P, i64, i64, P, i64, f32, P, P, P, P, sz, P]
    lib.hscale_output_error.restype = ctypes.c_int
    AD = ctypes.POINTER(HScaleAdapters)
    lib.hscale_adapted_linear_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    lib.hscale_adapted_linear_workspace_bytes.restype = sz
    lib.hscale_adapted_linear.argtypes = [P, i64, i64, i64, i64, f32, P, P, AD, P, i64, P, sz, P]
    lib.hscale_adapted_linear.restype = ctypes.c_int
    lib.hscale_pack_activations.argtypes = [P, i64, i64, i64, P, P, P]
    lib.hscale_pack_activations.restype = ctypes.c_int
    lib.hscale_unpack_activations.argtypes = [P, P, i64, i64, P, i64, P]
    lib.hscale_unpack_activations.restype = ctypes.c_int
    lib.hscale_adapted_linear_grad_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    lib.hscale_adapted_linear_grad_workspace_bytes.restype = sz
    lib.hscale_adapted_linear_grad.argtypes = [P, i64, i64, i64, P, P, i64, f32, P, P, AD, P, i64, P, P, P, sz, P]
    lib.hscale_adapted_linear_grad.restype = ctypes.c_int
    lib.hscale_token_loss_workspace_bytes.argtypes = [i64, i64, i64]
    lib.hscale_token_loss_workspace_bytes.restype = sz
    lib.hscale_token_loss.argtypes = [P, i64, i64, i64, P, i64, P, P, P, P, sz, P]
    lib.hscale_token_loss.restype = ctypes.c_int
    lib.hscale_token_loss_grad_workspace_bytes.argtypes = [i64, i64, i64]
    lib.hscale_token_loss_grad_workspace_bytes.restype = sz
    lib.hscale_token_loss_grad.argtypes = [P, i64, i64, i64, P, i64, P, P, P, P, i64, P, P, sz, P]
    lib.hscale_token_loss_grad.restype = ctypes.c_int
    lib.hscale_route_tokens.argtypes = [P, i32, i64, i32, i64, i32, i32, P, P, P]
    lib.hscale_route_tokens.restype = ctypes.c_int
    lib.hscale_expert_layer_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    lib.hscale_expert_layer_workspace_bytes.restype = sz
    lib.hscale_expert_layer.argtypes = [P, i64, i64, i64, i64, i32, P, P, P, P, P, i32, P, i64, P, sz, P]
    lib.hscale_expert_layer.restype = ctypes.c_int
    lib.hscale_adjust_logits.argtypes = [ctypes.POINTER(HScaleLogitRules), P, i32, i64, i64, i64, P, i64, P]
    lib.hscale_adjust_logits.restype = ctypes.c_int
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().hscale_status_string(int(status)).decode()


def hscale_hdiag_workspace_bytes(tokens: int, in_: int) -> int:
    return int(load().hscale_hdiag_workspace_bytes(int(tokens), int(in_)))


def hscale_hdiag(X: int, tokens: int, in_: int, h: int, workspace: int, workspace_bytes: int,
                 stream: int) -> int:
    return load().hscale_hdiag(X or None, tokens, in_, h or None, workspace or None,
                               workspace_bytes, stream or None)


def hscale_hdiag_noalloc(X: int, tokens: int, in_: int, h: int, stream: int) -> int:
    return load().hscale_hdiag_noalloc(X or None, tokens, in_, h or None, stream or None)


def hscale_search(W: int, out: int, in_: int, h: int, window: int, global_scale: float,
                  scale_codes: int, packed_e2m1: int, stream: int) -> int:
    return load().hscale_search(W or None, out, in_, h or None, window, global_scale,
                                scale_codes or None, packed_e2m1 or None, stream or None)


def hscale_search_du(W: int, out: int, in_: int, h: int, down: int, up: int, global_scale: float,
                     scale_codes: int, packed_e2m1: int, stream: int) -> int:
    return load().hscale_search_du(W or None, out, in_, h or None, down, up, global_scale,
                                   scale_codes or None, packed_e2m1 or None, stream or None)


def hscale_quantize(W: int, out: int, in_: int, global_scale: float, scale_codes: int,
                    packed_e2m1: int, stream: int) -> int:
    return load().hscale_quantize(W or None, out, in_, global_scale, scale_codes or None,
                                  packed_e2m1 or None, stream or None)


def hscale_hdiag_accumulate(X: int, tokens: int, in_: int, h64: int, workspace: int,
                            workspace_bytes: int, stream: int) -> int:
    return load().hscale_hdiag_accumulate(X or None, tokens, in_, h64 or None, workspace or None,
                                          workspace_bytes, stream or None)


def hscale_hdiag_finalize(h64: int, in_: int, h: int, stream: int) -> int:
    return load().hscale_hdiag_finalize(h64 or None, in_, h or None, stream or None)


def hscale_search_4over6(W: int, out: int, in_: int, h: int, down: int, up: int, global_scale: float,
                         scale_codes: int, packed_e2m1: int, stream: int) -> int:
    return load().hscale_search_4over6(W or None, out, in_, h or None, down, up, global_scale,
                                       scale_codes or None, packed_e2m1 or None, stream or None)


def hscale_search_from(W: int, out: int, in_: int, h: int, down: int, up: int, global_scale: float,
                       init_codes: int, scale_codes: int, packed_e2m1: int, stream: int) -> int:
    return load().hscale_search_from(W or None, out, in_, h or None, down, up, global_scale,
                                     init_codes or None, scale_codes or None, packed_e2m1 or None,
                                     stream or None)


def hscale_search_block(W: int, ldw: int, out: int, cols: int, h: int, down: int, up: int,
                        global_scale: float, init_mode: int, init_codes: int, ldi: int, scale_codes: int,
                        ldc: int, packed_e2m1: int, ldp: int, stream: int) -> int:
    return load().hscale_search_block(W or None, ldw, out, cols, h or None, down, up, global_scale,
                                      init_mode, init_codes or None, ldi, scale_codes or None, ldc,
                                      packed_e2m1 or None, ldp, stream or None)


def hscale_search_layers(layers, down: int, up: int, init_mode: int, stream: int) -> int:
    """layers: sequence of (W, out, in, h, global_scale, init_codes, scale_codes, packed_e2m1)
    with device addresses as ints (0 for NULL)."""
    arr = (HScaleLayer * max(len(layers), 1))()
    for k, (W, out, in_, h, s_g, init, codes, packed) in enumerate(layers):
        arr[k] = HScaleLayer(W or None, out, in_, h or None, s_g, init or None, codes or None, packed or None)
    return load().hscale_search_layers(arr if layers else None, len(layers), down, up, init_mode, stream or None)


def hscale_search_stats(W: int, out: int, in_: int, h: int, down: int, up: int, global_scale: float,
                        init_mode: int, init_codes: int, scale_codes: int, packed_e2m1: int, shift: int,
                        err_best: int, err_init: int, stream: int) -> int:
    return load().hscale_search_stats(W or None, out, in_, h or None, down, up, global_scale, init_mode,
                                      init_codes or None, scale_codes or None, packed_e2m1 or None,
                                      shift or None, err_best or None, err_init or None, stream or None)


def hscale_shift_summary_workspace_bytes(groups: int, down: int, up: int) -> int:
    return load().hscale_shift_summary_workspace_bytes(groups, down, up)


def hscale_shift_summary(shift: int, err_best: int, err_init: int, groups: int, down: int, up: int,
                         count: int, sum_init: int, sum_best: int, sum_rel: int, workspace: int,
                         workspace_bytes: int, stream: int) -> int:
    return load().hscale_shift_summary(shift or None, err_best or None, err_init or None, groups, down, up,
                                       count or None, sum_init or None, sum_best or None, sum_rel or None,
                                       workspace or None, workspace_bytes, stream or None)


def hscale_output_error_workspace_bytes(tokens: int, in_: int, out: int) -> int:
    return load().hscale_output_error_workspace_bytes(tokens, in_, out)


def hscale_output_error_least_workspace_bytes(tokens: int, in_: int, out: int) -> int:
    return load().hscale_output_error_least_workspace_bytes(tokens, in_, out)


def hscale_output_error(X: int, tokens: int, in_: int, W: int, out: int, global_scale: float, scale_codes: int,
                        packed_e2m1: int, row_err: int, workspace: int, workspace_bytes: int, stream: int) -> int:
    return load().hscale_output_error(X or None, tokens, in_, W or None, out, global_scale, scale_codes or None,
                                      packed_e2m1 or None, row_err or None, workspace or None, workspace_bytes,
                                      stream or None)


# The entry points of a stored layer in use.  They are called once a layer and
# token, where microseconds count: pointers go as they are (c_void_p takes 0 for
# NULL).


def _adapters(adapters):
    """A pointer to struct hscale_adapters of (count, rank, A, B, alpha, adapter), or NULL for None."""
    return None if adapters is None else ctypes.byref(HScaleAdapters(*adapters))


def hscale_adapted_linear_workspace_bytes(tokens: int, in_: int, out: int, count: int, rank: int) -> int:
    return (_lib or load()).hscale_adapted_linear_workspace_bytes(tokens, in_, out, count, rank)


def hscale_adapted_linear(X: int, tokens: int, in_: int, ldx: int, out: int, global_scale: float, scale_codes: int,
                          packed_e2m1: int, adapters, Y: int, ldy: int, workspace: int, workspace_bytes: int,
                          stream: int) -> int:
    return (_lib or load()).hscale_adapted_linear(X, tokens, in_, ldx, out, global_scale, scale_codes, packed_e2m1,
                                                  _adapters(adapters), Y, ldy, workspace, workspace_bytes, stream)


def hscale_pack_activations(X: int, tokens: int, in_: int, ldx: int, q: int, scale: int, stream: int) -> int:
    return (_lib or load()).hscale_pack_activations(X, tokens, in_, ldx, q, scale, stream)


def hscale_unpack_activations(q: int, scale: int, tokens: int, in_: int, X: int, ldx: int, stream: int) -> int:
    return (_lib or load()).hscale_unpack_activations(q, scale, tokens, in_, X, ldx, stream)


def hscale_adapted_linear_grad_workspace_bytes(tokens: int, in_: int, out: int, count: int, rank: int) -> int:
    return (_lib or load()).hscale_adapted_linear_grad_workspace_bytes(tokens, in_, out, count, rank)


def hscale_adapted_linear_grad(dY: int, tokens: int, out: int, lddy: int, q: int, scale: int, in_: int,
                               global_scale: float, scale_codes: int, packed_e2m1: int, adapters, dX: int, lddx: int,
                               dA: int, dB: int, workspace: int, workspace_bytes: int, stream: int) -> int:
    return (_lib or load()).hscale_adapted_linear_grad(dY, tokens, out, lddy, q, scale, in_, global_scale,
                                                       scale_codes, packed_e2m1, _adapters(adapters), dX, lddx, dA,
                                                       dB, workspace, workspace_bytes, stream)


def hscale_token_loss_workspace_bytes(tokens: int, d: int, vocab: int) -> int:
    return (_lib or load()).hscale_token_loss_workspace_bytes(tokens, d, vocab)


def hscale_token_loss(X: int, tokens: int, d: int, ldx: int, W: int, vocab: int, target: int, loss: int, lse: int,
                      workspace: int, workspace_bytes: int, stream: int) -> int:
    return (_lib or load()).hscale_token_loss(X, tokens, d, ldx, W, vocab, target, loss, lse, workspace,
                                              workspace_bytes, stream)


def hscale_token_loss_grad_workspace_bytes(tokens: int, d: int, vocab: int) -> int:
    return (_lib or load()).hscale_token_loss_grad_workspace_bytes(tokens, d, vocab)


def hscale_token_loss_grad(X: int, tokens: int, d: int, ldx: int, W: int, vocab: int, target: int, lse: int,
                           weight: int, dX: int, lddx: int, dW: int, workspace: int, workspace_bytes: int,
                           stream: int) -> int:
    return (_lib or load()).hscale_token_loss_grad(X, tokens, d, ldx, W, vocab, target, lse, weight, dX, lddx, dW,
                                                   workspace, workspace_bytes, stream)


def hscale_route_tokens(logits: int, type_: int, tokens: int, experts: int, ld: int, k: int, normalize: int,
                        expert: int, weight: int, stream: int) -> int:
    return (_lib or load()).hscale_route_tokens(logits, type_, tokens, experts, ld, k, normalize, expert, weight,
                                                stream)


def hscale_expert_layer_workspace_bytes(tokens: int, in_: int, hidden: int, experts: int, k: int) -> int:
    return (_lib or load()).hscale_expert_layer_workspace_bytes(tokens, in_, hidden, experts, k)


_ThreeExperts = HScaleExperts * 3
_EXPERTS_BYTES = ctypes.sizeof(HScaleExperts)


def hscale_expert_layer(X: int, tokens: int, in_: int, ldx: int, hidden: int, experts: int, gate, up, down,
                        expert: int, weight: int, k: int, Y: int, ldy: int, workspace: int, workspace_bytes: int,
                        stream: int) -> int:
    """gate, up, down: (global_scale, scale_codes, packed_e2m1) as addresses, or None for NULL."""
    m = _ThreeExperts(gate or (), up or (), down or ())
    at = ctypes.addressof(m)
    return (_lib or load()).hscale_expert_layer(X, tokens, in_, ldx, hidden, experts, at if gate else 0,
                                                at + _EXPERTS_BYTES if up else 0, at + 2 * _EXPERTS_BYTES if down else 0,
                                                expert, weight, k, Y, ldy, workspace, workspace_bytes, stream)


def hscale_adjust_logits(rules, logits: int, type_: int, rows: int, vocab: int, ld: int, out: int, ldo: int,
                         stream: int) -> int:
    """rules: the fields of struct hscale_logit_rules in order, addresses as ints (0 for NULL), or None."""
    r = None if rules is None else ctypes.byref(HScaleLogitRules(*rules))
    return (_lib or load()).hscale_adjust_logits(r, logits, type_, rows, vocab, ld, out, ldo, stream)
