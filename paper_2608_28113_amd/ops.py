"""Torch-tensor front end of the C ABI.

PyTorch supplies device memory and the current stream; these functions only
check tensor metadata, allocate outputs and pass raw pointers to
libhscale.so.  All arithmetic happens in the library's HIP kernels.

The C ABI cannot see buffer sizes or devices, so every tensor handed to it
here (inputs, caller-provided outputs and workspaces) is checked for dtype,
shape, contiguity and device first: a wrong buffer raises ValueError and
nothing is launched.

A call given `stream` runs there.  New outputs and scratch are allocated for
it; the tensors that are passed in are the caller's to order and to keep: what
wrote them comes before on that stream, and they are not dropped while it may
still read them (torch.Tensor.record_stream).
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

from . import _lib
from ._lib import HScaleError


def _check(status: int, where: str) -> None:
    if status != _lib.HSCALE_OK:
        raise HScaleError(status, where)


def _stream(stream, device) -> int:
    """Handle of `stream`, or of `device`'s current stream when None.  A
    torch stream must belong to `device`, the device the operands are on."""
    if stream is None:
        # The handle itself: building a torch.cuda.Stream around it costs 2 us
        # of a call that takes 4.
        return torch._C._cuda_getCurrentRawStream(device.index)
    if isinstance(stream, torch.cuda.Stream) and stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the operands on {device}")
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _elsewhere(stream, device):
    """`stream` as a torch stream if it is another than `device`'s current one, else None."""
    if stream is None or device.type != "cuda":
        return None
    handle = _stream(stream, device)
    if handle == torch._C._cuda_getCurrentRawStream(device.index):
        return None
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)


def _new(shape, dtype, device, stream, zeros=False, scratch=False) -> torch.Tensor:
    """A new tensor of a call on `stream`.  The allocator hands memory out again
    in the order of the stream that it was allocated on, so memory of a call on
    another stream than the current one is allocated on that one: nothing that
    pends on the current stream still uses it, and scratch that is dropped when
    the call returns is not given to the current stream while the call runs.
    What is returned is recorded on the current stream too, where the caller
    will use and drop it."""
    make = torch.zeros if zeros else torch.empty
    if stream is None or (side := _elsewhere(stream, device)) is None:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(side):
        t = make(shape, dtype=dtype, device=device)
    if not scratch:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def _call(device, fn, *args) -> int:
    """Calls the library with `device` current, so that its launches go to
    the device that holds the operands."""
    if torch._C._cuda_getDevice() == device.index:  # already current: no context to enter (1.3 us)
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _on_device(t) -> bool:
    """t is a tensor in GPU memory (the only memory the kernels may touch)."""
    return isinstance(t, torch.Tensor) and t.is_cuda


def _bf16_matrix(t, name: str) -> None:
    if (not _on_device(t) or t.dtype != torch.bfloat16 or t.dim() != 2 or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous 2-D bf16 CUDA tensor")


def _tensor(t, name: str, dtype, shape, device) -> torch.Tensor:
    """t must be a contiguous tensor of this dtype and shape (a tuple) on `device`."""
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or t.device != device
            or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return t


def _out(t, name: str, dtype, shape, device, stream) -> torch.Tensor:
    """A caller-provided output (checked) or a new one of a call on `stream`."""
    if t is None:
        return _new(shape, dtype, device, stream)
    return _tensor(t, name, dtype, shape, device)


def _workspace(ws, need: int, device, stream) -> tuple[int, int, torch.Tensor | None]:
    """(pointer, bytes, tensor) of a caller-provided scratch tensor (any dtype,
    contiguous, on `device`) or of a new one of a call on `stream`; the library
    checks the size.  The caller holds the tensor until its launches are queued,
    so that no other thread is given the memory before them."""
    if ws is None:
        if need <= 0:
            return 0, 0, None
        ws = _new((need,), torch.uint8, device, stream, scratch=True)
    elif not isinstance(ws, torch.Tensor) or ws.device != device or not ws.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return ws.data_ptr(), ws.numel() * ws.element_size(), ws


def _row_view(t, dtype, shape, device, name: str) -> int:
    """A 2-D view with unit column stride; returns its row stride."""
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or t.device != device
            or (shape[1] > 1 and t.stride(1) != 1)):
        raise ValueError(f"{name} must be a 2-D {dtype} view of shape {tuple(shape)} on {device} "
                         "with unit column stride")
    return t.stride(0) if shape[0] > 1 else shape[1]


def _init_mode(init, shape, device):
    """(init_mode, initial-code tensor or None) of an `init` argument."""
    if isinstance(init, str):
        modes = {"maxabs": _lib.HSCALE_INIT_MAXABS, "rtn": _lib.HSCALE_INIT_MAXABS,
                 "4over6": _lib.HSCALE_INIT_4OVER6}
        if init not in modes:
            raise ValueError("init must be 'maxabs', '4over6' or a uint8 tensor of codes")
        return modes[init], None
    if isinstance(init, torch.Tensor):
        return _lib.HSCALE_INIT_GIVEN, _tensor(init, "initial codes", torch.uint8, shape, device)
    raise ValueError("init must be 'maxabs', '4over6' or a uint8 tensor of codes")


def _window(window, down, up) -> tuple[int, int]:
    if window is not None:
        if down is not None or up is not None:
            raise ValueError("give either window or down/up")
        return int(window), int(window)
    if down is None or up is None:
        raise ValueError("give window or both down and up")
    return int(down), int(up)


def hdiag_workspace_bytes(tokens: int, in_features: int) -> int:
    """Bytes of scratch hdiag needs for a [tokens, in_features] X."""
    return _lib.hscale_hdiag_workspace_bytes(tokens, in_features)


def hdiag(X: torch.Tensor, h: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
          stream=None) -> torch.Tensor:
    """h = diag(X^T X) (Sec. 3.2, Eq. 4) of bf16 X [tokens, in] as fp32 [in]."""
    _bf16_matrix(X, "X")
    T, n = X.shape
    dev = X.device
    h = _out(h, "h", torch.float32, (n,), dev, stream)
    ws_ptr, ws_bytes, held = _workspace(workspace, hdiag_workspace_bytes(T, n), dev, stream)
    _check(_call(dev, _lib.hscale_hdiag, X.data_ptr(), T, n, h.data_ptr(), ws_ptr, ws_bytes,
                 _stream(stream, dev)), "hscale_hdiag")
    return h


def hdiag_noalloc(X: torch.Tensor, h: torch.Tensor, stream=None) -> torch.Tensor:
    """hdiag into a caller-provided fp32 h [in] with the library's static
    scratch instead of a workspace: the call allocates no device memory
    (problems up to 2^20 columns; calls that may overlap on one GPU race)."""
    _bf16_matrix(X, "X")
    T, n = X.shape
    dev = X.device
    _tensor(h, "h", torch.float32, (n,), dev)
    _check(_call(dev, _lib.hscale_hdiag_noalloc, X.data_ptr(), T, n, h.data_ptr(), _stream(stream, dev)),
           "hscale_hdiag_noalloc")
    return h


def search(W: torch.Tensor, h: torch.Tensor, global_scale: float, window: int | None = None,
           down: int | None = None, up: int | None = None, init="maxabs",
           scale_codes: torch.Tensor | None = None, packed_e2m1: torch.Tensor | None = None, stream=None):
    """The per-group NVFP4 scale search (Sec. 3.3).  Returns
    (scale_codes uint8 [out, in/16], packed_e2m1 uint8 [out, in/2]).

    ``window`` gives the symmetric shift set -window..+window; ``down``/``up``
    the paper's asymmetric one.  ``init`` is "maxabs" (Eq. 7), "4over6", or a
    uint8 tensor [out, in/16] of initial codes (it may be ``scale_codes``
    itself, to refine in place).
    """
    _bf16_matrix(W, "W")
    m, n = W.shape
    dev = W.device
    _tensor(h, "h", torch.float32, (n,), dev)
    down, up = _window(window, down, up)
    mode, init_t = _init_mode(init, (m, n // 16), dev)
    scale_codes = _out(scale_codes, "scale_codes", torch.uint8, (m, n // 16), dev, stream)
    packed_e2m1 = _out(packed_e2m1, "packed_e2m1", torch.uint8, (m, n // 2), dev, stream)
    s = _stream(stream, dev)
    if mode == _lib.HSCALE_INIT_MAXABS:
        st = _call(dev, _lib.hscale_search_du, W.data_ptr(), m, n, h.data_ptr(), down, up, float(global_scale),
                   scale_codes.data_ptr(), packed_e2m1.data_ptr(), s)
        _check(st, "hscale_search_du")
    elif mode == _lib.HSCALE_INIT_4OVER6:
        st = _call(dev, _lib.hscale_search_4over6, W.data_ptr(), m, n, h.data_ptr(), down, up, float(global_scale),
                   scale_codes.data_ptr(), packed_e2m1.data_ptr(), s)
        _check(st, "hscale_search_4over6")
    else:
        st = _call(dev, _lib.hscale_search_from, W.data_ptr(), m, n, h.data_ptr(), down, up, float(global_scale),
                   init_t.data_ptr(), scale_codes.data_ptr(), packed_e2m1.data_ptr(), s)
        _check(st, "hscale_search_from")
    return scale_codes, packed_e2m1


def search_layers(layers, window: int | None = None, down: int | None = None, up: int | None = None,
                  init="maxabs", outputs=None, stream=None):
    """The search of several layers in one launch (per up to 32 layers):
    ``layers`` is a sequence of (W, h, global_scale), all on one device;
    ``init`` is "maxabs", "4over6" or a sequence of per-layer uint8 code
    tensors; ``outputs`` optionally a sequence of (scale_codes, packed_e2m1)
    to write.  Returns the list of (scale_codes, packed_e2m1), each equal to
    what ``search`` returns for that layer alone."""
    layers = list(layers)
    down, up = _window(window, down, up)
    if outputs is not None:
        outputs = list(outputs)
        if len(outputs) != len(layers):
            raise ValueError("give one (scale_codes, packed_e2m1) pair per layer")
    given = None
    if isinstance(init, str):
        mode, _ = _init_mode(init, None, None)
    else:
        given = list(init)
        if len(given) != len(layers):
            raise ValueError("give one initial-code tensor per layer")
        mode = _lib.HSCALE_INIT_GIVEN
    dev = None
    args, result = [], []
    for k, layer in enumerate(layers):
        if len(layer) != 3:
            raise ValueError("each layer is (W, h, global_scale)")
        W, h, s_g = layer
        _bf16_matrix(W, f"W of layer {k}")
        if dev is None:
            dev = W.device
        elif W.device != dev:
            raise ValueError("all layers must be on one device")
        m, n = W.shape
        _tensor(h, f"h of layer {k}", torch.float32, (n,), dev)
        codes, packed = (None, None) if outputs is None else outputs[k]
        codes = _out(codes, f"scale_codes of layer {k}", torch.uint8, (m, n // 16), dev, stream)
        packed = _out(packed, f"packed_e2m1 of layer {k}", torch.uint8, (m, n // 2), dev, stream)
        iptr = 0
        if given is not None:
            iptr = _tensor(given[k], f"initial codes of layer {k}", torch.uint8, (m, n // 16), dev).data_ptr()
        args.append((W.data_ptr(), m, n, h.data_ptr(), float(s_g), iptr, codes.data_ptr(), packed.data_ptr()))
        result.append((codes, packed))
    if not layers:
        return result
    _check(_call(dev, _lib.hscale_search_layers, args, down, up, mode, _stream(stream, dev)), "hscale_search_layers")
    return result


def search_block(W: torch.Tensor, h: torch.Tensor, global_scale: float, down: int, up: int,
                 scale_codes: torch.Tensor, packed_e2m1: torch.Tensor, init="maxabs", stream=None):
    """The search on a column block given as strided views: W = Wfull[:, a:b]
    (bf16), h = hfull[a:b], scale_codes = codes[:, a/16:b/16] and
    packed_e2m1 = packed[:, a/2:b/2] (uint8), as in the paper's GPTQ
    combination (App. B).  Outputs are written in place."""
    if not _on_device(W) or W.dim() != 2:
        raise ValueError("W must be a 2-D bf16 CUDA view")
    m, cols = W.shape
    dev = W.device
    ldw = _row_view(W, torch.bfloat16, (m, cols), dev, "W")
    ldc = _row_view(scale_codes, torch.uint8, (m, cols // 16), dev, "scale_codes")
    ldp = _row_view(packed_e2m1, torch.uint8, (m, cols // 2), dev, "packed_e2m1")
    _tensor(h, "h", torch.float32, (cols,), dev)
    if isinstance(init, torch.Tensor):
        ldi = _row_view(init, torch.uint8, (m, cols // 16), dev, "initial codes")
        mode, iptr = _lib.HSCALE_INIT_GIVEN, init.data_ptr()
    else:
        mode, _ = _init_mode(init, None, dev)
        iptr, ldi = 0, 0
    st = _call(dev, _lib.hscale_search_block, W.data_ptr(), ldw, m, cols, h.data_ptr(), int(down), int(up),
               float(global_scale), mode, iptr, ldi, scale_codes.data_ptr(), ldc, packed_e2m1.data_ptr(), ldp,
               _stream(stream, dev))
    _check(st, "hscale_search_block")
    return scale_codes, packed_e2m1


def hdiag_accumulate(X: torch.Tensor, h64: torch.Tensor, workspace: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """h64 += diag(X^T X) for one calibration batch (fp64 accumulator)."""
    _bf16_matrix(X, "X")
    T, n = X.shape
    dev = X.device
    _tensor(h64, "h64", torch.float64, (n,), dev)
    ws_ptr, ws_bytes, held = _workspace(workspace, hdiag_workspace_bytes(T, n), dev, stream)
    _check(_call(dev, _lib.hscale_hdiag_accumulate, X.data_ptr(), T, n, h64.data_ptr(), ws_ptr, ws_bytes,
                 _stream(stream, dev)), "hscale_hdiag_accumulate")
    return h64


def hdiag_finalize(h64: torch.Tensor, h: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """h = fp32(h64)."""
    if not _on_device(h64) or h64.dim() != 1:
        raise ValueError("h64 must be a 1-D fp64 CUDA tensor")
    n = h64.shape[0]
    dev = h64.device
    _tensor(h64, "h64", torch.float64, (n,), dev)
    h = _out(h, "h", torch.float32, (n,), dev, stream)
    _check(_call(dev, _lib.hscale_hdiag_finalize, h64.data_ptr(), n, h.data_ptr(),
                 _stream(stream, dev)), "hscale_hdiag_finalize")
    return h


def quantize(W: torch.Tensor, global_scale: float, scale_codes: torch.Tensor,
             packed_e2m1: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Packed E2M1 codes of W at the given scale codes (final re-quantization)."""
    _bf16_matrix(W, "W")
    m, n = W.shape
    dev = W.device
    _tensor(scale_codes, "scale_codes", torch.uint8, (m, n // 16), dev)
    packed_e2m1 = _out(packed_e2m1, "packed_e2m1", torch.uint8, (m, n // 2), dev, stream)
    _check(_call(dev, _lib.hscale_quantize, W.data_ptr(), m, n, float(global_scale), scale_codes.data_ptr(),
                 packed_e2m1.data_ptr(), _stream(stream, dev)), "hscale_quantize")
    return packed_e2m1


def search_stats(W: torch.Tensor, h: torch.Tensor, global_scale: float, down: int, up: int, init="maxabs",
                 stream=None):
    """The search with per-group statistics.  Returns a dict of
    scale_codes, packed_e2m1, shift (int8 [out, in/16], the chosen shift),
    err_best and err_init (fp32 [out, in/16], the score at the chosen shift
    and at shift 0)."""
    _bf16_matrix(W, "W")
    m, n = W.shape
    dev = W.device
    _tensor(h, "h", torch.float32, (n,), dev)
    G = (m, n // 16)
    mode, init_t = _init_mode(init, G, dev)
    out = dict(scale_codes=_new(G, torch.uint8, dev, stream),
               packed_e2m1=_new((m, n // 2), torch.uint8, dev, stream),
               shift=_new(G, torch.int8, dev, stream),
               err_best=_new(G, torch.float32, dev, stream),
               err_init=_new(G, torch.float32, dev, stream))
    st = _call(dev, _lib.hscale_search_stats, W.data_ptr(), m, n, h.data_ptr(), int(down), int(up),
               float(global_scale), mode, init_t.data_ptr() if init_t is not None else 0,
               out["scale_codes"].data_ptr(), out["packed_e2m1"].data_ptr(), out["shift"].data_ptr(),
               out["err_best"].data_ptr(), out["err_init"].data_ptr(), _stream(stream, dev))
    _check(st, "hscale_search_stats")
    return out


def shift_summary(shift: torch.Tensor, err_best: torch.Tensor, err_init: torch.Tensor, down: int, up: int,
                  stream=None) -> dict:
    """Per-shift counts and fp64 sums of initial errors, chosen errors and
    relative reductions over the groups (bins d = -down..up), as tensors of
    length down + up + 1 on the device."""
    if not _on_device(shift):
        raise ValueError("shift must be an int8 CUDA tensor")
    groups = shift.numel()
    dev = shift.device
    for t, dt, name in ((shift, torch.int8, "shift"), (err_best, torch.float32, "err_best"),
                        (err_init, torch.float32, "err_init")):
        if (not isinstance(t, torch.Tensor) or t.dtype != dt or t.device != dev or not t.is_contiguous()
                or t.numel() != groups):
            raise ValueError(f"{name} must be a contiguous {dt} tensor on {dev} with one entry per group")
    K = int(down) + int(up) + 1
    # counts are uint64 in the C ABI; int64 holds them (< 2^63) with full torch support
    out = dict(count=_new((K,), torch.int64, dev, stream), sum_init=_new((K,), torch.float64, dev, stream),
               sum_best=_new((K,), torch.float64, dev, stream), sum_rel=_new((K,), torch.float64, dev, stream))
    need = _lib.hscale_shift_summary_workspace_bytes(groups, int(down), int(up))
    ws = _new((max(need, 8),), torch.uint8, dev, stream, scratch=True)
    st = _call(dev, _lib.hscale_shift_summary, shift.data_ptr(), err_best.data_ptr(), err_init.data_ptr(), groups,
               int(down), int(up), out["count"].data_ptr(), out["sum_init"].data_ptr(), out["sum_best"].data_ptr(),
               out["sum_rel"].data_ptr(), ws.data_ptr(), need, _stream(stream, dev))
    _check(st, "hscale_shift_summary")
    return out


def output_error_workspace_bytes(tokens: int, in_features: int, out_features: int) -> int:
    """Bytes of scratch with which output_error is fastest."""
    return _lib.hscale_output_error_workspace_bytes(tokens, in_features, out_features)


def output_error(X: torch.Tensor, W: torch.Tensor, global_scale: float, scale_codes: torch.Tensor,
                 packed_e2m1: torch.Tensor, row_err: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Eq. 3 per output row: row_err[r] += sum_t (X dW^T)_tr^2 with dW = W - W^
    the rounding error of the stored NVFP4 tensor (scale_codes, packed_e2m1).
    row_err is fp64 [out] (zeros when not given); the layer's L_full is its
    sum.  Without a workspace it allocates one of output_error_workspace_bytes,
    or the least one that the library accepts where that much is not free."""
    _bf16_matrix(X, "X")
    _bf16_matrix(W, "W")
    T, n = X.shape
    m = W.shape[0]
    dev = X.device
    if W.shape[1] != n or W.device != dev:
        raise ValueError("X and W must share in_features and device")
    _tensor(scale_codes, "scale_codes", torch.uint8, (m, n // 16), dev)
    _tensor(packed_e2m1, "packed_e2m1", torch.uint8, (m, n // 2), dev)
    if row_err is None:
        row_err = _new((m,), torch.float64, dev, stream, zeros=True)
    _tensor(row_err, "row_err", torch.float64, (m,), dev)
    need = output_error_workspace_bytes(T, n, m)
    try:
        ws_ptr, ws_bytes, held = _workspace(workspace, need, dev, stream)
    except torch.OutOfMemoryError:
        least = _lib.hscale_output_error_least_workspace_bytes(T, n, m)
        if least == need:
            raise
        ws_ptr, ws_bytes, held = _workspace(None, least, dev, stream)
    _check(_call(dev, _lib.hscale_output_error, X.data_ptr(), T, n, W.data_ptr(), m, float(global_scale),
                 scale_codes.data_ptr(), packed_e2m1.data_ptr(), row_err.data_ptr(), ws_ptr, ws_bytes,
                 _stream(stream, dev)), "hscale_output_error")
    return row_err


# ---------------------------------------------------------------------------
# A stored layer in use
# ---------------------------------------------------------------------------

CHECKPOINT_BLOCK = 128  # activations per checkpoint scale


def _no_graph(where: str, *tensors, grad: bool = True) -> None:
    """Refuses tensors whose gradient or tangent would be expected and lost: the calls record no graph."""
    if torch.is_grad_enabled():
        for t in tensors:
            if isinstance(t, torch.Tensor) and t.requires_grad:
                if not grad:
                    raise ValueError(f"{where} records no graph and has no gradient: call it under torch.no_grad() "
                                     "or with detached tensors")
                raise ValueError(f"{where} records no graph: call it under torch.no_grad(), in an autograd function "
                                 f"or with detached tensors, and take the gradients from {where}_grad")
    # Forward mode: no_grad leaves it on, an autograd function's forward turns it off.
    if forward_ad._current_level >= 0 and torch._C._is_fwd_grad_enabled():
        for t in tensors:
            if isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError(f"{where} would lose a tangent: call it with torch.autograd.forward_ad.unpack_dual's "
                                 "primal, or in an autograd function with a jvp")


def _rows_in(t, name: str) -> int:
    """t is a 2-D bf16 CUDA view with unit column stride; its row stride."""
    if not _on_device(t) or t.dtype is not torch.bfloat16 or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D bf16 CUDA tensor")
    row, col = t.stride()
    rows, cols = t.shape
    if col != 1 and cols > 1:
        raise ValueError(f"{name} must have unit column stride")
    return row if rows > 1 else cols


def _rows_out(t, name: str, shape, device, stream) -> tuple[torch.Tensor, int]:
    """A caller-provided bf16 view of rows (checked) or a new tensor, and its row stride."""
    if t is None:
        return _new(shape, torch.bfloat16, device, stream), shape[1]
    return t, _row_view(t, torch.bfloat16, shape, device, name)


def _stored(scale_codes, packed_e2m1, n: int, device) -> int:
    """The stored layer's tensors, for `n` inputs; its outputs."""
    if not isinstance(packed_e2m1, torch.Tensor) or packed_e2m1.dim() != 2:
        raise ValueError("packed_e2m1 must be a 2-D uint8 tensor")
    m = packed_e2m1.shape[0]
    _tensor(packed_e2m1, "packed_e2m1", torch.uint8, (m, n // 2), device)
    _tensor(scale_codes, "scale_codes", torch.uint8, (m, n // 16), device)
    return m


def _adapters(A, B, alpha, adapter, tokens: int, n: int, m: int, device):
    """The adapters' checked (count, rank, pointers...) for the library, or None."""
    if A is None or B is None:
        if not (A is None and B is None and alpha is None and adapter is None):
            raise ValueError("alpha and adapter need both A and B")
        return None
    if not isinstance(A, torch.Tensor) or A.dim() != 3:
        raise ValueError("A must be a 3-D bf16 tensor [adapters, rank, in]")
    count, rank = A.shape[0], A.shape[1]
    _tensor(A, "A", torch.bfloat16, (count, rank, n), device)
    _tensor(B, "B", torch.bfloat16, (count, m, rank), device)
    if alpha is not None:
        _tensor(alpha, "alpha", torch.float32, (count,), device)
    if adapter is not None:
        _tensor(adapter, "adapter", torch.int32, (tokens,), device)
    elif count != 1:
        raise ValueError("adapter (int32, one number a token) is required unless there is exactly one adapter")
    return (count, rank, A.data_ptr(), B.data_ptr(), 0 if alpha is None else alpha.data_ptr(),
            0 if adapter is None else adapter.data_ptr())


def adapted_linear_workspace_bytes(tokens: int, in_features: int, out_features: int, adapters: int = 0,
                                   rank: int = 0) -> int:
    """Bytes of scratch adapted_linear needs."""
    return _lib.hscale_adapted_linear_workspace_bytes(tokens, in_features, out_features, adapters, rank)


def adapted_linear(X: torch.Tensor, global_scale: float, scale_codes: torch.Tensor, packed_e2m1: torch.Tensor,
                   A: torch.Tensor | None = None, B: torch.Tensor | None = None, alpha: torch.Tensor | None = None,
                   adapter: torch.Tensor | None = None, Y: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y = X W^T of a stored NVFP4 layer, and each token's low-rank adapter
    beside it: Y[t] += alpha[a] B[a] (A[a] X[t]), a = adapter[t].

    X is bf16 [tokens, in] (rows may be strided, 16-byte aligned), Y bf16
    [tokens, out] (rows may be strided).  A is bf16 [adapters, rank, in], B
    bf16 [adapters, out, rank] (rank a multiple of 8 up to 256), alpha fp32
    [adapters] (1 when None), adapter int32 [tokens], where a number outside
    0 .. adapters - 1 means none; with one adapter it may be None: all use it.

    No graph is recorded: tensors that require a gradient are refused where
    torch would record one (adapted_linear_grad returns the gradients), and
    tensors with a tangent where torch would carry it on.
    """
    ldx = _rows_in(X, "X")
    T, n = X.shape
    dev = X.device
    m = _stored(scale_codes, packed_e2m1, n, dev)
    ad = _adapters(A, B, alpha, adapter, T, n, m, dev)
    _no_graph("adapted_linear", X, A, B, alpha)
    Y, ldy = _rows_out(Y, "Y", (T, m), dev, stream)
    need = adapted_linear_workspace_bytes(T, n, m, *(ad[:2] if ad else (0, 0)))
    ws_ptr, ws_bytes, held = _workspace(workspace, need, dev, stream)
    _check(_call(dev, _lib.hscale_adapted_linear, X.data_ptr(), T, n, ldx, m, float(global_scale),
                 scale_codes.data_ptr(), packed_e2m1.data_ptr(), ad, Y.data_ptr(), ldy, ws_ptr, ws_bytes,
                 _stream(stream, dev)), "hscale_adapted_linear")
    return Y


def pack_activations(X: torch.Tensor, q: torch.Tensor | None = None, scale: torch.Tensor | None = None, stream=None):
    """A checkpoint of bf16 X [tokens, in] (rows may be strided) in 8 bits:
    (q int8 [tokens, in], scale fp32 [tokens, ceil(in / 128)])."""
    ldx = _rows_in(X, "X")
    T, n = X.shape
    dev = X.device
    q = _out(q, "q", torch.int8, (T, n), dev, stream)
    scale = _out(scale, "scale", torch.float32, (T, -(-n // CHECKPOINT_BLOCK)), dev, stream)
    _check(_call(dev, _lib.hscale_pack_activations, X.data_ptr(), T, n, ldx, q.data_ptr(), scale.data_ptr(),
                 _stream(stream, dev)), "hscale_pack_activations")
    return q, scale


def _checkpoint(q, scale) -> tuple[int, int]:
    """The checked checkpoint's (tokens, in)."""
    if not _on_device(q) or q.dtype != torch.int8 or q.dim() != 2 or not q.is_contiguous():
        raise ValueError("q must be a contiguous 2-D int8 CUDA tensor")
    T, n = q.shape
    _tensor(scale, "scale", torch.float32, (T, -(-n // CHECKPOINT_BLOCK)), q.device)
    return T, n


def unpack_activations(q: torch.Tensor, scale: torch.Tensor, X: torch.Tensor | None = None, stream=None):
    """The bf16 [tokens, in] values that a checkpoint stands for."""
    T, n = _checkpoint(q, scale)
    dev = q.device
    X, ldx = _rows_out(X, "X", (T, n), dev, stream)
    _check(_call(dev, _lib.hscale_unpack_activations, q.data_ptr(), scale.data_ptr(), T, n, X.data_ptr(), ldx,
                 _stream(stream, dev)), "hscale_unpack_activations")
    return X


def adapted_linear_grad_workspace_bytes(tokens: int, in_features: int, out_features: int, adapters: int,
                                        rank: int) -> int:
    """Bytes of scratch adapted_linear_grad needs."""
    return _lib.hscale_adapted_linear_grad_workspace_bytes(tokens, in_features, out_features, adapters, rank)


def adapted_linear_grad(dY: torch.Tensor, q: torch.Tensor, scale: torch.Tensor, global_scale: float,
                        scale_codes: torch.Tensor, packed_e2m1: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                        alpha: torch.Tensor | None = None, adapter: torch.Tensor | None = None,
                        dX: torch.Tensor | None = None, dA: torch.Tensor | None = None,
                        dB: torch.Tensor | None = None, need_dX: bool = True, workspace: torch.Tensor | None = None,
                        stream=None):
    """Gradients (dX, dA, dB) of adapted_linear, all bf16, at the checkpoint
    (q, scale) that pack_activations made of its X, from dY bf16 [tokens, out]
    (rows may be strided).  The stored layer is frozen.  need_dX=False skips
    dX (None is returned for it)."""
    lddy = _rows_in(dY, "dY")
    T, m = dY.shape
    dev = dY.device
    if _checkpoint(q, scale)[0] != T or q.device != dev:
        raise ValueError(f"the checkpoint must have dY's {T} tokens, on {dev}")
    n = q.shape[1]
    if _stored(scale_codes, packed_e2m1, n, dev) != m:
        raise ValueError(f"the stored layer must have dY's {m} outputs")
    ad = _adapters(A, B, alpha, adapter, T, n, m, dev)
    if ad is None:
        raise ValueError("A and B are required")
    if not need_dX and dX is not None:
        raise ValueError("dX given although need_dX is False")
    dX, lddx = _rows_out(dX, "dX", (T, n), dev, stream) if need_dX else (None, n)
    dA = _out(dA, "dA", torch.bfloat16, A.shape, dev, stream)
    dB = _out(dB, "dB", torch.bfloat16, B.shape, dev, stream)
    ws_ptr, ws_bytes, held = _workspace(workspace, adapted_linear_grad_workspace_bytes(T, n, m, *ad[:2]), dev, stream)
    _check(_call(dev, _lib.hscale_adapted_linear_grad, dY.data_ptr(), T, m, lddy, q.data_ptr(), scale.data_ptr(), n,
                 float(global_scale), scale_codes.data_ptr(), packed_e2m1.data_ptr(), ad,
                 0 if dX is None else dX.data_ptr(), lddx, dA.data_ptr(), dB.data_ptr(), ws_ptr, ws_bytes,
                 _stream(stream, dev)), "hscale_adapted_linear_grad")
    return dX, dA, dB


def token_loss_workspace_bytes(tokens: int, d: int, vocab: int) -> int:
    """Bytes of scratch token_loss needs."""
    return _lib.hscale_token_loss_workspace_bytes(tokens, d, vocab)


def _head(X, W, target) -> None:
    if not isinstance(W, torch.Tensor) or W.dim() != 2:
        raise ValueError("W must be a 2-D bf16 tensor [vocab, d]")
    _tensor(W, "W", torch.bfloat16, (W.shape[0], X.shape[1]), X.device)
    _tensor(target, "target", torch.int64, (X.shape[0],), X.device)


def token_loss(X: torch.Tensor, W: torch.Tensor, target: torch.Tensor, loss: torch.Tensor | None = None,
               lse: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """Softmax cross entropy of each token over the vocabulary, without the
    logits X W^T in memory: (loss, lse), fp32 [tokens].  X is bf16 [tokens, d]
    (rows may be strided), W bf16 [vocab, d], target int64 [tokens]; a target
    outside 0 .. vocab - 1 is not scored (loss 0).  Tensors that require a
    gradient are refused where torch would record a graph (token_loss_grad
    returns the gradients), and tensors with a tangent where torch would carry
    it on."""
    ldx = _rows_in(X, "X")
    T, d = X.shape
    dev = X.device
    _head(X, W, target)
    _no_graph("token_loss", X, W)
    loss = _out(loss, "loss", torch.float32, (T,), dev, stream)
    lse = _out(lse, "lse", torch.float32, (T,), dev, stream)
    ws_ptr, ws_bytes, held = _workspace(workspace, token_loss_workspace_bytes(T, d, W.shape[0]), dev, stream)
    _check(_call(dev, _lib.hscale_token_loss, X.data_ptr(), T, d, ldx, W.data_ptr(), W.shape[0], target.data_ptr(),
                 loss.data_ptr(), lse.data_ptr(), ws_ptr, ws_bytes, _stream(stream, dev)), "hscale_token_loss")
    return loss, lse


def token_loss_grad_workspace_bytes(tokens: int, d: int, vocab: int) -> int:
    """Bytes of scratch token_loss_grad needs."""
    return _lib.hscale_token_loss_grad_workspace_bytes(tokens, d, vocab)


def token_loss_grad(X: torch.Tensor, W: torch.Tensor, target: torch.Tensor, lse: torch.Tensor, weight: torch.Tensor,
                    dX: torch.Tensor | None = None, dW: torch.Tensor | None = None, need_dX: bool = True,
                    need_dW: bool = True, workspace: torch.Tensor | None = None, stream=None):
    """(dX, dW), bf16, of sum_t weight[t] loss[t], from the lse of token_loss
    on the same X, W and target.  weight is fp32 [tokens] (1 / n for a mean
    over n tokens).  What is not needed is not computed (None)."""
    ldx = _rows_in(X, "X")
    T, d = X.shape
    dev = X.device
    _head(X, W, target)
    _tensor(lse, "lse", torch.float32, (T,), dev)
    _tensor(weight, "weight", torch.float32, (T,), dev)
    if (not need_dX and dX is not None) or (not need_dW and dW is not None):
        raise ValueError("an output was given that is not needed")
    dX, lddx = _rows_out(dX, "dX", (T, d), dev, stream) if need_dX else (None, d)
    dW = _out(dW, "dW", torch.bfloat16, tuple(W.shape), dev, stream) if need_dW else None
    ws_ptr, ws_bytes, held = _workspace(workspace, token_loss_grad_workspace_bytes(T, d, W.shape[0]), dev, stream)
    _check(_call(dev, _lib.hscale_token_loss_grad, X.data_ptr(), T, d, ldx, W.data_ptr(), W.shape[0],
                 target.data_ptr(), lse.data_ptr(), weight.data_ptr(), 0 if dX is None else dX.data_ptr(), lddx,
                 0 if dW is None else dW.data_ptr(), ws_ptr, ws_bytes, _stream(stream, dev)),
           "hscale_token_loss_grad")
    return dX, dW


# ---------------------------------------------------------------------------
# A decode step through stored experts and onto the vocabulary
# ---------------------------------------------------------------------------

_LOGIT_TYPES = {torch.bfloat16: _lib.HSCALE_BF16, torch.float32: _lib.HSCALE_F32}


def _logits(t, name: str) -> tuple[int, int]:
    """t is a 2-D bf16 or fp32 CUDA view with unit column stride; the library's type and its row stride."""
    if not _on_device(t) or (kind := _LOGIT_TYPES.get(t.dtype)) is None or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D bf16 or fp32 CUDA tensor")
    row, col = t.stride()
    rows, cols = t.shape
    if col != 1 and cols > 1:
        raise ValueError(f"{name} must have unit column stride")
    return kind, row if rows > 1 else cols


def route_tokens(logits: torch.Tensor, k: int, normalize: bool = True, expert: torch.Tensor | None = None,
                 weight: torch.Tensor | None = None, stream=None):
    """(expert int32 [tokens, k], weight fp32 [tokens, k]) of a router's logits,
    bf16 or fp32 [tokens, experts] (rows may be strided): the k largest, the
    lowest number first where they are equal, and their shares of the softmax
    of the k (normalize) or of all experts.

    A logit of -inf or NaN is never chosen; a token with fewer than k others
    gets -1 and weight 0 for the rest.  NaN or +inf among a token's logits make
    its weights NaN.  No graph is recorded: tensors that require a gradient are
    refused where torch would record one, and tensors with a tangent where torch
    would carry it on.
    """
    kind, ld = _logits(logits, "logits")
    T, E = logits.shape
    dev = logits.device
    _no_graph("route_tokens", logits, weight, grad=False)
    k = int(k)
    if not 1 <= k <= E:
        raise ValueError(f"k must be in 1 .. {E}, the number of experts")
    expert = _out(expert, "expert", torch.int32, (T, k), dev, stream)
    weight = _out(weight, "weight", torch.float32, (T, k), dev, stream)
    _check(_call(dev, _lib.hscale_route_tokens, logits.data_ptr(), kind, T, E, ld, k, int(bool(normalize)),
                 expert.data_ptr(), weight.data_ptr(), _stream(stream, dev)), "hscale_route_tokens")
    return expert, weight


def _expert_matrix(matrix, name: str, device, E: int, m: int, n: int) -> tuple[torch.Tensor, tuple[int, int, int]]:
    """The checked (global_scale, scale_codes, packed_e2m1) of E matrices of m x n: the scales, and the addresses."""
    try:
        scale, codes, packed = matrix
        # One pass over what must hold: a call has nine of these tensors, and a token's time for them.
        if (packed.dtype is torch.uint8 and codes.dtype is torch.uint8 and scale.dtype is torch.float32
                and packed.shape == (E, m, n // 2) and codes.shape == (E, m, n // 16) and scale.shape == (E,)
                and packed.device == device and codes.device == device and scale.device == device
                and packed.is_contiguous() and codes.is_contiguous() and scale.is_contiguous()):
            return scale, (scale.data_ptr(), codes.data_ptr(), packed.data_ptr())
    except (TypeError, ValueError, AttributeError):
        raise ValueError(f"{name} must be three tensors (global_scale, scale_codes, packed_e2m1)") from None
    raise ValueError(f"{name} must be contiguous (global_scale fp32 [{E}], scale_codes uint8 [{E}, {m}, {n // 16}], "
                     f"packed_e2m1 uint8 [{E}, {m}, {n // 2}]) on {device}")


def expert_layer_workspace_bytes(tokens: int, in_features: int, hidden: int, experts: int, k: int) -> int:
    """Bytes of scratch expert_layer needs."""
    return _lib.hscale_expert_layer_workspace_bytes(tokens, in_features, hidden, experts, k)


def expert_layer(X: torch.Tensor, expert: torch.Tensor, weight: torch.Tensor, gate, up, down,
                 Y: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y[t] = sum_j weight[t, j] D_e (silu(G_e X[t]) * (U_e X[t])), e = expert[t, j]:
    a gated layer of experts stored in NVFP4, for the tokens of a decode step or
    a chunk of a prompt.

    X is bf16 [tokens, in] (rows may be strided, 16-byte aligned), expert int32
    and weight fp32 [tokens, k] as route_tokens returns them; a number outside
    0 .. experts - 1 means no expert.  gate, up (hidden x in) and down
    (in x hidden) are each (global_scale fp32 [experts], scale_codes uint8
    [experts, out, in / 16], packed_e2m1 uint8 [experts, out, in / 2]): what
    search writes of each expert, stacked.  Y is bf16 [tokens, in] (rows may be
    strided).

    The stored experts are frozen and no graph is recorded: tensors that require
    a gradient, the experts' scales among them, are refused where torch would
    record one, and tensors with a tangent where torch would carry it on.
    """
    ldx = _rows_in(X, "X")
    T, n = X.shape
    dev = X.device
    if not isinstance(expert, torch.Tensor) or expert.dim() != 2:
        raise ValueError("expert must be a 2-D int32 tensor [tokens, k]")
    k = expert.shape[1]
    _tensor(expert, "expert", torch.int32, (T, k), dev)
    _tensor(weight, "weight", torch.float32, (T, k), dev)
    if not isinstance(gate, (tuple, list)) or len(gate) != 3 or not isinstance(gate[2], torch.Tensor) or gate[2].dim() != 3:
        raise ValueError("gate must be (global_scale, scale_codes, packed_e2m1), the last uint8 [experts, hidden, in / 2]")
    E, hidden, _ = gate[2].shape
    gate_scale, gate = _expert_matrix(gate, "gate", dev, E, hidden, n)
    up_scale, up = _expert_matrix(up, "up", dev, E, hidden, n)
    down_scale, down = _expert_matrix(down, "down", dev, E, n, hidden)
    _no_graph("expert_layer", X, weight, gate_scale, up_scale, down_scale, Y, grad=False)
    Y, ldy = _rows_out(Y, "Y", (T, n), dev, stream)
    need = expert_layer_workspace_bytes(T, n, hidden, E, k)
    ws_ptr, ws_bytes, held = _workspace(workspace, need, dev, stream)
    _check(_call(dev, _lib.hscale_expert_layer, X.data_ptr(), T, n, ldx, hidden, E, gate, up, down,
                 expert.data_ptr(), weight.data_ptr(), k, Y.data_ptr(), ldy, ws_ptr, ws_bytes,
                 _stream(stream, dev)), "hscale_expert_layer")
    return Y


def _each_row(t, name: str, dtype, rows: int, device) -> int:
    """The checked address of one number a row, 0 for None."""
    if t is None:
        return 0
    return _tensor(t, name, dtype, (rows,), device).data_ptr()


def _rows_of(t, row, name: str, dtype, width: int, rows: int, device) -> tuple[int, int, int]:
    """How many biases or masks [count, width] there are, and the checked
    addresses of them and of each row's number."""
    if t is None:
        if row is not None:
            raise ValueError(f"{name}_row needs {name}")
        return 0, 0, 0
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D {dtype} tensor")
    count = t.shape[0]
    _tensor(t, name, dtype, (count, width), device)
    if row is None and count != 1:
        raise ValueError(f"{name}_row (int32, one number a row) is required unless there is exactly one {name}")
    return count, t.data_ptr(), _each_row(row, f"{name}_row", torch.int32, rows, device)


def adjust_logits(logits: torch.Tensor, history: torch.Tensor | None = None, length: torch.Tensor | None = None,
                  prompt: torch.Tensor | None = None, repetition: torch.Tensor | None = None,
                  frequency: torch.Tensor | None = None, presence: torch.Tensor | None = None,
                  bias: torch.Tensor | None = None, bias_row: torch.Tensor | None = None,
                  mask: torch.Tensor | None = None, mask_row: torch.Tensor | None = None,
                  out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Logits, bf16 or fp32 [rows, vocab] (rows may be strided), with each row's
    penalties for repeated words, its bias and its mask, in this order:

        l > 0 ? l * (1 / repetition) : l * repetition   of words in the history
        l - frequency * count - presence          of words in the answer, said count times
        l + bias[v],  -inf where the mask's bit is clear

    history is int32 [rows, any length] (rows may be strided), of which the first
    length[row] words count (all when None) and the first prompt[row] of those
    are the prompt's, the rest the answer's (all when None); words outside the
    vocabulary are passed over.  repetition (normal, > 0), frequency and presence
    are fp32 [rows].  bias is fp32 [biases, vocab], mask int32 [masks,
    ceil(vocab / 32)] whose bit v % 32 of number v / 32 allows word v; bias_row
    and mask_row (int32 [rows]) say which row uses which, any number outside
    for none; with exactly one they may be None: all rows use it.

    Returns `out`, new when None; out=logits works in place.  No graph is
    recorded: tensors that require a gradient are refused where torch would
    record one, and tensors with a tangent where torch would carry it on.
    """
    kind, ld = _logits(logits, "logits")
    R, V = logits.shape
    dev = logits.device
    _no_graph("adjust_logits", logits, repetition, frequency, presence, bias, out, grad=False)
    if history is None and not (length is None and prompt is None and repetition is None and frequency is None
                                and presence is None):
        raise ValueError("repetition, frequency, presence, length and prompt need a history")
    words = ldh = at_history = 0
    if history is not None:
        if not isinstance(history, torch.Tensor) or history.dim() != 2:
            raise ValueError("history must be a 2-D int32 tensor [rows, length]")
        words = history.shape[1]
        ldh = _row_view(history, torch.int32, (R, words), dev, "history")
        at_history = history.data_ptr()
    biases, at_bias, at_bias_row = _rows_of(bias, bias_row, "bias", torch.float32, V, R, dev)
    masks, at_mask, at_mask_row = _rows_of(mask, mask_row, "mask", torch.int32, -(-V // 32), R, dev)
    rules = (at_history, words, ldh, _each_row(length, "length", torch.int32, R, dev),
             _each_row(prompt, "prompt", torch.int32, R, dev), _each_row(repetition, "repetition", torch.float32, R, dev),
             _each_row(frequency, "frequency", torch.float32, R, dev),
             _each_row(presence, "presence", torch.float32, R, dev), at_bias, biases, at_bias_row, at_mask, masks,
             at_mask_row)
    if out is None:
        out, ldo = _new((R, V), logits.dtype, dev, stream), V
    else:
        ldo = _row_view(out, logits.dtype, (R, V), dev, "out")
    _check(_call(dev, _lib.hscale_adjust_logits, rules, logits.data_ptr(), kind, R, V, ld, out.data_ptr(), ldo,
                 _stream(stream, dev)), "hscale_adjust_logits")
    return out
