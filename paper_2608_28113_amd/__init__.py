"""MI355X (gfx950) implementation of the H-Scale hot path.

H-Scale refines NVFP4 per-group scales with a diagonal second-order proxy:
``hdiag`` computes h = diag(X^T X) from calibration activations and
``search`` picks, for every 16-weight group, the E4M3 scale among a window of
neighbours of the max-abs scale that minimises the h-weighted reconstruction
error, returning NVFP4 scale bytes and packed E2M1 codes.

The stored layer is then served and trained through: ``adapted_linear``
applies it to the tokens of many requests, each with a low-rank adapter of its
own or none; ``pack_activations`` keeps its input in 8 bits for the backward
pass, ``token_loss`` and ``token_loss_grad`` are the cross entropy over a large
vocabulary and its gradient without stored logits, and ``adapted_linear_grad``
returns the gradients of the adapters and of the layer's input.

Layers of stored experts are served by ``route_tokens`` (the router's choice)
and ``expert_layer`` (the experts' products, for the tokens of a decode step or
a chunk of a prompt), and ``adjust_logits`` applies a request's penalties,
biases and masks to the logits before a token is chosen.

The compute is in ``libhscale.so`` (hand-written HIP, C ABI in
``include/hscale.h``); this package is its thin Python binding.
"""
from ._lib import HScaleError, EXPORTS  # noqa: F401
from .ops import (hdiag, hdiag_accumulate, hdiag_finalize, hdiag_noalloc, hdiag_workspace_bytes, quantize,  # noqa: F401
                  output_error, output_error_workspace_bytes, search, search_block, search_layers, search_stats,
                  shift_summary, adapted_linear, adapted_linear_workspace_bytes, adapted_linear_grad,
                  adapted_linear_grad_workspace_bytes, pack_activations, unpack_activations, token_loss,
                  token_loss_workspace_bytes, token_loss_grad, token_loss_grad_workspace_bytes, route_tokens,
                  expert_layer, expert_layer_workspace_bytes, adjust_logits)
