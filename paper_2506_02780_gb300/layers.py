"""A target layer's weight products, as a server keeps them beside the cache.

A verification pass (EfficientEdit, arXiv 2506.02780, Sec. III-A) runs every layer of
the target model over a draft's tokens.  The attention's side of a layer is
``VerifyStep``'s and ``PromptIntake``'s; these are its projections and feed-forward
layers, whose time is the stream of their weights:

    BlockLinear   ee_fp8_quantize -> ee_fp8_linear    y = x W^T (+ bias), W in e4m3 blocks
    Experts       ee_moe_layer                        a mixture-of-experts layer

Each owns its weights' codes and scales (made once, at load), its scratch and its
workspace.  Calls enqueue kernels on one stream and allocate nothing, so a layer can
be captured into a CUDA graph; what they return is valid until the object's next call.
Calls of one object must be ordered on one stream.
"""
from __future__ import annotations

import torch

from . import (EE_BLOCK, ee_fp8_linear, ee_fp8_quantize, ee_fp8_quantize_weights, ee_moe_layer, ee_read_errors,
               new_linear_workspace, new_moe_workspace)


def _blocks(n):
    return -(-n // EE_BLOCK)


def quantize_weights(w, stream=None):
    """(codes, scales) of bf16 weights [..., rows, cols]: float8_e4m3fn of w's shape and
    float32 [..., ceil(rows / 128), ceil(cols / 128)]."""
    *lead, rows, cols = w.shape
    q = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device=w.device)
    scale = torch.empty((*lead, _blocks(rows), _blocks(cols)), dtype=torch.float32, device=w.device)
    ee_fp8_quantize_weights(w, q, scale, stream=stream)
    return q, scale


class BlockLinear:
    """y = x W^T (+ bias) with W [N, K] in 8 bits: bf16 weights, quantised here, or codes with
    their ``scale`` [ceil(N / 128), ceil(K / 128)].  max_tokens: rows of one call at most."""

    def __init__(self, weight, bias=None, *, scale=None, max_tokens):
        if weight.dim() != 2:
            raise ValueError("weight must be [N, K]")
        if (scale is None) != (weight.dtype is torch.bfloat16):
            raise ValueError("codes come with their scale, bf16 weights without one")
        self.N, self.K = weight.shape
        self.w, self.w_scale = quantize_weights(weight) if scale is None else (weight, scale)
        self.bias = bias
        n, dev = int(max_tokens), weight.device
        self._q = torch.empty(n * self.K, dtype=torch.float8_e4m3fn, device=dev)
        self._scale = torch.empty(n * _blocks(self.K), dtype=torch.float32, device=dev)
        self._out = torch.empty((n, self.N), dtype=torch.bfloat16, device=dev)
        self.ws = new_linear_workspace(device=dev)

    def __call__(self, x, gated=False, out=None, stream=None):
        """x bf16 [n, K], or with ``gated`` [n, 2 K]: silu of the first half times the second goes
        in.  Returns bf16 [n, N] (``out``, if given: rows may be views of wider ones)."""
        n = x.shape[0]
        if n > self._out.shape[0]:
            raise ValueError(f"at most {self._out.shape[0]} tokens")
        q, scale = self._q[:n * self.K].view(n, self.K), self._scale[:n * _blocks(self.K)].view(_blocks(self.K), n)
        out = self._out[:n] if out is None else out
        if n:
            ee_fp8_quantize(x, q, scale, gated=gated, stream=stream)
            ee_fp8_linear(q, scale, self.w, self.w_scale, out, self.ws, bias=self.bias, stream=stream)
        return out

    def errors(self, stream=None):
        """Synchronise, return and clear the device error word (0 = none)."""
        return ee_read_errors(self.ws, stream=stream)


class Experts:
    """A mixture-of-experts layer (``ee_moe_layer``): router bf16 [E, H], w1 [E, 2 I, H] (gate rows, then up
    rows) and w2 [E, H, I], bf16 or codes with their scales; ``quantize``: bf16 weights are
    quantised here.  After a call ``ids`` and ``probs`` [n, k] hold each token's experts."""

    def __init__(self, router, w1, w2, k, *, renorm=True, w1_scale=None, w2_scale=None, quantize=False, max_tokens):
        if w1.dim() != 3 or w2.dim() != 3 or w1.shape[0] != w2.shape[0] or w1.shape[1:] != (2 * w2.shape[2], w2.shape[1]):
            raise ValueError("w1 must be [E, 2 I, H] and w2 [E, H, I]")
        self.E, self.H, self.I = w2.shape
        self.k, self.renorm = int(k), bool(renorm)
        if router.shape != (self.E, self.H):
            raise ValueError("router must be [E, H]")
        n, dev = int(max_tokens), w1.device
        self.ws = new_moe_workspace(n, self.H, self.I, self.E, self.k, device=dev)   # (refuses sizes that a call would)
        if quantize:
            if w1_scale is not None or w2_scale is not None:
                raise ValueError("quantize takes bf16 weights without scales")
            w1, w1_scale = quantize_weights(w1.view(self.E, 2, self.I, self.H))
            w1 = w1.view(self.E, 2 * self.I, self.H)
            w2, w2_scale = quantize_weights(w2)
        self.router, self.w1, self.w2, self.w1_scale, self.w2_scale = router, w1, w2, w1_scale, w2_scale
        self._out = torch.empty((n, self.H), dtype=torch.bfloat16, device=dev)
        self._ids = torch.empty(n * self.k, dtype=torch.int32, device=dev)
        self._probs = torch.empty(n * self.k, dtype=torch.float32, device=dev)

    def __call__(self, x, live=None, out=None, stream=None):
        """x bf16 [n, H]; live (device int32 [1]): only its first tokens are computed, what is behind them
        stays.  Returns bf16 [n, H] (``out``, if given: rows may be views of wider ones)."""
        n = x.shape[0]
        if n > self._out.shape[0]:
            raise ValueError(f"at most {self._out.shape[0]} tokens")
        out = self._out[:n] if out is None else out
        self.ids, self.probs = self._ids[:n * self.k].view(n, self.k), self._probs[:n * self.k].view(n, self.k)
        if n:
            ee_moe_layer(x, self.router, self.w1, self.w2, self.k, out, self.ws, w1_scale=self.w1_scale,
                         w2_scale=self.w2_scale, renorm=self.renorm, live=live, ids=self.ids, probs=self.probs,
                         stream=stream)
        return out

    def errors(self, stream=None):
        """Synchronise, return and clear the device error word (0 = none)."""
        return ee_read_errors(self.ws, stream=stream)
