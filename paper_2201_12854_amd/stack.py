"""A stack of MCA attention layers with synthetic weights: how the estimate's error grows
with depth (Sec. "Integration with Compressed Transformers": MCA's error accumulates over
attention layers, so a 6-layer model loses less than a 12-layer one) and how it behaves
with 16-bit weights (Sec. "Performance-Accuracy Trade-off", the quantised models).

Each layer l maps hidden states h [B, n, d] to LayerNorm(h + Y_l) with
Y_l = MCA(Q = h W_q, K = h W_k, X = h, W_v) through libmca; the projections, the residual
and the normalisation are plain torch operations around the library call (model wiring,
not part of the attention path). The exact stack runs the same layers in the paper's
regular mode (every token's count set to d_in, so H~ = X W_v exactly). Weights are drawn
N(0, 0.02^2) per layer from a seed; the layer-norm has no learned scale or shift.

``exact_forward`` and ``gradients`` are the same stack with the attention that MCA approximates
(``exact_attention_forward`` and ``exact_attention_backward`` on V = h W_v, instead of H~ through the
estimator's kernels), as it is trained before MCA serves its weights; there the layers may share a
learned relative position bias, which the estimator's count rule has no term for.
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

from . import binding


@dataclass
class StackLayer:
    Wq: object
    Wk: object
    Wv: object
    prepared: object


class SyntheticEncoder:
    """L attention layers of width d with H heads of 64, weights N(0, 0.02^2), in
    float32 or bfloat16, on one device."""

    def __init__(self, layers: int, d: int, heads: int, dtype: str = "bf16", seed: int = 0, device="cuda:0", *,
                 relative_buckets: int = 0, max_distance: int = 128):
        import torch

        if heads * 64 != d:
            raise ValueError("d must equal heads * 64")
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.d, self.heads = d, heads
        self.device = torch.device(device)
        rng = np.random.default_rng(seed)
        self.layers = []
        for _ in range(layers):
            W = [torch.from_numpy((0.02 * rng.standard_normal((d, d))).astype(np.float32)).to(self.device)
                 .to(self.dtype).contiguous() for _ in range(3)]
            self.layers.append(StackLayer(W[0], W[1], W[2], binding.prepare_weights(W[2])))
        self.bias = None
        if relative_buckets:
            table = torch.from_numpy(rng.standard_normal((relative_buckets, heads)).astype(np.float32))
            self.bias = binding.RelativeBias(table.to(self.device).to(self.dtype).contiguous(), max_distance)

    def layer_inputs(self, h, l: int):
        """Q = h W_q and K = h W_k of layer l (torch matmul in the stack's dtype)."""
        B, n, d = h.shape
        L = self.layers[l]
        q = (h.reshape(B * n, d) @ L.Wq).reshape(B, n, d).contiguous()
        k = (h.reshape(B * n, d) @ L.Wk).reshape(B, n, d).contiguous()
        return q, k

    def forward(self, x, seq_lens, alpha: float, seed: int = 0, *, exact: bool = False, keep: bool = False,
                sampling: str = "token", window: int = 0):
        """Runs the stack on x [B, n, d] (the stack's dtype). Layer l draws with seed + l.
        ``exact``: regular mode (r_j = d_in for every token). Returns the final hidden
        states, or the list of every layer's output when ``keep``."""
        import torch

        if self.bias is not None:
            raise ValueError("MCA has no relative bias: run exact_forward")
        B, n, d = x.shape
        h = x.contiguous()
        r_full = torch.full((B, n), d, dtype=torch.int32, device=x.device) if exact else None
        outs = []
        for l, L in enumerate(self.layers):
            q, k = self.layer_inputs(h, l)
            res = binding.attention_forward(q, k, h, L.Wv, L.prepared, alpha, seed + l, heads=self.heads,
                                            seq_lens=seq_lens, r_in=r_full, sampling=sampling, window=window)
            y = torch.nn.functional.layer_norm(h.float() + res.Y, (d,))
            h = y.to(self.dtype).contiguous()
            if keep:
                outs.append(h)
        return outs if keep else h

    def _exact_layer(self, h, l: int, seq_lens, window: int):
        """Layer l with exact attention: its inputs, results and the sum that is normalised."""
        import torch

        B, n, d = h.shape
        q, k = self.layer_inputs(h, l)
        v = (h.reshape(B * n, d) @ self.layers[l].Wv).reshape(B, n, d).contiguous()
        kw = dict(heads=self.heads, q_lens=seq_lens, kv_lens=seq_lens, window=window, bias=self.bias)
        a = binding.exact_attention_forward(q, k, v, **kw)
        z = h.float() + a.Y.float()
        return (h, q, k, v, a, z, kw), torch.nn.functional.layer_norm(z, (d,)).to(self.dtype).contiguous()

    def exact_forward(self, x, seq_lens=None, *, window: int = 0):
        """Final hidden states of the stack with exact attention (padded rows attend nothing: their Y
        is 0). seq_lens: int32 [B] or None."""
        h = x.contiguous()
        for l in range(len(self.layers)):
            _, h = self._exact_layer(h, l, seq_lens, window)
        return h

    def gradients(self, x, d_out, seq_lens=None, *, window: int = 0) -> dict:
        """Gradients of sum(d_out * exact_forward(x)) in float32: "x", per layer "Wq", "Wk", "Wv" (lists),
        and "bias" of the shared table (None without one). Rounding to the stack's type counts as the
        identity."""
        B, n, d = x.shape
        h, saved = x.contiguous(), []
        for l in range(len(self.layers)):
            s, h = self._exact_layer(h, l, seq_lens, window)
            saved.append(s)
        g = d_out.float()
        out = {"Wq": [], "Wk": [], "Wv": [], "bias": None}
        for L, (h, q, k, v, a, z, kw) in zip(reversed(self.layers), reversed(saved)):
            # layer norm: t = (z - mean) / s
            z = z - z.mean(-1, keepdim=True)
            s = (z.square().mean(-1, keepdim=True) + 1e-5).sqrt()
            t = z / s
            g = (g - g.mean(-1, keepdim=True) - t * (g * t).mean(-1, keepdim=True)) / s
            a = binding.exact_attention_backward(g.to(self.dtype).contiguous(), q, k, v, a.Y, a.lse, **kw)
            hf = h.reshape(B * n, d).float()
            for name, dy, W in (("Wq", a.dQ, L.Wq), ("Wk", a.dK, L.Wk), ("Wv", a.dV, L.Wv)):
                dy = dy.reshape(B * n, d).float()
                out[name].insert(0, hf.t() @ dy)
                g = g + (dy @ W.float().t()).reshape(B, n, d)
            if self.bias is not None:
                out["bias"] = a.dbias.float() if out["bias"] is None else out["bias"] + a.dbias.float()
        out["x"] = g
        return out


def depth_error(enc: SyntheticEncoder, x, seq_lens, alpha: float, seeds, **kw):
    """Mean over seeds of the relative Frobenius error of every layer's output (valid rows
    only) of the MCA stack against the exact stack, and the exact stack's outputs."""
    import torch

    exact = enc.forward(x, seq_lens, alpha, 0, exact=True, keep=True, **kw)
    B, n, d = x.shape
    mask = (torch.arange(n, device=x.device)[None, :] < seq_lens[:, None]).float()[..., None]
    errs = np.zeros(len(enc.layers))
    for s in seeds:
        outs = enc.forward(x, seq_lens, alpha, s, keep=True, **kw)
        for l, (a, e) in enumerate(zip(outs, exact)):
            diff = ((a.float() - e.float()) * mask).norm().item()
            errs[l] += diff / max((e.float() * mask).norm().item(), 1e-30) / len(seeds)
    return errs
