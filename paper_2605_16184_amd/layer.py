"""One LLaMA-style decoder layer, forward and backward, as a source of weight gradients: the matrices of
``workloads.llama_1b_matrices`` get the gradients of a layer that has run on packed sequences, in place of random matrices of
their spectrum.  Norm, dropout and attention are the library's operators; the plain products go to torch.

    r -> norm -> q, k, v -> causal attention -> o -> dropout -> + r = H -> norm -> gate, up -> silu(gate) up -> down -> dropout -> + H

Order enters by the causal mask alone (no rotary positions).  Nothing of the optimizer lives here.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Tuple

import torch

from . import binding as B
from . import workloads as W


class DecoderLayer:
    """Weights (out x in, as stored) and the buffers of one layer for a fixed number of rows.

    ``dropout``: probability before each residual addition; the masks follow (seed, offset) and the step, which the caller passes
    to ``forward`` and which ``backward`` reuses.  All matrices and activations have ``dtype``; the residual stream is fp32."""

    MATRICES = ("q", "k", "v", "o", "gate", "up", "down")

    def __init__(self, rows: int, d: int = 2048, heads: int = 32, kv_heads: int = 4, ffn: int = 5632, dtype=torch.bfloat16,
                 device="cuda", dropout: float = 0.0, seed: int = 0, eps: float = 1e-6):
        if d % heads or heads % kv_heads:
            raise ValueError("d must be a multiple of heads, heads of kv_heads")
        self.rows, self.d, self.heads, self.kv_heads, self.ffn = rows, d, heads, kv_heads, ffn
        self.dim, self.dtype, self.eps, self.dropout, self.seed = d // heads, dtype, eps, dropout, seed
        kv = kv_heads * self.dim
        g = W._gen(device, 5, d, ffn, seed)

        def matrix(m, n):
            return (torch.randn(m, n, generator=g, device=device) * n ** -0.5).to(dtype)

        # q, k and v are one matrix, so that one product leaves them side by side, as attention reads them
        self.qkv, self.o = matrix(d + 2 * kv, d), matrix(d, d)
        self.gate_up, self.down = matrix(2 * ffn, d), matrix(d, ffn)
        self.norm1, self.norm2 = (torch.ones(d, dtype=dtype, device=device) for _ in range(2))

        def rows_of(*shape, dtype=dtype):
            return torch.zeros(rows, *shape, dtype=dtype, device=device)

        self.y1, self.y2, self.H = rows_of(d), rows_of(d), rows_of(d, dtype=torch.float32)
        self.O, self.lse = rows_of(heads, self.dim), torch.zeros(heads, rows, device=device)
        self.dqkv = rows_of(heads + 2 * kv_heads, self.dim)
        self.ws = None
        self._saved = None

    def _split(self, qkv):
        h, k = self.heads, self.kv_heads
        return qkv[:, :h], qkv[:, h:h + k], qkv[:, h + k:]

    def forward(self, r: torch.Tensor, cu: Optional[torch.Tensor] = None, step: int = 0) -> torch.Tensor:
        """The residual stream behind the layer (fp32, rows x d) from the one before it; ``cu`` as in ``attention``.  Rows of no
        sequence attend to nothing."""
        p, seed = self.dropout, self.seed
        B.rms_norm(r, self.y1, W=self.norm1, eps=self.eps)
        qkv = (self.y1 @ self.qkv.T).view(self.rows, self.heads + 2 * self.kv_heads, self.dim)
        if cu is not None:
            self.O.zero_()                         # rows of no sequence
        B.attention(*self._split(qkv), self.O, lse=self.lse, cu=cu)
        a = self.O.view(self.rows, self.d) @ self.o.T
        B.rms_norm(a, self.y2, W=self.norm2, R=r, H=self.H, eps=self.eps, p=p, seed=seed, offset=2 * step)
        gu = self.y2 @ self.gate_up.T
        gate, up = gu[:, :self.ffn].float(), gu[:, self.ffn:].float()
        s = (gate * torch.sigmoid(gate) * up).to(self.dtype)
        f = s @ self.down.T
        if p:
            B.dropout(f, f, p, seed=seed, offset=2 * step + 1)
        self._saved = (r, cu, step, qkv, gu, s)
        return self.H + f

    def backward(self, dout: torch.Tensor) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
        """(gradient of the residual stream before the layer, gradients of the matrices and norm weights by name) for the last
        ``forward``; dout: fp32, rows x d."""
        r, cu, step, qkv, gu, s = self._saved
        p, seed, ffn, rows, d = self.dropout, self.seed, self.ffn, self.rows, self.d
        df = dout.to(self.dtype, copy=True)
        if p:
            B.dropout(df, df, p, seed=seed, offset=2 * step + 1)
        ds = (df @ self.down).float()
        gate, up = gu[:, :ffn].float(), gu[:, ffn:].float()
        sg = torch.sigmoid(gate)
        dgu = torch.cat([ds * up * sg * (1 + gate * (1 - sg)), ds * gate * sg], 1).to(self.dtype)
        dy2 = dgu @ self.gate_up
        da, dH, dnorm2 = torch.empty_like(dy2), torch.empty_like(dout), torch.empty_like(self.norm2)
        B.rms_norm_backward(self.H, dy2, W=self.norm2, dH=dout, dX=da, dR=dH, dW=dnorm2, eps=self.eps, p=p, seed=seed, offset=2 * step)
        dO = (da @ self.o).view(rows, self.heads, self.dim)
        q, k, v = self._split(qkv)
        need = B.attention_backward_workspace_bytes(q, k, v, self.O, self.lse, cu)
        if self.ws is None or self.ws.numel() < need:       # fewer sequences may take more
            self.ws = torch.empty(need, dtype=torch.uint8, device=dout.device)
        if cu is not None:
            self.dqkv.zero_()
        B.attention_backward(q, k, v, self.O, self.lse, dO, *self._split(self.dqkv), cu=cu, ws=self.ws)
        dqkv = self.dqkv.view(rows, -1)
        dy1, dr, dnorm1 = dqkv @ self.qkv, torch.empty_like(dout), torch.empty_like(self.norm1)
        B.rms_norm_backward(r, dy1, W=self.norm1, dH=dH, dR=dr, dW=dnorm1, eps=self.eps)
        gqkv, ggu = dqkv.T @ self.y1, dgu.T @ self.y2
        kv = self.kv_heads * self.dim
        grads = {"q": gqkv[:d], "k": gqkv[d:d + kv], "v": gqkv[d + kv:], "o": da.T @ self.O.view(rows, d), "gate": ggu[:ffn], "up": ggu[ffn:],
                 "down": df.T @ s, "norm1": dnorm1, "norm2": dnorm2}
        return dr, grads


def gradient_blocks(grads: Dict[str, torch.Tensor], cap: int = 1024) -> List[torch.Tensor]:
    """The matrices' gradients cut into blocks of at most cap x cap (views), in the order of ``workloads.block_shapes``: what
    ``stats_update`` and ``precondition`` take as G."""
    out = []
    for name in DecoderLayer.MATRICES:
        G = grads[name]
        at = 0
        for m in W.split_dim(G.shape[0], cap):
            col = 0
            for n in W.split_dim(G.shape[1], cap):
                out.append(G[at:at + m, col:col + n])
                col += n
            at += m
    return out
