"""AQDecoderBlock: one decoder block served at any prefix m, for one new token per sequence.

The seven projections are AQLinear layers (additive codebooks, App. C); between them run the RMS
norms, the paged key-value cache and the attention of libaq. The rotary embedding and the gate's
activation are elementwise torch operations.
"""
import torch

from .linear import gemv_group
from .norm import rmsnorm


def rope_angles(positions, head_dim, theta=500000.0):
    """(cos, sin), each [n][1][head_dim / 2] in fp32, of int positions [n]."""
    inv = theta ** (-torch.arange(0, head_dim, 2, device=positions.device, dtype=torch.float64) / head_dim)
    a = (positions.double()[:, None] * inv)[:, None]
    return a.cos().float(), a.sin().float()


def _rotate(x, rope):
    # Pairs (i, i + head_dim / 2), in fp32, rounded once.
    cos, sin = rope
    a, b = x.float().chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)


class AQDecoderBlock:
    """layers: a dict of AQLinear, "q", "k", "v", "o", "gate", "up" and "down"; attn_norm, mlp_norm:
    the norms' weights ([hidden]); layer: this block's layer of the cache."""

    def __init__(self, layers, attn_norm, mlp_norm, q_heads, kv_heads, layer=0, eps=1e-5):
        self.p, self.attn_norm, self.mlp_norm = layers, attn_norm, mlp_norm
        self.q_heads, self.kv_heads, self.layer, self.eps = q_heads, kv_heads, layer, eps

    def _products(self, names, x, m):
        lins = [self.p[n] for n in names]
        return gemv_group(lins, x, m) if x.shape[0] <= 16 else [lin(x, m) for lin in lins]

    def step(self, x, residual, m, cache, seqs, rope):
        """x: [n][hidden], what the block before added to the residual stream; residual: the stream
        before that ([n][hidden]), or None at the first block (x is then the embedding). The new
        token's slot must be reserved (cache.reserve(seqs), once for all blocks); rope:
        rope_angles of the tokens' positions. Returns (this block's addition, the stream before
        it): the stream itself is their sum, which the next norm takes."""
        n = x.shape[0]
        y, h = rmsnorm(x, self.attn_norm, self.eps, residual=residual)
        residual = x if residual is None else h
        q, k, v = self._products(("q", "k", "v"), y, m)
        q = _rotate(q.view(n, self.q_heads, -1), rope)
        k = _rotate(k.view(n, self.kv_heads, -1), rope)
        cache.write(k, v.view(n, self.kv_heads, -1), seqs, layer=self.layer)
        a = cache.attend(q, seqs, layer=self.layer)
        o = self.p["o"](a.view(n, -1), m)
        y, residual = rmsnorm(o, self.mlp_norm, self.eps, residual=residual)
        g, u = self._products(("gate", "up"), y, m)
        return self.p["down"](torch.nn.functional.silu(g) * u, m), residual
