"""Shared pieces of the tests of trees and eviction: random trees, a pool without a model's weights, plain forms in 64 bits."""
from __future__ import annotations

import contextlib
import math

import numpy as np
import torch

from paper_2506_09397_amd import sled, synth

BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


def random_tree(rng, n, kind="mixed"):
    """parent[j] of n nodes (parent[0] = -1)."""
    if kind == "chain":
        return [-1] + list(range(n - 1))
    if kind == "star":
        return [-1] + [0] * (n - 1)
    p = [-1]
    for j in range(1, n):
        p.append(int(rng.integers(max(0, j - 3), j)) if rng.random() < 0.6 else int(rng.integers(0, j)))
    return p


def depths(parent):
    d = [0]
    for j in range(1, len(parent)):
        d.append(d[parent[j]] + 1)
    return d


def ancestors(parent, j):
    """j and its ancestors, root first."""
    out = [j]
    while out[-1] != 0:
        out.append(parent[out[-1]])
    return out[::-1]


def seen_matrix(parent):
    n = len(parent)
    m = np.zeros((n, n), dtype=bool)
    for j in range(n):
        m[j, ancestors(parent, j)] = True
    return torch.from_numpy(m)


class Pool:
    """A pool of `layers` layers with the given heads; the model behind it holds no weights worth mentioning."""

    def __init__(self, hq, hkv, D, dtype, layers=1, n_pages=256, max_requests=16, invariant=False):
        self.shape = synth.ModelShape(layers, 256, hq, hkv, D, 256, 1024, dtype, 10000.0, k_max=min(8, max(0, 80 // (hq // hkv) - 1)))
        self.model = sled.sled_model_create(self.shape)
        if invariant:
            sled.sled_model_set_batch_invariant(self.model, True)
        self.pool = sled.sled_kvpool_create(self.model, n_pages, max_requests)
        self.dt = self.shape.torch_dtype

    def open(self, L, g, scale=1.0):
        """A request with L random context tokens; returns (id, K, V)."""
        s = self.shape
        r = sled.sled_kvpool_open(self.pool)
        K = (scale * torch.randn(s.n_layers, L, s.n_kv_heads, s.head_dim, generator=g, device="cuda")).to(self.dt)
        V = torch.randn(s.n_layers, L, s.n_kv_heads, s.head_dim, generator=g, device="cuda").to(self.dt)
        if L:
            sled.sled_kv_append(self.pool, [r], [L], [K], [V])
        return r, K, V

    def read(self, r, first, n):
        s = self.shape
        K = torch.empty(s.n_layers, n, s.n_kv_heads, s.head_dim, dtype=self.dt, device="cuda")
        V = torch.empty_like(K)
        sled.sled_kv_read(self.pool, r, first, n, K, V)
        return K, V

    def workspace(self, B, T, ctx):
        return sled.workspace(sled.sled_tree_workspace_bytes(self.model, B, T, ctx))

    def destroy(self):
        torch.cuda.synchronize()
        sled.sled_kvpool_destroy(self.pool)
        sled.sled_model_destroy(self.model)


@contextlib.contextmanager
def pool(*a, **kw):
    p = Pool(*a, **kw)
    try:
        yield p
    finally:
        p.destroy()


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def plain_attention(q, K, V, k, v, parent):
    """One layer, one request, in 64 bits.  q [n, Hq, D], K and V [L, Hkv, D], k and v [n, Hkv, D].
    Returns (out [n, Hq, D], lse [n, Hq], weights [n, Hq, L + n], largest sum |q||k| / sqrt(D) [n, Hq], largest |V| seen [n, Hq])."""
    n, hq, D = q.shape
    hkv, L = k.shape[1], K.shape[0]
    G = hq // hkv
    keys = torch.cat([K, k]).double().repeat_interleave(G, dim=1).permute(1, 0, 2).contiguous()     # [Hq, L + n, D]
    vals = torch.cat([V, v]).double().repeat_interleave(G, dim=1).permute(1, 0, 2).contiguous()
    qd = q.double().permute(1, 0, 2).contiguous()                                                   # [Hq, n, D]
    see = torch.cat([torch.ones(n, L, dtype=torch.bool), seen_matrix(parent)], dim=1).to(q.device)
    x = torch.matmul(qd, keys.transpose(1, 2).contiguous()) / math.sqrt(D)
    big = torch.matmul(qd.abs(), keys.abs().transpose(1, 2).contiguous()) / math.sqrt(D)
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    big = torch.where(see, big, torch.zeros_like(big)).amax(dim=2)
    lse = torch.logsumexp(x, dim=2)
    w = torch.exp(x - lse[:, :, None])
    out = torch.matmul(w, vals)
    vmax = torch.where(see[None, :, :, None], vals.abs()[:, None], torch.zeros((), dtype=torch.float64, device=q.device)).amax(dim=(2, 3)) \
        if n * (L + n) * hq * D < 2**27 else vals.abs().amax() * torch.ones_like(lse)
    return out.permute(1, 0, 2), lse.t(), w.permute(1, 0, 2), big.t(), vmax.t()


def attention_bounds(out, lse, big, vmax, D, bf16):
    """How far a result may lie from the exact one.  A score is a float32 sum of D products (exact for bf16), each addition off by at most
    half a step of 2^-24 of what has been summed: (D + 4) 2^-24 of the sum of magnitudes, the scaling and the exponential's argument
    included.  A weight is then off by that much (numerator and denominator: twice), by the pair's 2^-16 (bf16), and by a few
    float32 roundings in its exponential and sums; the result is rounded once to its type."""
    score = (D + 8) * 2.0**-24 * big + 2.0**-20
    weight = 2.0 * score + (2.0**-15 if bf16 else 0.0)
    tol = weight[:, :, None] * vmax[:, :, None] + (BF16_HALF_STEP if bf16 else 2.0**-24) * out.abs()
    return tol * 1.01, score + 2.0**-22 * lse.abs()
