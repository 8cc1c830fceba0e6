"""Plain forms of the cache's operators in 64 bits (numpy), written from their definitions, and inputs for them."""
from __future__ import annotations

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# half a step of rounding to the type, relative
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def f64(t):
    return t.detach().cpu().double().numpy()


def visible(n, T, causal):
    """[T] rows that query t sees of a cache of n rows."""
    return [max(0, min(n, n - T + t + 1)) if causal else n for t in range(T)]


def decode(Q, K, V, own_K, own_V, lens, own_lens, scale):
    """Q [Z,B,H,T,D] .. in 64 bits.  -> O, lse, and A = sum_j p_j |v_j| / sum_j p_j, what O's error is measured against."""
    Z, B, H, T, D = Q.shape
    G = H // (K if K is not None else own_K).shape[-3]
    O, A = np.zeros(Q.shape), np.zeros(Q.shape)
    lse = np.full((Z, B, H, T), -np.inf)
    for z in range(Z):
        for b in range(B):
            own = visible(own_lens[z][b], T, True) if own_K is not None else [0] * T
            for h in range(H):
                for t in range(T):
                    k = [K[z, h // G, :lens[z]]] if K is not None else []
                    v = [V[z, h // G, :lens[z]]] if K is not None else []
                    if own_K is not None:
                        k.append(own_K[z, b, h // G, :own[t]])
                        v.append(own_V[z, b, h // G, :own[t]])
                    k, v = np.concatenate(k), np.concatenate(v)
                    if len(k) == 0:
                        continue
                    x = scale * (k @ Q[z, b, h, t])
                    m = x.max()
                    e = np.exp(x - m)
                    O[z, b, h, t] = e @ v / e.sum()
                    A[z, b, h, t] = e @ np.abs(v) / e.sum()
                    lse[z, b, h, t] = m + np.log(e.sum())
    return O, lse, A


def key_weights(Q, K, lens, causal, scale, lse=None, prev=None):
    """-> [Z,Hkv,L] (entries behind lens: 0)"""
    Z, B, H, T, D = Q.shape
    Hkv, L = K.shape[1], K.shape[2]
    w = np.zeros((Z, Hkv, L))
    for z in range(Z):
        n = lens[z]
        sees = visible(n, T, causal)
        for h in range(H):
            g = h // (H // Hkv)
            for b in range(B):
                x = scale * (Q[z, b, h] @ K[z, g, :n].T)                     # [T, n]
                for t in range(T):
                    if sees[t] == 0:
                        continue
                    y = x[t, :sees[t]]
                    a = lse[z, b, h, t] if lse is not None else y.max() + np.log(np.exp(y - y.max()).sum())
                    if np.isfinite(a):
                        w[z, g, :sees[t]] += np.exp(y - a)
        if prev is not None:
            w[z, :, :n] += prev[z, :, :n]
    return w


def evict(weights, lens, keep, sink, recent):
    """-> [[indices of (z, g)]]"""
    out = []
    for z in range(weights.shape[0]):
        n, row = lens[z], []
        for g in range(weights.shape[1]):
            w = weights[z, g, :n].astype(np.float64)
            w = np.where(np.isnan(w), -np.inf, w)
            sure = [i for i in range(n) if i < sink or i >= n - recent]
            rest = sorted((i for i in range(n) if sink <= i < n - recent), key=lambda i: (-w[i], i))
            row.append(np.array(sorted(sure + rest[:min(n, keep) - len(sure)]), dtype=np.int64))
        out.append(row)
    return out


def randn(gen, *shape, dtype="bf16", token=False, gain=1.0):
    """[.., heads, rows, D] on the GPU; token: stored [.., rows, heads, D]."""
    x = (torch.randn(shape, generator=gen) * gain).to(DTYPES[dtype]).to("cuda:0")
    if token:
        x = x.transpose(-3, -2).contiguous().transpose(-3, -2)
    return x


def strides(x):
    return tuple(x.stride()[:-1])
