"""CPU oracle of the multi-head block's operators beside its projections, in binary64: layer norm and linear
attention with a decay for each head, both with their gradients.

TEST INFRASTRUCTURE ONLY: tests and the smoke check may import this; the GPU library never does, and this
module imports nothing from the GPU package.

attention evaluates the definition token by token; attention_sums the same as explicit sums over pairs of
tokens, O(T^2), which is what the gradients are written from.
"""
from __future__ import annotations

import numpy as np


def layer_norm(x, weight=None, bias=None, eps=1e-5, groups=1):
    """x: [M][groups n].  -> y, mean [M][groups], rstd [M][groups]"""
    x = np.asarray(x, dtype=np.float64)
    z = x.reshape(x.shape[0], groups, -1)
    mean = z.mean(-1)
    rstd = 1.0 / np.sqrt(((z - mean[..., None]) ** 2).mean(-1) + eps)
    y = ((z - mean[..., None]) * rstd[..., None]).reshape(x.shape)
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, mean, rstd


def layer_norm_backward(dy, x, weight=None, eps=1e-5, groups=1):
    """-> dx, dweight, dbias"""
    dy = np.asarray(dy, dtype=np.float64)
    xhat, _, rstd = layer_norm(x, None, None, eps, groups)
    shape = (dy.shape[0], groups, -1)
    g = (dy if weight is None else dy * weight).reshape(shape)
    z = xhat.reshape(shape)
    dx = rstd[..., None] * (g - g.mean(-1, keepdims=True) - z * (g * z).mean(-1, keepdims=True))
    return dx.reshape(dy.shape), (dy * xhat).sum(0), dy.sum(0)


def attention(r, k, v, w, u, state=None):
    """One sequence.  r, k, v: [T][H][D]; w: [H]; u: [H][D]; state: [H][D][D] (channel of k, channel of v).
    -> out [T][H][D], the state behind the last token"""
    r, k, v = (np.asarray(a, dtype=np.float64) for a in (r, k, v))
    T, H, D = r.shape
    S = np.zeros((H, D, D)) if state is None else np.array(state, dtype=np.float64)
    lam = np.exp(-np.asarray(w, dtype=np.float64))[:, None, None]
    out = np.empty((T, H, D))
    for t in range(T):
        kv = k[t][:, :, None] * v[t][:, None, :]
        out[t] = np.einsum("hc,hcj->hj", r[t], S + u[:, :, None] * kv)
        S = lam * S + kv
    return out, S


def weights(T, w):
    """exp(-(t-1-i) w) for t > i, 0 elsewhere, [H][T][T], and the lags t-1-i."""
    t = np.arange(T)
    lag = t[:, None] - 1 - t[None, :]
    return np.where(lag >= 0, np.exp(-np.maximum(lag, 0) * np.asarray(w, dtype=np.float64)[:, None, None]), 0.0), lag


def attention_sums(r, k, v, w, u, state=None):
    """attention() as sums over pairs of tokens: [T][H][D] outputs only."""
    r, k, v = (np.asarray(a, dtype=np.float64).transpose(1, 0, 2) for a in (r, k, v))
    H, T, D = r.shape
    W, _ = weights(T, w)
    out = (r @ k.transpose(0, 2, 1) * W) @ v + (r * u[:, None] * k).sum(-1, keepdims=True) * v
    if state is not None:
        out = out + np.exp(-np.arange(T) * w[:, None])[..., None] * (r @ np.asarray(state, dtype=np.float64))
    return out.transpose(1, 0, 2)


def attention_backward(r, k, v, dout, w, u, state=None, dstate=None):
    """-> dr, dk, dv [T][H][D], dw [H], du [H][D], dstate_in [H][D][D]"""
    r, k, v, do = (np.asarray(a, dtype=np.float64).transpose(1, 0, 2) for a in (r, k, v, dout))
    H, T, D = r.shape
    w, u = np.asarray(w, dtype=np.float64), np.asarray(u, dtype=np.float64)
    S = np.zeros((H, D, D)) if state is None else np.asarray(state, dtype=np.float64)
    G = np.zeros((H, D, D)) if dstate is None else np.asarray(dstate, dtype=np.float64)
    W, lag = weights(T, w)
    n = np.arange(T)
    past = np.exp(-n * w[:, None])[..., None]                      # weight of `state` in the output of token t
    left = np.exp(-(T - 1 - n) * w[:, None])[..., None]            # weight of token i in the state behind
    whole = np.exp(-T * w)[:, None, None]
    A = r @ k.transpose(0, 2, 1)
    X = do @ v.transpose(0, 2, 1)
    now = (do * v).sum(-1, keepdims=True)
    dr = (X * W) @ k + now * u[:, None] * k + past * (do @ S.transpose(0, 2, 1))
    dk = (X * W).transpose(0, 2, 1) @ r + now * u[:, None] * r + left * (v @ G.transpose(0, 2, 1))
    dv = (A * W).transpose(0, 2, 1) @ do + (r * u[:, None] * k).sum(-1, keepdims=True) * do + left * (k @ G)
    dw = -((A * X * W * lag).sum((1, 2)) + (n[:, None] * past * (r @ S) * do).sum((1, 2))
           + ((T - 1 - n)[:, None] * left * (k @ G) * v).sum((1, 2)) + T * (whole * S * G).sum((1, 2)))
    du = (r * k * now).sum(1)
    dS = whole * G + (past * r).transpose(0, 2, 1) @ do
    return dr.transpose(1, 0, 2), dk.transpose(1, 0, 2), dv.transpose(1, 0, 2), dw, du, dS
