"""CPU oracle of the layer's gradients around the experts: plain numpy in 64 bits, from the chain rule.

TEST INFRASTRUCTURE ONLY.  With y[t] = sum_j w[t, j] o[inv[t K + j]], w = softmax of the chosen logits, logits = x W_g^T:
"""
from __future__ import annotations

import numpy as np


def combine_backward(dy, o_perm, inv_perm, topk_w):
    """-> (d_o_perm [A, H], d_topk_w [T, K]); assignments whose sorted row is outside [0, A) have none."""
    dy, o_perm, w = (np.asarray(v, dtype=np.float64) for v in (dy, o_perm, topk_w))
    T, K = w.shape
    d_o, d_w = np.zeros((T * K, dy.shape[1])), np.zeros((T, K))
    for t in range(T):
        for j in range(K):
            p = int(inv_perm[t * K + j])
            if 0 <= p < T * K:
                d_o[p] = w[t, j] * dy[t]
                d_w[t, j] = dy[t] @ o_perm[p]
    return d_o, d_w


def permute_backward(d_x_perm, inv_perm, T, add=None):
    d = np.asarray(d_x_perm, dtype=np.float64)
    dx = d[np.asarray(inv_perm)].reshape(T, -1, d.shape[1]).sum(axis=1)
    return dx if add is None else dx + np.asarray(add, dtype=np.float64)


def route_backward(topk_idx, topk_w, d_topk_w, n_experts):
    w, dw = np.asarray(topk_w, dtype=np.float64), np.asarray(d_topk_w, dtype=np.float64)
    part = w * (dw - (w * dw).sum(axis=1, keepdims=True))
    d = np.zeros((w.shape[0], n_experts))
    for t in range(w.shape[0]):
        for j in range(w.shape[1]):
            if 0 <= topk_idx[t, j] < n_experts:
                d[t, topk_idx[t, j]] += part[t, j]
    return d


def router_backward(x, w_g, d_logits, add=None):
    """-> (dx [T, H], d_w_g [E, H])"""
    x, w_g, d = (np.asarray(v, dtype=np.float64) for v in (x, w_g, d_logits))
    dx = d @ w_g
    return (dx if add is None else dx + np.asarray(add, dtype=np.float64)), d.T @ x
