"""CPU oracle of the expert FFN in 8-bit integers (HMOE_BF16_I8).

TEST INFRASTRUCTURE ONLY: the library's quantisers and kernels are written separately.

  * a row v (of a weight matrix [N, K], of the tokens, of the intermediate h) has  amax = max(max |v|, 2^-100),
    scale amax / 127 and codes rint(127 v / amax) (nearest even);
  * a product of two rows is scale * scale' * sum of products of codes;
  * g, u from the token's codes, h = silu(g) u, quantised again over its F values, then the down projection.

Everything in 64 bits.  For rows of bfloat16 values the codes are those of an evaluation in fp32 as well: 127 v and (2n + 1) amax
/ 2 are whole multiples of one power of two below 2^16, so a quotient that is not half a code away is at least 2^-17 of
its size away from being so, which is more than the rounding of a division.
"""
from __future__ import annotations

from typing import Sequence, Tuple

import numpy as np


def quantize_rows(v: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """[N, K] -> codes (whole numbers, float64) [N, K], scales [N]."""
    v = np.asarray(v, dtype=np.float64)
    amax = np.maximum(np.abs(v).max(axis=1), 2.0 ** -100)
    return np.rint(127.0 * v / amax[:, None]), amax / 127.0


def expert_ffn(x: np.ndarray, w_gate: np.ndarray, w_up: np.ndarray, w_down: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """x [M, H], values as float64 -> (o [M, H], slack [M, H]).

    slack bounds what an evaluation in fp32 may differ by before its last rounding.  The sums are exact; h has a relative
    error of at most 2^-18 there (three roundings in g and u each; the exponential of up to |g| = 32 in fp32: 32 * 1.45 *
    2^-24 < 2^-18.4), so 127 h / amax is off by at most 2 * 127 * 2^-18 < 2^-10 and only codes that close to a half can
    be another whole number.  Each changes the result by scale * scale' * |code'| <= scale * scale' * 127.
    """
    qx, sx = quantize_rows(x)
    (qg, sg), (qu, su), (qd, sd) = (quantize_rows(w) for w in (w_gate, w_up, w_down))
    g = sx[:, None] * sg[None, :] * (qx @ qg.T)
    u = sx[:, None] * su[None, :] * (qx @ qu.T)
    h = g / (1.0 + np.exp(-g)) * u
    qh, sh = quantize_rows(h)
    at = 127.0 * np.abs(h) / np.maximum(np.abs(h).max(axis=1), 2.0 ** -100)[:, None]
    near = (np.abs(at - np.floor(at) - 0.5) < 2.0 ** -10).sum(axis=1)
    o = sh[:, None] * sd[None, :] * (qh @ qd.T)
    slack = (near * sh)[:, None] * (127.0 * sd)[None, :] + 2.0 ** -17 * np.abs(o)
    return o, slack


def moe_layer(x: np.ndarray, topk_idx: np.ndarray, topk_w: np.ndarray, experts: Sequence, shared: Sequence = ()):
    """-> (y [T, H], bound [T, H]): the weighted sum over the chosen experts (and the shared experts, packed as one FFN of their
    widths together), and how far a result may be off whose expert outputs and sum are each rounded to bfloat16 (half a
    step is 2^-8 of the value)."""
    x = np.asarray(x, dtype=np.float64)
    y, bound = np.zeros_like(x), np.zeros_like(x)
    parts = [(e, np.nonzero((topk_idx == e).any(axis=1))[0]) for e in range(len(experts))]
    for e, rows in parts:
        if len(rows):
            o, slack = expert_ffn(x[rows], *experts[e])
            w = np.where(topk_idx[rows] == e, topk_w[rows].astype(np.float64), 0.0).sum(axis=1)[:, None]
            y[rows] += w * o
            bound[rows] += w * (slack + 2.0 ** -8 * (np.abs(o) + slack))
    if len(shared):
        o, slack = expert_ffn(x, np.concatenate([s[0] for s in shared]), np.concatenate([s[1] for s in shared]),
                              np.concatenate([s[2] for s in shared], axis=1))
        y += o
        bound += slack + 2.0 ** -8 * (np.abs(o) + slack)
    return y, bound + 2.0 ** -8 * (np.abs(y) + bound)
