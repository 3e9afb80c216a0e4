"""Attention on changed scores, and the norm and the axes of rotary positions, in float64.

TEST INFRASTRUCTURE (see oracle/__init__.py).  Plain numpy.

attend_scored: Eq. 1 with the score of query row r and key j, s = scale * q.k, replaced by c tanh(s / c) where there is a
cap c, and then by s + slope[head] * (pos(j) - pos(r)) where there are slopes, pos being the position ids of Eq. 4 that the
token table keeps.  Mask, softmax and log-sum-exp as in attention.py.

Beside the results it gives what a bound on a lower-precision evaluation is made of: how much of |v| a row's weights carry,
and the same with every weight times its own share of error (a caller says what a score's error is).

norm_rotate: x / sqrt(mean(x^2) + eps) * w per head, then the rotation of rope.py with a position per pair.
"""
from __future__ import annotations

import numpy as np
import torch

from .attention import _rows_f64


def attend_scored(table, meta, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, softcap: float = 0.0,
                  slopes=None, scale: float | None = None, rows=None, shared_mask: bool = False, score_error=None):
    """Returns a dict of float64 arrays over the packed rows (NaN for rows not asked for): out [NQ][Hq][D], lse [NQ][Hq];
    mass = sum_j p_j |v_j| [NQ][Hq][D]; keys [NQ] the keys a row sees; with score_error(s_abs, s, bias, spread), the error of a
    score whose products' absolute values sum to s_abs, spread being |slope| times the range of the rows' positions: error_mass = sum_j p_j e_j |v_j| and error = sum_j p_j e_j."""
    NQ, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    qf = q.to(torch.float64).numpy()
    got = {n: np.full((NQ, Hq, D), np.nan) for n in ("out", "mass", "error_mass")}
    got.update({n: np.full((NQ, Hq), np.nan) for n in ("lse", "error")}, keys=np.zeros(NQ))
    want = np.arange(NQ) if rows is None else np.asarray(rows, dtype=np.int64)
    for s in np.unique(meta.q_seq[want]):
        idx = want[meta.q_seq[want] == s]
        slots = meta.logical_slot[idx]
        mask = table.dense_mask(int(s), slots, shared=shared_mask)
        pos = np.asarray(table.pos[int(s)], dtype=np.float64)
        far = pos[None, :] - pos[slots][:, None]
        phys = table.physical_slots(int(s))
        got["keys"][idx] = mask.sum(1)
        for h in range(Hq):
            k = np.nan_to_num(_rows_f64(k_cache, phys, h // G, table.block_size))
            v = np.nan_to_num(_rows_f64(v_cache, phys, h // G, table.block_size))
            x = qf[idx, h] @ k.T * scale
            if softcap:
                x = softcap * np.tanh(x / softcap)
            bias = np.zeros_like(far) if slopes is None else float(slopes[h]) * far
            x = np.where(mask, x + bias, -np.inf)
            m = x.max(axis=1, keepdims=True)
            p = np.exp(x - m)
            l = p.sum(axis=1, keepdims=True)
            p /= l
            got["out"][idx, h] = p @ v
            got["lse"][idx, h] = (m + np.log(l))[:, 0]
            got["mass"][idx, h] = p @ np.abs(v)
            if score_error is not None:
                e = p * score_error(np.abs(qf[idx, h]) @ np.abs(k).T * scale, np.where(mask, x - bias, 0.0), np.where(mask, bias, 0.0),
                                    0.0 if slopes is None else abs(float(slopes[h])) * (pos[slots].max() - pos[slots].min()))
                got["error_mass"][idx, h] = e @ np.abs(v)
                got["error"][idx, h] = e.sum(1)
    return got


def norm_rotate(x: np.ndarray, positions: np.ndarray, theta: float, weight=None, eps: float = 0.0, offset: float = 0.0) -> np.ndarray:
    """x [n][H][D] float64; positions [n] or [n][D/2], one per pair; theta 0: nothing turns; weight [D] or None: no norm."""
    n, H, D = x.shape
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * (offset + np.asarray(weight, dtype=np.float64))
    if theta == 0:
        return y
    p = np.broadcast_to(positions.reshape(n, -1), (n, D // 2)).astype(np.float64)
    phi = p * float(theta) ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(phi)[:, None], np.sin(phi)[:, None]
    a, b = y[..., :D // 2], y[..., D // 2:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)
