"""Gradients of the MoE hot path, and the 8-bit form in which it keeps activations, in plain numpy fp64.

Same role and rules as moe_oracle: written from the formulas, slow, and shared with nothing on the CUDA side.  Inputs may
be bf16 bits (uint16) or real arrays; padding rows (row_pair < 0) never enter a sum and are zero in the results.
"""
from __future__ import annotations

import numpy as np

from .moe_oracle import _values

BLOCK = 32                       # columns of a row that share one scale
E4M3_MAX = 448.0


def e4m3_round(v: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value (ties to the even code) of |v| <= 448: 3 mantissa bits, least exponent -6."""
    v = np.asarray(v, dtype=np.float64)
    _, e = np.frexp(v)                                  # |v| = m 2^e, m in [0.5, 1)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)     # spacing of the codes around v
    return np.round(v / step) * step                    # numpy rounds ties to even


def act8_encode(v):
    """(codes as the values they stand for before scaling [rows, P], scale bytes [P/32, rows]) of v [rows, cols]."""
    v = np.asarray(v, dtype=np.float64)
    rows, cols = v.shape
    P = (cols + BLOCK - 1) // BLOCK * BLOCK
    codes, scale = np.zeros((rows, P)), np.zeros((P // BLOCK, rows), dtype=np.int64)
    for r in range(rows):
        for b in range(P // BLOCK):
            block = v[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(block).all():
                scale[b, r] = 255
                codes[r, b * BLOCK:(b + 1) * BLOCK] = np.nan
                continue
            top = np.abs(block).max()
            k = -127
            while top > E4M3_MAX * 2.0 ** k:
                k += 1
            scale[b, r] = k + 127
            codes[r, b * BLOCK:b * BLOCK + block.size] = e4m3_round(block / 2.0 ** k)
    return codes, scale


def act8_decode(codes, scale, cols: int) -> np.ndarray:
    """Values [rows, cols] of codes (as values) [rows, P] and scale bytes [P/32, rows]."""
    s = np.where(np.asarray(scale) == 255, np.nan, np.ldexp(1.0, np.asarray(scale, dtype=np.int64) - 127))
    return (np.asarray(codes, dtype=np.float64) * np.repeat(s.T, BLOCK, axis=1))[:, :cols]


def _sigmoid(z):
    return 1.0 / (1.0 + np.exp(-z))


def _experts(slot_row_off, slot_expert, row_pair):
    """(expert, its slot's occupied rows) for every slot that has some."""
    row_pair = np.asarray(row_pair).reshape(-1)
    for s, e in enumerate(np.asarray(slot_expert).reshape(-1).tolist()):
        rows = np.arange(int(slot_row_off[s]), int(slot_row_off[s + 1]))
        rows = rows[row_pair[rows] >= 0]
        if e >= 0 and rows.size:
            yield e, rows


def gate_up(xp, slot_row_off, slot_expert, row_pair, w_gate, w_up):
    """(g, u) [Rcap, F]."""
    x, w1, w3 = _values(xp), _values(w_gate), _values(w_up)
    g, u = np.zeros((x.shape[0], w1.shape[1])), np.zeros((x.shape[0], w1.shape[1]))
    for e, rows in _experts(slot_row_off, slot_expert, row_pair):
        g[rows], u[rows] = x[rows] @ w1[e].T, x[rows] @ w3[e].T
    return g, u


def expert_ffn_backward(dyp, xp, g, u, slot_row_off, slot_expert, row_pair, w_gate, w_up, w_down):
    """dict of dxp, dw_gate, dw_up, dw_down, and of what lies between: dgate, dup, h.  g, u: as decoded, [Rcap, F]."""
    dy, x, w1, w3, w2 = _values(dyp), _values(xp), _values(w_gate), _values(w_up), _values(w_down)
    out = dict(dxp=np.zeros(x.shape), dw_gate=np.zeros(w1.shape), dw_up=np.zeros(w3.shape), dw_down=np.zeros(w2.shape),
               dgate=np.zeros(g.shape), dup=np.zeros(g.shape), h=np.zeros(g.shape))
    for e, rows in _experts(slot_row_off, slot_expert, row_pair):
        s = _sigmoid(g[rows])
        dh = dy[rows] @ w2[e]
        dg = dh * u[rows] * s * (1.0 + g[rows] * (1.0 - s))
        du = dh * g[rows] * s
        h = g[rows] * s * u[rows]
        out["dgate"][rows], out["dup"][rows], out["h"][rows] = dg, du, h
        out["dxp"][rows] = dg @ w1[e] + du @ w3[e]
        out["dw_gate"][e] += dg.T @ x[rows]
        out["dw_up"][e] += du.T @ x[rows]
        out["dw_down"][e] += dy[rows].T @ h
    return out


def combine_backward(dout, yp, pair_row, topk_w):
    """(dyp [Rcap, D], dtopk_w [T, K])."""
    d, y, w = _values(dout), _values(yp), np.asarray(topk_w, dtype=np.float64)
    T, K = w.shape
    rows = np.asarray(pair_row).reshape(T, K)
    dyp, dw = np.zeros(y.shape), np.zeros((T, K))
    for t in range(T):
        for j in range(K):
            dyp[rows[t, j]] = w[t, j] * d[t]
            dw[t, j] = d[t] @ y[rows[t, j]]
    return dyp, dw


def dispatch_backward(dxp, pair_row, T: int, K: int, topk_idx=None, dlogit=None, w_router=None):
    """dx [T, D]."""
    d = _values(dxp)
    rows = np.asarray(pair_row).reshape(T, K)
    dx = np.zeros((T, d.shape[1]))
    for t in range(T):
        for j in range(K):
            dx[t] += d[rows[t, j]]
            if dlogit is not None:
                dx[t] += float(dlogit[t, j]) * _values(w_router)[int(topk_idx[t, j])]
    return dx


def route_backward(x, w_router, bias, topk_idx, topk_w, dtopk_w, gate_mode: int):
    """(dlogit [T, K] of the selected logits, dw_router [E, D], dbias [E])."""
    xv, wr = _values(x), _values(w_router)
    w, dw = np.asarray(topk_w, dtype=np.float64), np.asarray(dtopk_w, dtype=np.float64)
    T, K = w.shape
    dl = np.zeros((T, K))
    dwr, db = np.zeros(wr.shape), np.zeros(wr.shape[0])
    for t in range(T):
        m = float(w[t] @ dw[t])
        for j in range(K):
            e = int(topk_idx[t, j])
            dl[t, j] = w[t, j] * (dw[t, j] - m)
            if gate_mode == 1:
                dl[t, j] *= 1.0 - _sigmoid(xv[t] @ wr[e] + (0.0 if bias is None else float(bias[e])))
            dwr[e] += dl[t, j] * xv[t]
            db[e] += dl[t, j]
    return dl, dwr, db
