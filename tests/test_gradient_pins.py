"""The gradient oracle against central differences of the forward oracle, and the 8-bit form against its definition.

Central differences in fp64 with step h have an error of about h^2 |f'''| / 6 + 2^-52 |f| / h; with h = 2^-14 and functions
of order 1 whose third derivatives are of order 10 that is below 1e-7, so 1e-6 of the largest entry is asked for.
"""
import numpy as np
import pytest
import torch

import oracle

H = 2.0 ** -14


def numeric(f, v):
    """Gradient of the scalar f with respect to the array v (changed in place and put back)."""
    out = np.zeros(v.shape)
    for i in np.ndindex(*v.shape):
        keep = v[i]
        v[i] = keep + H
        hi = f()
        v[i] = keep - H
        lo = f()
        v[i] = keep
        out[i] = (hi - lo) / (2 * H)
    return out


def close(got, want):
    assert np.abs(got - want).max() <= 1e-6 * max(1e-3, np.abs(want).max())


def layout(T, D, E, K, S, A, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, D))
    wr = rng.standard_normal((E, D)) / np.sqrt(D)
    b = 0.3 * rng.standard_normal(E)
    idx, w, logits = oracle.route(x, wr, b, K, 0)
    hist = oracle.histogram(idx, E)
    replicas, slot_off, slot_expert, _ = oracle.plan(hist, S)
    slot_row_off, row_pair, pair_row, _ = oracle.dispatch(None, idx, hist, replicas, slot_off, S, A)
    return rng, x, wr, b, idx, w, slot_expert, slot_row_off, row_pair, pair_row.reshape(T, K)


def test_expert_gradient_against_differences():
    T, D, F, E, K, S, A = 5, 3, 4, 3, 2, 4, 2
    rng, x, _, _, idx, w, slot_expert, off, row_pair, pair_row = layout(T, D, E, K, S, A, 1)
    xp = np.zeros((row_pair.size, D))
    xp[row_pair >= 0] = x[row_pair[row_pair >= 0] // K]
    w1, w3, w2 = (rng.standard_normal(s) for s in ((E, F, D), (E, F, D), (E, D, F)))
    dyp = rng.standard_normal(xp.shape) * (row_pair >= 0)[:, None]

    def f():
        return float((oracle.expert_ffn(xp, off, slot_expert, w1, w3, w2)[row_pair >= 0] * dyp[row_pair >= 0]).sum())

    g, u = oracle.gate_up(xp, off, slot_expert, row_pair, w1, w3)
    got = oracle.expert_ffn_backward(dyp, xp, g, u, off, slot_expert, row_pair, w1, w3, w2)
    close(got["dxp"], numeric(f, xp))
    close(got["dw_gate"], numeric(f, w1))
    close(got["dw_up"], numeric(f, w3))
    close(got["dw_down"], numeric(f, w2))


def test_shuffle_gradients_against_differences():
    T, D, E, K, S, A = 6, 3, 4, 3, 5, 4
    rng, x, wr, _, idx, w, _, off, row_pair, pair_row = layout(T, D, E, K, S, A, 2)
    yp, dout = rng.standard_normal((row_pair.size, D)), rng.standard_normal((T, D))
    dyp, dw = oracle.combine_backward(dout, yp, pair_row, w)
    f = lambda: float((oracle.combine(yp, pair_row, w) * dout).sum())  # noqa: E731
    close(dyp, numeric(f, yp))
    close(dw, numeric(f, w))
    dxp, dl = rng.standard_normal((row_pair.size, D)), rng.standard_normal((T, K))

    def g():   # <xp, dxp> with xp[row] = x[token], and <selected logits, dl>
        s = sum(float(x[t] @ dxp[pair_row[t, j]]) for t in range(T) for j in range(K))
        return s + sum(float(x[t] @ wr[idx[t, j]]) * dl[t, j] for t in range(T) for j in range(K))

    close(oracle.dispatch_backward(dxp, pair_row, T, K, idx, dl, wr), numeric(g, x))


@pytest.mark.parametrize("mode", [0, 1])
def test_router_gradient_against_differences(mode):
    T, D, E, K = 7, 5, 6, 3
    rng = np.random.default_rng(3)
    x, wr, b = rng.standard_normal((T, D)), rng.standard_normal((E, D)), rng.standard_normal(E)
    idx, w, _ = oracle.route(x, wr, b, K, mode)
    dw = rng.standard_normal((T, K))

    def f():
        z = np.take_along_axis(x @ wr.T + b, idx.astype(np.int64), 1)
        s = np.exp(z) if mode == 0 else 1 / (1 + np.exp(-z))
        return float((s / s.sum(1, keepdims=True) * dw).sum())

    dl, dwr, db = oracle.route_backward(x, wr, b, idx, w, dw, mode)
    close(dwr, numeric(f, wr))
    close(db, numeric(f, b))
    assert dl.shape == (T, K) and np.allclose(dl.sum(), db.sum())


def test_e4m3_rounding_is_the_formats():
    codes = torch.arange(256, dtype=torch.uint8)
    values = codes.view(torch.float8_e4m3fn).double().numpy()
    finite = np.sort(np.unique(values[np.isfinite(values)]))
    assert finite.max() == 448 and np.array_equal(oracle.e4m3_round(finite), finite)
    rng = np.random.default_rng(4)
    v = np.concatenate([rng.uniform(-448, 448, 4000), rng.uniform(-1, 1, 4000) * 2.0 ** rng.integers(-14, 8, 4000),
                        (finite[1:] + finite[:-1]) / 2])          # the ties among them
    assert np.array_equal(oracle.e4m3_round(v), torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy())


def test_act8_round_trip():
    rng = np.random.default_rng(5)
    v = rng.standard_normal((9, 75)) * 2.0 ** rng.integers(-20, 20, (9, 1))
    v[2] = 0
    v[3, 40] = np.inf
    v[4, 70] = np.nan
    v[5, 1] = 448.0 * 2.0 ** 3
    codes, scale = oracle.act8_encode(v)
    back = oracle.act8_decode(codes, scale, 75)
    assert codes.shape == (9, 96) and scale.shape == (3, 9)
    assert scale[1, 3] == 255 and scale[2, 4] == 255 and (scale[:, 2] == 0).all()
    assert np.isnan(back[3, 32:64]).all() and np.isnan(back[4, 64:]).all()
    ok = np.isfinite(back)
    assert ok.sum() == 9 * 75 - 32 - 11
    unit = np.repeat(np.ldexp(1.0, np.minimum(scale, 254) - 127).T, 32, 1)[:, :75]
    assert (np.abs(back - v)[ok] <= np.maximum(np.abs(v) / 16, unit * 2.0 ** -10)[ok]).all()
