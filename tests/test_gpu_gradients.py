"""The training step's kernels against the fp64 gradient oracle: gate+up with kept activations, the experts' gradient, and
the gradients of combine, dispatch and route.

Bounds (u = 2^-8, bf16's unit roundoff; fp32 sums of n terms: n 2^-24 of the sum of magnitudes, with 2^-13 taken for every
matrix product here, whose sums have at most 2048 terms):
  * a stored bf16 result r: u |r| + its sum's error;
  * dgate, dup and h are rounded before they are used, so a product over them gets u (and the error of dh) times the sum of
    magnitudes on top.
Beside these worst cases the 2-norm of the error is held to 4e-3 of the result's where there are 1000 values or more: two
independent roundings have a root mean square of about 2.4e-3.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2506_07366_b200 import binding
from tests import harness as hz

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, ACC = 2.0 ** -8, 2.0 ** -13

# T, D, F, E, K, S, row_align
SHAPES = [
    (1, 8, 8, 1, 1, 1, 1),            # the smallest
    (1, 64, 40, 4, 2, 4, 16),         # one token: two experts without rows, a partial block of 32
    (3, 136, 64, 2, 1, 4, 1),         # copies without rows
    (257, 72, 264, 5, 3, 7, 1),       # odd widths, slots that start anywhere
    (300, 520, 104, 4, 2, 6, 16),
    (129, 256, 512, 3, 2, 3, 128),
    (513, 512, 328, 8, 8, 10, 32),    # every expert takes every token
    (700, 2048, 1408, 6, 2, 9, 16),
]


def bf(a):
    return hz.f64_to_bf16_tensor(a, DEV)


class Case:
    """Tables, inputs (bf16) and garbage in every place that must not matter."""

    def __init__(self, T, D, F, E, K, S, A, mode=0, seed=0, hot=0.0):
        rng = np.random.default_rng(seed)
        self.rng, self.dims = rng, (T, D, F, E, K, S)
        self.shape = binding.Shape(T, D, F, E, K, S, mode, A)
        self.x, self.wr = bf(rng.standard_normal((T, D))), bf(rng.standard_normal((E, D)) / np.sqrt(D))
        self.bias = (rng.standard_normal(E) - hot * np.log1p(np.arange(E))).astype(np.float32)
        idx, w, _ = oracle.route(hz.bits(self.x), hz.bits(self.wr), self.bias, K, mode)
        hist = oracle.histogram(idx, E)
        self.replicas, self.slot_off, self.slot_expert, _ = oracle.plan(hist, S)
        self.slot_row_off, self.row_pair, pair_row, _ = oracle.dispatch(None, idx, hist, self.replicas, self.slot_off, S, A)
        self.pair_row, self.idx, self.w = pair_row.reshape(T, K), idx, w.astype(np.float32)
        self.occ = self.row_pair >= 0
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(DEV)  # noqa: E731
        self.t = {n: i32(getattr(self, n)) for n in ("slot_off", "slot_expert", "slot_row_off", "row_pair", "pair_row", "idx")}
        self.t["w"] = torch.from_numpy(self.w).to(DEV)
        self.ctx = binding.Context(self.shape)

    def rows(self, std, width):
        """Rows in slot order; every row that holds no token is NaN."""
        v = self.rng.standard_normal((self.row_pair.size, width)) * std
        v[~self.occ] = np.nan
        return bf(v)

    def clean(self, t):
        v = hz.bits(t).copy()
        v[~self.occ] = 0
        return v

    def weights(self):
        _, D, F, E, _, _ = self.dims
        return [bf(self.rng.standard_normal(s) * 0.05) for s in ((E, F, D), (E, F, D), (E, D, F))]

    def kept(self):
        s = self.shape
        u8 = dict(dtype=torch.uint8, device=DEV)
        return [torch.full(d, 0xAA, **u8) for d in ((s.Rcap, s.P), (s.Rcap, s.P), (s.P // 32, s.Rcap), (s.P // 32, s.Rcap))]

    def save(self, xp, w1, w3):
        h = torch.full((self.shape.Rcap, self.shape.F), float("nan"), dtype=torch.bfloat16, device=DEV)
        kept = self.kept()
        self.ctx.expert_ffn_gate_up_save(xp, self.t["slot_row_off"], self.t["slot_expert"], w1, w3, h, *kept)
        return h, kept

    def decoded(self, kept):
        g, u = (oracle.act8_decode(c.view(torch.float8_e4m3fn).double().cpu().numpy(), s.cpu().numpy(), self.shape.F)
                for c, s in ((kept[0], kept[2]), (kept[1], kept[3])))
        g[~self.occ] = 0
        u[~self.occ] = 0
        return g, u

    def backward(self, dyp, xp, ws, kept, stream=None):
        s = self.shape
        nan = lambda *d: torch.full(d, float("nan"), dtype=torch.bfloat16, device=DEV)  # noqa: E731
        mid = [nan(s.Rcap, s.F) for _ in range(3)]
        out = dict(dxp=nan(s.Rcap, s.D), dw_gate=nan(s.E, s.F, s.D), dw_up=nan(s.E, s.F, s.D), dw_down=nan(s.E, s.D, s.F))
        t = self.t
        self.ctx.expert_ffn_backward(dyp, xp, t["slot_row_off"], t["slot_off"], t["slot_expert"], t["row_pair"], *ws, *kept,
                                     *mid, *out.values(), stream=stream)
        return out


def f64(t):
    return t.double().cpu().numpy()


def within(got, ref, bound, what):
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - ref) - bound
    assert over.max() <= 0, f"{what}: {over.max():.3e} over its bound"
    if ref.size >= 1000 and np.linalg.norm(ref) > 0:
        rel = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert rel <= 4e-3, f"{what}: {rel:.2e} of the norm"


@pytest.mark.parametrize("dims", SHAPES, ids=lambda d: "x".join(map(str, d)))
def test_gate_up_save(dims):
    c = Case(*dims, seed=11)
    xp, (w1, w3, _) = c.rows(1.0, c.shape.D), c.weights()
    h, kept = c.save(xp, w1, w3)
    plain = torch.full_like(h, float("nan"))
    c.ctx.expert_ffn_gate_up(xp, c.t["slot_row_off"], c.t["slot_expert"], w1, w3, plain)
    c.ctx.check_status()
    occ = torch.from_numpy(c.occ).to(DEV)
    assert torch.equal(h[occ], plain[occ])                       # the forward pass is the same, bit for bit
    outside = np.arange(c.row_pair.size) >= c.slot_row_off[-1]
    assert (kept[0].cpu().numpy()[outside] == 0xAA).all() and (kept[2].cpu().numpy()[:, outside] == 0xAA).all()
    x = c.clean(xp)
    g, u = oracle.gate_up(x, c.slot_row_off, c.slot_expert, c.row_pair, hz.bits(w1), hz.bits(w3))
    mag = [oracle.gate_up(np.abs(oracle.bf16_bits_to_f64(x)), c.slot_row_off, c.slot_expert, c.row_pair,
                          np.abs(oracle.bf16_bits_to_f64(hz.bits(w))), np.zeros(w.shape))[0] for w in (w1, w3)]
    for v, m, dec, codes, scale in zip((g, u), mag, c.decoded(kept), kept[:2], kept[2:]):
        _, want = oracle.act8_encode(v)
        sc = scale.cpu().numpy().astype(int)
        # the block maximum may sit on either side of a step of the scale by its own error: one step at most, and rarely
        off = (sc != want)[:, c.occ]
        assert off.mean() <= 1e-3 + 2 / off.size and (np.abs(sc - want)[:, c.occ] <= 1).all()
        unit = np.repeat(np.ldexp(1.0, sc - 127).T, 32, axis=1)[:, :c.shape.F]
        within_8 = np.maximum(np.abs(v) / 16, unit * 2.0 ** -10) + 1.1 * ACC * m
        assert (np.abs(dec - v) <= within_8)[c.occ].all()
        stored = codes.view(torch.float8_e4m3fn).float().cpu().numpy()[c.occ]
        top = np.abs(stored).reshape(stored.shape[0], -1, 32).max(-1)
        # the largest value, above 224 before it is rounded (else the scale would be smaller), is 224 or more after
        assert ((top >= 224) | (sc.T[c.occ] == 0)).all()
        assert (codes[:, c.shape.F:].cpu().numpy()[c.occ] == 0).all()


def gradient_bounds(c, dyp, x, g, u, ws, ref):
    """Worst-case errors of the four results (see the module's text)."""
    dy, xv = (np.abs(oracle.bf16_bits_to_f64(a)) for a in (dyp, x))
    w1, w3, w2 = (np.abs(f64(w)) for w in ws)
    out = {k: np.zeros(ref[k].shape) for k in ("dxp", "dw_gate", "dw_up", "dw_down")}
    s = 1 / (1 + np.exp(-g))
    slope, act = np.abs(u * s * (1 + g * (1 - s))), np.abs(g * s)
    for e, rows in oracle.moe_gradients._experts(c.slot_row_off, c.slot_expert, c.row_pair):
        dh = ACC * (dy[rows] @ w2[e])
        eg = 1.01 * U * np.abs(ref["dgate"][rows]) + dh * slope[rows] + 2.0 ** -18 * np.abs(u[rows]) * (dy[rows] @ w2[e])
        eu = 1.01 * U * np.abs(ref["dup"][rows]) + dh * act[rows]
        eh = 1.01 * U * np.abs(ref["h"][rows])
        ag, au, ah = (np.abs(ref[k][rows]) for k in ("dgate", "dup", "h"))
        out["dxp"][rows] = (eg + ACC * ag) @ w1[e] + (eu + ACC * au) @ w3[e]
        out["dw_gate"][e] += (eg + ACC * ag).T @ xv[rows]
        out["dw_up"][e] += (eu + ACC * au).T @ xv[rows]
        out["dw_down"][e] += dy[rows].T @ (eh + ACC * ah)
    return {k: 1.01 * v + U * np.abs(ref[k]) + 1e-37 for k, v in out.items()}


@pytest.mark.parametrize("hot", [0.0, 2.0])
@pytest.mark.parametrize("dims", SHAPES, ids=lambda d: "x".join(map(str, d)))
def test_expert_backward(dims, hot):
    c = Case(*dims, seed=12, hot=hot)
    xp, dyp, ws = c.rows(1.0, c.shape.D), c.rows(0.01, c.shape.D), c.weights()
    _, kept = c.save(xp, ws[0], ws[1])
    out = c.backward(dyp, xp, ws, kept)
    c.ctx.check_status()
    g, u = c.decoded(kept)
    x, dy = c.clean(xp), c.clean(dyp)
    ref = oracle.expert_ffn_backward(dy, x, g, u, c.slot_row_off, c.slot_expert, c.row_pair, *map(hz.bits, ws))
    bound = gradient_bounds(c, dy, x, g, u, ws, ref)
    within(f64(out["dxp"])[c.occ], ref["dxp"][c.occ], bound["dxp"][c.occ], "dxp")
    for k in ("dw_gate", "dw_up", "dw_down"):
        within(f64(out[k]), ref[k], bound[k], k)
    again = c.backward(dyp, xp, ws, kept)                        # fixed summation order
    occ = torch.from_numpy(c.occ).to(DEV)
    assert all(torch.equal(out[k], again[k]) if k != "dxp" else torch.equal(out[k][occ], again[k][occ]) for k in out)


def test_expert_backward_steps_and_streams():
    c = Case(300, 520, 104, 4, 2, 6, 16, seed=13)
    xp, dyp, ws = c.rows(1.0, c.shape.D), c.rows(0.01, c.shape.D), c.weights()
    _, kept = c.save(xp, ws[0], ws[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = c.backward(dyp, xp, ws, kept, stream=side)             # tensors of the current stream, work on another
    side.synchronize()
    s, t = c.shape, c.t
    e = lambda *d: torch.empty(d, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    dgate, dup, h, dxp = e(s.Rcap, s.F), e(s.Rcap, s.F), e(s.Rcap, s.F), e(s.Rcap, s.D)
    dw = e(s.E, s.F, s.D), e(s.E, s.F, s.D), e(s.E, s.D, s.F)
    c.ctx.expert_ffn_backward_act(dyp, t["slot_row_off"], t["slot_expert"], ws[2], *kept, dgate, dup, h)
    c.ctx.expert_ffn_backward_input(dgate, dup, t["slot_row_off"], t["slot_expert"], ws[0], ws[1], dxp)
    c.ctx.expert_ffn_backward_weights(dyp, xp, dgate, dup, h, t["slot_row_off"], t["slot_off"], t["row_pair"], *dw)
    c.ctx.check_status()
    occ = torch.from_numpy(c.occ).to(DEV)
    assert torch.equal(dxp[occ], out["dxp"][occ])
    assert all(torch.equal(a, out[k]) for a, k in zip(dw, ("dw_gate", "dw_up", "dw_down")))


def test_not_a_number_stays_with_its_expert():
    c = Case(200, 64, 96, 4, 1, 4, 1, seed=14)                   # slots are neighbours: tiles read into the next one
    ws = c.weights()
    xp, dyp = c.rows(1.0, c.shape.D), c.rows(0.01, c.shape.D)
    bad = int(c.slot_row_off[1])                                  # first row of the second expert
    e = int(c.slot_expert[1])
    assert c.slot_row_off[2] > bad
    clean = c.backward(dyp, xp, ws, c.save(xp, ws[0], ws[1])[1])
    xp[bad, 3] = float("nan")
    xp[bad, 5] = float("inf")
    _, kept = c.save(xp, ws[0], ws[1])
    assert (kept[2][:, bad] == 255).all() and (kept[3][:, bad] == 255).all()
    assert (kept[2][:, bad + 1] != 255).all() and (kept[2][:, bad - 1] != 255).all()
    out = c.backward(dyp, xp, ws, kept)
    c.ctx.check_status()
    keep = torch.arange(c.row_pair.size, device=DEV) != bad
    assert out["dxp"][bad].isnan().all() and torch.equal(out["dxp"][keep], clean["dxp"][keep])
    for k in ("dw_gate", "dw_up", "dw_down"):
        assert out[k][e].isnan().any()
        others = [i for i in range(4) if i != e]
        assert torch.equal(out[k][others], clean[k][others])


@pytest.mark.parametrize("dims", SHAPES, ids=lambda d: "x".join(map(str, d)))
def test_combine_backward(dims):
    c = Case(*dims, seed=15)
    T, D, _, _, K, _ = c.dims
    dout, yp = bf(c.rng.standard_normal((T, D))), c.rows(0.5, D)
    dyp = torch.full_like(yp, 7.0)
    dw = torch.full((T, K), float("nan"), device=DEV)
    c.ctx.combine_backward(dout, yp, c.t["pair_row"], c.t["w"], dyp, dw)
    c.ctx.check_status()
    want_dyp, want_dw = oracle.combine_backward(hz.bits(dout), c.clean(yp), c.pair_row, c.w)
    assert np.array_equal(f64(dyp)[c.occ], f64((c.t["w"][..., None] * dout[:, None].float()).to(torch.bfloat16))[
        c.row_pair[c.occ] // K, c.row_pair[c.occ] % K])           # one product, rounded once
    within(f64(dyp)[c.occ], want_dyp[c.occ], U * np.abs(want_dyp)[c.occ], "dyp")
    assert (dyp.float().cpu().numpy()[~c.occ] == 7).all()         # padding rows are not written
    mag = oracle.combine_backward(np.abs(f64(dout)), np.abs(oracle.bf16_bits_to_f64(c.clean(yp))), c.pair_row, c.w)[1]
    within(f64(dw), want_dw, (D / 32 + 8) * 2.0 ** -24 * mag, "dtopk_w")


@pytest.mark.parametrize("router", [False, True])
@pytest.mark.parametrize("dims", SHAPES, ids=lambda d: "x".join(map(str, d)))
def test_dispatch_backward(dims, router):
    c = Case(*dims, seed=16)
    T, D, _, _, K, _ = c.dims
    dxp = c.rows(0.01, D)
    dl = c.rng.standard_normal((T, K)).astype(np.float32) * 0.01 if router else None
    args = (c.idx, dl, f64(c.wr)) if router else ()
    dx = torch.full((T, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    c.ctx.dispatch_backward(dxp, c.t["pair_row"], c.t["idx"] if router else None,
                            torch.from_numpy(dl).to(DEV) if router else None, c.wr if router else None, dx)
    c.ctx.check_status()
    rows = oracle.bf16_bits_to_f64(c.clean(dxp))
    want = oracle.dispatch_backward(rows, c.pair_row, T, K, *args)
    mag = oracle.dispatch_backward(np.abs(rows), c.pair_row, T, K, *((c.idx, np.abs(dl), np.abs(f64(c.wr))) if router else ()))
    within(f64(dx), want, U * np.abs(want) + 17 * 2.0 ** -24 * mag, "dx")


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dims", SHAPES + [(900, 264, 8, 256, 8, 288, 16)], ids=lambda d: "x".join(map(str, d)))
def test_route_backward(dims, mode):
    c = Case(*dims, mode=mode, seed=17, hot=1.0)
    T, D, _, E, K, _ = c.dims
    dw = c.rng.standard_normal((T, K)).astype(np.float32)
    f32 = dict(dtype=torch.float32, device=DEV)
    dl, dwr, db = (torch.full(d, float("nan"), **f32) for d in ((T, K), (E, D), (E,)))
    ws = torch.full((binding.route_backward_workspace_bytes(c.shape),), 0xFF, dtype=torch.uint8, device=DEV)
    bias = torch.from_numpy(c.bias).to(DEV)
    router = (c.wr, bias, c.t["idx"]) if mode == 1 else (None, None, None)   # softmax reads none of them
    c.ctx.route_backward(c.x, *router, c.t["w"], torch.from_numpy(dw).to(DEV), c.t["slot_row_off"], c.t["slot_off"],
                         c.t["row_pair"], dl, dwr, db, ws)
    c.ctx.check_status()
    want = oracle.route_backward(hz.bits(c.x), hz.bits(c.wr), c.bias, c.idx, c.w, dw, mode)
    # dl = w (dw - m) [(1 - s)]: nine roundings, and with a sigmoid the error of its logit
    m = (np.abs(c.w) * np.abs(dw)).sum(1, keepdims=True)
    err = 16 * 2.0 ** -24 * np.abs(c.w) * (np.abs(dw) + m)
    if mode == 1:
        z = np.abs(f64(c.x)) @ np.abs(f64(c.wr)).T + np.abs(c.bias)
        err = err + np.abs(want[0]) * ((D / 32 + 8) * 2.0 ** -24 * np.take_along_axis(z, c.idx.astype(np.int64), 1) + 2.0 ** -20)
    within(f64(dl), want[0], err, "dlogit")
    dense, xa = np.zeros((T, E)), np.abs(f64(c.x))
    size = np.zeros((T, E))
    np.put_along_axis(dense, c.idx.astype(np.int64), err, 1)
    np.put_along_axis(size, c.idx.astype(np.int64), np.abs(want[0]), 1)
    acc = (80 + T / 64) * 2.0 ** -24
    within(f64(dwr), want[1], (dense + acc * size).T @ xa + 1e-37, "dw_router")
    within(f64(db), want[2], (dense + acc * size).sum(0) + 1e-37, "dbias")


def test_long_buffers_pass_32_bit_offsets():
    """163840 rows x 14336 columns: offsets of elements pass 2^31, of bytes 2^32.  Checked on the last rows."""
    T, D, F, E, K = 81920, 64, 14336, 2, 2
    shape = binding.Shape(T, D, F, E, K, E, 0, 1)
    ctx = binding.Context(shape)
    gen = torch.Generator(device=DEV).manual_seed(5)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device=DEV) * std).to(torch.bfloat16)  # noqa: E731
    xp, dyp = rnd(2 * T, D), rnd(2 * T, D, std=0.01)
    ws = rnd(E, F, D, std=0.05), rnd(E, F, D, std=0.05), rnd(E, D, F, std=0.05)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    off, slot_off, expert = i32([0, T, 2 * T]), i32([0, 1, 2]), i32([0, 1])
    row_pair = torch.arange(2 * T, dtype=torch.int32, device=DEV)
    mid = [torch.empty(2 * T, F, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    kept = [torch.empty(2 * T, F, dtype=torch.uint8, device=DEV) for _ in range(2)] + [
        torch.empty(F // 32, 2 * T, dtype=torch.uint8, device=DEV) for _ in range(2)]
    ctx.expert_ffn_gate_up_save(xp, off, expert, ws[0], ws[1], mid[2], *kept)
    dxp, dw = torch.empty_like(xp), [torch.empty_like(w) for w in ws]
    ctx.expert_ffn_backward(dyp, xp, off, slot_off, expert, row_pair, *ws, *kept, *mid, dxp, *dw)
    ctx.check_status()
    last = slice(2 * T - 8, 2 * T)
    x, dy, w1, w3, w2 = (v.double() for v in (xp[last], dyp[last], ws[0][1], ws[1][1], ws[2][1]))
    unit = lambda s: torch.exp2(s[:, last].double() - 127).T.repeat_interleave(32, 1)  # noqa: E731
    g, u = (k[last].view(torch.float8_e4m3fn).double() * unit(s) for k, s in ((kept[0], kept[2]), (kept[1], kept[3])))
    assert ((g - x @ w1.T).abs() <= (x @ w1.T).abs() / 16 + unit(kept[2]) * 2.0 ** -9).all()
    assert ((u - x @ w3.T).abs() <= (x @ w3.T).abs() / 16 + unit(kept[3]) * 2.0 ** -9).all()
    s = torch.sigmoid(g)
    dh = dy @ w2
    dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
    for got, want in ((mid[0][last], dg), (mid[1][last], du), (mid[2][last], g * s * u), (dxp[last], dg @ w1 + du @ w3)):
        assert (got.double() - want).norm() <= 4e-3 * want.norm()


def test_no_tokens():
    shape = binding.Shape(0, 64, 32, 3, 2, 4, 1, 1)
    ctx = binding.Context(shape)
    e = lambda *d, dtype=torch.bfloat16: torch.empty(d, dtype=dtype, device=DEV)  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    off, slot_off, expert, none = i32([0] * 5), i32([0, 2, 3, 4]), i32([0, 0, 1, 2]), i32([])
    w = [torch.randn(s, device=DEV).to(torch.bfloat16) for s in ((3, 32, 64), (3, 32, 64), (3, 64, 32))]
    kept = [e(0, 32, dtype=torch.uint8), e(0, 32, dtype=torch.uint8), e(1, 0, dtype=torch.uint8), e(1, 0, dtype=torch.uint8)]
    mid = [e(0, 32) for _ in range(3)]
    dw = [torch.full_like(v, float("nan")) for v in w]
    ctx.expert_ffn_gate_up_save(e(0, 64), off, expert, w[0], w[1], mid[2], *kept)
    ctx.expert_ffn_backward(e(0, 64), e(0, 64), off, slot_off, expert, none, *w, *kept, *mid, e(0, 64), *dw)
    assert all((v == 0).all() for v in dw)
    f32 = dict(dtype=torch.float32, device=DEV)
    dwr, db, wr = torch.full((3, 64), float("nan"), **f32), torch.full((3,), float("nan"), **f32), e(3, 64)
    ws = torch.empty(binding.route_backward_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    ctx.route_backward(e(0, 64), wr, None, none.view(0, 2), e(0, 2, dtype=torch.float32), e(0, 2, dtype=torch.float32), off,
                       slot_off, none, e(0, 2, dtype=torch.float32), dwr, db, ws)
    assert (dwr == 0).all() and (db == 0).all()
    ctx.combine_backward(e(0, 64), e(0, 64), none.view(0, 2), e(0, 2, dtype=torch.float32), e(0, 64), e(0, 2, dtype=torch.float32))
    ctx.dispatch_backward(e(0, 64), none.view(0, 2), None, None, None, e(0, 64))
    ctx.check_status()


def test_refusals():
    c = Case(64, 64, 64, 4, 2, 4, 16, seed=18)
    s, t = c.shape, c.t
    xp, dyp, ws = c.rows(1.0, s.D), c.rows(1.0, s.D), c.weights()
    h, kept = c.save(xp, ws[0], ws[1])
    dout, dyp2, dw = bf(np.zeros((s.T, s.D))), torch.empty_like(dyp), torch.empty(s.T, s.K, device=DEV)
    n = c.ctx.launch_count()
    with pytest.raises(TypeError):
        c.ctx.expert_ffn_gate_up_save(xp.float(), t["slot_row_off"], t["slot_expert"], ws[0], ws[1], h, *kept)
    with pytest.raises(ValueError):                               # scales are [blocks, rows]
        c.ctx.expert_ffn_gate_up_save(xp, t["slot_row_off"], t["slot_expert"], ws[0], ws[1], h, *kept[:3],
                                      kept[3].T.contiguous())
    with pytest.raises(ValueError):
        c.ctx.combine_backward(dout, xp.T.contiguous().T, t["pair_row"], t["w"], dyp2, dw)     # not contiguous
    with pytest.raises(ValueError):
        c.ctx.combine_backward(dout, None, t["pair_row"], t["w"], dyp2, dw)
    with pytest.raises(TypeError):
        c.ctx.dispatch_backward(dyp, t["pair_row"].cpu(), None, None, None, dout)
    with pytest.raises(ValueError):                               # the router's part needs its weights
        c.ctx.dispatch_backward(dyp, t["pair_row"], t["idx"], t["w"], None, dout)
    odd = torch.empty(s.T * s.D + 1, dtype=torch.bfloat16, device=DEV)[1:].view(s.T, s.D)
    with pytest.raises(binding.MoegpsError) as err:               # not 16-byte aligned
        c.ctx.combine_backward(odd, xp, t["pair_row"], t["w"], dyp2, dw)
    assert err.value.code == binding.ERR_INVALID_ARG
    f32 = dict(dtype=torch.float32, device=DEV)
    with pytest.raises(binding.MoegpsError) as err:
        c.ctx.route_backward(c.x, None, None, None, t["w"], dw, t["slot_row_off"], t["slot_off"], t["row_pair"], dw,
                             torch.empty(s.E, s.D, **f32), torch.empty(s.E, **f32),
                             torch.empty(16, dtype=torch.uint8, device=DEV))
    assert err.value.code == binding.ERR_WORKSPACE_TOO_SMALL
    assert c.ctx.launch_count() == n                              # a failing call launches nothing


def test_bad_tables_are_reported():
    c = Case(64, 64, 64, 4, 2, 4, 16, seed=19)
    s, t = c.shape, c.t
    xp, dyp, ws = c.rows(1.0, s.D), c.rows(1.0, s.D), c.weights()
    _, kept = c.save(xp, ws[0], ws[1])
    c.ctx.check_status()
    good = c.backward(dyp, xp, ws, kept)
    keep = t["slot_row_off"].clone()
    t["slot_row_off"][4] = s.Rcap + 64                            # the last slot would leave the buffers
    out = c.backward(dyp, xp, ws, kept)
    assert c.ctx.status() == binding.ERR_BAD_INDEX
    for k in ("dw_gate", "dw_up", "dw_down"):
        assert torch.equal(out[k][:3], good[k][:3]) and (out[k][3] == 0).all()
    t["slot_row_off"] = keep
    rows = t["pair_row"].clone()
    rows[5, 1], rows[6, 0] = s.Rcap, -1
    dout, dyp2 = bf(c.rng.standard_normal((s.T, s.D))), torch.zeros_like(dyp)
    dw = torch.empty(s.T, s.K, device=DEV)
    c.ctx.combine_backward(dout, xp, rows, t["w"], dyp2, dw)
    assert c.ctx.status() == binding.ERR_BAD_INDEX
    assert dw[5, 1] == 0 and dw[6, 0] == 0 and dw[5, 0] != 0
    dx = torch.empty_like(dout)
    c.ctx.dispatch_backward(dyp2, rows, None, None, None, dx)
    assert c.ctx.status() == binding.ERR_BAD_INDEX


def test_checks_without_the_compiled_module(monkeypatch):
    """Where _marshal has not been built the same checks run in Python: same results, same refusals."""
    assert binding._marshal() is not None
    monkeypatch.setattr(binding, "_marshal", lambda: None)
    c = Case(64, 64, 64, 4, 2, 4, 16, seed=20)
    s, t = c.shape, c.t
    dout, yp = bf(c.rng.standard_normal((s.T, s.D))), c.rows(0.5, s.D)
    got = torch.zeros_like(yp), torch.empty(s.T, s.K, device=DEV)
    c.ctx.combine_backward(dout, yp, t["pair_row"], t["w"], *got)
    monkeypatch.undo()
    other = binding.Context(s)
    want = torch.zeros_like(yp), torch.empty(s.T, s.K, device=DEV)
    other.combine_backward(dout, yp, t["pair_row"], t["w"], *want, stream=torch.cuda.current_stream())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for ctx in (c.ctx, other):
        with pytest.raises(TypeError, match="topk_w must be torch.float32"):
            ctx.combine_backward(dout, yp, t["pair_row"], t["w"].double(), *got)
        with pytest.raises(ValueError, match="dtopk_w must have shape"):
            ctx.combine_backward(dout, yp, t["pair_row"], t["w"], got[0], got[1][:-1])
        with pytest.raises(TypeError, match="yp must be a CUDA tensor"):
            ctx.combine_backward(dout, "yp", t["pair_row"], t["w"], *got)
        with pytest.raises(AttributeError):
            ctx.combine_backward(dout, yp, t["pair_row"], t["w"], *got, stream=object())
        ctx.close()
        with pytest.raises(binding.MoegpsError) as err:
            ctx.combine_backward(dout, yp, t["pair_row"], t["w"], *got)
        assert err.value.code == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("given", [True, False])
def test_route_backward_keeps_bad_tokens_to_their_experts(given):
    """A token with infinities or NaN in x adds nothing to the experts that it did not choose."""
    T, D, _, E, K, S, A = 500, 264, 8, 20, 3, 24, 16
    c = Case(T, D, 8, E, K, S, A, seed=21)
    dw = c.rng.standard_normal((T, K)).astype(np.float32)
    x = c.x.clone()
    x[7, 3], x[7, 200], x[499] = float("inf"), float("nan"), float("nan")
    dl, dwr, db = (torch.full(d, float("nan"), device=DEV) for d in ((T, K), (E, D), (E,)))
    ws = torch.empty(binding.route_backward_workspace_bytes(c.shape), dtype=torch.uint8, device=DEV)
    c.ctx.route_backward(x, None, None, c.t["idx"] if given else None, c.t["w"], torch.from_numpy(dw).to(DEV),
                         c.t["slot_row_off"], c.t["slot_off"], c.t["row_pair"], dl, dwr, db, ws)
    c.ctx.check_status()
    xz = f64(x)
    bad = np.zeros((E, D), dtype=bool)
    for t, cols in ((7, [3, 200]), (499, range(D))):
        for e in c.idx[t]:
            bad[e, list(cols)] = True
    xz[~np.isfinite(xz)] = 0
    want = oracle.route_backward(xz, hz.bits(c.wr), c.bias, c.idx, c.w, dw, 0)
    got = f64(dwr)
    assert (~np.isfinite(got) == bad).all()
    dense = np.zeros((T, E))
    np.put_along_axis(dense, c.idx.astype(np.int64), np.abs(want[0]) + np.abs(c.w) * np.abs(dw).sum(1, keepdims=True), 1)
    bound = (96 + T) * 2.0 ** -24 * dense.T @ np.abs(xz) + 1e-37      # one sum of up to T terms
    assert (np.abs(got - want[1]) <= bound)[~bad].all()
    assert torch.isfinite(db).all()


@pytest.mark.parametrize("mode", [0, 1])
def test_route_backward_reports_bad_indices(mode):
    c = Case(200, 64, 8, 6, 2, 6, 16, mode=mode, seed=22)
    s, t = c.shape, c.t
    f32 = dict(dtype=torch.float32, device=DEV)
    dw = torch.randn(s.T, s.K, **f32)
    ws = torch.empty(binding.route_backward_workspace_bytes(s), dtype=torch.uint8, device=DEV)

    def run(idx, row_pair):
        out = torch.empty(s.T, s.K, **f32), torch.empty(s.E, s.D, **f32), torch.empty(s.E, **f32)
        c.ctx.route_backward(c.x, c.wr, torch.from_numpy(c.bias).to(DEV), idx, t["w"], dw, t["slot_row_off"], t["slot_off"],
                             row_pair, *out, ws)
        return out

    good = run(t["idx"], t["row_pair"])
    c.ctx.check_status()
    idx = t["idx"].clone()
    e = int(idx[9, 1])
    idx[9, 1] = s.E
    dl, dwr, _ = run(idx, t["row_pair"])
    assert c.ctx.status() == binding.ERR_BAD_INDEX
    assert dl[9, 1] == 0 and torch.equal(dl[9, 0], good[0][9, 0])
    others = [i for i in range(s.E) if i != e]
    assert torch.equal(dwr[others], good[1][others]) and torch.isfinite(dwr).all()
    rows = t["row_pair"].clone()
    rows[0] = s.R
    _, dwr, _ = run(t["idx"], rows)
    assert c.ctx.status() == binding.ERR_BAD_INDEX and torch.equal(dwr, good[1])


@pytest.mark.parametrize("T", [64, 1300])                         # four warps for each token, and one
def test_skipped_pairs_add_nothing_where_values_are_not_finite(T):
    """A pair whose row or expert is outside its range is skipped: its dtopk_w is 0, and dx is the other pairs' sum, also
    where the value that it would have been multiplied with is an infinity or a NaN."""
    c = Case(T, 64, 8, 4, 2, 4, 16, seed=23)
    s, t = c.shape, c.t
    yp, dxp = c.rows(1.0, s.D), c.rows(1.0, s.D)
    dout = bf(c.rng.standard_normal((s.T, s.D)))
    dout[5, 3], dout[6, 1] = float("inf"), float("nan")
    rows = t["pair_row"].clone()
    rows[5, 1], rows[6, 0] = s.Rcap, -1
    dyp, dw = torch.zeros_like(yp), torch.empty(s.T, s.K, device=DEV)
    c.ctx.combine_backward(dout, yp, rows, t["w"], dyp, dw)
    assert c.ctx.status() == binding.ERR_BAD_INDEX
    assert dw[5, 1] == 0 and dw[6, 0] == 0
    assert not torch.isfinite(dw[5, 0]) and not torch.isfinite(dw[6, 1])
    idx, dl = t["idx"].clone(), torch.randn(s.T, s.K, device=DEV)
    idx[7, 1], idx[8, 0], dl[7, 1], dl[8, 0] = s.E, -1, float("inf"), float("nan")
    got, want = torch.empty_like(dout), torch.empty_like(dout)
    c.ctx.dispatch_backward(dxp, t["pair_row"], idx, dl, c.wr, got)
    assert c.ctx.status() == binding.ERR_BAD_INDEX
    dl[7, 1] = dl[8, 0] = 0
    c.ctx.dispatch_backward(dxp, t["pair_row"], t["idx"], dl, c.wr, want)
    c.ctx.check_status()
    assert torch.equal(got, want)


def test_weight_gradient_over_more_rows_than_a_second_lasts():
    """400 million tokens, all but a thousand of one expert: its sums take longer than the kernels' plain waiting limit.  All
    rows are zero but for some, whose products are small whole numbers: the sums are exact."""
    T, D, F = 400_000_005, 8, 8
    first = T - 1001                                              # neither part is whole blocks of 16 rows
    shape = binding.Shape(T, D, F, 2, 1, 2, 0, 1)
    ctx = binding.Context(shape)
    i32 = dict(dtype=torch.int32, device=DEV)
    dyp, xp, dgate, dup, h = (torch.zeros(T, 8, dtype=torch.bfloat16, device=DEV) for _ in range(5))
    rows = [0, 15, 77_777_777, 268_435_456, first - 1, first, T - 2, T - 1]
    rng = np.random.default_rng(24)
    small = rng.integers(-3, 4, (5, len(rows), 8)).astype(np.float64)
    for t, v in zip((dyp, xp, dgate, dup, h), small):
        t[rows] = bf(v)
    dw = [torch.full((2, 8, 8), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    ctx.expert_ffn_backward_weights(dyp, xp, dgate, dup, h, torch.tensor([0, first, T], **i32), torch.tensor([0, 1, 2], **i32),
                                    torch.arange(T, **i32), *dw)
    ctx.check_status()
    dy, x, dg, du, hh = small
    for e, part in enumerate((slice(0, 5), slice(5, 8))):
        for got, want in zip(dw, (dg[part].T @ x[part], du[part].T @ x[part], dy[part].T @ hh[part])):
            assert np.array_equal(f64(got[e]), want)
    del dyp, xp, dgate, dup, h
    torch.cuda.empty_cache()


def test_route_backward_of_many_short_parts():
    """67.2 million tokens: more parts than a grid's second or third dimension holds.  dl is zero but for some tokens, whose
    products are exact."""
    T, D, E = 67_200_000, 8, 2
    shape = binding.Shape(T, D, 8, E, 2, E, 0, 1)
    ctx = binding.Context(shape)
    i32 = dict(dtype=torch.int32, device=DEV)
    x, dw = torch.zeros(T, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, 2, device=DEV)
    rng = np.random.default_rng(25)
    at = [0, 63, 64, 1023, 1024, 33_554_432, 67_107_839, 67_107_840, T - 1]      # (the 65536th part starts at 67107840)
    xs, ds = rng.integers(-3, 4, (len(at), D)).astype(np.float64), rng.integers(-8, 9, len(at)).astype(np.float64) * 4
    x[at] = bf(xs)
    dw[at, 0] = torch.from_numpy(ds).float().to(DEV)
    idx = torch.tensor([[0, 1]], **i32).expand(T, 2).contiguous()
    w = torch.full((T, 2), 0.5, device=DEV)
    row_pair = torch.arange(2 * T, **i32).view(T, 2).T.contiguous().view(-1)
    off, slot_off = torch.tensor([0, T, 2 * T], **i32), torch.tensor([0, 1, 2], **i32)
    dl, dwr, db = (torch.full(d, float("nan"), device=DEV) for d in ((T, 2), (E, D), (E,)))
    ws = torch.empty(binding.route_backward_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    ctx.route_backward(x, None, None, idx, w, dw, off, slot_off, row_pair, dl, dwr, db, ws)
    ctx.check_status()
    assert np.array_equal(f64(dl[at]), np.stack([ds / 4, -ds / 4], 1)) and int((dl != 0).sum()) == 2 * int((ds != 0).sum())
    assert np.array_equal(f64(dwr), np.stack([ds @ xs, -ds @ xs]) / 4) and np.array_equal(f64(db), np.array([1, -1]) * ds.sum() / 4)
    del x, dw, idx, w, row_pair, dl, ws
    torch.cuda.empty_cache()


def traced(monkeypatch, shape):
    """A context whose launches are logged to stderr."""
    monkeypatch.setenv("MOEGPS_TRACE", "1")
    ctx = binding.Context(shape)
    monkeypatch.delenv("MOEGPS_TRACE")
    return ctx


# T, D, E, K and the cut: columns of a tile, parts of the tokens, steps of 64 tokens in a part.  (The last part has 13, 12, 8 and
# 9 steps, so the ring of dl tiles ends on either stage; no T is whole steps.)
LONG_ROUTES = [
    (4099, 7168, 256, 8, 256, 5, 13),
    (3401, 7160, 250, 3, 208, 4, 14),
    (8131, 2048, 64, 6, 128, 9, 15),
    (5003, 2056, 130, 1, 176, 6, 14),
]


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dims", LONG_ROUTES, ids=lambda d: "x".join(map(str, d)))
def test_route_backward_over_many_steps(dims, mode, monkeypatch, capfd):
    """Sums over many steps of 64 tokens, as training batches have them, against the definition in 64 bits on the GPU.

    Bounds for dw_router, M being the sum of the terms' magnitudes: an accumulation on the tensor core truncates, so it is off
    by at most 2^-23 of the running sum, as is each of the 16 products that it aligns with it; a sum runs over at most 64
    accumulations, the sum of the two small parts of dl over 128 of 2^-8 the size.  (64 + 1)(16 + 1) 2^-23 M at worst.  The
    2-norm of the error is held to 64 2^-24 of the result's: 64 truncations by half a unit on average of a running sum, which
    is smaller than the result on average.  dbias: fp32, at most T K terms in 256 threads and a tree."""
    T, D, E, K, cols, parts, steps = dims
    gen = torch.Generator(device=DEV).manual_seed(26)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    x, wr, bias = rnd(T, D).to(torch.bfloat16), (rnd(E, D) / D ** 0.5).to(torch.bfloat16), -torch.log1p(torch.arange(E, device=DEV).float())
    logits = x.double() @ wr.double().T + bias.double()
    top, idx = torch.topk(logits, K, dim=1)
    s = torch.sigmoid(top)
    w = (torch.softmax(top, 1) if mode == 0 else s / s.sum(1, keepdim=True)).float()
    dw = rnd(T, K)
    # the pairs in the order of their experts, one slot for each
    order = torch.argsort(idx.view(-1), stable=True)
    off = torch.nn.functional.pad(torch.bincount(idx.view(-1), minlength=E).cumsum(0), (1, 0)).to(torch.int32)
    shape = binding.Shape(T, D, 8, E, K, E, mode, 1)
    ctx = traced(monkeypatch, shape)
    dl, dwr, db = (torch.full(d, float("nan"), device=DEV) for d in ((T, K), (E, D), (E,)))
    ws = torch.full((binding.route_backward_workspace_bytes(shape),), 0xFF, dtype=torch.uint8, device=DEV)
    idx32, slot_off = idx.to(torch.int32), torch.arange(E + 1, dtype=torch.int32, device=DEV)
    for given in ([idx32] if mode else [idx32, None]):
        capfd.readouterr()
        ctx.route_backward(x, wr, bias, given, w, dw, off, slot_off, order.to(torch.int32), dl, dwr, db, ws)
        ctx.check_status()
        assert f"cols={cols} parts={parts} steps={steps}" in capfd.readouterr().err
        m = (w.double() * dw.double()).sum(1, keepdim=True)
        want = w.double() * (dw.double() - m) * (1 if mode == 0 else 1 - torch.sigmoid(top))
        err = 16 * 2.0 ** -24 * w.double() * (dw.abs().double() + (w * dw.abs()).double().sum(1, keepdim=True))
        if mode:
            z = (x.double().abs() @ wr.double().abs().T + bias.abs()).gather(1, idx)
            err += want.abs() * ((D / 32 + 8) * 2.0 ** -24 * z + 2.0 ** -20)
        within(f64(dl), f64(want), f64(err), "dlogit")
        # the sums, of the dl that the call itself has returned
        dense = torch.zeros(T, E, dtype=torch.float64, device=DEV).scatter_(1, idx, dl.double())
        ref, mag = dense.T @ x.double(), dense.abs().T @ x.double().abs()
        within(f64(dwr), f64(ref), f64(65 * 17 * 2.0 ** -23 * mag) + 1e-37, "dw_router")
        assert (dwr.double() - ref).norm() <= 64 * 2.0 ** -24 * ref.norm()
        within(f64(db), f64(dense.sum(0)), f64((T * K / 256 + 16) * 2.0 ** -24 * dense.abs().sum(0)) + 1e-37, "dbias")


def test_weight_gradients_over_long_sums():
    """90001 rows of one expert in two of its three slots and 70 of another, all values checked against 64 bits.  A running sum
    is truncated at each of up to 5626 accumulations (2^-24 of it on average) and the result rounded to bf16 (1.7e-3 of the
    norm): together below 2e-3."""
    D, F = 264, 328
    off = [0, 50_001, 50_001, 90_001, 90_071]                     # the second slot of the first expert is empty
    R = off[-1]
    shape = binding.Shape(R, D, F, 2, 1, 4, 0, 1)
    ctx = binding.Context(shape)
    gen = torch.Generator(device=DEV).manual_seed(27)
    rnd = lambda n: torch.randn(R, n, generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
    dyp, xp, dgate, dup, h = rnd(D), rnd(D), rnd(F), rnd(F), rnd(F)
    i32 = dict(dtype=torch.int32, device=DEV)
    dw = [torch.full(s, float("nan"), dtype=torch.bfloat16, device=DEV) for s in ((2, F, D), (2, F, D), (2, D, F))]
    ctx.expert_ffn_backward_weights(dyp, xp, dgate, dup, h, torch.tensor(off, **i32), torch.tensor([0, 3, 4], **i32),
                                    torch.arange(R, **i32), *dw)
    ctx.check_status()
    for e, part in enumerate((slice(0, off[3]), slice(off[3], R))):
        for got, a, b in zip(dw, (dgate, dup, dyp), (xp, xp, h)):
            ref = a[part].double().T @ b[part].double()
            assert (got[e].double() - ref).norm() <= 2e-3 * ref.norm()


def check_layer(ctx, idx, seed):
    """save and backward on a layer with these selections, NaN in every padding row and result; against 64 bits on the GPU, to
    4e-3 of the norm as above, for every expert by itself.  Returns the experts without rows."""
    s = ctx.shape
    hist = oracle.histogram(idx, s.E)
    replicas, slot_off, slot_expert, _ = oracle.plan(hist, s.S)
    slot_row_off, row_pair, _, _ = oracle.dispatch(None, idx, hist, replicas, slot_off, s.S, s.row_align)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(DEV)  # noqa: E731
    gen = torch.Generator(device=DEV).manual_seed(seed)
    occ = i32(row_pair) >= 0

    def rows(n, std):
        v = torch.randn(s.Rcap, n, generator=gen, device=DEV) * std
        v[~occ] = float("nan")
        return v.to(torch.bfloat16)

    D, F, E = s.D, s.F, s.E
    xp, dyp = rows(D, 1.0), rows(D, 0.01)
    ws = [(torch.randn(d, generator=gen, device=DEV) * 0.03).to(torch.bfloat16) for d in ((E, F, D), (E, F, D), (E, D, F))]
    u8 = dict(dtype=torch.uint8, device=DEV)
    kept = [torch.empty(d, **u8) for d in ((s.Rcap, s.P), (s.Rcap, s.P), (s.P // 32, s.Rcap), (s.P // 32, s.Rcap))]
    nan = lambda *d: torch.full(d, float("nan"), dtype=torch.bfloat16, device=DEV)  # noqa: E731
    mid, dxp, dw = [nan(s.Rcap, F) for _ in range(3)], nan(s.Rcap, D), [nan(E, F, D), nan(E, F, D), nan(E, D, F)]
    off, expert = i32(slot_row_off), i32(slot_expert)
    ctx.expert_ffn_gate_up_save(xp, off, expert, ws[0], ws[1], mid[2], *kept)
    ctx.expert_ffn_backward(dyp, xp, off, i32(slot_off), expert, i32(row_pair), *ws, *kept, *mid, dxp, *dw)
    ctx.check_status()
    unit = lambda c, sc: (c.view(torch.float8_e4m3fn).double()  # noqa: E731
                          * torch.exp2(sc.double() - 127).T.repeat_interleave(32, 1))
    close = lambda got, ref: (got.double() - ref).norm() <= 4e-3 * ref.norm()  # noqa: E731
    idle = []
    for e in range(E):
        at = torch.arange(slot_row_off[slot_off[e]], slot_row_off[slot_off[e + 1]], device=DEV)
        at = at[occ[at]]
        if at.numel() == 0:
            assert hist[e] == 0 and all((v[e] == 0).all() for v in dw)
            idle.append(e)
            continue
        g, u = (unit(c[at], sc[:, at])[:, :F] for c, sc in ((kept[0], kept[2]), (kept[1], kept[3])))
        x, dy, w1, w3, w2 = (v.double() for v in (xp[at], dyp[at], ws[0][e], ws[1][e], ws[2][e]))
        sig = torch.sigmoid(g)
        dh = dy @ w2
        dg, du = dh * u * sig * (1 + g * (1 - sig)), dh * g * sig
        assert close(dxp[at], dg @ w1 + du @ w3)
        assert close(dw[0][e], dg.T @ x) and close(dw[1][e], du.T @ x)
        assert close(dw[2][e], dy.T @ (g * sig * u))
    return idle


def test_expert_gradient_of_a_large_layer_with_idle_experts():
    """4096 tokens over 6 of 40 experts (13 to 3458 pairs each): the others have no rows in slots of their own, and zero
    weight gradients."""
    T, D, F, E, K, S, A = 4096, 1000, 712, 40, 2, 48, 16
    rng = np.random.default_rng(28)
    busy = rng.permutation(E)[:11]
    score = rng.random((T, 11)) + np.linspace(0, 2, 11)
    idx = busy[np.argsort(-score, axis=1)[:, :K]].astype(np.int32)
    assert len(check_layer(binding.Context(binding.Shape(T, D, F, E, K, S, 0, A)), idx, 29)) == E - 6


# T, D, F, E, K, S, A and the tiles that the data gradients of such a layer take: every shape of them, for either
TILES = [
    (257, 72, 264, 5, 3, 7, 1, "128x64", "128x64"),
    (600, 1032, 1000, 40, 2, 48, 16, "128x128", "128x128"),
    (1500, 1032, 520, 30, 2, 36, 16, "128x256", "128x128"),
    (520, 1416, 2056, 40, 4, 50, 1, "128x128", "128x256"),        # 42 rows a slot: not by pairs of CTAs, though two rounds
    (900, 2056, 1032, 12, 4, 14, 16, "256x256", "256x256"),
]


@pytest.mark.parametrize("dims", TILES, ids=lambda d: "x".join(map(str, d[:7])))
def test_expert_gradient_on_every_tile_shape(dims, monkeypatch, capfd):
    T, D, F, E, K, S, A, act, data = dims
    ctx = traced(monkeypatch, binding.Shape(T, D, F, E, K, S, 0, A))
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the tiles are those for 148 SMs")
    idx = np.argsort(np.random.default_rng(30).random((T, E)) - 0.3 * np.exp(-np.arange(E)), axis=1)[:, :K].astype(np.int32)
    capfd.readouterr()
    check_layer(ctx, idx, 31)
    err = capfd.readouterr().err
    assert f"act tile={act}\n" in err and f"input tile={data}\n" in err


# T, D, K and the warps that a token gets in combine, in dispatch and in dispatch with the router's part
SHUFFLES = [
    (1301, 72, 1, 1, 1, 1), (1301, 136, 2, 1, 1, 1), (1301, 520, 3, 1, 1, 1), (1301, 264, 5, 1, 1, 1), (1301, 1032, 8, 1, 1, 1),
    (1301, 1032, 4, 1, 4, 1), (1301, 1544, 2, 1, 4, 1), (1301, 2048, 6, 4, 4, 1), (1301, 2056, 7, 4, 4, 4), (9, 8, 2, 4, 4, 4),
]


@pytest.mark.parametrize("dims", SHUFFLES, ids=lambda d: "x".join(map(str, d[:3])))
def test_shuffle_gradients_with_every_team_of_warps(dims, monkeypatch, capfd):
    """Against 64 bits on the GPU.  dyp is one product rounded once; dtopk_w a sum of D terms, (D / 32 + 8) 2^-24 of their
    magnitudes; dx an fp32 sum of at most 2 K terms rounded once."""
    T, D, K, *warps = dims
    E, S, A = 9, 11, 16
    idx = np.argsort(np.random.default_rng(32).random((T, E)), axis=1)[:, :K].astype(np.int32)
    hist = oracle.histogram(idx, E)
    replicas, slot_off, _, _ = oracle.plan(hist, S)
    _, row_pair, pair_row, _ = oracle.dispatch(None, idx, hist, replicas, slot_off, S, A)
    ctx = traced(monkeypatch, binding.Shape(T, D, 8, E, K, S, 0, A))
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the teams are those for 148 SMs")
    gen = torch.Generator(device=DEV).manual_seed(33)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(DEV)  # noqa: E731
    rows, at, pad = i32(pair_row).view(T, K), i32(pair_row).view(T, K).long(), i32(row_pair) < 0
    dout, wr, w, dl = rnd(T, D).to(torch.bfloat16), rnd(E, D).to(torch.bfloat16), torch.softmax(rnd(T, K), 1), rnd(T, K)
    buf = rnd(ctx.shape.Rcap, D).to(torch.bfloat16)
    buf[pad] = float("nan")
    dyp, dw, dx = torch.full_like(buf, 7.0), torch.full((T, K), float("nan"), device=DEV), torch.full_like(dout, float("nan"))
    capfd.readouterr()
    ctx.combine_backward(dout, buf, rows, w, dyp, dw)
    assert f"warps={warps[0]}\n" in capfd.readouterr().err
    assert torch.equal(dyp[at], (w[..., None] * dout[:, None].float()).to(torch.bfloat16)) and (dyp[pad] == 7).all()
    terms = buf[at].double() * dout[:, None].double()
    assert ((dw.double() - terms.sum(-1)).abs() <= (D / 32 + 8) * 2.0 ** -24 * terms.abs().sum(-1)).all()
    ctx.dispatch_backward(buf, rows, None, None, None, dx)
    assert f"warps={warps[1]}\n" in capfd.readouterr().err
    parts = buf[at].double()
    off = lambda p: (dx.double() - p.sum(1)).abs() - U * p.sum(1).abs() - 17 * 2.0 ** -24 * p.abs().sum(1)  # noqa: E731
    assert off(parts).max() <= 0
    ctx.dispatch_backward(buf, rows, i32(idx), dl, wr, dx)
    assert f"warps={warps[2]}\n" in capfd.readouterr().err
    assert off(torch.cat([parts, dl[..., None].double() * wr[i32(idx).long()].double()], 1)).max() <= 0
    ctx.check_status()
