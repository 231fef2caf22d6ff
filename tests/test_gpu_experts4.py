"""Experts in 4 bits on the GPU: rounding and reading back (exact), the FFN on them, the layer.

Tolerances of the FFN, derived here and applied element by element (`bound`):
 - sums: an MMA adds 32 products and the accumulator, each cut off at 2^-24 of the largest, so at most 33 2^-24 of the sum of
   magnitudes S for each MMA; two MMAs for 32 inputs.
 - a row's values below 2^-15 of their block's largest are off by at most 2^-21 of that.
 - h is kept to 2^-9 relative (two e4m3 terms: a half step 2^-4 each, and half of that at the top of a binade), silu's exp and
   division to 2^-19 (26 ulp at |g| = 20); |silu'| <= 1.1.
 - y is rounded to bf16 once: 2^-8.
 - products, h and y below 2^-126 may vanish: sums of at most 2^13 of them, times weights below 2^6, stay below 2^-100.
The norm of the error over a whole output is asked to be below 2.6e-3 of the output's: independent roundings, uniform in a half
step, have a root mean square of at most 2^-8 / sqrt(3) (y) and 2^-9 / sqrt(3) (h), together 2.53e-3.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2506_07366_b200 import binding, workloads as wl
from paper_2506_07366_b200.layer import HostPipeline, MoeLayer, MoeLayer4
from tests import harness as hz

pytestmark = pytest.mark.gpu
DEV = "cuda"
F64 = torch.float64


def pair(shape, down=False, fill=0xEE):
    return tuple(torch.full(n, fill, dtype=torch.uint8, device=DEV) for n in shape.w4_shapes(down))


def normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------- weights
def special_matrix(E, N, C, seed):
    """Normal weights whose rows have scales over the whole range, ties, zero blocks, blocks with infinities and NaN."""
    rng = np.random.default_rng(seed)
    w = rng.standard_normal((E, N, C)) * 2.0 ** rng.integers(-12, 3, (E, N, 1))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    w[:, ::5] = rng.choice(ties, w[:, ::5].shape) * rng.choice([-1, 1], w[:, ::5].shape) * 2.0 ** -7
    w[:, 1::11] = 0.0
    w[:, 2::11] *= 2.0 ** -118
    w[:, 3::11] *= 2.0 ** 120
    t = torch.from_numpy(w.astype(np.float32)).to(torch.bfloat16)
    flat = t.view(-1)
    for v in (float("inf"), float("-inf"), float("nan"), 3.3e38, -2.0 ** -133, 2.0 ** -126):
        flat[int(rng.integers(flat.numel()))] = v
    return t


@pytest.mark.parametrize("E,D,F", [(1, 8, 8), (3, 136, 264), (2, 128, 384), (5, 40, 1000), (2, 1416, 24)])
@pytest.mark.parametrize("down", [False, True])
def test_quantize_and_back_are_exact(E, D, F, down):
    shape = binding.Shape(4, D, F, E, 1, E)
    ctx = binding.Context(shape)
    N, C = (D, F) if down else (F, D)
    w = special_matrix(E, N, C, 7 * E + D)
    code, scale = oracle.weights4_encode(w.double().numpy())
    codes, scales = oracle.weights4_pack(code, scale)
    w4, w4s = pair(shape, down)
    ctx.weights_quantize4(w.to(DEV), w4, w4s, down)
    assert np.array_equal(w4.cpu().numpy(), codes)
    assert np.array_equal(w4s.cpu().numpy(), scales)
    back = torch.full((E, N, C), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.weights_dequantize4(w4, w4s, back, down)
    ctx.check_status()
    want = oracle.weights4_decode(code, scale, C)
    assert np.array_equal(back.double().cpu().numpy(), want, equal_nan=True)
    assert ctx.launch_count() == 2


def test_refusals_of_the_weight_calls():
    shape = binding.Shape(4, 64, 96, 2, 1, 2)
    ctx = binding.Context(shape)
    w = torch.zeros(2, 96, 64, dtype=torch.bfloat16, device=DEV)
    w4, w4s = pair(shape)
    for bad in (lambda: ctx.weights_quantize4(w.float(), w4, w4s), lambda: ctx.weights_quantize4(w.cpu(), w4, w4s),
                lambda: ctx.weights_quantize4(w, w4.view(torch.int8), w4s)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ctx.weights_quantize4(w, w4, w4s, down=True), lambda: ctx.weights_quantize4(w, w4[:1], w4s),
                lambda: ctx.weights_quantize4(w, w4, w4s[..., :256]), lambda: ctx.weights_quantize4(None, w4, w4s),
                lambda: ctx.weights_dequantize4(w4, w4s, w.transpose(1, 2)), lambda: ctx.weights_dequantize4(w4, None, w)):
        with pytest.raises(ValueError):
            bad()
    shifted = torch.zeros(w4.numel() + 16, dtype=torch.uint8, device=DEV)[16:].view(w4.shape)
    with pytest.raises(binding.MoegpsError) as e:                      # 16-byte aligned is not enough for codes
        ctx.weights_quantize4(w, shifted, w4s)
    assert e.value.code == binding.ERR_INVALID_ARG
    assert ctx.launch_count() == 0


# ------------------------------------------------------------------------------------------- FFN
def slots(rows_of_slot, experts, align):
    off = [0]
    for r in rows_of_slot:
        off.append(off[-1] + (r + align - 1) // align * align)
    i32 = dict(dtype=torch.int32, device=DEV)
    return torch.tensor(off, **i32), torch.tensor(experts, **i32)


def make(shape, seed, std=0.05):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ctx = binding.Context(shape)
    packed, dense = [], []
    for n, c, down in ((shape.F, shape.D, False), (shape.F, shape.D, False), (shape.D, shape.F, True)):
        w = normal(g, shape.E, n, c, std=std)
        p = pair(shape, down)
        ctx.weights_quantize4(w, *p, down)
        ctx.weights_dequantize4(*p, w, down)
        packed.append(p)
        dense.append(w)
    ws = torch.full((binding.expert_ffn4_workspace_bytes(shape),), 0xFF, dtype=torch.uint8, device=DEV)
    return ctx, g, packed, dense, ws


def call(ctx, xp, off, expert, packed, yp, ws, stream=None):
    (g, gs), (u, us), (d, ds) = packed
    ctx.expert_ffn4(xp, off, expert, g, u, d, gs, us, ds, yp, ws, stream=stream)


def bound(x, wg, wu, wd):
    """(y, largest error) of one expert's rows in 64 bits; see the top of the file."""
    x, wg, wu, wd = (t.to(F64) for t in (x, wg, wu, wd))
    cut = lambda c: 2 * ((c + 31) // 32) * 33 * 2.0 ** -24  # noqa: E731
    small = 2.0 ** -21 * x.abs().amax(1, keepdim=True)
    off = lambda w: cut(x.shape[1]) * (x.abs() @ w.abs().T) + small * w.abs().sum(1)  # noqa: E731
    g, u, dg, du = x @ wg.T, x @ wu.T, off(wg), off(wu)
    h = g / (1 + torch.exp(-g)) * u
    silu = (g / (1 + torch.exp(-g))).abs()
    dh = 1.1 * dg * (u.abs() + du) + silu * du
    dh = dh + (2.0 ** -9 + 2.0 ** -18) * (h.abs() + dh) + 2.0 ** -21 * h.abs().amax(1, keepdim=True)
    y = h @ wd.T
    dy = dh @ wd.abs().T + cut(h.shape[1]) * ((h.abs() + dh) @ wd.abs().T)
    return y, dy + 2.0 ** -8 * (y.abs() + dy) + 2.0 ** -100


def check(xp, off, expert, dense, yp, fill, used=None):
    """Every row of every slot against the formula; rows outside the slots as they were."""
    off, expert = off.tolist(), expert.tolist()
    inside = torch.zeros(yp.shape[0], dtype=torch.bool, device=DEV)
    err = norm = 0.0
    for s, e in enumerate(expert):
        lo, hi = off[s], off[s + 1]
        if e < 0 or hi <= lo:
            continue
        inside[lo:hi] = True
        if used is not None:
            hi = lo + used[s]
        y, most = bound(xp[lo:hi], *(w[e] for w in dense))
        d = (yp[lo:hi].to(F64) - y).abs()
        assert torch.isfinite(d).all() and (d <= most).all(), (s, float((d / most).max()))
        err += float((d ** 2).sum())
        norm += float((y ** 2).sum())
    assert (yp[~inside] == fill).all()
    assert err ** 0.5 <= 2.6e-3 * norm ** 0.5


# rows of each slot: the shape's T * K of them in all, so that every choice that goes by rows per slot is met
CASES = [
    # one token: one and several experts
    dict(D=64, F=96, E=3, K=1, rows=[0, 1, 0], align=1),
    dict(D=512, F=1024, E=8, K=2, rows=[0, 1, 0, 0, 0, 0, 1, 0], align=16),
    # widths below a block, a chunk, a tile, and just above them
    dict(D=8, F=8, E=2, K=1, rows=[3, 2], align=1),
    dict(D=136, F=136, E=2, K=1, rows=[5, 9], align=4),
    dict(D=264, F=1000, E=4, K=2, rows=[7, 0, 16, 17], align=1),
    # a serving batch
    dict(D=512, F=640, E=6, K=2, rows=[31, 33, 0, 64, 65, 1], align=1),
    # more rows than a tile, slots that end inside one, long and short slots side by side
    dict(D=256, F=384, E=4, K=2, rows=[300, 1, 129, 210], align=1),
    dict(D=1000, F=1416, E=3, K=3, rows=[777, 0, 113], align=16),
    dict(D=128, F=128, E=2, K=1, rows=[2000, 48], align=128),
    # long slots over odd numbers of tiles, chunks and blocks
    dict(D=264, F=392, E=2, K=1, rows=[700, 31], align=1),
    dict(D=392, F=40, E=1, K=1, rows=[449], align=8),
    # long sums, few rows
    dict(D=4096, F=2048, E=2, K=1, rows=[1, 15], align=1),
    dict(D=24, F=7168, E=2, K=1, rows=[20, 4], align=8),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "D{D}-F{F}-E{E}-A{align}-".format(**c) + "_".join(map(str, c["rows"])))
def test_ffn_against_64_bits(c):
    total = sum(c["rows"])
    T = -(-total // c["K"])
    shape = binding.Shape(T, c["D"], c["F"], c["E"], c["K"], c["E"], 0, c["align"])
    ctx, g, packed, dense, ws = make(shape, 11)
    off, expert = slots(c["rows"], list(range(c["E"])), c["align"])
    xp = torch.full((shape.Rcap, shape.D), float("nan"), dtype=torch.bfloat16, device=DEV)
    for s, r in enumerate(c["rows"]):
        xp[int(off[s]):int(off[s]) + r] = normal(g, r, shape.D)
    yp = torch.full((shape.Rcap, shape.D), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    check(xp, off, expert, dense, yp, 13.0, used=c["rows"])
    again = torch.full_like(yp, 13.0)
    ws.fill_(0x3C)                                       # nothing depends on what the workspace held
    call(ctx, xp, off, expert, packed, again, ws)
    ctx.check_status()
    assert torch.equal(again.view(torch.int16), yp.view(torch.int16)) or torch.equal(
        again.nan_to_num(5.0), yp.nan_to_num(5.0))       # the same bits (rows of the padding may be any NaN)


@pytest.mark.parametrize("align", [1, 16])
def test_short_and_long_slots_in_one_call(align, monkeypatch, capfd):
    """Heavy weights, and some slots with more rows than the launch for short slots takes: both kinds of launches run.  Copies of an
    expert side by side, some short by themselves and long together, and apart."""
    monkeypatch.setenv("MOEGPS_TRACE", "1")
    rng = np.random.default_rng(4)
    E, S = 128, 160
    rows = [int(v) for v in rng.choice([0, 1, 5, 16, 17, 31, 32, 33, 47], S - 8)] + [49, 64, 112, 223, 224, 225, 500, 900]
    rng.shuffle(rows)
    experts = sorted(list(range(E)) + [int(v) for v in rng.integers(0, E, S - E)])
    experts[3], experts[150] = experts[150], experts[3]
    experts[20:40] = [7] * 20
    shape = binding.Shape(sum(rows), 2560, 4000, E, 1, S, 0, align)
    ctx, g, packed, dense, ws = make(shape, 31)
    off, expert = slots(rows, experts, align)
    xp = normal(g, shape.Rcap, shape.D)
    yp = torch.full((shape.Rcap, shape.D), 13.0, dtype=torch.bfloat16, device=DEV)
    capfd.readouterr()
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    launched = capfd.readouterr().err
    for kernel in ("launch_split", "launch_wide", "launch_short"):
        assert kernel in launched
    check(xp, off, expert, dense, yp, 13.0)


@pytest.mark.parametrize("align", [1, 4])
@pytest.mark.parametrize("rows,experts", [
    ([5, 9, 0, 30, 2, 40, 1, 3, 3, 0], [1, 1, 1, 1, 0, 2, 2, 1, 1, 1]),             # copies side by side, with empty ones, and apart
    ([20, 7, 0, 9, 11, 0, 6], [0, 0, -1, 0, 0, 2, 0]),                              # a slot without expert, another expert's empty one
    ([300, 500, 100, 1, 224, 224, 223], [2, 2, 0, 0, 1, 1, 1]),                     # long ones
    ([1] * 70 + [9, 8, 7, 0], [0] * 35 + [1] * 35 + [2, 2, 2, 2]),                  # more slots than a warp has lanes
])
def test_copies_side_by_side(rows, experts, align):
    shape = binding.Shape(sum(rows), 264, 392, 3, 1, len(rows), 0, align)
    ctx, g, packed, dense, ws = make(shape, 17)
    off, expert = slots(rows, experts, align)
    xp = normal(g, shape.Rcap, 264)
    yp = torch.full((shape.Rcap, 264), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    check(xp, off, expert, dense, yp, 13.0)


def test_values_over_a_wide_range():
    """Rows with magnitudes from 2^-60 to 2^30 beside each other, zero rows, single large values, weights with scales from 2^-40 up."""
    shape = binding.Shape(40, 256, 160, 2, 1, 2, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 3)
    for (w, p, down) in zip(dense, packed, (False, False, True)):
        w *= 2.0 ** torch.randint(-40, 3, (2, w.shape[1], 1), generator=g, device=DEV)
        ctx.weights_quantize4(w, *p, down)
        ctx.weights_dequantize4(*p, w, down)
    xp = normal(g, shape.Rcap, shape.D) * 2.0 ** torch.randint(-60, 30, (shape.Rcap, 1), generator=g, device=DEV)
    xp[3] = 0.0
    xp[4] = 0.0
    xp[4, 100] = 2.0 ** 40
    xp[5, ::7] *= 2.0 ** -20
    xp[6] = 2.0 ** -126
    xp = xp.to(torch.bfloat16)
    off, expert = slots([13, 27], [1, 0], 1)
    yp = torch.full((shape.Rcap, shape.D), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    check(xp, off, expert, dense, yp, 13.0)
    assert (yp[3] == 0).all()


def test_rows_that_are_not_finite_stay_apart():
    shape = binding.Shape(30, 200, 136, 2, 1, 2, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 5)
    xp = normal(g, 30, 200)
    off, expert = slots([17, 13], [0, 1], 1)
    yp = torch.zeros(30, 200, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    bad = xp.clone()
    bad[2, 150], bad[16, 0], bad[20, 199] = float("inf"), float("nan"), float("-inf")
    got = torch.zeros_like(yp)
    call(ctx, bad, off, expert, packed, got, ws)
    ctx.check_status()
    rows = torch.tensor([2, 16, 20], device=DEV)
    assert torch.isnan(got[rows]).all()
    keep = torch.ones(30, dtype=torch.bool, device=DEV)
    keep[rows] = False
    assert torch.equal(got[keep], yp[keep])


@pytest.mark.parametrize("T", [50, 700])                 # short and long slots
def test_the_result_over_its_rows(T):
    """yp = xp gives the same; in long slots too, rows that are not finite stay apart."""
    shape = binding.Shape(T, 200, 136, 2, 1, 2, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 15)
    xp = normal(g, T, 200)
    xp[7, 150], xp[T - 1, 0] = float("inf"), float("nan")
    off, expert = slots([T - 17, 17], [0, 1], 1)
    yp = torch.zeros_like(xp)
    call(ctx, xp, off, expert, packed, yp, ws)
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[[7, T - 1]] = False
    y, most = bound(xp[:T - 17], *(w[0] for w in dense))
    ok = keep[:T - 17]
    assert ((yp[:T - 17].to(F64) - y).abs() <= most)[ok].all()
    assert torch.isnan(yp[~keep]).all() and torch.isfinite(yp[keep]).all()
    call(ctx, xp, off, expert, packed, xp, ws)
    ctx.check_status()
    assert torch.equal(xp[keep], yp[keep]) and torch.isnan(xp[~keep]).all()


def test_weights_that_are_not_finite():
    """A NaN block makes its output NaN for that expert's rows, and no other output."""
    shape = binding.Shape(8, 64, 64, 2, 1, 2, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 6)
    dense[2][1, 40, 3] = float("nan")
    ctx.weights_quantize4(dense[2], *packed[2], True)
    xp = normal(g, 8, 64)
    off, expert = slots([4, 4], [0, 1], 1)
    yp = torch.zeros(8, 64, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    nan = torch.isnan(yp)
    assert nan[4:, 40].all() and int(nan.sum()) == 4


def test_slots_without_expert_and_bad_tables():
    """Empty copies, copies of one expert, extents outside the buffers, an expert that does not exist."""
    shape = binding.Shape(60, 72, 56, 3, 1, 6, 0, 4)
    ctx, g, packed, dense, ws = make(shape, 9)
    xp = normal(g, shape.Rcap, 72)
    i32 = dict(dtype=torch.int32, device=DEV)
    off = torch.tensor([0, 20, 20, 24, 30, 44, 60], **i32)
    expert = torch.tensor([2, 0, -1, 1, 2, 2], **i32)
    yp = torch.full((shape.Rcap, 72), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    check(xp, off, expert, dense, yp, 13.0)
    for bad_off, bad_expert, good in (([0, 20, 10, 24, 30, 44, 60], expert.tolist(), (0, 2, 3, 4, 5)),
                                      ([0, 20, 24, 30, 44, 50, shape.Rcap + 1], expert.tolist(), (0, 1, 3, 4)),
                                      ([0, 20, 24, 30, 44, 50, -3], expert.tolist(), (0, 1, 3, 4)),
                                      ([-8, 20, 24, 30, 44, 50, 60], expert.tolist(), (1, 3, 4, 5)),
                                      (off.tolist(), [2, 0, -1, 1, 3, 2], (0, 3, 5))):
        yp.fill_(13.0)
        call(ctx, xp, torch.tensor(bad_off, **i32), torch.tensor(bad_expert, **i32), packed, yp, ws)
        assert ctx.status() == binding.ERR_BAD_INDEX
        want = torch.full_like(yp, 13.0)
        for s in good:
            if bad_expert[s] >= 0 and bad_off[s + 1] > bad_off[s]:
                lo, hi = bad_off[s], bad_off[s + 1]
                y, most = bound(xp[lo:hi], *(w[bad_expert[s]] for w in dense))
                assert ((yp[lo:hi].to(F64) - y).abs() <= most).all(), (bad_off, s)
                yp[lo:hi] = 13.0
        assert torch.equal(yp, want)


@pytest.mark.parametrize("T,rows", [(64, 60), (3000, 2900), (12000, 11900)])
def test_overlapping_slots_stay_inside_the_workspace(T, rows):
    """Tables that no plan makes: every other slot is the same rows.  More tiles than there is room for are left out and
    reported; the first slots are right, and nothing behind the workspace or the result is touched."""
    S = 40
    shape = binding.Shape(T, 128, 128, 1, 1, S, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 8)
    xp = normal(g, shape.Rcap, 128)
    off = torch.tensor([0, rows] * (S // 2) + [0], dtype=torch.int32, device=DEV)
    expert = torch.zeros(S, dtype=torch.int32, device=DEV)
    room = torch.full((ws.numel() + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
    out = torch.full((shape.Rcap + 500, 128), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, out[:shape.Rcap], room[:ws.numel()])
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert (room[ws.numel():] == 0x5A).all() and (out[rows:] == 13.0).all()
    y, most = bound(xp[:rows], *(w[0] for w in dense))
    assert ((out[:rows].to(F64) - y).abs() <= most).all()


def test_overlapping_slots_whose_sum_passes_32_bits():
    """Half of 1024 slots are the same 16.7 million rows each: in the units of 64 to a tile in which they are dealt their sum is above 2^31."""
    T, S = 1 << 21, 1024
    shape = binding.Shape(T, 8, 8, 8, 8, S, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 9)
    rows = shape.Rcap - 100
    assert S // 2 * (-(-rows // 224) * 64) > 2 ** 31
    xp = normal(g, shape.Rcap, 8)
    off = torch.tensor([0, rows] * (S // 2) + [0], dtype=torch.int32, device=DEV)
    expert = torch.zeros(S, dtype=torch.int32, device=DEV)
    out = torch.full((shape.Rcap, 8), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, out, ws)
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert (out[rows:] == 13.0).all()
    for lo in (0, rows // 2, rows - 500):
        y, most = bound(xp[lo:lo + 500], *(w[0] for w in dense))
        assert ((out[lo:lo + 500].to(F64) - y).abs() <= most).all()


def test_refusals_of_the_ffn():
    shape = binding.Shape(6, 64, 96, 2, 1, 2, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 1)
    n0 = ctx.launch_count()
    off, expert = slots([3, 3], [0, 1], 1)
    xp = normal(g, 6, 64)
    yp = torch.zeros(6, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(binding.MoegpsError) as e:
        call(ctx, xp, off, expert, packed, yp, ws[:-1])
    assert e.value.code == binding.ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(TypeError):
        call(ctx, xp.float(), off, expert, packed, yp, ws)
    with pytest.raises(ValueError):
        call(ctx, xp[:5], off, expert, packed, yp, ws)
    with pytest.raises(ValueError):
        call(ctx, xp, off, expert, [packed[2], packed[1], packed[0]], yp, ws)
    codes = torch.zeros(packed[0][0].numel() + 16, dtype=torch.uint8, device=DEV)[16:].view(packed[0][0].shape)
    with pytest.raises(binding.MoegpsError) as e:
        call(ctx, xp, off, expert, [(codes, packed[0][1]), packed[1], packed[2]], yp, ws)
    assert e.value.code == binding.ERR_INVALID_ARG
    assert ctx.launch_count() == n0
    empty = binding.Shape(0, 64, 96, 2, 1, 2, 0, 1)
    c0 = binding.Context(empty)
    none = torch.zeros(0, 64, dtype=torch.bfloat16, device=DEV)
    call(c0, none, torch.zeros(3, dtype=torch.int32, device=DEV), expert, packed, none, ws)
    assert c0.launch_count() == 0


def test_two_streams_and_a_graph():
    """Two contexts on two streams at once, and captured calls replayed with other rows, tables and weights."""
    shape = binding.Shape(96, 256, 384, 4, 1, 4, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 21)
    other, ws2 = binding.Context(shape), torch.empty_like(ws)
    off, expert = slots([50, 3, 0, 43], [0, 1, 2, 3], 1)
    xa, xb = normal(g, 96, 256), normal(g, 96, 256)
    ya, yb = (torch.full((96, 256), 13.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        call(ctx, xa, off, expert, packed, ya, ws, stream=s1)
        call(other, xb, off, expert, packed, yb, ws2, stream=s2)
    torch.cuda.synchronize()
    check(xa, off, expert, dense, ya, 13.0)
    check(xb, off, expert, dense, yb, 13.0)
    ctx.check_status()
    other.check_status()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ctx, xa, off, expert, packed, ya, ws)
    for rows in ([50, 3, 0, 43], [0, 0, 96, 0], [1, 0, 0, 0]):
        new_off, _ = slots(rows, [0, 1, 2, 3], 1)
        off.copy_(new_off)
        xa.copy_(normal(g, 96, 256))
        w = normal(g, *dense[0].shape, std=0.05)
        ctx.weights_quantize4(w, *packed[0])
        ctx.weights_dequantize4(*packed[0], dense[0])
        ya.fill_(13.0)
        graph.replay()
        ctx.check_status()
        check(xa, off, expert, dense, ya, 13.0)


@pytest.mark.parametrize("rows", [[50, 3, 0, 43], [700, 1, 0, 500]])          # short and long slots
def test_one_context_on_two_streams_and_in_two_branches_of_a_graph(rows):
    """Calls that overlap, each with its workspace; the context's first call is a captured one."""
    T = sum(rows)
    shape = binding.Shape(T, 256, 384, 4, 1, 4, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 22)
    ctx = binding.Context(shape)
    off, expert = slots(rows, [0, 1, 2, 3], 1)
    x = [normal(g, T, 256) for _ in range(2)]
    y = [torch.full((T, 256), 13.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    w = [ws, torch.empty_like(ws)]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        for i, stream in enumerate((here, side)):
            call(ctx, x[i], off, expert, packed, y[i], w[i], stream=stream)
        here.wait_stream(side)
    for _ in range(10):
        graph.replay()
    torch.cuda.synchronize()
    ctx.check_status()
    captured = [v.clone() for v in y]
    for i in range(2):
        check(x[i], off, expert, dense, y[i], 13.0)
        y[i].fill_(13.0)
    streams = [torch.cuda.Stream(), side]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            call(ctx, x[i], off, expert, packed, y[i], w[i], stream=streams[i])
    torch.cuda.synchronize()
    ctx.check_status()
    assert all(torch.equal(a, b) for a, b in zip(y, captured))


# ------------------------------------------------------------------------------------------- layer
LAYERS = [
    (wl.WORKLOADS["tiny"].scaled(sigma_x=1.0, S=11), 16),
    (wl.WORKLOADS["many_expert"].scaled(T=1, D=264, F=104, E=24, K=6, S=30), 1),
    (wl.WORKLOADS["fine_grained"].scaled(T=200, D=448, F=136, E=40, K=8, S=50), 128),
]


@pytest.mark.parametrize("w,A", LAYERS, ids=lambda v: v if isinstance(v, int) else v.name)
def test_layer(w, A):
    """Route, dispatch, FFN and combine together, as they are used; the same layer on the weights that the codes stand for."""
    wr, bias = wl.router(w, "cpu")
    x, _ = hz.screened_activations(w, wr, bias)
    ws = wl.expert_weights(w, "cpu")
    shape = binding.Shape(w.T, w.D, w.F, w.E, w.K, w.S, w.gate_mode, A)
    layer = MoeLayer4(shape, wr.to(DEV), bias.to(DEV), *(v.to(DEV) for v in ws))
    idx, _, _ = oracle.route(hz.bits(x), hz.bits(wr), bias.numpy(), w.K, w.gate_mode)
    layer.plan(torch.from_numpy(oracle.histogram(idx, w.E)))
    layer.xp.fill_(float("nan"))
    out = layer.forward(x.to(DEV)).clone()
    layer.ctx.check_status()
    dense = layer.dense_experts()
    for v, d in zip(ws, dense):
        code, scale = oracle.weights4_encode(v.double().numpy())
        assert np.array_equal(d.double().cpu().numpy(), oracle.weights4_decode(code, scale, v.shape[-1]))
    ref = oracle.moe_layer(hz.bits(x), hz.bits(wr), bias.numpy(), *(hz.bits(d) for d in dense), layer.pred.cpu().numpy(), K=w.K,
                           S=w.S, gate_mode=w.gate_mode, row_align=A)
    got = out.double().cpu().numpy()
    # yp and out are rounded to bf16 and h to 2^-9, independently: (2 * 2^-16 + 2^-18)^(1/2) / sqrt(3)
    assert np.isfinite(got).all() and np.linalg.norm(got - ref["out"]) <= 3.5e-3 * np.linalg.norm(ref["out"])
    plain = MoeLayer(shape, wr.to(DEV), bias.to(DEV), *dense)
    plain.plan(layer.pred)
    same = plain.forward(x.to(DEV)).double().cpu().numpy()
    assert np.linalg.norm(got - same) <= 8e-3 * np.linalg.norm(same)
    again = MoeLayer4(shape, wr.to(DEV), bias.to(DEV), layer.w_gate, layer.w_up, layer.w_down)
    again.plan(layer.pred)
    assert torch.equal(again.forward(x.to(DEV)), out)
    graph = again.capture(x.to(DEV))
    again.out.zero_()
    graph.replay()
    assert torch.equal(again.out, out)
    host_in, host_out = x.pin_memory(), torch.empty(x.shape, dtype=torch.bfloat16).pin_memory()
    pipe = HostPipeline(layer)
    for _ in range(3):
        pipe.submit(host_in, host_out)
    pipe.drain()
    torch.cuda.synchronize()
    assert torch.equal(host_out, out.cpu())
    layer.ctx.check_status()


def test_large_layer_by_slots():
    """Long slots and single rows over wide experts, 64 bits on the GPU."""
    shape = binding.Shape(1200, 2048, 1408, 4, 2, 8, 0, 16)
    ctx, g, packed, dense, ws = make(shape, 77, std=0.02)
    rows = [1000, 500, 1, 17, 0, 600, 250, 32]
    off, expert = slots(rows, [0, 0, 1, 1, 2, 2, 3, 3], 16)
    xp = normal(g, shape.Rcap, 2048)
    yp = torch.full((shape.Rcap, 2048), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    check(xp, off, expert, dense, yp, 13.0)


@pytest.mark.parametrize("D,F", [(4096, 264), (520, 4096)])
def test_runs_worked_in_groups_of_rows(D, F):
    """Runs whose rows do not stay in L2 together, over several tiles of outputs: 4096 inputs in groups of 13 row tiles, the last
    group not full, its last tile neither.  The first size meets it in gate + up, the second in down."""
    rows = [7000, 0, 2912, 13]
    shape = binding.Shape(sum(rows), D, F, 2, 1, 4, 0, 1)
    ctx, g, packed, dense, ws = make(shape, 41, std=0.02)
    off, expert = slots(rows, [0, 1, 1, 0], 1)
    xp = normal(g, shape.Rcap, D)
    yp = torch.full((shape.Rcap, D), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    check(xp, off, expert, dense, yp, 13.0)


@pytest.mark.parametrize("align", [1, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("T", [1, 40])
def test_few_tokens_at_any_alignment(align, T):
    """Slots that hold a row or two each, of weights that are read in 40 us: all ways that the alignment leads to."""
    shape = binding.Shape(T, 1024, 2560, 64, 4, 70, 0, align)
    ctx, g, packed, dense, ws = make(shape, 51, std=0.03)
    counts = torch.bincount(torch.randint(0, 70, (4 * T,), generator=g, device=DEV), minlength=70).tolist()
    experts = sorted(list(range(64)) + [3, 3, 3, 10, 10, 63])
    off, expert = slots(counts, experts, align)
    xp = torch.zeros(shape.Rcap, 1024, dtype=torch.bfloat16, device=DEV)
    for s, n in enumerate(counts):
        xp[int(off[s]):int(off[s]) + n] = normal(g, n, 1024)
    yp = torch.full((shape.Rcap, 1024), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    check(xp, off, expert, dense, yp, 13.0, used=counts)


@pytest.mark.parametrize("most", [3, 40])                # below and above what heavy weights turn to launches of both kinds at
def test_many_experts_of_heavy_weights(most):
    shape_of = lambda T: binding.Shape(T, 2560, 4000, 128, 1, 128, 0, 1)  # noqa: E731
    rng = np.random.default_rng(most)
    rows = [int(v) for v in rng.integers(0, most + 1, 126)] + [50, 130]
    shape = shape_of(sum(rows))
    ctx, g, packed, dense, ws = make(shape, 52)
    off, expert = slots(rows, [int(v) for v in rng.permutation(128)], 1)
    xp = normal(g, shape.Rcap, shape.D)
    yp = torch.full((shape.Rcap, shape.D), 13.0, dtype=torch.bfloat16, device=DEV)
    call(ctx, xp, off, expert, packed, yp, ws)
    ctx.check_status()
    assert ctx.launch_count() - 6 == (1 if sum(rows) <= 128 * 12 else 4)
    check(xp, off, expert, dense, yp, 13.0)
