"""The operators of 4-bit experts, as cases that can be timed and compared.

Two operators: an expert matrix rounded to 4 bits with a scale for each 32 weights and read back (`weights`), and the
experts' SwiGLU products on such weights over slots of any length, from the two or eight experts of a single token to long
prompts (`ffn`).  With `own` false they run in plain torch operations in 32 bits; with `own` true through the framework's
calls.
"""
import math

import torch

own = False

# tokens, width, hidden, experts, chosen, slots of the layers that the cases stand for
_TINY = dict(T=256, D=512, F=1024, E=8, K=2, S=8, zipf=1.0, align=16)
_RAGGED = dict(T=777, D=1000, F=1416, E=13, K=3, S=17, zipf=1.2, align=16)
_MIXTRAL = dict(D=4096, F=14336, E=8, K=2, align=16)
_MANY = dict(D=2048, F=1408, E=64, K=6, S=80, zipf=1.2, align=16)
_FINE = dict(D=7168, F=2048, E=256, K=8, S=288, zipf=1.0, align=16)
_BLOCK = 32       # weights along the contraction that share one scale
_CHUNK = 128      # a row of codes is whole chunks of so many weights
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)       # of the codes 0 to 7 (e2m1); codes 8 to 15 are their negatives


def listed():
    return [
        # one matrix of a unit-test sized layer: latency
        dict(name="weights tiny", op="weights", E=8, N=1024, C=512),
        # widths that neither a block nor a chunk divides
        dict(name="weights ragged", op="weights", E=13, N=1000, C=1416),
        # the gate matrices of a large layer, as they are laid out once when a model is loaded
        dict(name="weights mixtral", op="weights", E=8, N=14336, C=4096),
        # unit-test sized layer: latency
        dict(_TINY, name="ffn tiny", op="ffn"),
        # odd sizes, 13 experts of different loads, more than one row tile for some
        dict(_RAGGED, name="ffn ragged", op="ffn"),
        # one token being generated: two matrix-vector products through two large experts
        dict(_MIXTRAL, name="ffn mixtral 1 token", op="ffn", T=1, S=8, zipf=0.8),
        # the same through eight of 256 experts
        dict(_FINE, name="ffn fine_grained 1 token", op="ffn", T=1),
        # a small serving batch over many experts: most of them have a few rows
        dict(_MANY, name="ffn many_expert 48 tokens", op="ffn", T=48),
        # a serving batch over large experts: some 32 rows each
        dict(_MIXTRAL, name="ffn mixtral 128 tokens", op="ffn", T=128, S=8, zipf=0.8),
        # a prompt over 256 experts, most with fewer than 64 rows: weights and products weigh the same
        dict(_FINE, name="ffn fine_grained 4096 tokens", op="ffn", T=4096),
        # a batch of prompts over 64 experts
        dict(_MANY, name="ffn many_expert 8192 tokens", op="ffn", T=8192),
        # long prompts, 16 slots for 8 experts of very different loads: the largest work here
        dict(_MIXTRAL, name="ffn mixtral_skew 16384 tokens", op="ffn", T=16384, S=16, zipf=1.5),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if rng.random() < 0.25:
        while True:
            case = dict(op="weights", E=spread(1, 64), N=8 * spread(1, 1792), C=8 * spread(1, 1792))
            if case["E"] * case["N"] * case["C"] <= 8 * 14336 * 4096:
                return case
    while True:
        E = spread(2, 256)
        case = dict(op="ffn", T=spread(1, 16384), D=8 * spread(8, 896), F=8 * spread(8, 1792), E=E, K=rng.randint(1, min(8, E)),
                    S=E + rng.randint(0, max(1, E // 4)), zipf=round(rng.uniform(0.0, 1.5), 3), align=rng.choice([1, 16, 16, 128]))
        rows = case["T"] * case["K"]
        if (rows * case["D"] * case["F"] <= 32768 * 4096 * 14336 and E * case["D"] * case["F"] <= 256 * 2048 * 7168
                and rows * max(case["D"], case["F"]) <= 32768 * 14336):
            return case


def _selected(case, g, device):
    """The experts of each token: the largest of normal logits with popular experts ahead."""
    T, E, K = case["T"], case["E"], case["K"]
    bias = -case["zipf"] * torch.log(torch.randperm(E, generator=g, device=device).float() + 1)
    return torch.topk(torch.randn(T, E, generator=g, device=device) + bias, K, dim=1).indices


def work(case):
    if case["op"] == "weights":
        n = case["E"] * case["N"] * case["C"]
        return {"bytes": 4 * n + n // 2 + n // _BLOCK, "flops": 2 * n}
    R, D, F = case["T"] * case["K"], case["D"], case["F"]
    active = _selected(case, torch.Generator().manual_seed(0), "cpu").unique().numel()   # experts with rows, nearly the same for all seeds
    weights = 3 * active * D * F
    return {"bytes": 4 * R * D + weights // 2 + weights // _BLOCK, "flops": 6 * R * D * F}


# ------------------------------------------------------------------------------------------- inputs
def _normal(g, shape, std):
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 27):
        part = flat[lo:lo + (1 << 27)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda").mul_(std))
    return out


def _placement(case, idx):
    """The slot tables that plan and dispatch leave behind for these selections, and which rows hold a token."""
    E, S, A = case["E"], case["S"], case["align"]
    n = torch.bincount(idx.reshape(-1), minlength=E).tolist()
    copies = [1] * E
    for _ in range(S - E):                              # each spare slot to the largest load for each copy
        e = max(range(E), key=lambda i: (n[i] / copies[i], -copies[i], -i))
        copies[e] += 1
    off, expert, used = [0], [], []
    for e in range(E):
        for c in range(copies[e]):
            rows = (c + 1) * n[e] // copies[e] - c * n[e] // copies[e]
            expert.append(e)
            used.append((off[-1], off[-1] + rows))
            off.append(off[-1] + (rows + A - 1) // A * A)
    held = torch.zeros(case["T"] * case["K"] + S * (A - 1), dtype=torch.bool)
    for lo, hi in used:
        held[lo:hi] = True
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    extents = [(lo, hi, e) for e, lo, hi in zip(expert, off, off[1:]) if hi > lo]
    return dict(slot_row_off=ints(off), slot_expert=ints(expert), held=held.cuda(), extents=extents)


def _power(k, dtype):
    """2^k, exactly, for whole k >= -127."""
    bits = k.to(torch.int64)
    if dtype == torch.float64:
        return (bits + 1023 << 52).view(dtype)
    return torch.where(bits == -127, 1 << 22, bits + 127 << 23).to(torch.int32).view(dtype)      # 2^-127 is subnormal


def _to_4_bits(w):
    """(codes packed two to a byte, the even one low [rows, chunks * 64], scale bytes [rows, chunks * 4]) of w [rows, columns]."""
    rows, cols = w.shape
    blocks = torch.nn.functional.pad(w.float(), (0, -cols % _CHUNK)).view(rows, -1, _BLOCK)
    m, e = torch.frexp(blocks.abs().amax(-1))           # amax = m 2^e, 0.5 <= m < 1; 6 = 0.75 2^3
    k = torch.where(m == 0, torch.full_like(e, -127), (e - 3 + (m > 0.75).int()).clamp(-127, 125))
    v = blocks * _power(-k, torch.float32)[..., None]
    a = v.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)       # steps between neighbours; a tie goes to the even code
    for step, tie_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= step) if tie_up else (a > step)
    code += 8 * torch.signbit(v).to(torch.uint8)
    code = code.view(rows, -1, 2)
    return code[..., 0] | code[..., 1] << 4, (k + 127).to(torch.uint8)


def _from_4_bits(codes, scale, cols, dtype):
    """w [rows, columns] in `dtype`."""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), dtype=dtype, device=codes.device)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).view(codes.shape[0], -1, _BLOCK)
    return (v * _power(scale.long() - 127, dtype)[..., None]).reshape(codes.shape[0], -1)[:, :cols]


def _expert_matrix(g, E, N, C):
    """An expert matrix in 4 bits: codes [E, N, chunks * 64], scale bytes [E, N, chunks * 4]."""
    chunks = -(-C // _CHUNK)
    codes = torch.empty(E, N, chunks * _CHUNK // 2, dtype=torch.uint8, device="cuda")
    scale = torch.empty(E, N, chunks * _CHUNK // _BLOCK, dtype=torch.uint8, device="cuda")
    for e in range(E):
        codes[e], scale[e] = _to_4_bits(torch.randn(N, C, generator=g, device="cuda").mul_(0.02))
    return codes, scale


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "weights":
        return {"case": case, "w": _normal(g, (case["E"], case["N"], case["C"]), 0.02)}
    D, F, E = (case[k] for k in "DFE")
    s = {"case": case}
    s.update(_placement(case, _selected(case, g, "cuda")))
    s["xp"] = _normal(g, (s["held"].numel(), D), 1.0).mul_(s["held"][:, None])       # zero where no token sits
    for name, n, c in (("gate", F, D), ("up", F, D), ("down", D, F)):
        s[name], s[name + "_scale"] = _expert_matrix(g, E, n, c)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2506_07366_b200 import binding
        u8 = dict(dtype=torch.uint8, device="cuda")
        if case["op"] == "weights":                     # as the gate matrix of a layer of this size
            shape = binding.Shape(1, case["C"], case["N"], case["E"], 1, case["E"])
            codes, scale = shape.w4_shapes()
            s.update(ctx=binding.Context(shape), codes=torch.empty(codes, **u8), scale=torch.empty(scale, **u8),
                     back=torch.empty_like(s["w"]))
        else:
            T, D, F, E, K, S = (case[k] for k in "TDFEKS")
            shape = binding.Shape(T, D, F, E, K, S, 0, case["align"])
            s["ctx"] = binding.Context(shape)
            for name in ("gate", "up", "down"):
                s[name + "_scale"] = binding.w4_scale_tiles(s[name + "_scale"])
            s["yp"] = torch.zeros(shape.Rcap, D, dtype=torch.bfloat16, device="cuda")    # rows outside the slots are not written
            s["workspace"] = torch.empty(binding.expert_ffn4_workspace_bytes(shape), **u8)
    return s


# ------------------------------------------------------------------------------------------- one pass
def run(s):
    if s["case"]["op"] == "weights":
        return _own_weights(s) if own else _plain_weights(s)
    return _own_ffn(s) if own else _plain_ffn(s)


def _own_weights(s):
    s["ctx"].weights_quantize4(s["w"], s["codes"], s["scale"])
    s["ctx"].weights_dequantize4(s["codes"], s["scale"], s["back"])
    return s["back"]


def _own_ffn(s):
    s["ctx"].expert_ffn4(s["xp"], s["slot_row_off"], s["slot_expert"], s["gate"], s["up"], s["down"], s["gate_scale"],
                         s["up_scale"], s["down_scale"], s["yp"], s["workspace"])
    return s["yp"]


def _plain_weights(s):
    back = torch.empty_like(s["w"])
    for e, w in enumerate(s["w"]):
        back[e] = _from_4_bits(*_to_4_bits(w), w.shape[1], torch.float32)
    return back


def _plain_ffn(s):
    D, F = s["case"]["D"], s["case"]["F"]
    yp = torch.zeros_like(s["xp"])
    for lo, hi, e in s["extents"]:                       # the slots hold different numbers of rows
        x = s["xp"][lo:hi].float()
        g = x @ _from_4_bits(s["gate"][e], s["gate_scale"][e], D, torch.float32).T
        u = x @ _from_4_bits(s["up"][e], s["up_scale"][e], D, torch.float32).T
        yp[lo:hi] = (g * torch.sigmoid(g) * u) @ _from_4_bits(s["down"][e], s["down_scale"][e], F, torch.float32).T
    return yp


# ------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions in 64 bits: the nearest of the fifteen values, and the products of the experts."""
    s = _inputs(case, seed)
    d = torch.float64
    if case["op"] == "weights":
        back = torch.empty(s["w"].shape, dtype=d, device="cuda")
        for e in range(case["E"]):
            for lo in range(0, case["N"], 2048):
                w = s["w"][e, lo:lo + 2048].to(d)
                blocks = torch.zeros(w.shape[0], -(-w.shape[1] // _BLOCK) * _BLOCK, dtype=d, device="cuda")
                blocks[:, :w.shape[1]] = w
                blocks = blocks.unflatten(1, (-1, _BLOCK))
                top = blocks.abs().amax(-1, keepdim=True)
                m, k = torch.frexp(top / 6)              # m 2^k, 0.5 <= m < 1: the power of two at or above it
                unit = _power(torch.where(top > 0, k - (m == 0.5).int(), torch.zeros_like(k)), d)
                a = blocks.abs() / unit
                # spacing of the values: 1/2 below 2, 1 up to 4, 2 beyond; round() takes ties to the even multiple
                step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(d)
                near = torch.round(a / step) * step
                back[e, lo:lo + 2048] = (torch.sign(blocks) * near * unit).flatten(1)[:, :w.shape[1]]
        return back
    D, F = case["D"], case["F"]
    value = torch.tensor(_VALUES, dtype=d, device="cuda")

    def matrix(name, e, cols):
        c = s[name][e]
        both = torch.empty(c.shape[0], 2 * c.shape[1], dtype=torch.int64, device="cuda")
        both[:, 0::2], both[:, 1::2] = c.long() % 16, c.long() // 16
        w = value[both % 8] * (1 - 2 * (both // 8)).to(d)
        return (w * _power(s[name + "_scale"][e].long() - 127, d).repeat_interleave(_BLOCK, 1))[:, :cols]

    yp = torch.zeros(s["xp"].shape, dtype=d, device="cuda")
    last = None
    for lo, hi, e in s["extents"]:
        if e != last:
            gate, up, down, last = matrix("gate", e, D), matrix("up", e, D), matrix("down", e, F), e
        x = s["xp"][lo:hi].to(d)
        g = torch.einsum("rd,fd->rf", x, gate)
        h = g / (1 + torch.exp(-g)) * torch.einsum("rd,fd->rf", x, up)
        yp[lo:hi] = torch.einsum("rf,df->rd", h, down)
    return yp
