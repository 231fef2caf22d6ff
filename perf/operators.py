"""The operators of the layer's training step, as cases that can be timed and compared.

Five operators: the gate+up product that keeps its activations in 8 bits (`save`), the gradient of the experts'
products that reads them (`backward`), and the gradients of the weighted way back to token order (`combine`), of the
sorting by expert (`dispatch`) and of the router (`route`).  With `own` false they run in plain torch operations in 32
bits; with `own` true through the framework's calls.
"""
import math

import torch

own = False

# (tokens, width, hidden, experts, chosen, slots, gate mode) of the layers that the cases stand for
_TINY = dict(T=256, D=512, F=1024, E=8, K=2, S=8, mode=0, zipf=1.0)
_RAGGED = dict(T=777, D=1000, F=1416, E=13, K=3, S=17, mode=1, zipf=1.2)
_MANY = dict(T=8192, D=2048, F=1408, E=64, K=6, S=80, mode=0, zipf=1.2)
_SKEW = dict(T=16384, D=4096, F=14336, E=8, K=2, S=16, mode=0, zipf=1.5)
_FINE = dict(T=4096, D=7168, F=2048, E=256, K=8, S=288, mode=1, zipf=1.0)
_ALIGN = 16       # slots start at multiples of 16 rows, as in the framework's layer
_BLOCK = 32       # columns that share one scale in the 8-bit activations


def listed():
    return [
        # a debugging or unit-test sized layer: the call's own latency counts
        dict(_TINY, name="save tiny", op="save"),
        # 64 small experts: the kept activations are written next to a short product
        dict(_MANY, name="save many_expert", op="save"),
        # small layer: launches and latency
        dict(_TINY, name="backward tiny", op="backward"),
        # widths that no tile divides, experts with few rows, a last partial block of 32 columns
        dict(_RAGGED, name="backward ragged", op="backward"),
        # 64 small experts of very different loads, 16 of the slots copies of popular ones
        dict(_MANY, name="backward many_expert", op="backward"),
        # two large popular experts among eight, 16 slots: the largest work here
        dict(_SKEW, name="backward mixtral_skew", op="backward"),
        # small batch: latency
        dict(_TINY, name="combine tiny", op="combine"),
        # eight rows for each token, wide: memory
        dict(_FINE, name="combine fine_grained", op="combine"),
        # odd sizes, with the router's part of the gradient
        dict(_RAGGED, name="dispatch ragged", op="dispatch", router=True),
        # long batch, two rows for each token, router frozen
        dict(_SKEW, name="dispatch mixtral_skew", op="dispatch", router=False),
        # softmax gates over 6 of 64 experts
        dict(_MANY, name="route many_expert", op="route"),
        # sigmoid gates over 8 of 256 experts: the selected logits come into it
        dict(_FINE, name="route fine_grained", op="route"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["save", "backward", "combine", "dispatch", "route"])
    products = op in ("save", "backward")
    while True:
        E = spread(2, 64 if products else 256)
        case = dict(op=op, T=spread(1, 16384), D=8 * spread(8, 896), F=8 * spread(8, 1792), E=E, K=rng.randint(1, min(8, E)),
                    S=E + rng.randint(0, max(1, E // 4)), mode=rng.randint(0, 1), zipf=round(rng.uniform(0.0, 1.5), 3))
        rows = case["T"] * case["K"]
        if products and (rows * case["D"] * case["F"] > 32768 * 4096 * 14336 or E * case["D"] * case["F"] > 8 * 4096 * 14336
                         or rows * case["F"] > 32768 * 14336):
            continue
        if rows * case["D"] > 4096 * 8 * 7168:
            continue
        if op == "dispatch":
            case["router"] = rng.random() < 0.5
        return case


def work(case):
    T, D, F, E, K = (case[k] for k in "TDFEK")
    R = T * K
    active = min(E, R)                                   # experts that can have rows
    kept = 2 * R * F + 2 * R * ((F + _BLOCK - 1) // _BLOCK)
    if case["op"] == "save":
        return {"bytes": 2 * R * D + 4 * active * F * D + 2 * R * F + kept, "flops": 4 * R * D * F}
    if case["op"] == "backward":
        return {"bytes": 6 * R * D + kept + 6 * active * F * D + 6 * E * F * D, "flops": 12 * R * D * F}
    if case["op"] == "combine":
        return {"bytes": 2 * T * D + 4 * R * D + 12 * R, "flops": 3 * R * D}
    if case["op"] == "dispatch":
        more = 8 * R + 2 * active * D if case["router"] else 0
        return {"bytes": 2 * R * D + 2 * T * D + 4 * R + more, "flops": (3 if case["router"] else 1) * R * D}
    scores = 2 * active * D if case["mode"] == 1 else 0
    return {"bytes": 2 * T * D + 4 * E * D + 16 * R + scores, "flops": (4 if case["mode"] == 1 else 2) * R * D}


# ------------------------------------------------------------------------------------------- inputs
def _normal(g, shape, std, dtype=torch.bfloat16):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 27):
        part = flat[lo:lo + (1 << 27)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda").mul_(std))
    return out


def _routing(case, g, x, w_router, bias):
    """Selected experts and their gate weights, from the router's own logits (or, without one, from normal ones)."""
    T, E, K = case["T"], case["E"], case["K"]
    logits = torch.randn(T, E, generator=g, device="cuda") if x is None else x.float() @ w_router.float().T
    top, idx = torch.topk(logits + bias, K, dim=1)
    s = torch.sigmoid(top)
    w = torch.softmax(top, dim=1) if case["mode"] == 0 else s / s.sum(1, keepdim=True)
    return idx.to(torch.int32), w


def _placement(case, idx):
    """The tables that plan and dispatch leave behind for these selections."""
    T, E, K, S = (case[k] for k in "TEKS")
    flat = idx.reshape(-1).long()
    n = torch.bincount(flat, minlength=E).tolist()
    copies = [1] * E
    for _ in range(S - E):                              # each spare slot to the largest load for each copy
        e = max(range(E), key=lambda i: (n[i] / copies[i], -copies[i], -i))
        copies[e] += 1
    starts, slot_off, slot_expert, slot_row_off, begin = [], [0], [], [0], []
    for e in range(E):
        for c in range(copies[e]):
            first, last = c * n[e] // copies[e], (c + 1) * n[e] // copies[e]
            begin.append(first)
            slot_expert.append(e)
            slot_row_off.append(slot_row_off[-1] + (last - first + _ALIGN - 1) // _ALIGN * _ALIGN)
        slot_off.append(len(slot_expert))
    dev = dict(device="cuda")
    count, first_pair = torch.tensor(n, **dev), torch.tensor([0] + n, **dev).cumsum(0)
    order = torch.argsort(flat, stable=True)
    rank = torch.empty_like(flat)
    rank[order] = torch.arange(T * K, **dev) - first_pair[flat[order]]
    r = torch.tensor(copies, **dev)[flat]
    slot = torch.tensor(slot_off, **dev)[flat] + ((rank + 1) * r - 1) // count[flat].clamp(min=1)
    row = torch.tensor(slot_row_off, **dev)[slot] + rank - torch.tensor(begin, **dev)[slot]
    row_pair = torch.full((T * K + S * (_ALIGN - 1),), -1, dtype=torch.int32, device="cuda")
    row_pair[row] = torch.arange(T * K, dtype=torch.int32, **dev)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, **dev)  # noqa: E731
    return dict(pair_row=row.to(torch.int32).view(T, K), row_pair=row_pair, slot_off=ints(slot_off), slot_expert=ints(slot_expert),
                slot_row_off=ints(slot_row_off), extents=[(slot_row_off[slot_off[e]], slot_row_off[slot_off[e + 1]]) for e in range(E)])


def _to_8_bits(v):
    """(codes e4m3 [rows, blocks * 32], scale bytes [blocks, rows]) of v [rows, columns] fp32: 32 columns of a row share one."""
    rows, cols = v.shape
    blocks = torch.nn.functional.pad(v, (0, -cols % _BLOCK)).view(rows, -1, _BLOCK)
    m, e = torch.frexp(blocks.abs().amax(-1))           # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    k = torch.where(m == 0, torch.full_like(e, -127), (e - 9 + (m > 0.875).int()).clamp(-127, 127))
    codes = torch.ldexp(blocks, -k[..., None]).to(torch.float8_e4m3fn).view(rows, -1)
    return codes, (k + 127).to(torch.uint8).T


def _from_8_bits(codes, scale, cols, dtype):
    v = codes.view(torch.float8_e4m3fn).to(dtype).view(codes.shape[0], -1, _BLOCK)
    return torch.ldexp(v, scale.T.to(torch.int32)[..., None] - 127).reshape(codes.shape[0], -1)[:, :cols]


def _rows_by_expert(case, g, p, width, std):
    """Rows in slot order, zero where no token sits."""
    rows = _normal(g, (p["row_pair"].numel(), width), std)
    return rows.mul_((p["row_pair"] >= 0)[:, None])


def _inputs(case, seed):
    T, D, F, E, K, S = (case[k] for k in "TDFEKS")
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    bias = -case["zipf"] * torch.log(torch.randperm(E, generator=g, device="cuda").float() + 1)
    x = w_router = None
    if case["op"] == "route":
        x, w_router = _normal(g, (T, D), 1.0), _normal(g, (E, D), 1 / math.sqrt(D))
    s["topk_idx"], s["topk_w"] = _routing(case, g, x, w_router, bias)
    s.update(x=x, w_router=w_router, bias=bias)
    s.update(_placement(case, s["topk_idx"]))
    if case["op"] in ("save", "backward"):
        s["xp"] = _rows_by_expert(case, g, s, D, 1.0)
        s["w_gate"], s["w_up"] = _normal(g, (E, F, D), 0.02), _normal(g, (E, F, D), 0.02)
    if case["op"] == "backward":
        s["w_down"] = _normal(g, (E, D, F), 0.02)
        s["dyp"] = _rows_by_expert(case, g, s, D, 0.01)
        std = 0.02 * math.sqrt(D)                        # what the gate and up products of such rows spread over
        for name in ("gate", "up"):
            wide = -(-F // _BLOCK) * _BLOCK
            codes = torch.empty(s["xp"].shape[0], wide, dtype=torch.uint8, device="cuda")
            scale = torch.empty(wide // _BLOCK, s["xp"].shape[0], dtype=torch.uint8, device="cuda")
            for lo in range(0, codes.shape[0], 4096):
                hi = min(lo + 4096, codes.shape[0])
                v = torch.randn(hi - lo, F, generator=g, device="cuda").mul_(std).mul_((s["row_pair"][lo:hi] >= 0)[:, None])
                c, k = _to_8_bits(v)
                codes[lo:hi], scale[:, lo:hi] = c.view(torch.uint8), k
            s[name + "8"], s[name + "_scale"] = codes, scale
    if case["op"] == "combine":
        s["dout"], s["yp"] = _normal(g, (T, D), 0.01), _rows_by_expert(case, g, s, D, 0.5)
    if case["op"] == "dispatch":
        s["dxp"] = _rows_by_expert(case, g, s, D, 0.01)
        s["dlogit"] = s["w_router"] = None
        if case["router"]:
            s["dlogit"] = torch.randn(T, K, generator=g, device="cuda").mul_(0.01)
            s["w_router"] = _normal(g, (E, D), 1 / math.sqrt(D))
    if case["op"] == "route":
        s["dtopk_w"] = torch.randn(T, K, generator=g, device="cuda").mul_(0.01)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2506_07366_b200 import binding
        T, D, F, E, K, S = (case[k] for k in "TDFEKS")
        shape = binding.Shape(T, D, F, E, K, S, case["mode"], _ALIGN)
        s["ctx"] = binding.Context(shape)
        rows, wide = shape.Rcap, -(-F // _BLOCK) * _BLOCK
        bf, u8 = dict(dtype=torch.bfloat16, device="cuda"), dict(dtype=torch.uint8, device="cuda")
        fl = dict(dtype=torch.float32, device="cuda")
        if case["op"] == "save":                        # rows that hold no token are not written
            s["h"] = torch.zeros(rows, F, **bf)
            for name in ("gate", "up"):
                s[name + "8"] = torch.zeros(rows, wide, **u8)
                s[name + "_scale"] = torch.zeros(wide // _BLOCK, rows, **u8)
        if case["op"] == "backward":
            s["dgate"], s["dup"], s["h"] = (torch.empty(rows, F, **bf) for _ in range(3))
            s["dxp"] = torch.zeros(rows, D, **bf)
            s["dw_gate"], s["dw_up"], s["dw_down"] = (torch.empty_like(s[k]) for k in ("w_gate", "w_up", "w_down"))
        if case["op"] == "combine":
            s["dyp"], s["dtopk_w"] = torch.zeros(rows, D, **bf), torch.empty(T, K, **fl)
        if case["op"] == "dispatch":
            s["dx"] = torch.empty(T, D, **bf)
        if case["op"] == "route":
            s["dlogit"], s["dw_router"], s["dbias"] = torch.empty(T, K, **fl), torch.empty(E, D, **fl), torch.empty(E, **fl)
            s["workspace"] = torch.empty(binding.route_backward_workspace_bytes(shape), **u8)
    return s


# ------------------------------------------------------------------------------------------- one pass
def run(s):
    return (_RUN_OWN if own else _RUN_PLAIN)[s["case"]["op"]](s)


def _own_save(s):
    s["ctx"].expert_ffn_gate_up_save(s["xp"], s["slot_row_off"], s["slot_expert"], s["w_gate"], s["w_up"], s["h"], s["gate8"],
                                     s["up8"], s["gate_scale"], s["up_scale"])
    return (s["h"], s["gate8"].view(torch.float8_e4m3fn), s["up8"].view(torch.float8_e4m3fn),
            s["gate_scale"].view(torch.float8_e8m0fnu), s["up_scale"].view(torch.float8_e8m0fnu))


def _own_backward(s):
    s["ctx"].expert_ffn_backward(s["dyp"], s["xp"], s["slot_row_off"], s["slot_off"], s["slot_expert"], s["row_pair"], s["w_gate"],
                                 s["w_up"], s["w_down"], s["gate8"], s["up8"], s["gate_scale"], s["up_scale"], s["dgate"],
                                 s["dup"], s["h"], s["dxp"], s["dw_gate"], s["dw_up"], s["dw_down"])
    return s["dxp"], s["dw_gate"], s["dw_up"], s["dw_down"]


def _own_combine(s):
    s["ctx"].combine_backward(s["dout"], s["yp"], s["pair_row"], s["topk_w"], s["dyp"], s["dtopk_w"])
    return s["dyp"], s["dtopk_w"]


def _own_dispatch(s):
    s["ctx"].dispatch_backward(s["dxp"], s["pair_row"], s["topk_idx"], s["dlogit"], s["w_router"], s["dx"])
    return s["dx"]


def _own_route(s):
    s["ctx"].route_backward(s["x"], s["w_router"], s["bias"], s["topk_idx"], s["topk_w"], s["dtopk_w"], s["slot_row_off"],
                            s["slot_off"], s["row_pair"], s["dlogit"], s["dw_router"], s["dbias"], s["workspace"])
    return s["dlogit"], s["dw_router"], s["dbias"]


def _plain_save(s):
    xp, F = s["xp"], s["w_gate"].shape[1]
    rows, wide = xp.shape[0], -(-F // _BLOCK) * _BLOCK
    h = torch.zeros(rows, F, dtype=torch.bfloat16, device="cuda")
    codes = torch.zeros(2, rows, wide, dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.zeros(2, wide // _BLOCK, rows, dtype=torch.uint8, device="cuda")
    for e, (lo, hi) in enumerate(s["extents"]):          # the experts hold different numbers of rows
        if hi > lo:
            x = xp[lo:hi].float()
            g, u = x @ s["w_gate"][e].float().T, x @ s["w_up"][e].float().T
            h[lo:hi] = g * torch.sigmoid(g) * u
            codes[0, lo:hi], scale[0, :, lo:hi] = _to_8_bits(g)
            codes[1, lo:hi], scale[1, :, lo:hi] = _to_8_bits(u)
    return h, codes[0], codes[1], scale[0].view(torch.float8_e8m0fnu), scale[1].view(torch.float8_e8m0fnu)


def _plain_backward(s):
    F = s["w_gate"].shape[1]
    dxp = torch.zeros_like(s["xp"])
    dw_gate, dw_up, dw_down = (torch.empty_like(s[k]) for k in ("w_gate", "w_up", "w_down"))
    for e, (lo, hi) in enumerate(s["extents"]):
        x, dy = s["xp"][lo:hi].float(), s["dyp"][lo:hi].float()
        g = _from_8_bits(s["gate8"][lo:hi], s["gate_scale"][:, lo:hi], F, torch.float32)
        u = _from_8_bits(s["up8"][lo:hi], s["up_scale"][:, lo:hi], F, torch.float32)
        sig = torch.sigmoid(g)
        act = g * sig
        dh = dy @ s["w_down"][e].float()
        dup = dh * act
        dgate = dh * u * (sig * (1 + g * (1 - sig)))
        dxp[lo:hi] = dgate @ s["w_gate"][e].float() + dup @ s["w_up"][e].float()
        dw_gate[e] = dgate.T @ x
        dw_up[e] = dup.T @ x
        dw_down[e] = dy.T @ (act * u)
    return dxp, dw_gate, dw_up, dw_down


def _plain_combine(s):
    T, K = s["topk_w"].shape
    at = s["pair_row"].long()
    dout = s["dout"].float()
    dyp = torch.zeros_like(s["yp"])
    dyp[at.view(-1)] = (s["topk_w"][..., None] * dout[:, None]).to(torch.bfloat16).view(T * K, -1)
    return dyp, (s["yp"][at].float() * dout[:, None]).sum(-1)


def _plain_dispatch(s):
    dx = s["dxp"][s["pair_row"].long()].float().sum(1)
    if s["dlogit"] is not None:
        dx = dx + (s["dlogit"][..., None] * s["w_router"][s["topk_idx"].long()].float()).sum(1)
    return dx.to(torch.bfloat16)


def _plain_route(s):
    idx, w, dw = s["topk_idx"].long(), s["topk_w"], s["dtopk_w"]
    x = s["x"].float()
    dl = w * (dw - (w * dw).sum(1, keepdim=True))
    if s["case"]["mode"] == 1:
        logits = torch.gather(x @ s["w_router"].float().T + s["bias"], 1, idx)
        dl = dl * (1 - torch.sigmoid(logits))
    dense = torch.zeros(x.shape[0], s["bias"].numel(), device="cuda").scatter_(1, idx, dl)
    return dl, dense.T @ x, dense.sum(0)


_RUN_OWN = {"save": _own_save, "backward": _own_backward, "combine": _own_combine, "dispatch": _own_dispatch, "route": _own_route}
_RUN_PLAIN = {"save": _plain_save, "backward": _plain_backward, "combine": _plain_combine, "dispatch": _plain_dispatch,
              "route": _plain_route}


# ------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions in 64 bits.  The codes of `save` are given before they are rounded to 8 bits: what is kept is
    measured against what it stands for.  A scale is a choice of representation and has no such value."""
    s = _inputs(case, seed)
    d = torch.float64
    op = case["op"]
    if op in ("save", "backward"):
        E, F, D = s["w_gate"].shape
        rows = s["xp"].shape[0]
        zeros = lambda *shape: torch.zeros(*shape, dtype=d, device="cuda")  # noqa: E731
        if op == "save":
            wide = -(-F // _BLOCK) * _BLOCK
            h, kept = zeros(rows, F), [zeros(rows, wide), zeros(rows, wide)]
            for e, (lo, hi) in enumerate(s["extents"]):
                pre = [torch.einsum("rd,fd->rf", s["xp"][lo:hi].to(d), s[k][e].to(d)) for k in ("w_gate", "w_up")]
                h[lo:hi] = pre[0] / (1 + torch.exp(-pre[0])) * pre[1]
                for v, to in zip(pre, kept):
                    top = torch.nn.functional.pad(v.abs(), (0, wide - F)).unflatten(1, (-1, _BLOCK)).amax(-1)
                    unit = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 448)))
                    to[lo:hi, :F] = v / unit.repeat_interleave(_BLOCK, 1)[:, :F]
            return h, kept[0], kept[1], None, None
        dxp, grads = zeros(rows, D), [zeros(E, F, D), zeros(E, F, D), zeros(E, D, F)]
        for e, (lo, hi) in enumerate(s["extents"]):
            g, u = (_from_8_bits(s[k + "8"][lo:hi], s[k + "_scale"][:, lo:hi], F, d) for k in ("gate", "up"))
            x, dy = s["xp"][lo:hi].to(d), s["dyp"][lo:hi].to(d)
            ex = torch.exp(-g)
            slope = (1 + ex + g * ex) / (1 + ex) ** 2     # derivative of g / (1 + exp(-g))
            dh = torch.einsum("rd,df->rf", dy, s["w_down"][e].to(d))
            dg, du = dh * u * slope, dh * g / (1 + ex)
            dxp[lo:hi] = torch.einsum("rf,fd->rd", dg, s["w_gate"][e].to(d)) + torch.einsum("rf,fd->rd", du, s["w_up"][e].to(d))
            grads[0][e] = torch.einsum("rf,rd->fd", dg, x)
            grads[1][e] = torch.einsum("rf,rd->fd", du, x)
            grads[2][e] = torch.einsum("rd,rf->df", dy, g / (1 + ex) * u)
        return (dxp, *grads)
    T, K = s["topk_w"].shape
    rows = s["pair_row"].reshape(-1).long()
    if op == "combine":
        dout = s["dout"].to(d).repeat_interleave(K, 0)
        dyp = torch.zeros(s["yp"].shape, dtype=d, device="cuda")
        dyp.index_copy_(0, rows, s["topk_w"].to(d).reshape(-1, 1) * dout)
        return dyp, torch.einsum("pd,pd->p", dout, s["yp"].index_select(0, rows).to(d)).view(T, K)
    if op == "dispatch":
        dx = torch.zeros(T, case["D"], dtype=d, device="cuda")
        for j in range(K):
            dx += s["dxp"].index_select(0, s["pair_row"][:, j].long()).to(d)
            if s["dlogit"] is not None:
                dx += s["dlogit"][:, j:j + 1].to(d) * s["w_router"].index_select(0, s["topk_idx"][:, j].long()).to(d)
        return dx
    w, dw, x = s["topk_w"].to(d), s["dtopk_w"].to(d), s["x"].to(d)
    flat = s["topk_idx"].reshape(-1).long()
    dl = torch.empty(T, K, dtype=d, device="cuda")
    mean = torch.einsum("tk,tk->t", w, dw)
    for j in range(K):
        e = s["topk_idx"][:, j].long()
        dl[:, j] = w[:, j] * (dw[:, j] - mean)
        if case["mode"] == 1:
            dl[:, j] /= 1 + torch.exp(torch.einsum("td,td->t", x, s["w_router"].to(d)[e]) + s["bias"].to(d)[e])
    by_expert = torch.zeros(case["E"], case["D"], dtype=d, device="cuda")
    for j in range(K):
        by_expert.index_add_(0, s["topk_idx"][:, j].long(), dl[:, j:j + 1] * x)
    return dl, by_expert, torch.zeros(case["E"], dtype=d, device="cuda").index_add_(0, flat, dl.reshape(-1))
