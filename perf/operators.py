"""Cases of the microscaled 4-bit operators and of the mixture-of-experts layer
around them: quantisation, the product, tokens sorted by expert and back, and
the experts' products.

A microscaled (MX) matrix holds blocks of 32 values along a row that share one
power of two: 4-bit elements E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
negatives) and an 8-bit scale E8M0, 2^(code - 127).  The scale of a block is
2^(floor(log2 max|x|) - 2), at least 2^-127; an element is the nearest E2M1 value of x over
that scale, ties to the even code, at most 6 in magnitude.  Rows whose length
is no multiple of 32 are padded with zeros.

The families, and what each stands for:

  quant         a matrix to 4 bits and the values it then stands for, blocks
                along its rows (activations before a product), along its
                columns (the transposed operand of a gradient), or both (an
                output gradient, which both gradient products read)
  linear        x W^T, activations bf16 (cast to 4 bits within the call),
                weights kept in 4 bits: decode steps, batches, prefill
  linear_grad   the gradients of that layer in training: dx = dy W and
                dW = dy^T x, all four operands cast within the call
  route         tokens sorted by expert, their rows gathered, and the experts'
                rows summed back with the router's weights
  route_grad    the gradient of the gather and of the weighted sum
  experts       gathered rows to 4 bits, times the weights of each row's expert
  experts_grad  the gradients of that product: rows times the experts' transposed
                weights, and dW of each expert over its own rows
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases ---------------------------------------------------------------------------------


def _quant(rows, cols, kind, axis):
    return {"family": "quant", "rows": rows, "cols": cols, "type": kind, "axis": axis}


def _linear(M, N, K, out):
    return {"family": "linear", "M": M, "N": N, "K": K, "out": out}


def _linear_grad(M, N, K):
    return {"family": "linear_grad", "M": M, "N": N, "K": K}


def _route(T, topk, E, D, kind, grad, align=1, dropped=False):
    return {"family": "route_grad" if grad else "route", "T": T, "topk": topk, "E": E, "D": D, "type": kind,
            "align": align, "dropped": dropped}


def _experts(T, topk, E, N, K, out, skew):
    return {"family": "experts", "T": T, "topk": topk, "E": E, "N": N, "K": K, "out": out, "skew": skew}


def _experts_grad(T, topk, E, N, K, skew):
    return {"family": "experts_grad", "T": T, "topk": topk, "E": E, "N": N, "K": K, "skew": skew}


def listed():
    def named(name, case):
        return dict(case, name=name)

    return [
        # the activations of a decode step: latency
        named("quant16x4096_bf16_rows", _quant(16, 4096, "bf16", "rows")),
        # an output gradient of a training step, blocks both ways (dx and dW read it)
        named("quant8192x4096_bf16_both", _quant(8192, 4096, "bf16", "both")),
        # an fp32 weight of odd sides, transposed
        named("quant5003x2049_f32_cols", _quant(5003, 2049, "f32", "cols")),
        # a few tokens times an up-projection: the weights are read once
        named("linear16x14336x4096_bf16", _linear(16, 14336, 4096, "bf16")),
        # a batch of odd sides, a row length that needs padding
        named("linear333x5003x2047_f32", _linear(333, 5003, 2047, "f32")),
        # a long prompt times the up-projection
        named("linear4096x14336x4096_bf16", _linear(4096, 14336, 4096, "bf16")),
        # the gradients of a square projection
        named("linear_grad8192x4096x4096", _linear_grad(8192, 4096, 4096)),
        # routing of a decode step
        named("route16x4096_2of8", _route(16, 2, 8, 4096, "bf16", False)),
        # gradient of routing a training batch
        named("route_grad8191x4096_2of8", _route(8191, 2, 8, 4096, "bf16", True, align=32)),
        # a decode step's experts: about two rows each, all weights read once
        named("experts32x2048x4096_4of64", _experts(32, 4, 64, 2048, 4096, "bf16", 0.0)),
        # experts of a prompt, uneven loads
        named("experts4096x14336x4096_2of8", _experts(4096, 2, 8, 14336, 4096, "bf16", 1.0)),
        # gradients of the experts' product in training, uneven loads
        named("experts_grad4096x2048x4096", _experts_grad(4096, 2, 8, 2048, 4096, 1.0)),
    ]


def _log(rng, lo, hi, mult=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(mult, int(round(v / mult)) * mult))


_MAX_FLOPS = 8192.0 * 14336 * 4096 * 2.0
_MAX_BYTES = 6.0e8


def draw(rng):
    """One more case of the families above, sizes spread over their ranges."""
    family = rng.choice(["quant", "quant", "linear", "linear", "linear", "linear_grad", "route", "route", "route_grad",
                         "experts", "experts", "experts_grad"])
    kind = rng.choice(["bf16", "bf16", "f32"])
    while True:
        if family == "quant":
            c = _quant(_log(rng, 1, 8192), _log(rng, 32, 16384), kind, rng.choice(["rows", "cols", "both"]))
        elif family == "linear":
            # every third one a few tokens
            M = _log(rng, 1, 64) if rng.random() < 0.34 else _log(rng, 65, 8192)
            c = _linear(M, _log(rng, 64, 16384), _log(rng, 64, 16384, rng.choice([1, 32, 64])), kind)
        elif family == "linear_grad":
            c = _linear_grad(_log(rng, 64, 8192), _log(rng, 64, 8192), _log(rng, 64, 8192))
        elif family in ("route", "route_grad"):
            E = rng.choice([4, 8, 16, 60, 64, 128])
            c = _route(_log(rng, 1, 16384), rng.choice([1, 2, 4]), E, _log(rng, 64, 8192, rng.choice([1, 8])), kind,
                       family == "route_grad", rng.choice([1, 16, 32]), rng.random() < 0.3)
        elif family == "experts":
            E = rng.choice([4, 8, 16, 60, 64])
            # every third one a decode step
            T = _log(rng, 1, 64) if rng.random() < 0.34 else _log(rng, 65, 8192)
            c = _experts(T, rng.choice([1, 2, 4]), E, _log(rng, 256, 14336, rng.choice([1, 16])),
                         _log(rng, 256, 8192, rng.choice([1, 32])), kind, rng.choice([0.0, 1.0]))
        else:
            E = rng.choice([4, 8, 16])
            c = _experts_grad(_log(rng, 64, 8192), rng.choice([1, 2]), E, _log(rng, 256, 4096), _log(rng, 256, 4096),
                              rng.choice([0.0, 1.0]))
        w = work(c)
        if w["flops"] <= _MAX_FLOPS and w["bytes"] <= _MAX_BYTES:
            return c


# ---- what a pass cannot do without -----------------------------------------------------------


def _up(v, m):
    return (v + m - 1) // m * m


def _mx_bytes(rows, cols):
    return rows * _up(cols, 32) * 17 / 32


def _sorted_rows(c):
    """Rows of the sorted arrays: every slot, and the padding of each expert's rows."""
    return c["T"] * c["topk"] + c["E"] * (c["align"] - 1)


def work(case):
    c, f = case, case["family"]
    if f == "quant":
        size = 4 if c["type"] == "f32" else 2
        n = 2 if c["axis"] == "both" else 1
        # the matrix, its 4-bit forms, and the bf16 values they stand for
        return {"bytes": c["rows"] * c["cols"] * (size + 2 * n) + _mx_bytes(c["rows"], c["cols"]) * n,
                "flops": float(c["rows"] * c["cols"] * n)}
    if f == "linear":
        size = 4 if c["out"] == "f32" else 2
        return {"bytes": c["M"] * c["K"] * 2 + _mx_bytes(c["N"], c["K"]) + c["M"] * c["N"] * size,
                "flops": 2.0 * c["M"] * c["N"] * c["K"]}
    if f == "linear_grad":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": 2.0 * (M * N + M * K + N * K) + 2.0 * M * K + 4.0 * N * K, "flops": 4.0 * M * N * K}
    slots = c["T"] * c["topk"]
    if f == "route":
        size = 4 if c["type"] == "f32" else 2
        rows = _sorted_rows(c)
        # ids, order, positions; x and the gathered rows; the experts' rows, weights and sums
        return {"bytes": 4.0 * (2 * slots + rows) + (c["T"] + rows) * c["D"] * size + (slots + c["T"]) * c["D"] * size
                + 4.0 * slots, "flops": 2.0 * slots * c["D"]}
    if f == "route_grad":
        size = 4 if c["type"] == "f32" else 2
        rows = _sorted_rows(c)
        # dy, the experts' rows, their gradient; the gathered rows' gradient and its sum
        return {"bytes": (c["T"] + slots + rows) * c["D"] * size + (slots + c["T"]) * c["D"] * size
                + 4.0 * (3 * slots + rows), "flops": 4.0 * slots * c["D"]}
    if f == "experts":
        size = 4 if c["out"] == "f32" else 2
        used = min(c["E"], slots)
        return {"bytes": c["T"] * c["K"] * 2.0 + used * _mx_bytes(c["N"], c["K"]) + slots * c["N"] * size,
                "flops": 2.0 * slots * c["N"] * c["K"]}
    used = min(c["E"], slots)
    return {"bytes": slots * c["N"] * 2.0 + c["T"] * c["K"] * 2.0 + used * _mx_bytes(c["K"], c["N"])
            + slots * c["K"] * 2.0 + 4.0 * c["E"] * c["N"] * c["K"], "flops": 4.0 * slots * c["N"] * c["K"]}


# ---- inputs ------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, rows, cols, kind):
    """Normal values under channel gains that spread over a few octaves, some channels large."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    x *= torch.exp2(1.5 * torch.randn((1, cols), generator=g, device="cuda"))
    return x.to(_TYPES[kind])


def _normal(g, shape, scale, kind):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(_TYPES[kind])


def _mx_weights(g, lead, rows, cols):
    """A trained weight in 4 bits, as a checkpoint holds it: codes (.., rows, cols/2), two to a
    byte, the even column in the low bits, and scale codes (.., rows, cols/32), rows of scales
    a multiple of 4 bytes apart."""
    cp, blocks = _up(cols, 32), _up(cols, 32) // 32
    codes = torch.empty(lead + (rows, cp // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full(lead + (rows, _up(blocks, 4)), 127, dtype=torch.uint8, device="cuda")[..., :blocks]
    for i in range(lead[0] if lead else 1):
        w = torch.randn((rows, cols), generator=g, device="cuda") * 0.02
        c, s = _codes(torch.nn.functional.pad(w, (0, cp - cols)))
        (codes[i] if lead else codes).copy_(c[:, 0::2] | (c[:, 1::2] << 4))
        (scales[i] if lead else scales).copy_(s)
    return codes, scales


def _routing(c, g):
    """Experts of every token, distinct within a token, loads uneven with `skew`."""
    load = torch.exp(c.get("skew", 0.0) * torch.randn((1, c["E"]), generator=g, device="cuda"))
    noise = torch.empty((c["T"], c["E"]), device="cuda").exponential_(generator=g)
    k = min(c["topk"], c["E"])
    ids = (load / noise).topk(k, dim=1).indices.to(torch.int32)
    if c.get("dropped"):
        # slots that a capacity limit took away
        ids = torch.where(torch.rand(ids.shape, generator=g, device="cuda") < 0.1, -1, ids)
    return ids


def _sort(ids, E, align, rows):
    """Stable order of the slots by expert: segment starts, slot of every sorted row (-1:
    padding), sorted row of every slot (-1: dropped)."""
    flat = ids.reshape(-1).long()
    hot = flat[:, None] == torch.arange(E, device=flat.device)[None, :]
    seen = hot.to(torch.int32).cumsum(0)
    counts = seen[-1].long() if flat.numel() else torch.zeros(E, dtype=torch.long, device=flat.device)
    starts = torch.zeros(E + 1, dtype=torch.long, device=flat.device)
    starts[1:] = ((counts + align - 1) // align * align).cumsum(0)
    valid = (flat >= 0) & (flat < E)
    e = flat.clamp(0, E - 1)
    pos = starts[e] + seen.gather(1, e[:, None])[:, 0] - 1
    pos = torch.where(valid, pos, -1)
    order = torch.full((rows + 1,), -1, dtype=torch.long, device=flat.device)
    order[torch.where(valid, pos, rows)] = torch.arange(flat.numel(), device=flat.device)
    return starts.to(torch.int32), order[:rows].to(torch.int32), pos.to(torch.int32)


def prepare(case, seed):
    c, f, g = case, case["family"], _gen(seed)
    s = {"case": c}
    if f == "quant":
        s["x"] = _activations(g, c["rows"], c["cols"], c["type"])
    elif f == "linear":
        s["x"] = _activations(g, c["M"], c["K"], "bf16")
        s["w"] = _mx_weights(g, (), c["N"], c["K"])
    elif f == "linear_grad":
        s["x"] = _activations(g, c["M"], c["K"], "bf16")
        s["dy"] = _normal(g, (c["M"], c["N"]), 1e-3, "bf16")
        s["w"] = _normal(g, (c["N"], c["K"]), 0.02, "bf16")
    elif f in ("route", "route_grad"):
        rows = _sorted_rows(c)
        s["ids"] = _routing(c, g)
        s["weights"] = torch.softmax(torch.randn((c["T"], s["ids"].shape[1]), generator=g, device="cuda"), 1)
        s["ys"] = _normal(g, (rows, c["D"]), 1.0, c["type"])
        if f == "route":
            s["x"] = _activations(g, c["T"], c["D"], c["type"])
        else:
            s["dy"] = _normal(g, (c["T"], c["D"]), 1e-3, c["type"])
            s["dxs"] = _normal(g, (rows, c["D"]), 1e-3, c["type"])
            _, s["order"], s["pos"] = _sort(s["ids"], c["E"], c["align"], rows)
    else:
        align = 32 if f == "experts_grad" else 1
        s["ids"] = _routing(c, g)
        s["rows"] = s["ids"].numel() + c["E"] * (align - 1)
        s["offsets"], s["order"], _ = _sort(s["ids"], c["E"], align, s["rows"])
        s["x"] = _activations(g, c["T"], c["K"], "bf16")
        if f == "experts":
            s["w"] = _mx_weights(g, (c["E"],), c["N"], c["K"])
        else:
            s["dys"] = _normal(g, (s["rows"], c["N"]), 1e-3, "bf16")
            s["dys"][s["order"] < 0] = 0
            s["wt"] = _mx_weights(g, (c["E"],), c["K"], c["N"])
    return s


# ---- the plain form ------------------------------------------------------------------------------


def _codes(x):
    """E2M1 and scale codes of an fp32 matrix whose row length is a multiple of 32."""
    b = x.reshape(x.shape[0], -1, 32)
    field = b.abs().amax(-1).view(torch.int32) >> 23
    s = torch.where(field == 255, 255, (field - 2).clamp(min=0))
    inverse = ((254 - s).clamp(min=1) << 23).view(torch.float32)
    m = (b * inverse[..., None]).abs()
    # steps of 1/2 below 2, of 1 below 4, of 2 above; torch.round takes ties to even
    v = torch.where(m < 2, torch.round(m * 2), torch.where(m < 4, torch.round(m) + 2, torch.round(m * 0.5) + 4))
    code = v.clamp(max=7).nan_to_num().to(torch.uint8) | (torch.signbit(b).to(torch.uint8) << 3)
    return code.reshape(x.shape), s.to(torch.uint8)


def _grid():
    v = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return torch.tensor(v + [-a for a in v], device="cuda")


def _power(s):
    bits = s.to(torch.int32)
    return torch.where(bits == 255, float("nan"), torch.where(bits == 0, 1 << 22, bits << 23).view(torch.float32))


def _values(code, s):
    v = _grid()[code.long()].reshape(code.shape[0], -1, 32)
    return (v * _power(s)[..., None]).reshape(code.shape)


def _unpack(packed, s):
    """fp32 values of packed codes and their scales."""
    code = torch.stack((packed & 15, packed >> 4), dim=-1).reshape(packed.shape[0], -1)
    return _values(code, s)


def _rounded(x):
    """The fp32 values that a matrix stands for in 4 bits, rows padded to whole blocks."""
    x = x.float()
    return _values(*_codes(torch.nn.functional.pad(x, (0, -x.shape[1] % 32))))


def _gather(x, order, topk):
    rows = x[(order.long().clamp(min=0) // topk)].float()
    return torch.where(order[:, None] >= 0, rows, 0.0)


def _combine(rows, pos, weights):
    """Sum over a token's slots of its sorted rows, times the weights if there are any."""
    T, k = pos.shape
    y = torch.zeros((T, rows.shape[1]), device="cuda")
    for j in range(k):
        p = pos[:, j].long()
        v = torch.where(p[:, None] >= 0, rows[p.clamp(min=0)].float(), 0.0)
        y += v if weights is None else v * weights[:, j:j + 1]
    return y


def _plain(s):
    c, f = s["case"], s["case"]["family"]
    if f == "quant":
        x = s["x"]
        out = []
        if c["axis"] in ("rows", "both"):
            out.append(_rounded(x)[:, :c["cols"]].to(torch.bfloat16))
        if c["axis"] in ("cols", "both"):
            out.append(_rounded(x.t().contiguous())[:, :c["rows"]].to(torch.bfloat16))
        return out
    if f == "linear":
        return (_rounded(s["x"]) @ _unpack(*s["w"]).t()).to(_TYPES[c["out"]])
    if f == "linear_grad":
        dx = _rounded(s["dy"]) @ _rounded(s["w"].t().contiguous()).t()
        dw = _rounded(s["dy"].t().contiguous()) @ _rounded(s["x"].t().contiguous()).t()
        return [dx.to(torch.bfloat16), dw]
    if f == "route":
        rows, k = _sorted_rows(c), s["ids"].shape[1]
        offsets, order, pos = _sort(s["ids"], c["E"], c["align"], rows)
        xs = _gather(s["x"], order, k)
        y = _combine(s["ys"], pos.view(-1, k), s["weights"])
        return [offsets, order, pos, xs.to(_TYPES[c["type"]]), y.to(_TYPES[c["type"]])]
    if f == "route_grad":
        k = s["ids"].shape[1]
        order, pos = s["order"].long(), s["pos"].view(-1, k).long()
        w = torch.where(order >= 0, s["weights"].reshape(-1)[order.clamp(min=0)], 0.0)
        dys = _gather(s["dy"], order, k) * w[:, None]
        dw = torch.zeros(pos.shape, device="cuda")
        for j in range(k):
            p = pos[:, j]
            dot = (s["dy"].float() * s["ys"][p.clamp(min=0)].float()).sum(1)
            dw[:, j] = torch.where(p >= 0, dot, 0.0)
        dx = _combine(s["dxs"], pos, None)
        return [dys.to(_TYPES[c["type"]]), dw, dx.to(_TYPES[c["type"]])]
    at = s["offsets"].tolist()
    k = s["ids"].shape[1]
    if f == "experts":
        xs = _rounded(_gather(s["x"], s["order"], k))
        y = torch.zeros((s["rows"], c["N"]), device="cuda")
        for e in range(c["E"]):
            y[at[e]:at[e + 1]] = xs[at[e]:at[e + 1]] @ _unpack(s["w"][0][e], s["w"][1][e]).t()
        return y.to(_TYPES[c["out"]])
    dys = _rounded(s["dys"])
    dyt = _rounded(s["dys"].t().contiguous())
    xst = _rounded(_gather(s["x"], s["order"], k).t().contiguous())
    dxs = torch.zeros((s["rows"], c["K"]), device="cuda")
    dw = torch.zeros((c["E"], c["N"], c["K"]), device="cuda")
    for e in range(c["E"]):
        dxs[at[e]:at[e + 1]] = dys[at[e]:at[e + 1]] @ _unpack(s["wt"][0][e], s["wt"][1][e]).t()
        dw[e] = dyt[:, at[e]:at[e + 1]] @ xst[:, at[e]:at[e + 1]].t()
    return [dxs.to(torch.bfloat16), dw]


# ---- the framework's calls -------------------------------------------------------------------------


def _kernels(s):
    from paper_2601_16294_amd import sfcops as so

    c, f = s["case"], s["case"]["family"]

    def new(shape, kind):
        return torch.empty(shape, dtype=_TYPES.get(kind, kind), device="cuda")

    if f == "quant":
        R, C = c["rows"], c["cols"]
        q = so.mx4_empty(R, C) if c["axis"] in ("rows", "both") else (None, None)
        t = so.mx4_empty(C, R) if c["axis"] in ("cols", "both") else (None, None)
        so.sfc_mx4_quant(s["x"], *q, *t)
        out = []
        if q[0] is not None:
            out.append(new((R, C), "bf16"))
            so.sfc_mx4_dequant(*q, out[-1])
        if t[0] is not None:
            out.append(new((C, R), "bf16"))
            so.sfc_mx4_dequant(*t, out[-1])
        return out
    if f == "linear":
        y = new((c["M"], c["N"]), c["out"])
        so.sfc_mx4_linear(s["x"], *s["w"], y)
        return y
    if f == "linear_grad":
        M, N, K = c["M"], c["N"], c["K"]
        dyq, dyt, wt, xt = so.mx4_empty(M, N), so.mx4_empty(N, M), so.mx4_empty(K, N), so.mx4_empty(K, M)
        so.sfc_mx4_quant(s["dy"], *dyq, *dyt)
        so.sfc_mx4_quant(s["w"], None, None, *wt)
        so.sfc_mx4_quant(s["x"], None, None, *xt)
        dx, dw = new((M, K), "bf16"), new((N, K), "f32")
        so.sfc_gemm_mx4_ex(*dyq, *wt, dx)
        so.sfc_gemm_mx4_ex(*dyt, *xt, dw)
        return [dx, dw]
    k = s["ids"].shape[1]
    if f == "route":
        rows = _sorted_rows(c)
        offsets, order, pos = new((c["E"] + 1,), torch.int32), new((rows,), torch.int32), new((s["ids"].numel(),), torch.int32)
        so.sfc_moe_sort(s["ids"], offsets, order, pos, align=c["align"])
        xs, y = new((rows, c["D"]), c["type"]), new((c["T"], c["D"]), c["type"])
        so.sfc_moe_dispatch(s["x"], order, xs, topk=k)
        so.sfc_moe_combine(s["ys"], pos, y, weights=s["weights"])
        return [offsets, order, pos, xs, y]
    if f == "route_grad":
        dys, dw = new(tuple(s["ys"].shape), c["type"]), new((c["T"], k), "f32")
        dx = new((c["T"], c["D"]), c["type"])
        so.sfc_moe_combine_grad(s["dy"], s["ys"], s["order"], s["pos"], s["weights"], dys, dw)
        so.sfc_moe_combine(s["dxs"], s["pos"], dx)
        return [dys, dw, dx]
    if f == "experts":
        xq = so.mx4_empty(s["rows"], c["K"])
        so.sfc_mx4_quant(s["x"], *xq, order=s["order"], topk=k)
        y = new((s["rows"], c["N"]), c["out"])
        so.sfc_moe_gemm_mx4_ex(*xq, *s["w"], s["offsets"], y)
        return y
    rows, N, K = s["rows"], c["N"], c["K"]
    dq, dt, xt = so.mx4_empty(rows, N), so.mx4_empty(N, rows), so.mx4_empty(K, rows)
    so.sfc_mx4_quant(s["dys"], *dq, *dt)
    so.sfc_mx4_quant(s["x"], None, None, *xt, order=s["order"], topk=k)
    dxs, dw = new((rows, K), "bf16"), new((c["E"], N, K), "f32")
    so.sfc_moe_gemm_mx4_ex(*dq, *s["wt"], s["offsets"], dxs)
    so.sfc_moe_wgrad_mx4_ex(*dt, *xt, s["offsets"], dw)
    return [dxs, dw]


def run(state):
    return _kernels(state) if own else _plain(state)


# ---- 64 bits ---------------------------------------------------------------------------------------


def _power64(exponent):
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def _mx64(x):
    """Values of a matrix in 4 bits from the definition: nearest of the 8 magnitudes, ties to
    the one of even index, over the block's power of two.  In strips, for memory."""
    R, C = x.shape
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    out = torch.zeros((R, _up(C, 32)), dtype=torch.float64, device=x.device)
    strip = max(1, (1 << 26) // max(1, out.shape[1]))
    for r in range(0, R, strip):
        b = torch.zeros((min(strip, R - r), out.shape[1]), dtype=torch.float64, device=x.device)
        b[:, :C] = x[r:r + strip].double()
        b = b.view(b.shape[0], -1, 32)
        top = b.abs().amax(-1, keepdim=True)
        exponent = torch.frexp(top).exponent - 1
        scale = _power64(torch.where(top == 0, -127, (exponent - 2).clamp(min=-127)))
        m = b.abs() / scale
        # index of the nearest: how many midpoints lie below (or at, where the upper one is even)
        index = torch.zeros_like(m, dtype=torch.int64)
        for i in range(7):
            mid = (grid[i] + grid[i + 1]) / 2
            index += (m >= mid) if i % 2 == 1 else (m > mid)
        out[r:r + strip] = (torch.sign(b) * grid[index] * scale).view(b.shape[0], -1)
    return out


def _decode64(packed, scales):
    low, high = (packed & 15).long(), (packed >> 4).long()
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=packed.device)
    out = torch.empty((packed.shape[0], packed.shape[1] * 2), dtype=torch.float64, device=packed.device)
    for i, code in enumerate((low, high)):
        out[:, i::2] = grid[code % 8] * (1 - 2 * (code // 8)).double()
    return out * _power64(scales.long() - 127).repeat_interleave(32, dim=1)


def exact(case, seed):
    c, f = case, case["family"]
    s = prepare(case, seed)
    if f == "quant":
        out = []
        if c["axis"] != "cols":
            out.append(_mx64(s["x"])[:, :c["cols"]])
        if c["axis"] != "rows":
            out.append(_mx64(s["x"].t())[:, :c["rows"]])
        return out
    if f == "linear":
        return torch.mm(_mx64(s["x"]), _decode64(*s["w"]).t())
    if f == "linear_grad":
        return [torch.mm(_mx64(s["dy"]), _mx64(s["w"].t()).t()), torch.mm(_mx64(s["dy"].t()), _mx64(s["x"].t()).t())]
    T, k = s["ids"].shape
    if f == "route":
        # expert by expert, the slots in ascending order
        flat = s["ids"].reshape(-1).cpu()
        order, starts, pos = [], [0], torch.full((T * k,), -1, dtype=torch.int32)
        for e in range(c["E"]):
            slots = torch.nonzero(flat == e)[:, 0].tolist()
            for i, v in enumerate(slots):
                pos[v] = starts[-1] + i
            order += slots + [-1] * (-len(slots) % c["align"])
            starts.append(len(order))
        order += [-1] * (_sorted_rows(c) - len(order))
        order = torch.tensor(order, dtype=torch.int32, device="cuda")
        pos = pos.cuda()
        xs = torch.zeros((order.numel(), c["D"]), dtype=torch.float64, device="cuda")
        xs[order >= 0] = s["x"].double()[order[order >= 0].long() // k]
        y = torch.zeros((T, c["D"]), dtype=torch.float64, device="cuda")
        kept = torch.nonzero(pos >= 0)[:, 0]
        y.index_add_(0, kept // k, s["ys"].double()[pos[kept].long()] * s["weights"].reshape(-1)[kept].double()[:, None])
        return [torch.tensor(starts, dtype=torch.int32, device="cuda"), order, pos, xs, y]
    if f == "route_grad":
        pos = s["pos"]
        kept = torch.nonzero(pos >= 0)[:, 0]
        row = pos[kept].long()
        dy = s["dy"].double()[kept // k]
        dys = torch.zeros((s["ys"].shape[0], c["D"]), dtype=torch.float64, device="cuda")
        dys[row] = dy * s["weights"].reshape(-1)[kept].double()[:, None]
        dw = torch.zeros(T * k, dtype=torch.float64, device="cuda")
        dw[kept] = (dy * s["ys"].double()[row]).sum(1)
        dx = torch.zeros((T, c["D"]), dtype=torch.float64, device="cuda")
        dx.index_add_(0, kept // k, s["dxs"].double()[row])
        return [dys, dw.view(T, k), dx]
    at = s["offsets"].tolist()
    xs = torch.zeros((s["rows"], c["K"]), dtype=torch.float64, device="cuda")
    kept = s["order"] >= 0
    xs[kept] = s["x"].double()[s["order"][kept].long() // k]
    if f == "experts":
        a = _mx64(xs)
        y = torch.zeros((s["rows"], c["N"]), dtype=torch.float64, device="cuda")
        for e in range(c["E"]):
            torch.mm(a[at[e]:at[e + 1]], _decode64(s["w"][0][e], s["w"][1][e]).t(), out=y[at[e]:at[e + 1]])
        return y
    a, at_, bt = _mx64(s["dys"]), _mx64(s["dys"].t()), _mx64(xs.t())
    dxs = torch.zeros((s["rows"], c["K"]), dtype=torch.float64, device="cuda")
    dw = torch.zeros((c["E"], c["N"], c["K"]), dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        lo, hi = at[e], at[e + 1]
        torch.mm(a[lo:hi], _decode64(s["wt"][0][e], s["wt"][1][e]).t(), out=dxs[lo:hi])
        dw[e] = torch.mm(at_[:, lo:hi], bt[:, lo:hi].t())
    return [dxs, dw]
