"""Cases of the bf16 experts' products and of the low-rank adapters: products whose
weights depend on the row.

Experts: rows sorted by expert (segments offsets[e] .. offsets[e+1]-1, as the sort by
expert leaves them) times the weights of each row's expert, bf16 with fp32 sums.
Adapters: row t of a batch belongs to adapter a = ids[t] (a request's; -1: none) and
gets, beside what a shared projection gave it,

    y[t] = base[t] + V[t] B[a]^T,   V[t] = s[a] x[t] A[a]^T

with A[a] of R x K, B[a] of N x R, and R between a few and a few hundred.

The families, and what each stands for:

  experts        a layer's up-projection: tokens gathered in sorted order times the weights
                 (N x K, as a linear layer holds them) of each row's expert
  experts_grad   its gradients in training: dxs[p] = dys[p] W[e], dW[e] = dys[seg]^T xs[seg]
  adapters       the adapters' part of a projection: decode steps, where every row is a
                 request of its own, and prompts, where a request is a run of rows
  adapters_grad  its gradients: dx = dbase + U A with U[t] = s[a] dy[t] B[a], and
                 dA[a] = U^T x, dB[a] = dy^T V over the adapter's rows
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases ---------------------------------------------------------------------------------


def _experts(T, topk, E, N, K, out, skew):
    return {"family": "experts", "T": T, "topk": topk, "E": E, "N": N, "K": K, "out": out, "skew": skew}


def _experts_grad(T, topk, E, N, K, skew, out="f32"):
    return {"family": "experts_grad", "T": T, "topk": topk, "E": E, "N": N, "K": K, "out": out, "skew": skew}


def _adapters(T, requests, adapters, R, N, K, out):
    return {"family": "adapters", "T": T, "requests": requests, "adapters": adapters, "R": R, "N": N, "K": K, "out": out}


def _adapters_grad(T, requests, adapters, R, N, K):
    return {"family": "adapters_grad", "T": T, "requests": requests, "adapters": adapters, "R": R, "N": N, "K": K,
            "out": "bf16"}


def listed():
    def named(name, case):
        return dict(case, name=name)

    return [
        # a decode step of many experts: about two rows each, their weights are read once
        named("experts32x2048x4096_4of64", _experts(32, 4, 64, 2048, 4096, "bf16", 0.0)),
        # a token alone: two experts' weights, latency
        named("experts1x4096x4096_2of8", _experts(1, 2, 8, 4096, 4096, "bf16", 0.0)),
        # a batch of odd sides over uneven loads, rows of odd length
        named("experts333x1407x2047_3of60_f32", _experts(333, 3, 60, 1407, 2047, "f32", 1.0)),
        # a long prompt through the up-projection, uneven loads
        named("experts4096x14336x4096_2of8", _experts(4096, 2, 8, 14336, 4096, "bf16", 1.0)),
        # both gradients in training
        named("experts_grad8192x4096x4096_2of8", _experts_grad(8192, 2, 8, 4096, 4096, 1.0)),
        # the same for small experts of odd sides
        named("experts_grad2000x1001x1503_2of16", _experts_grad(2000, 2, 16, 1001, 1503, 1.0, "bf16")),
        # a decode step, every row a request of its own
        named("adapters32x4096x4096_r16", _adapters(32, 32, 16, 16, 4096, 4096, "bf16")),
        # prompts of a batch through the up-projection, higher rank
        named("adapters4096x14336x4096_r64", _adapters(4096, 24, 8, 64, 14336, 4096, "bf16")),
        # odd sides and rank, fp32
        named("adapters1003x5003x2047_r12_f32", _adapters(1003, 17, 5, 12, 5003, 2047, "f32")),
        # training of a few adapters at once
        named("adapters_grad8192x4096x4096_r16", _adapters_grad(8192, 8, 4, 16, 4096, 4096)),
        # training of one adapter of higher rank, odd sides
        named("adapters_grad2001x2047x4097_r40", _adapters_grad(2001, 1, 1, 40, 2047, 4097)),
    ]


def _log(rng, lo, hi, mult=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(mult, int(round(v / mult)) * mult))


_MAX_FLOPS = 8192.0 * 2 * 4096 * 4096 * 4.0
_MAX_BYTES = 1.2e9


def draw(rng):
    """One more case of the families above, sizes spread over their ranges."""
    family = rng.choice(["experts", "experts", "experts_grad", "adapters", "adapters", "adapters_grad"])
    out = rng.choice(["bf16", "bf16", "f32"])
    while True:
        if family in ("experts", "experts_grad"):
            E = rng.choice([1, 4, 8, 16, 60, 64])
            mult = rng.choice([1, 8, 64])
            N, K = _log(rng, 64, 14336, mult), _log(rng, 64, 8192, mult)
            skew = rng.choice([0.0, 1.0])
            if family == "experts":
                # every third one a decode step
                T = _log(rng, 1, 64) if rng.random() < 0.34 else _log(rng, 65, 8192)
                c = _experts(T, rng.choice([1, 2, 4]), E, N, K, out, skew)
            else:
                c = _experts_grad(_log(rng, 16, 8192), rng.choice([1, 2]), E, N, K, skew, out)
        else:
            R = rng.choice([4, 8, 16, 16, 24, 32, 64, 100, 128, 256])
            mult = rng.choice([1, 8, 64])
            N, K = _log(rng, 64, 16384, mult), _log(rng, 64, 16384, mult)
            adapters = _log(rng, 1, 64)
            if family == "adapters" and rng.random() < 0.4:
                T = _log(rng, 1, 256)
                c = _adapters(T, T, adapters, R, N, K, out)
            elif family == "adapters":
                T = _log(rng, 64, 16384)
                c = _adapters(T, min(T, _log(rng, 1, 64)), adapters, R, N, K, out)
            else:
                T = _log(rng, 64, 16384)
                c = _adapters_grad(T, min(T, _log(rng, 1, 64)), min(8, adapters), R, N, K)
        w = work(c)
        if w["flops"] <= _MAX_FLOPS and w["bytes"] <= _MAX_BYTES:
            return c


# ---- what a pass cannot do without -----------------------------------------------------------


def work(case):
    c, f = case, case["family"]
    size = 4 if c["out"] == "f32" else 2
    N, K = c["N"], c["K"]
    if f in ("experts", "experts_grad"):
        slots = c["T"] * min(c["topk"], c["E"])
        used = min(c["E"], slots)
        if f == "experts":
            return {"bytes": c["T"] * K * 2.0 + used * N * K * 2.0 + slots * N * size + 4.0 * slots,
                    "flops": 2.0 * slots * N * K}
        return {"bytes": slots * (N + K) * 2.0 + used * N * K * 2.0 + slots * K * 2.0 + c["E"] * N * K * size,
                "flops": 4.0 * slots * N * K}
    T, R = c["T"], c["R"]
    used = min(c["adapters"], c["requests"])
    if f == "adapters":
        # x, ids, the adapters, the shared projection's rows; V and the sums
        return {"bytes": T * K * 2.0 + 4.0 * T + used * R * (N + K) * 2.0 + 2.0 * T * N * size + 4.0 * T * R,
                "flops": 2.0 * T * R * (N + K)}
    # dy, x, V, ids, the adapters, dbase; dx, dA, dB
    return {"bytes": T * (N + K) * 2.0 + 4.0 * T * R + 4.0 * T + used * R * (N + K) * 2.0 + 2.0 * T * K * size
            + 4.0 * c["adapters"] * R * (N + K), "flops": 4.0 * T * R * (N + K)}


# ---- inputs ------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, rows, cols):
    """Normal values under channel gains that spread over a few octaves, some channels large."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    x *= torch.exp2(torch.randn((1, cols), generator=g, device="cuda"))
    return x.to(torch.bfloat16)


def _normal(g, shape, scale, kind="bf16"):
    if len(shape) < 3:
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(_TYPES[kind])
    # stacks of weights one by one, for memory
    out = torch.empty(shape, dtype=_TYPES[kind], device="cuda")
    for w in out:
        w.copy_(torch.randn(shape[1:], generator=g, device="cuda") * scale)
    return out


def _routing(c, g):
    """Slots sorted by expert (stable): segment starts, and the slot of every sorted row.
    A token's experts are distinct; loads are uneven with `skew`."""
    load = torch.exp(c["skew"] * torch.randn((1, c["E"]), generator=g, device="cuda"))
    noise = torch.empty((c["T"], c["E"]), device="cuda").exponential_(generator=g)
    ids = (load / noise).topk(min(c["topk"], c["E"]), dim=1).indices
    order = torch.sort(ids.reshape(-1), stable=True).indices
    starts = torch.zeros(c["E"] + 1, dtype=torch.int64, device="cuda")
    starts[1:] = torch.bincount(ids.reshape(-1), minlength=c["E"]).cumsum(0)
    return starts.to(torch.int32), order.to(torch.int32)


def _requests(c, g):
    """The adapter of every row: requests are runs of rows, some without an adapter."""
    T, q = c["T"], c["requests"]
    cuts = torch.randperm(T - 1, generator=g, device="cuda")[:q - 1] + 1 if q > 1 else torch.zeros(0, device="cuda")
    mark = torch.zeros(T, dtype=torch.int64, device="cuda")
    mark[cuts.long()] = 1
    owner = torch.randint(0, c["adapters"], (q,), generator=g, device="cuda")
    if q > 1:
        owner = torch.where(torch.rand(q, generator=g, device="cuda") < 0.1, -1, owner)
    return owner[mark.cumsum(0)].to(torch.int32)


def prepare(case, seed):
    c, f, g = case, case["family"], _gen(seed)
    s = {"case": c}
    N, K = c["N"], c["K"]
    if f in ("experts", "experts_grad"):
        s["offsets"], s["order"] = _routing(c, g)
        s["topk"] = min(c["topk"], c["E"])
        s["w"] = _normal(g, (c["E"], N, K), 0.02)
        if f == "experts":
            s["x"] = _activations(g, c["T"], K)
        else:
            s["xs"] = _activations(g, c["T"], K)[s["order"].long() // s["topk"]]
            s["dys"] = _normal(g, (s["order"].numel(), N), 1e-3)
        return s
    T, R, n = c["T"], c["R"], c["adapters"]
    s["ids"] = _requests(c, g)
    s["a"] = _normal(g, (n, R, K), K ** -0.5)
    s["b"] = _normal(g, (n, N, R), 0.02)
    s["scales"] = torch.rand(n, generator=g, device="cuda") + 0.5
    s["x"] = _activations(g, T, K)
    if f == "adapters":
        s["base"] = _normal(g, (T, N), 1.0, c["out"])
    else:
        s["dy"] = _normal(g, (T, N), 1e-3)
        s["dbase"] = _normal(g, (T, K), 1e-3, c["out"])
        s["v"] = _down(s["x"], s["a"], s["ids"], s["scales"])     # as the forward pass left it
    return s


# ---- the plain form ------------------------------------------------------------------------------


def _rows_of(ids, adapters):
    """(adapter, its rows) of a batch."""
    for a in range(adapters):
        yield a, torch.nonzero(ids == a)[:, 0]


def _down(x, a, ids, scales):
    v = torch.zeros((x.shape[0], a.shape[1]), device="cuda")
    for i, rows in _rows_of(ids, a.shape[0]):
        v[rows] = x[rows].float() @ a[i].float().t() * scales[i]
    return v


def _up(v, b, ids, base):
    y = base.float()
    for i, rows in _rows_of(ids, b.shape[0]):
        y[rows] += v[rows] @ b[i].float().t()
    return y.to(base.dtype)


def _plain(s):
    c, f = s["case"], s["case"]["family"]
    N, K = c["N"], c["K"]
    if f in ("experts", "experts_grad"):
        at = s["offsets"].tolist()
        rows = s["order"].numel()
        if f == "experts":
            y = torch.empty((rows, N), device="cuda")
            source = s["order"].long() // s["topk"]
            for e in range(c["E"]):
                y[at[e]:at[e + 1]] = s["x"][source[at[e]:at[e + 1]]].float() @ s["w"][e].float().t()
            return y.to(_TYPES[c["out"]])
        dxs = torch.empty((rows, K), device="cuda")
        dw = torch.empty((c["E"], N, K), device="cuda")
        for e in range(c["E"]):
            dy = s["dys"][at[e]:at[e + 1]].float()
            dxs[at[e]:at[e + 1]] = dy @ s["w"][e].float()
            dw[e] = dy.t() @ s["xs"][at[e]:at[e + 1]].float()
        return [dxs.to(torch.bfloat16), dw.to(_TYPES[c["out"]])]
    if f == "adapters":
        v = _down(s["x"], s["a"], s["ids"], s["scales"])
        return [v, _up(v, s["b"], s["ids"], s["base"])]
    u = _down(s["dy"], s["b"].transpose(1, 2), s["ids"], s["scales"])
    dx = _up(u, s["a"].transpose(1, 2), s["ids"], s["dbase"])
    da = torch.zeros(s["a"].shape, device="cuda")
    db = torch.zeros(s["b"].shape, device="cuda")
    for i, rows in _rows_of(s["ids"], c["adapters"]):
        da[i] = u[rows].t() @ s["x"][rows].float()
        db[i] = s["dy"][rows].float().t() @ s["v"][rows]
    return [dx, da, db]


# ---- the framework's calls -------------------------------------------------------------------------


def _kernels(s):
    from paper_2601_16294_amd import sfcops as so

    c, f = s["case"], s["case"]["family"]

    def new(shape, kind):
        return torch.empty(shape, dtype=_TYPES[kind], device="cuda")

    N, K = c["N"], c["K"]
    if f == "experts":
        y = new((s["order"].numel(), N), c["out"])
        so.sfc_moe_gemm_ex(s["x"], s["w"], s["offsets"], y, order=s["order"], topk=s["topk"])
        return y
    if f == "experts_grad":
        dxs, dw = new((s["order"].numel(), K), "bf16"), new((c["E"], N, K), c["out"])
        so.sfc_moe_gemm_ex(s["dys"], s["w"], s["offsets"], dxs, layout=so.SFC_B_KN)
        so.sfc_moe_wgrad_ex(s["dys"], s["xs"], s["offsets"], dw)
        return [dxs, dw]
    T, R, n = c["T"], c["R"], c["adapters"]
    if f == "adapters":
        # (fp32 rows are added to where the shared projection left them, as the plain form does)
        v, y = new((T, R), "f32"), s["base"] if c["out"] == "f32" else new((T, N), c["out"])
        so.sfc_lora_down(s["x"], s["a"], s["ids"], v, scales=s["scales"])
        so.sfc_lora_up(v, s["b"], s["ids"], y, base=s["base"])
        return [v, y]
    u, dx = new((T, R), "f32"), new((T, K), c["out"])
    da, db = new((n, R, K), "f32"), new((n, N, R), "f32")
    so.sfc_lora_down(s["dy"], s["b"], s["ids"], u, scales=s["scales"], layout=so.SFC_B_KN)
    so.sfc_lora_up(u, s["a"], s["ids"], dx, base=s["dbase"], layout=so.SFC_B_KN)
    so.sfc_lora_wgrad(s["x"], u, s["ids"], da, layout=so.SFC_B_KN)
    so.sfc_lora_wgrad(s["dy"], s["v"], s["ids"], db)
    return [dx, da, db]


def run(state):
    return _kernels(state) if own else _plain(state)


# ---- 64 bits ---------------------------------------------------------------------------------------


def exact(case, seed):
    c, f = case, case["family"]
    s = prepare(case, seed)
    N, K = c["N"], c["K"]
    double = torch.float64
    if f in ("experts", "experts_grad"):
        starts = s["offsets"].cpu()
        rows = s["order"].numel()
        if f == "experts":
            y = torch.zeros((rows, N), dtype=double, device="cuda")
            x = s["x"].double()
            for e in range(c["E"]):
                lo, hi = int(starts[e]), int(starts[e + 1])
                token = torch.div(s["order"][lo:hi], s["topk"], rounding_mode="floor").long()
                torch.mm(x.index_select(0, token), s["w"][e].double().t(), out=y[lo:hi])
            return y
        dxs = torch.zeros((rows, K), dtype=double, device="cuda")
        dw = torch.zeros((c["E"], N, K), dtype=double, device="cuda")
        for e in range(c["E"]):
            lo, hi = int(starts[e]), int(starts[e + 1])
            dy, xs = s["dys"][lo:hi].double(), s["xs"][lo:hi].double()
            torch.mm(dy, s["w"][e].double(), out=dxs[lo:hi])
            torch.mm(dy.t(), xs, out=dw[e])
        return [dxs, dw]
    # the batch as one product of stacked adapters: column block a counts in the rows of adapter a
    n, R = c["adapters"], c["R"]
    ids = s["ids"].long()
    mine = (ids[:, None] == torch.arange(n, device="cuda")[None, :]).double()          # rows x adapters
    weight = mine * s["scales"].double()[None, :]

    def spread(rows, stack, factor):
        """rows times the transposed stack (adapters x R x columns), kept in each row's own block."""
        flat = torch.mm(rows.double(), stack.double().reshape(n * R, -1).t())
        return flat * factor.repeat_interleave(R, dim=1)

    a64, b64 = s["a"].double().reshape(n * R, K), s["b"].double().transpose(1, 2).reshape(n * R, N)
    if f == "adapters":
        wide = spread(s["x"], s["a"], weight)
        return [wide.view(-1, n, R).sum(1), torch.addmm(s["base"].double(), wide, b64)]
    wide = spread(s["dy"], s["b"].transpose(1, 2), weight)
    dx = torch.addmm(s["dbase"].double(), wide, a64)
    da = torch.mm(wide.t(), s["x"].double()).view(n, R, K)
    v = s["v"].double()[:, None, :] * mine[:, :, None]
    db = torch.mm(v.view(-1, n * R).t(), s["dy"].double()).view(n, R, N).transpose(1, 2).contiguous()
    return [dx, da, db]
