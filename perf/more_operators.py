"""Routing to experts, its counterpart behind them, and products of 8-bit integers, as cases that can be timed and compared.

A case is a dict of plain values with a "kind":

    route     T rows of E logits to `top` experts each, their weights, and the routes grouped by expert
    combine   the outputs of `top` routes of T tokens, N values each, weighted and added (and another output, where "add")
    swiglu    silu(gate) * up of M rows of (gate | up), rounded to the model dtype, to 8-bit codes and a scale for each row, and back to values
    linear    x W^T: W in 8-bit codes with a scale for each channel, x in the model dtype, quantised on the way with a scale for each row
    moe       the experts of a layer in 8 bits: routed gate | up, gated activation, routed down, combined

The choice of experts: scores are a softmax or sigmoids of the logits; with "bias" a value for each expert is added for the choice alone.  With
"groups" > 1 the experts fall into groups of neighbours, whose score is the sum of their two best; only the best `kept` groups stay.
Experts are taken in descending order; of equals (in 64 bits) the larger logit, then the lower index comes first.  A logit of -inf
is never chosen: the last "padded" rows have no other, and no routes.  Weights are the scores of the chosen, over their sum where "renormalise", times "scale".

8 bits: d = max(max|x|, 1e-10) / 127 of a row, codes x / d rounded to the nearest, halves away from zero.

"dtype" is the model dtype, "logits" that of the logits.  Sizes are those of this repository's configurations and benchmark (the
Llama-3-8B linears, the Llama-3-70B MLP, sixteen experts of 2816 x 2048 and 2048 x 1408), and generic ones in between.
"""
import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one token of single-stream decoding: launch and latency
        {"name": "route t1 e64", "kind": "route", "T": 1, "E": 64, "top": 4, "score": "softmax", "bias": False, "groups": 1, "kept": 1, "renormalise": True,
         "scale": 1.0, "padded": 0, "logits": "f32"},
        # a long prompt over many experts in groups, balanced by a bias
        {"name": "route t8192 e256 groups", "kind": "route", "T": 8192, "E": 256, "top": 8, "score": "sigmoid", "bias": True, "groups": 8, "kept": 4,
         "renormalise": True, "scale": 2.5, "padded": 100, "logits": "bf16"},
        # an odd decoding batch, its routes together again beside the output of a shared expert
        {"name": "combine t13 n2048", "kind": "combine", "T": 13, "N": 2048, "top": 4, "add": True, "padded": 2, "dtype": "bf16"},
        # the same for a prompt
        {"name": "combine t4096 n4096", "kind": "combine", "T": 4096, "N": 4096, "top": 8, "add": False, "padded": 0, "dtype": "bf16"},
        # between the products of an MLP, an odd decoding batch
        {"name": "swiglu m13 i14336", "kind": "swiglu", "M": 13, "I": 14336, "dtype": "bf16"},
        # the same for a long prompt, binary16 model
        {"name": "swiglu m4096 i14336 f16", "kind": "swiglu", "M": 4096, "I": 14336, "dtype": "f16"},
        # single-stream decoding, the smallest projection
        {"name": "linear o m1", "kind": "linear", "M": 1, "N": 4096, "K": 4096, "dtype": "bf16"},
        # a ragged batch, binary16 model, a long k
        {"name": "linear down m200 f16", "kind": "linear", "M": 200, "N": 4096, "K": 14336, "dtype": "f16"},
        # an ordinary prompt
        {"name": "linear qkv m1024", "kind": "linear", "M": 1024, "N": 6144, "K": 4096, "dtype": "bf16"},
        # the largest prefill product
        {"name": "linear 70b gate_up m4096", "kind": "linear", "M": 4096, "N": 57344, "K": 8192, "dtype": "bf16"},
        # the expert block of a small decoding batch: few rows for each of many matrices
        {"name": "moe e16 t8", "kind": "moe", "E": 16, "hidden": 2048, "inter": 1408, "T": 8, "top": 4, "dtype": "bf16"},
        # the same for a prompt, uneven loads of hundreds of rows
        {"name": "moe e16 t4096", "kind": "moe", "E": 16, "hidden": 2048, "inter": 1408, "T": 4096, "top": 2, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], evenly spread over the logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["route", "route", "combine", "swiglu", "linear", "linear", "linear", "moe", "moe"])
    dtype = rng.choice(["bf16", "bf16", "f16"])

    def wide(lo, hi):   # a length along k: a multiple of sixteen
        return _log(rng, lo // 16, hi // 16) * 16

    T = _log(rng, 1, 8192 if kind == "route" else 4096)
    padded = rng.choice([0, 0, rng.randint(0, T) // 4])
    if kind == "route":
        E = rng.choice([8, 16, 30, 60, 64, 72, 128, 160, 256])
        groups = rng.choice([1, 1] + [g for g in (2, 3, 4, 8) if E % g == 0 and E // g >= 2])
        kept = rng.randint(1, groups)
        return {"kind": kind, "T": T, "E": E, "top": rng.randint(1, min(8, E // groups * kept)), "score": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.5, "groups": groups, "kept": kept, "renormalise": rng.random() < 0.7, "scale": rng.choice([1.0, 2.5]),
                "padded": padded, "logits": rng.choice(["f32", "bf16", "f16"])}
    if kind == "combine":
        return {"kind": kind, "T": T, "N": _log(rng, 256, 4096), "top": rng.randint(1, 8), "add": rng.random() < 0.5, "padded": padded, "dtype": dtype}
    if kind == "swiglu":
        return {"kind": kind, "M": T, "I": wide(256, 14336), "dtype": dtype}
    if kind == "linear":
        N, K = _log(rng, 256, 57344), wide(256, 28672)
        while N * K > 470e6:
            N //= 2
        return {"kind": kind, "M": T, "N": N if rng.random() < 0.4 else max(8, N // 8 * 8), "K": K, "dtype": dtype}
    E = rng.choice([4, 8, 16, 32, 60])
    return {"kind": kind, "E": E, "hidden": wide(256, 2816), "inter": wide(256, 1408), "T": T, "top": rng.choice([1, 2, 4]), "dtype": dtype}


# ------------------------------------------------------------------ the plain form: elementary operations of torch
def _plain_choice(logits, bias, c):
    """Experts [T, top] (-1: none) and weights, decided in 64 bits."""
    l = logits.double()
    able = l > float("-inf")
    if c["score"] == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-l))
    else:
        e = torch.where(able, torch.exp(l - l.amax(dim=1, keepdim=True)), 0.0)
        s = e / e.sum(dim=1, keepdim=True)
    none = torch.full_like(l, float("-inf"))
    key = torch.where(able, s if bias is None else s + bias.double(), none)
    if c["groups"] > 1:
        of = key.unflatten(1, (c["groups"], -1))
        best = of.sort(dim=2, descending=True).values[..., :2]
        total = torch.where(best > float("-inf"), best, 0.0).sum(dim=2)
        total = torch.where(best[..., 0] > float("-inf"), total, float("-inf"))
        ahead = total.argsort(dim=1, descending=True, stable=True)[:, : c["kept"]]
        stays = torch.zeros_like(total, dtype=torch.bool).scatter_(1, ahead, True)
        key = torch.where(stays.unsqueeze(2), of, float("-inf")).flatten(1)
    by_logit = torch.where(able, l, none).argsort(dim=1, descending=True, stable=True)
    order = by_logit.gather(1, key.gather(1, by_logit).argsort(dim=1, descending=True, stable=True))[:, : c["top"]]
    there = key.gather(1, order) > float("-inf")
    w = torch.where(there, s.gather(1, order), 0.0)
    if c["renormalise"]:
        w = w / w.sum(dim=1, keepdim=True)
    return torch.where(there, order, -1), torch.where(there, w * c["scale"], 0.0).float()


def _plain_routes(expert, E):
    """The routes grouped by expert: tokens [T top] (-1 behind the last), first routes of the experts [E + 1], the place of each choice (-1: none)."""
    T, top = expert.shape
    flat = expert.flatten()
    order = torch.where(flat < 0, E, flat).argsort(stable=True)
    count = (flat.unsqueeze(1) == torch.arange(E, device=flat.device)).sum(dim=0)
    offset = torch.cat((count.new_zeros(1), count.cumsum(0)))
    token = torch.where(flat[order] < 0, -1, order // top)
    row = torch.empty_like(order)
    row[order] = torch.arange(T * top, device=flat.device)
    return token.to(torch.int32), offset.to(torch.int32), torch.where(flat < 0, -1, row).reshape(T, top).to(torch.int32)


def _plain_combine(routes, weight, row, add):
    total = torch.zeros((row.shape[0], routes.shape[1]), device=routes.device) if add is None else add.float()
    for j in range(row.shape[1]):
        there = (row[:, j] >= 0).unsqueeze(1)
        part = routes[row[:, j].clamp_min(0).long()].float() * weight[:, j].unsqueeze(1)
        total = total + torch.where(there, part, 0.0)
    return total.to(routes.dtype)


def _plain_codes(x):
    """Codes as fp32 numbers, and the scale of each row."""
    v = x.float()
    d = v.abs().amax(dim=-1, keepdim=True).clamp_min(1e-10) / 127.0
    u = v / d
    whole = torch.trunc(u)
    return (whole + torch.where((u - whole).abs() >= 0.5, torch.sign(u), 0.0)).clamp(-127.0, 127.0), d.squeeze(-1)


def _plain_product(codes, d, w8, dw):
    """codes [.., M, K] as fp32 numbers times 8-bit w8 [.., N, K]: sums of 1024 products are exact in 32 bits, those of the pieces are whole numbers."""
    total = 0
    for k in range(0, codes.shape[-1], 1024):
        total = total + (codes[..., k:k + 1024] @ w8[..., k:k + 1024].float().transpose(-1, -2)).to(torch.int32)
    return total.float() * (d.unsqueeze(-1) * dw.unsqueeze(-2))


def _plain_linear(x, w8, dw):
    codes, d = _plain_codes(x)
    out = torch.empty((x.shape[0], w8.shape[0]), dtype=x.dtype, device=x.device)
    for n in range(0, w8.shape[0], 8192):   # in pieces: whole sums take their room
        out[:, n:n + 8192] = _plain_product(codes, d, w8[n:n + 8192], dw[n:n + 8192]).to(x.dtype)
    return out


def _plain_gated(h):
    """silu(gate) * up in the model dtype: in 64 bits, since a value next to a rounding border decides a code."""
    gate, up = h.double().chunk(2, dim=-1)
    return (gate / (1.0 + torch.exp(-gate)) * up).float().to(h.dtype)


def _plain_experts(x, w8, dw, expert, place, most):
    """x [R, K], a row for each route; route r is row place[r] of matrix expert[r]."""
    codes, d = _plain_codes(x)
    E = w8.shape[0]
    rows, scales = torch.zeros((E, most, x.shape[1]), device=x.device), torch.zeros((E, most), device=x.device)
    rows[expert, place], scales[expert, place] = codes, d
    return _plain_product(rows, scales, w8, dw)[expert, place].to(x.dtype)


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 8765)
    return g


def _activations(g, M, K, dtype):
    """N(0, 1) with one column in a hundred twenty times larger, as activations of a trained model look."""
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, torch.randperm(K, generator=g, device="cuda")[: K // 100]] *= 20.0
    return x.to(DTYPE[dtype])


def _matrix(g, N, K):
    """A stored matrix: 8-bit codes [N, K] and the scale of each channel [N]."""
    codes = torch.empty((N, K), dtype=torch.int8, device="cuda")
    scale = torch.empty(N, device="cuda")
    rows = max(1, (1 << 26) // K)
    for r in range(0, N, rows):
        W = torch.randn((min(rows, N - r), K), generator=g, device="cuda").mul_(0.02)
        W.mul_(1.0 + 9.0 * (torch.rand((W.shape[0], 1), generator=g, device="cuda") < 0.01))   # a few rows are larger
        d = W.abs().amax(dim=1, keepdim=True) / 127.0
        codes[r:r + rows] = torch.round(W / d).to(torch.int8)
        scale[r:r + rows] = d.squeeze(1)
    return codes, scale


def _experts(g, E, N, K):
    parts = [_matrix(g, N, K) for _ in range(E)]
    return torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])


def _logits(g, T, E, padded, dtype):
    l = 1.5 * torch.randn((T, E), generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")   # some experts are preferred
    l = l.to(DTYPE[dtype])
    if padded:
        l[T - padded:] = float("-inf")
    return l


def _some_routes(g, c):
    """Weights, grouped tokens, offsets and places as a router leaves them, and which row of which matrix each route is."""
    l = _logits(g, c["T"], c.get("E", 16), c.get("padded", 0), "f32")
    how = {"score": "softmax", "groups": 1, "kept": 1, "top": c["top"], "renormalise": True, "scale": 1.0}
    expert, weight = _plain_choice(l, None, how)
    token, offset, row = _plain_routes(expert, l.shape[1])
    return {"expert": expert.to(torch.int32), "weight": weight, "token": token, "offset": offset, "row": row}


def _inputs(c, seed):
    g, kind = _generator(seed), c["kind"]
    if kind == "route":
        l = _logits(g, c["T"], c["E"], c["padded"], c["logits"])
        return {"l": l, "bias": 0.1 * torch.randn(c["E"], generator=g, device="cuda") if c["bias"] else None}
    if kind == "combine":
        r = _some_routes(g, c)
        routes = _activations(g, c["T"] * c["top"], c["N"], c["dtype"])
        return {"y": routes, "add": _activations(g, c["T"], c["N"], c["dtype"]) if c["add"] else None, **r}
    if kind == "swiglu":
        return {"h": _activations(g, c["M"], 2 * c["I"], c["dtype"])}
    if kind == "linear":
        w = _matrix(g, c["N"], c["K"])
        return {"w": w, "x": _activations(g, c["M"], c["K"], c["dtype"])}
    up, down = _experts(g, c["E"], 2 * c["inter"], c["hidden"]), _experts(g, c["E"], c["hidden"], c["inter"])
    x, r = _activations(g, c["T"], c["hidden"], c["dtype"]), _some_routes(g, c)
    matrix = torch.repeat_interleave(torch.arange(c["E"], device="cuda"), r["offset"].diff().long())
    place = torch.arange(matrix.numel(), device="cuda") - r["offset"][matrix]
    return {"up": up, "down": down, "x": x, "matrix": matrix, "place": place, "most": int(r["offset"].diff().max()), **r}


def prepare(case, seed):
    c, s = case, {"c": case, "kind": case["kind"], **_inputs(case, seed)}
    if own:   # what a program keeps from call to call: matrices laid out once, workspaces, buffers
        import paper_2608_06763_b200 as cq
        if c["kind"] == "route":
            s["out"] = cq.cq_routes_empty(c["T"], c["E"], c["top"])
            s["ws"] = cq.cq_route_workspace(c["T"], c["E"])
        elif c["kind"] == "combine":
            s["routes"] = cq.Routes(s["expert"], s["weight"], s["token"], s["offset"], s["row"])
            s["out"] = torch.empty((c["T"], c["N"]), dtype=s["y"].dtype, device="cuda")
        elif c["kind"] == "swiglu":
            s["q"] = cq.cq_i8_empty(c["M"], c["I"])
            s["out"] = torch.empty((c["M"], c["I"]), dtype=s["h"].dtype, device="cuda")
        elif c["kind"] == "linear":
            s["w"] = cq.cq_i8_pack(*s["w"])
            s["ws"] = cq.cq_i8_workspace(s["w"], c["M"])
            s["out"] = torch.empty((c["M"], c["N"]), dtype=s["x"].dtype, device="cuda")
        else:
            s["up"], s["down"] = cq.cq_i8_pack(*s["up"]), cq.cq_i8_pack(*s["down"])
            s["routes"] = cq.Routes(s["expert"], s["weight"], s["token"], s["offset"], s["row"])
            s["ws"] = cq.cq_i8_moe_workspace(s["up"], s["down"], c["T"], c["top"])
            s["out"] = torch.empty((c["T"], c["hidden"]), dtype=s["x"].dtype, device="cuda")
    return s


def run(state):
    s, c, kind = state, state["c"], state["kind"]
    if own:
        import paper_2608_06763_b200 as cq
        if kind == "route":
            r = cq.cq_route(s["l"], c["top"], cq.CQ_SIGMOID if c["score"] == "sigmoid" else cq.CQ_SOFTMAX, bias=s["bias"], groups=c["groups"], groups_kept=c["kept"],
                            renormalise=c["renormalise"], scale=c["scale"], workspace=s["ws"], out=s["out"])
            return r.expert, r.weight, r.token, r.offset, r.row
        if kind == "combine":
            return cq.cq_combine(s["y"], s["routes"], add=s["add"], out=s["out"])
        if kind == "swiglu":
            return cq.cq_i8_dequantize(cq.cq_i8_swiglu_quantize(s["h"], out=s["q"]), out=s["out"])
        if kind == "linear":
            return cq.cq_i8_gemm(s["w"], s["x"], workspace=s["ws"], out=s["out"])
        return cq.cq_i8_moe(s["up"], s["down"], s["x"], s["routes"], workspace=s["ws"], out=s["out"])
    if kind == "route":
        expert, weight = _plain_choice(s["l"], s["bias"], c)
        return (expert.to(torch.int32), weight, *_plain_routes(expert, c["E"]))
    if kind == "combine":
        return _plain_combine(s["y"], s["weight"], s["row"], s["add"])
    if kind == "swiglu":
        codes, d = _plain_codes(_plain_gated(s["h"]))
        return (codes * d.unsqueeze(-1)).to(s["h"].dtype)
    if kind == "linear":
        return _plain_linear(s["x"], *s["w"])
    where = (s["matrix"], s["place"], s["most"])
    rows = s["x"][s["token"].long()]
    a = _plain_gated(_plain_experts(rows, *s["up"], *where))
    return _plain_combine(_plain_experts(a, *s["down"], *where), s["weight"], s["row"], None)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, kind = case, case["kind"]
    if kind == "route":
        n = c["T"] * c["E"]
        return {"bytes": n * (4 if c["logits"] == "f32" else 2) + 16 * c["T"] * c["top"] + 4 * (c["E"] + 1) + (4 * c["E"] if c["bias"] else 0), "flops": 6.0 * n}
    if kind == "combine":
        live = c["T"] - c["padded"]
        return {"bytes": 2 * c["N"] * (live * c["top"] + c["T"] * (2 if c["add"] else 1)) + 8 * c["T"] * c["top"], "flops": 2.0 * live * c["top"] * c["N"]}
    if kind == "swiglu":
        n = c["M"] * c["I"]
        return {"bytes": n * (4 + 2), "flops": 9.0 * n}
    if kind == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": N * K + 4 * N + 2 * M * (K + N), "flops": 2.0 * M * N * K}
    R, per = c["T"] * c["top"], c["hidden"] * c["inter"] * 3
    met = min(c["E"], R)   # no more matrices than routes are met
    return {"bytes": met * per + 4 * c["T"] * c["hidden"] + 12 * R, "flops": 2.0 * R * per}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_route(l, bias, c):
    x, T, E = l.double(), c["T"], c["E"]
    none = float("-inf")
    out = ~(x > none)
    if c["score"] == "sigmoid":
        s = torch.sigmoid(x)
    else:
        s = torch.softmax(x.masked_fill(out, -1e300), dim=1)
    key = (s + (0.0 if bias is None else bias.double())).masked_fill(out, none)
    if c["groups"] > 1:
        left = key.reshape(T, c["groups"], -1).clone()
        total, alive = torch.zeros((T, c["groups"]), dtype=torch.float64, device=l.device), None
        for _ in range(2):
            m, at = left.max(dim=2)
            alive = m > none if alive is None else alive
            total += torch.where(m > none, m, 0.0)
            left.scatter_(2, at.unsqueeze(2), none)
        total = total.masked_fill(~alive, none)
        index = torch.arange(c["groups"], device=l.device)
        better = (total.unsqueeze(1) > total.unsqueeze(2)) | ((total.unsqueeze(1) == total.unsqueeze(2)) & (index.unsqueeze(0) < index.unsqueeze(1)))
        stays = better.sum(dim=2) < c["kept"]
        key = key.masked_fill(~stays.repeat_interleave(E // c["groups"], dim=1), none)
    chosen = []
    for _ in range(c["top"]):   # the largest, among its equals the largest logit, among those the first
        m = key.max(dim=1, keepdim=True).values
        same = (key == m) & (key > none)
        same &= x == x.masked_fill(~same, none).max(dim=1, keepdim=True).values
        at = torch.where(same, torch.arange(E, device=l.device), E).min(dim=1).values
        chosen.append(torch.where(at < E, at, -1))
        key = key.scatter(1, at.clamp_max(E - 1).unsqueeze(1), none)
    expert = torch.stack(chosen, dim=1)
    w = s.gather(1, expert.clamp_min(0)).masked_fill(expert < 0, 0.0)
    if c["renormalise"]:
        w = w / torch.where(w.sum(dim=1, keepdim=True) > 0, w.sum(dim=1, keepdim=True), 1.0)
    R = T * c["top"]
    token, row = torch.full((R,), -1, dtype=torch.int32), torch.full((T, c["top"]), -1, dtype=torch.int32)
    of = [[] for _ in range(E)]
    for t, picks in enumerate(expert.tolist()):
        for j, e in enumerate(picks):
            if e >= 0:
                of[e].append((t, j))
    offset, at = [0], 0
    flat = [p for group in of for p in group]
    for group in of:
        at += len(group)
        offset.append(at)
    if flat:
        pairs = torch.tensor(flat)
        token[: len(flat)] = pairs[:, 0].to(torch.int32)
        row[pairs[:, 0], pairs[:, 1]] = torch.arange(len(flat), dtype=torch.int32)
    dev = l.device
    return expert.to(torch.int32), w * c["scale"], token.to(dev), torch.tensor(offset, dtype=torch.int32, device=dev), row.to(dev)


def _exact_combine(y, weight, row, add):
    """The sum over the routes as a product with one weight for each place; y in 64 bits."""
    T, top = row.shape
    picked = torch.cat((y, y.new_zeros(1, y.shape[1])))[torch.where(row < 0, y.shape[0], row.long()).flatten()].reshape(T, top, -1)
    out = torch.bmm(weight.double().unsqueeze(1), picked).squeeze(1)
    return out if add is None else out + add.double()


def _exact_codes(x):
    """Codes and scales from the definition: the scale and the quotient are 32-bit numbers, correctly rounded, the decision exact."""
    v = x.double()
    d = (v.abs().max(dim=-1).values.clamp_min(float(torch.tensor(1e-10))) / 127.0).float().double()
    u = (v / d.unsqueeze(-1)).float().double()
    return (torch.sign(u) * torch.floor(u.abs() + 0.5)).clamp(-127, 127), d


def _exact_product(x, w8, dw):
    q, d = _exact_codes(x)
    out = torch.empty((x.shape[0], w8.shape[0]), dtype=torch.float64, device=x.device)
    rows = max(1, (1 << 25) // x.shape[1])
    for r in range(0, w8.shape[0], rows):
        out[:, r:r + rows] = (q @ w8[r:r + rows].double().T) * dw[r:r + rows].double()
    return out * d.unsqueeze(1)


def _exact_experts(x, w8, dw, matrix):
    out = torch.empty((x.shape[0], w8.shape[1]), dtype=torch.float64, device=x.device)
    for e in range(w8.shape[0]):
        mine = matrix == e
        if mine.any():
            out[mine] = _exact_product(x[mine], w8[e], dw[e])
    return out


def _exact_gated(h):
    gate, up = h[:, : h.shape[1] // 2].double(), h[:, h.shape[1] // 2:].double()
    return (gate * torch.sigmoid(gate) * up).to(h.dtype)


def exact(case, seed):
    c, kind = case, case["kind"]
    if kind == "linear" and 2.0 * c["M"] * c["N"] * c["K"] > 4e14:
        return None   # half a minute and more in 64 bits
    s = _inputs(case, seed)
    if kind == "route":
        return _exact_route(s["l"], s["bias"], c)
    if kind == "combine":
        return _exact_combine(s["y"].double(), s["weight"], s["row"], s["add"])
    if kind == "swiglu":
        q, d = _exact_codes(_exact_gated(s["h"]))
        return q * d.unsqueeze(1)
    if kind == "linear":
        return _exact_product(s["x"], *s["w"])
    h = _exact_experts(s["x"][s["token"].long()], *s["up"], s["matrix"]).to(s["x"].dtype)   # the products return the model dtype
    y = _exact_experts(_exact_gated(h), *s["down"], s["matrix"]).to(s["x"].dtype)
    return _exact_combine(y.double(), s["weight"], s["row"], None)
