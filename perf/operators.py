"""Operators on 4-bit floating point with block scales, as cases that can be timed and compared.

A value is an e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) times the scale of its block of consecutive k:

    "mx"   blocks of 32, the scale a power of two (e8m0):  e = floor(log2 max|x|) - 2
    "nv"   blocks of 16, the scale in e4m3, and one fp32 scale g for the whole tensor:  s = RNE(max|x| / (6 g))

A case is a dict of plain values with a "kind":

    quantise  M x K values to codes and scales, and back to the values they stand for
    swiglu    silu(gate) * up of M rows of (gate | up), rounded to the model dtype, to codes and scales, and back to values
    linear    x W^T: W stored in 4 bits, x in the model dtype, quantised on the way
    routed    T tokens, `top` routes each, through one of E matrices by the route; rows grouped by matrix, the groups' offsets on the GPU
    moe       the experts of a layer: routed gate | up, gated activation, routed down

"fmt" is the format, "dtype" the model dtype ("f32": a matrix still in training precision).  Sizes are those of this
repository's configurations and benchmark (the Llama-3-8B linears, the Llama-3-70B MLP, sixteen matrices of 2816 x 2048), and
generic ones in between.
"""
import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = {"mx": 32, "nv": 16}
BYTES = {"mx": 0.5 + 1 / 32, "nv": 0.5 + 1 / 16}   # of a stored value


def listed():
    return [
        # activations of one token in front of a projection: launch and latency
        {"name": "quantise m1 k4096 nv", "kind": "quantise", "M": 1, "K": 4096, "fmt": "nv", "dtype": "bf16"},
        # a trained matrix to 4 bits and back, to see what it loses
        {"name": "quantise 14336x4096 mx", "kind": "quantise", "M": 14336, "K": 4096, "fmt": "mx", "dtype": "f32"},
        # between the products of an MLP, an odd decoding batch
        {"name": "swiglu m13 i14336 nv", "kind": "swiglu", "M": 13, "I": 14336, "fmt": "nv", "dtype": "bf16"},
        # the same for a long prompt
        {"name": "swiglu m4096 i14336 mx", "kind": "swiglu", "M": 4096, "I": 14336, "fmt": "mx", "dtype": "bf16"},
        # single-stream decoding, the smallest projection
        {"name": "linear o m1 nv", "kind": "linear", "M": 1, "N": 4096, "K": 4096, "fmt": "nv", "dtype": "bf16"},
        # batched decoding, an odd batch
        {"name": "linear gate_up m13 mx", "kind": "linear", "M": 13, "N": 28672, "K": 4096, "fmt": "mx", "dtype": "bf16"},
        # a short prompt of ragged length, binary16 model
        {"name": "linear down m200 nv f16", "kind": "linear", "M": 200, "N": 4096, "K": 14336, "fmt": "nv", "dtype": "f16"},
        # an ordinary prompt
        {"name": "linear qkv m1024 mx", "kind": "linear", "M": 1024, "N": 6144, "K": 4096, "fmt": "mx", "dtype": "bf16"},
        # the largest prefill product
        {"name": "linear 70b gate_up m4096 nv", "kind": "linear", "M": 4096, "N": 57344, "K": 8192, "fmt": "nv", "dtype": "bf16"},
        # a decoding batch over the experts of a layer: few rows for each of many matrices
        {"name": "routed e16 t192 mx", "kind": "routed", "E": 16, "N": 2816, "K": 2048, "T": 192, "top": 2, "fmt": "mx", "dtype": "bf16"},
        # a prompt over the same experts, uneven loads of hundreds of rows
        {"name": "routed e16 t4096 nv", "kind": "routed", "E": 16, "N": 2816, "K": 2048, "T": 4096, "top": 2, "fmt": "nv", "dtype": "bf16"},
        # the whole expert block for a small decoding batch
        {"name": "moe e16 t8 nv", "kind": "moe", "E": 16, "hidden": 2048, "inter": 1408, "T": 8, "top": 4, "fmt": "nv", "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], evenly spread over the logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    fmt, dtype = rng.choice(["mx", "nv"]), rng.choice(["bf16", "bf16", "f16"])
    kind = rng.choice(["quantise", "swiglu", "linear", "linear", "linear", "routed", "routed", "moe"])
    block, how = BLOCK[fmt], {"fmt": fmt, "dtype": dtype}

    def wide(lo, hi):   # a length along k: whole blocks
        return max(1, _log(rng, lo, hi) // block) * block

    if kind == "quantise":
        how["dtype"] = rng.choice(["bf16", "f16", "f32"])
        return {"kind": kind, "M": _log(rng, 1, 14336), "K": wide(64, 4096), **how}
    if kind == "swiglu":
        return {"kind": kind, "M": _log(rng, 1, 4096), "I": wide(256, 14336), **how}
    if kind == "linear":
        M, N, K = _log(rng, 1, 4096), _log(rng, 256, 57344), wide(256, 28672)
        while N * K > 470e6:
            N //= 2
        return {"kind": kind, "M": M, "N": N if rng.random() < 0.4 else max(8, N // 8 * 8), "K": K, **how}
    E, T = rng.choice([4, 8, 16, 32]), _log(rng, 1, 4096)
    top = rng.choice([1, 2, 4])
    if kind == "routed":
        return {"kind": kind, "E": E, "N": _log(rng, 256, 4096), "K": wide(256, 4096), "T": T, "top": top, **how}
    return {"kind": kind, "E": E, "hidden": max(256, _log(rng, 256, 2816) // 32 * 32), "inter": max(256, _log(rng, 256, 1408) // 32 * 32), "T": T, "top": top, **how}


# ------------------------------------------------------------------ the plain form: elementary operations of torch
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _round_e2m1(u):
    """Codes 0 .. 7 of |u| and 8 for a sign; a value half way between two goes to the even code."""
    a = u.abs()
    code = (a > 0.25).to(torch.uint8)
    for above in (a >= 0.75, a > 1.25, a >= 1.75, a > 2.5, a >= 3.5, a > 5.0):
        code += above
    return code + 8 * (u < 0).to(torch.uint8)


def _power_of_two(e):
    """2^e in 64 bits, from the bits: pow and exp2 need not be exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x, fmt, g):
    """Codes [..., K] and scales [..., K / block] in fp32 (without g) of x; g: fp32, one for the last two axes, or None."""
    block = BLOCK[fmt]
    v = x.float().unflatten(-1, (-1, block))
    top = v.abs().amax(dim=-1, keepdim=True)
    if fmt == "mx":
        e = torch.frexp(top).exponent - 3
        e = torch.where(top > 0, e, -127).clamp(-127, 127)
        s = _power_of_two(e)
        u = v.double() / s   # far exponents leave the range of 32 bits on the way
        s = s.float()
    else:
        r = 1.0 / g.reshape(g.shape + (1,) * (v.dim() - g.dim()))
        s = ((top * r).double() / 6.0).float().clamp(2.0 ** -9, 448.0).to(torch.float8_e4m3fn).float()
        u = v * (r / s)
    return _round_e2m1(u).flatten(-2), s.squeeze(-1)


def _values(codes, s, fmt, g=None):
    """The fp32 values that codes and scales stand for."""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=codes.device)
    if g is not None:
        s = s * g.reshape(g.shape + (1,) * (s.dim() - g.dim()))
    return (table[codes.long()].unflatten(-1, (-1, BLOCK[fmt])) * s.unsqueeze(-1)).flatten(-2)


def _unpack(packed):
    """Codes one to a byte from two to a byte, the first in the low half."""
    return torch.stack((packed & 15, packed >> 4), dim=-1).flatten(-2)


def _stored_scale(stored, fmt):
    return _power_of_two(stored.long() - 127).float() if fmt == "mx" else stored.view(torch.float8_e4m3fn).float()


def _times(g, h):
    return 1.0 if g is None else g if h is None else g * h


def _matrix_values(w, fmt):
    codes, stored, _ = w
    out = torch.empty(codes.shape[:-1] + (codes.shape[-1] * 2,), device=codes.device)
    rows = max(1, (1 << 26) // out.shape[-1])
    flat, c, s = out.flatten(0, -2), codes.flatten(0, -2), stored.flatten(0, -2)
    for r in range(0, flat.shape[0], rows):   # in pieces: the table look-up wants eight bytes a code
        part = slice(r, r + rows)
        flat[part] = _values(_unpack(c[part]), _stored_scale(s[part], fmt), fmt)
    return out


def _plain_linear(w, x, g, fmt):
    codes, s = _quantise(x, fmt, g)
    return ((_values(codes, s, fmt) @ _matrix_values(w, fmt).T) * _times(w[2], g)).to(x.dtype)


def _plain_routed(w, x, g, fmt, expert, place, most):
    """x [R, K], a row for each route; route r is row place[r] of matrix expert[r]."""
    codes, s = _quantise(x, fmt, g)
    E, K = w[0].shape[0], x.shape[1]
    rows = torch.zeros((E, most, K), device=x.device)
    rows[expert, place] = _values(codes, s, fmt)
    y = torch.bmm(rows, _matrix_values(w, fmt).transpose(1, 2))
    if g is not None:
        y = y * (w[2] * g)[:, None, None]
    return y[expert, place].to(x.dtype)


def _gated(h):
    """silu(gate) * up in the model dtype: in 64 bits, since a value next to a rounding border decides a code."""
    gate, up = h.double().chunk(2, dim=-1)
    return (gate / (1.0 + torch.exp(-gate)) * up).float().to(h.dtype)


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 4321)
    return g


def _activations(g, M, K, dtype):
    """N(0, 1) with one column in a hundred twenty times larger, as activations of a trained model look."""
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, torch.randperm(K, generator=g, device="cuda")[: K // 100]] *= 20.0
    return x.to(DTYPE[dtype])


def _weights(g, N, K):
    W = torch.randn((N, K), generator=g, device="cuda").mul_(0.02)
    return W.mul_(1.0 + 9.0 * (torch.rand((N, 1), generator=g, device="cuda") < 0.01))   # a few rows are larger


def _tensor_scale(x, fmt):
    """The scale g that brings the largest value of x to the end of the range."""
    return x.abs().amax().float() / (448.0 * 6.0) if fmt == "nv" else None


def _matrix(g, N, K, fmt):
    """A stored matrix of a checkpoint: codes two to a byte [N, K / 2], scales a byte each [N, K / block], g or None."""
    codes = torch.empty((N, K // 2), dtype=torch.uint8, device="cuda")
    stored = torch.empty((N, K // BLOCK[fmt]), dtype=torch.uint8, device="cuda")
    scale = torch.tensor(0.02 * 5.5 * 10 / (448.0 * 6.0), device="cuda") if fmt == "nv" else None
    rows = max(1, (1 << 26) // K)
    for r in range(0, N, rows):
        c, s = _quantise(_weights(g, min(rows, N - r), K), fmt, scale)
        codes[r:r + rows] = c[:, 0::2] | (c[:, 1::2] << 4)
        stored[r:r + rows] = (torch.frexp(s).exponent + 126).to(torch.uint8) if fmt == "mx" else s.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, stored, scale


def _experts(g, E, N, K, fmt):
    parts = [_matrix(g, N, K, fmt) for _ in range(E)]
    scale = torch.stack([p[2] for p in parts]) * (0.75 + 0.5 * torch.rand(E, generator=g, device="cuda")) if fmt == "nv" else None
    return torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts]), scale


def _routes(g, c):
    """Token, matrix and row within the matrix of each route, routes grouped by matrix; the groups' offsets; the longest group."""
    load = torch.rand((c["T"], c["E"]), generator=g, device="cuda") + 0.5 * torch.rand(c["E"], generator=g, device="cuda")   # some matrices are preferred
    chosen = load.topk(c["top"], dim=1).indices.flatten()
    order = chosen.argsort(stable=True)
    expert = chosen[order]
    count = torch.bincount(chosen, minlength=c["E"])
    offset = torch.cat((count.new_zeros(1), count.cumsum(0)))
    place = torch.arange(order.numel(), device="cuda") - offset[expert]
    return {"token": (order // c["top"]).to(torch.int32), "expert": expert, "place": place, "offset": offset.to(torch.int32), "most": int(count.max())}


def _inputs(c, seed):
    g, kind, fmt = _generator(seed), c["kind"], c["fmt"]
    if kind == "quantise":
        x = _weights(g, c["M"], c["K"]) if c["dtype"] == "f32" else _activations(g, c["M"], c["K"], c["dtype"])
        return {"x": x, "g": _tensor_scale(x, fmt)}
    if kind == "swiglu":
        h = _activations(g, c["M"], 2 * c["I"], c["dtype"])
        g = torch.tensor(60.0 / 448.0, device="cuda") if fmt == "nv" else None   # calibrated beforehand: activations reach some 360
        return {"h": h, "g": g}
    if kind == "linear":
        w = _matrix(g, c["N"], c["K"], fmt)
        x = _activations(g, c["M"], c["K"], c["dtype"])
        return {"w": w, "x": x, "g": _tensor_scale(x, fmt)}
    if kind == "routed":
        w = _experts(g, c["E"], c["N"], c["K"], fmt)
        x = _activations(g, c["T"], c["K"], c["dtype"])
        return {"w": w, "x": x, "g": _tensor_scale(x, fmt), **_routes(g, c)}
    up = _experts(g, c["E"], 2 * c["inter"], c["hidden"], fmt)
    down = _experts(g, c["E"], c["hidden"], c["inter"], fmt)
    x = _activations(g, c["T"], c["hidden"], c["dtype"])
    g2 = torch.tensor(60.0 / 448.0, device="cuda") if fmt == "nv" else None
    return {"up": up, "down": down, "x": x, "g": _tensor_scale(x, fmt), "g2": g2, **_routes(g, c)}


def prepare(case, seed):
    s = {"kind": case["kind"], "fmt": case["fmt"], **_inputs(case, seed)}
    if own:   # what a program keeps from call to call: matrices laid out once, workspaces, buffers
        import paper_2608_06763_b200 as cq
        s["fp4"] = cq.CQ_MXFP4 if case["fmt"] == "mx" else cq.CQ_NVFP4
        if case["kind"] == "quantise":
            s["q"] = cq.cq_fp4_empty(s["fp4"], *s["x"].shape)
            s["out"] = torch.empty(s["x"].shape, dtype=_model_dtype(s["x"]), device="cuda")
        elif case["kind"] == "swiglu":
            s["q"] = cq.cq_fp4_empty(s["fp4"], case["M"], case["I"])
            s["out"] = torch.empty((case["M"], case["I"]), dtype=s["h"].dtype, device="cuda")
        else:
            for name in ("w", "up", "down"):
                if name in s:
                    codes, stored, scale = s[name]
                    s[name] = cq.cq_fp4_pack(codes, stored, s["fp4"], scale)
            if case["kind"] == "linear":
                s["ws"] = cq.cq_fp4_workspace(s["w"], case["M"])
                s["out"] = torch.empty((case["M"], case["N"]), dtype=s["x"].dtype, device="cuda")
            elif case["kind"] == "routed":
                s["ws"] = cq.cq_fp4_workspace(s["w"], s["token"].numel())
                s["out"] = torch.empty((s["token"].numel(), case["N"]), dtype=s["x"].dtype, device="cuda")
            else:
                R = s["token"].numel()
                s["ws"], s["ws2"] = cq.cq_fp4_workspace(s["up"], R), cq.cq_fp4_workspace(s["down"], R)
                s["h"] = torch.empty((R, 2 * case["inter"]), dtype=s["x"].dtype, device="cuda")
                s["q"] = cq.cq_fp4_empty(s["fp4"], R, case["inter"], groups=case["E"])
                s["out"] = torch.empty((R, case["hidden"]), dtype=s["x"].dtype, device="cuda")
    return s


def _model_dtype(x):
    return torch.bfloat16 if x.dtype == torch.float32 else x.dtype


def run(state):
    s, kind, fmt = state, state["kind"], state["fmt"]
    if own:
        import paper_2608_06763_b200 as cq
        if kind == "quantise":
            return cq.cq_fp4_dequantize(cq.cq_fp4_quantize(s["x"], s["fp4"], s["g"], out=s["q"]), out=s["out"])
        if kind == "swiglu":
            return cq.cq_fp4_dequantize(cq.cq_fp4_swiglu_quantize(s["h"], s["fp4"], s["g"], out=s["q"]), out=s["out"])
        if kind == "linear":
            return cq.cq_fp4_gemm(s["w"], s["x"], s["g"], workspace=s["ws"], out=s["out"])
        if kind == "routed":
            return cq.cq_fp4_gemm_routed(s["w"], s["x"], s["token"], s["offset"], s["g"], workspace=s["ws"], out=s["out"])
        h = cq.cq_fp4_gemm_routed(s["up"], s["x"], s["token"], s["offset"], s["g"], workspace=s["ws"], out=s["h"])
        a = cq.cq_fp4_swiglu_quantize(h, s["fp4"], s["g2"], expert_offset=s["offset"], out=s["q"])
        return cq.cq_fp4_gemm_routed(s["down"], a, None, s["offset"], workspace=s["ws2"], out=s["out"])
    if kind == "quantise":
        return _values(*_quantise(s["x"], fmt, s["g"]), fmt, s["g"]).to(_model_dtype(s["x"]))
    if kind == "swiglu":
        return _values(*_quantise(_gated(s["h"]), fmt, s["g"]), fmt, s["g"]).to(s["h"].dtype)
    if kind == "linear":
        return _plain_linear(s["w"], s["x"], s["g"], fmt)
    rows, where = s["x"][s["token"].long()], (s["expert"], s["place"], s["most"])
    if kind == "routed":
        return _plain_routed(s["w"], rows, s["g"], fmt, *where)
    return _plain_routed(s["down"], _gated(_plain_routed(s["up"], rows, s["g"], fmt, *where)), s["g2"], fmt, *where)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, kind, stored = case, case["kind"], BYTES[case["fmt"]]
    if kind == "quantise":
        n = c["M"] * c["K"]
        return {"bytes": n * ((4 if c["dtype"] == "f32" else 2) + 2), "flops": 4.0 * n}
    if kind == "swiglu":
        n = c["M"] * c["I"]
        return {"bytes": n * (4 + 2), "flops": 9.0 * n}
    if kind == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": N * K * stored + 2 * M * (K + N), "flops": 2.0 * M * N * K}
    R = c["T"] * c["top"]
    met = min(c["E"], R)   # no more matrices than routes are met
    if kind == "routed":
        return {"bytes": met * c["N"] * c["K"] * stored + 2 * c["T"] * c["K"] + 2 * R * c["N"], "flops": 2.0 * R * c["N"] * c["K"]}
    per = c["hidden"] * c["inter"] * 3
    return {"bytes": met * per * stored + 2 * c["T"] * c["hidden"] + 2 * R * c["hidden"], "flops": 2.0 * R * per}


# ------------------------------------------------------------------ the same in 64 bits
def _scaled(a, e):
    """a 2^e, exactly: two is squared, never raised to a power by a logarithm."""
    bit, factor = 2.0, torch.ones_like(a)
    for k in range(7):
        factor = factor * torch.where((e.abs() >> k) & 1 == 1, bit, 1.0).double()
        bit = bit * bit
    return torch.where(e >= 0, a * factor, a / factor)


def _to_grid(u, least, bits, most):
    """The nearest value with `bits` binary places below its leading one (no finer than those of `least`), even ones on ties."""
    a = u.double().abs().clamp_max(most)
    place = torch.frexp(a.clamp_min(least)).exponent - 1 - bits
    return _scaled(torch.round(_scaled(a, -place)), place) * torch.sign(u.double())


def _exact_values(x, fmt, g):
    """What quantising and reading back makes of x, from the definition: the factors are 32-bit numbers, the decisions exact."""
    v = x.double().reshape(*x.shape[:-1], -1, BLOCK[fmt])
    top = v.abs().amax(dim=-1, keepdim=True)
    if fmt == "mx":
        s = _scaled(torch.ones_like(top), (torch.frexp(top.clamp_min(2.0 ** -140)).exponent - 3).clamp(-127, 127))
        return (_to_grid(v / s, 1.0, 1, 6.0) * s).reshape(x.shape)
    r = (1.0 / g.double()).float().double()
    s = _to_grid((((top * r).float().double()) / 6.0).clamp_min(2.0 ** -9), 2.0 ** -6, 3, 448.0)
    u = (v * (r / s).float().double()).float()
    return (_to_grid(u, 1.0, 1, 6.0) * (s * g.double()).float().double()).reshape(x.shape)


def _exact_matrix(w, fmt):
    codes, stored, g = w
    low, high = (codes & 15).long(), (codes >> 4).long()
    both = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.long, device=codes.device)
    both[..., 0::2], both[..., 1::2] = low, high
    mag = (both & 7).double()
    # a code is two bits of exponent and one of fraction; exponent 0 is the subnormal half
    value = torch.where(mag < 2, mag * 0.5, _scaled(1 + 0.5 * (mag % 2), ((both & 7) >> 1) - 1))
    b = stored.long()
    if fmt == "mx":
        s = _scaled(torch.ones(b.shape, dtype=torch.float64, device=b.device), b - 127)
    else:
        s = torch.where(b >= 8, _scaled(1 + (b & 7).double() / 8, (b >> 3) - 7), (b & 7).double() * 2.0 ** -9)
    return value * (1 - 2 * (both >> 3)) * s.repeat_interleave(BLOCK[fmt], dim=-1)


def _exact_product(w, xv, fmt):
    """xv [rows, K] in 64 bits times a stored matrix, in pieces."""
    codes, stored, g = w
    out = torch.empty((xv.shape[0], codes.shape[0]), dtype=torch.float64, device=xv.device)
    rows = max(1, (1 << 25) // xv.shape[1])
    for r in range(0, codes.shape[0], rows):
        part = slice(r, r + rows)
        out[:, part] = xv @ _exact_matrix((codes[part], stored[part], g), fmt).T
    return out if g is None else out * g.double()


def _exact_routed(w, xv, fmt, expert):
    out = torch.empty((xv.shape[0], w[0].shape[1]), dtype=torch.float64, device=xv.device)
    for e in range(w[0].shape[0]):
        mine = expert == e
        out[mine] = _exact_product((w[0][e], w[1][e], None if w[2] is None else w[2][e]), xv[mine], fmt)
    return out


def _exact_gated(h, dtype):
    gate, up = h[:, : h.shape[1] // 2].double(), h[:, h.shape[1] // 2:].double()
    return (gate * torch.sigmoid(gate) * up).to(dtype)


def exact(case, seed):
    c, kind, fmt = case, case["kind"], case["fmt"]
    if kind == "linear" and 2.0 * c["M"] * c["N"] * c["K"] > 4e14:
        return None   # half a minute and more in 64 bits
    s = _inputs(case, seed)
    if kind == "quantise":
        return _exact_values(s["x"], fmt, s["g"])
    if kind == "swiglu":
        return _exact_values(_exact_gated(s["h"], s["h"].dtype), fmt, s["g"])
    if kind == "linear":
        return _exact_product(s["w"], _exact_values(s["x"], fmt, s["g"]), fmt)
    rows = _exact_values(s["x"], fmt, s["g"])[s["token"].long()]
    if kind == "routed":
        return _exact_routed(s["w"], rows, fmt, s["expert"])
    h = _exact_routed(s["up"], rows, fmt, s["expert"]).to(s["x"].dtype)   # the first product returns the model dtype
    return _exact_routed(s["down"], _exact_values(_exact_gated(h, h.dtype), fmt, s["g2"]), fmt, s["expert"])
