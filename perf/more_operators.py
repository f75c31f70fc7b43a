"""A feed-forward block in 8 bits and its optimiser's step: measured cases, plain forms and 64-bit values.

Next to the 8-bit norm, product and weight gradient, one training or serving step of such a block runs:

gemm   z = op(A) op(B) + bias, c = act(z) + r, both operands e4m3 numbers with a scale for each block of 128 along the summed
       index; z, c in bf16 or fp32, c also as e4m3 numbers with one power-of-two scale for 128 features of a token; and its
       gradient form c = op(A) op(B) act'(z), z given
act    the activation's backward pass, dz = dy act'(z), with the bias's gradient (dz summed over the tokens) and dz in 8 bits
adamw  one AdamW step over all tensors of some layers, its two moments in fp32 or in 8 bits (m and sqrt(v) as e4m3 numbers with
       one power-of-two scale for 128 consecutive elements, rounded at random by a hash of the elements' numbers)

Storage is the library's: column-major with leading dimensions, so a torch tensor of shape [cols, ld].  A token is one
column.  8-bit numbers and their scales are returned in their own floating types, i.e. as the values they stand for.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ---- the cases ------------------------------------------------------------------------------------------------------
def _gemm(name, m, n, k, act, **more):
    return {"name": name, "op": "gemm", "m": m, "n": n, "k": k, "ta": "T", "act": act, "grad": False, "bias": True, "res": False, "z": False, "c": True, "q": False,
            "out": "bf16", "scale": "e8m0", "ba": 128, "bb": 1, "pad": 0, **more}


def listed():
    return [
        # one decoding step of 8 sequences, first product of the block: latency and reading the weight
        _gemm("up_decode_16384x8x4096", 16384, 8, 4096, "gelu", c=False, q=True),
        # the same step's second product, onto the residual stream
        _gemm("down_decode_4096x8x16384", 4096, 8, 16384, "none", res=True),
        # a training micro-batch of 8192 tokens: pre-activations kept, result in 8 bits for the next product and for the weight gradient
        _gemm("up_train_16384x8192x4096", 16384, 8192, 4096, "gelu", z=True, c=False, q=True),
        # its second product with bias and residual: the largest
        _gemm("down_train_4096x8192x16384", 4096, 8192, 16384, "none", res=True),
        # its backward pass: gradient of the pre-activations, kept for the weight gradient and quantised for the next product
        _gemm("dgrad_16384x8192x4096", 16384, 8192, 4096, "gelu", ta="N", grad=True, bias=False, q=True),
        # odd everything: fp32 scales of single rows, fp32 results, everything in the epilogue
        _gemm("odd_1001x999x1003", 1001, 999, 1003, "silu", res=True, z=True, out="f32", scale="f32", ba=1, pad=32),
        # a few odd tokens of a small model in fp32
        {"name": "act_backward_33x1003", "op": "act", "d": 1003, "t": 33, "act": "silu", "dz": True, "q": True, "db": True, "type": "f32", "pad": 24},
        # the micro-batch: gradient of the pre-activations where the product before did not make it
        {"name": "act_backward_8192x16384", "op": "act", "d": 16384, "t": 8192, "act": "gelu_tanh", "dz": True, "q": True, "db": True, "type": "bf16", "pad": 0},
        # the gradient that reaches the block: quantised, and the second bias's gradient
        {"name": "bias_gradient_8192x4096", "op": "act", "d": 4096, "t": 8192, "act": "none", "dz": False, "q": True, "db": True, "type": "bf16", "pad": 0},
        # a small model's step: ten tensors, latency
        {"name": "adamw8_2x384x512", "op": "adamw", "layers": 2, "d": 384, "f": 512, "bits": 8, "param": "f32", "grad": "f32", "scaled": False, "offset": 0},
        # odd sizes, states in 32 bits, the gradient scaled (clipping), tensors that start anywhere
        {"name": "adamw32_24x515x1003", "op": "adamw", "layers": 24, "d": 515, "f": 1003, "bits": 32, "param": "f32", "grad": "f32", "scaled": True, "offset": 3},
        # 268 million parameters in fp32, bf16 gradients, states in 8 bits
        {"name": "adamw8_2x4096x16384", "op": "adamw", "layers": 2, "d": 4096, "f": 16384, "bits": 8, "param": "f32", "grad": "bf16", "scaled": True, "offset": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo=128, hi=16384):
    """Half of them multiples of 128 as layers have them, a quarter multiples of 16, a quarter anything."""
    v, kind = _log_int(rng, lo, hi), rng.random()
    if kind < 0.5:
        return max(128, v // 128 * 128)
    return max(16, v // 16 * 16) if kind < 0.75 else v


def draw(rng):
    op = rng.choice(["gemm", "gemm", "act", "adamw"])
    if op == "adamw":
        big = rng.random() < 0.3
        return {"op": op, "layers": rng.choice([1, 1, 2]) if big else _log_int(rng, 1, 16), "d": _features(rng, 128, 4096 if big else 1024),
                "f": _features(rng, 128, 16384 if big else 2048), "bits": rng.choice([8, 8, 32]), "param": rng.choice(["f32", "f32", "bf16"]),
                "grad": rng.choice(["f32", "bf16"]), "scaled": rng.random() < 0.5, "offset": rng.choice([0, 0, 0, 1, 8])}
    act, pad = rng.choice(ACTS), rng.choice([0, 0, 16, 48])
    if op == "act":
        dz, q, db = rng.choice([(True, True, True), (True, False, True), (False, True, True), (True, True, False), (False, False, True)])
        return {"op": op, "d": _features(rng), "t": _log_int(rng, 1, 8192), "act": act, "dz": dz, "q": q, "db": db, "type": rng.choice(["bf16", "bf16", "f32"]), "pad": pad}
    m, n, k = _features(rng), _log_int(rng, 1, 8192), _features(rng)
    while m * n * k > 4096 * 8192 * 16384:
        k = max(128, k // 256 * 128)
    grad = act != "none" and rng.random() < 0.3
    c, q = rng.choice([(True, False), (False, True), (True, True)])
    return {"op": op, "m": m, "n": n, "k": k, "ta": "N" if grad else rng.choice("TTTN"), "act": act, "grad": grad, "bias": not grad and rng.random() < 0.8, "res": rng.random() < 0.3,
            "z": not grad and rng.random() < 0.4, "c": c, "q": q, "out": rng.choice(["bf16", "bf16", "f32"]), "scale": rng.choice(["e8m0", "e8m0", "f32"]),
            "ba": rng.choice([128, 128, 1]), "bb": rng.choice([1, 1, 128]), "pad": pad}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _blocks(n, b=128):
    return (n + b - 1) // b


def _tile_amax(x, rows_per, cols_per=128):
    """Largest magnitude of every rows_per x cols_per tile of x, edge tiles included."""
    r, c = x.shape
    br, bc = _blocks(r, rows_per), _blocks(c, cols_per)
    p = torch.nn.functional.pad(x.abs(), (0, bc * cols_per - c, 0, br * rows_per - r))
    return p.view(br, rows_per, bc, cols_per).amax(dim=(1, 3))


def _spread(s, shape, rows_per, cols_per=128):
    """One value per tile to one value per element."""
    return s.repeat_interleave(rows_per, 0)[: shape[0]].repeat_interleave(cols_per, 1)[:, : shape[1]]


def _scale_e8m0(amax):
    """The smallest power of two that brings amax to 448 or below; 1 for a tile of zeros."""
    mant, expo = torch.frexp(amax)
    byte = (expo - 9 + (mant > 0.875)).clamp(-127, 127) + 127
    return torch.where(amax > 0, byte, 127).to(torch.uint8).view(E8)


def _quantise(x, rows_per, scale="e8m0"):
    """x (fp32) as e4m3 numbers and the scales of its rows_per x 128 tiles."""
    amax = _tile_amax(x, rows_per)
    s = _scale_e8m0(amax) if scale == "e8m0" else torch.where(amax > 0, amax / E4M3_MAX, 1.0)
    return (x / _spread(s.float(), x.shape, rows_per)).clamp(-E4M3_MAX, E4M3_MAX).to(F8), s


def _stored(x, ld):
    """x [cols, rows] in columns of ld elements; what lies between rows and ld is never read."""
    if ld == x.shape[1]:
        return x.contiguous()
    buf = torch.zeros(x.shape[0], ld, dtype=torch.uint8 if x.element_size() == 1 else x.dtype, device=x.device)
    buf[:, : x.shape[1]] = x.view(torch.uint8) if x.element_size() == 1 else x
    return buf.view(x.dtype)


def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _activations(g, t, d):
    """Tokens of different magnitudes and a few features that are larger than the rest, as residual streams have them."""
    x = _normal(g, t, d)
    x *= torch.exp(0.5 * _normal(g, t, 1))
    x *= 1.0 + 4.0 * (torch.rand(1, d, device="cuda", generator=g) < 0.01)
    return x


def _padded(n, pad):
    return _blocks(n, 16) * 16 + pad if pad else n


def _operand(x, trans, block, scale, pad):
    """A product's operand x, own index by summed index: the summed one contiguous (as 'T' has A and 'N' has B) or the own one."""
    q, s = _quantise(x, block, scale)
    if not trans:
        q, s = q.view(torch.uint8).t().contiguous().view(F8), s.view(torch.uint8 if s.dtype == E8 else s.dtype).t().contiguous().view(s.dtype)
    ld = _padded(q.shape[1], pad)
    return _stored(q, ld), ld, s


def _empty8(st, t, d, ld):
    st["q"], st["s"] = torch.empty(t, ld, dtype=F8, device="cuda"), torch.empty(t, _blocks(d), dtype=E8, device="cuda")


def _prepare_gemm(c, g):
    m, n, k, T = c["m"], c["n"], c["k"], TYPES[c["out"]]
    st = {"c": c, "ld": _padded(m, c["pad"])}
    st["A"], st["lda"], st["sa"] = _operand(k**-0.5 * _normal(g, m, k), c["ta"] == "T", c["ba"], c["scale"], c["pad"])
    st["B"], st["ldb"], st["sb"] = _operand(_activations(g, n, k), True, c["bb"], c["scale"], c["pad"])
    st["bias"] = 0.5 * _normal(g, m) if c["bias"] else None
    st["r"] = _stored(_activations(g, n, m).to(T), st["ld"]) if c["res"] else None
    st["z"] = _stored(_activations(g, n, m).to(T), st["ld"]) if c["grad"] else torch.empty(n, st["ld"], dtype=T, device="cuda") if c["z"] else None
    st["out"] = torch.empty(n, st["ld"], dtype=T, device="cuda") if c["c"] else None
    st["q"] = st["s"] = None
    if c["q"]:
        _empty8(st, n, m, st["ld"])
    return st


def _prepare_act(c, g):
    d, t, T = c["d"], c["t"], TYPES[c["type"]]
    st = {"c": c, "ld": _padded(d, c["pad"]), "q": None, "s": None}
    st["dy"] = _stored((1e-3 * _normal(g, t, d)).to(T), st["ld"])
    st["z"] = _stored(_activations(g, t, d).to(T), st["ld"]) if c["act"] != "none" else None
    st["dz"] = torch.empty(t, st["ld"], dtype=T, device="cuda") if c["dz"] else None
    st["db"] = torch.empty(d, dtype=torch.float32, device="cuda") if c["db"] else None
    if c["q"]:
        _empty8(st, t, d, st["ld"])
    return st


def _sizes(c):
    """Elements of every tensor of the layers: norm, first weight and bias, second weight and bias."""
    d, f = c["d"], c["f"]
    return [d, f * d, f, d * f, d] * c["layers"]


ADAMW = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "wd": 0.1, "step": 10}


def _prepare_adamw(c, g):
    """All tensors lie in one buffer, each from the next multiple of 128 elements (and an offset) on; so do their states, whose blocks of 128 follow on."""
    sizes = _sizes(c)
    first = [0]
    for n in sizes:
        first.append(first[-1] + _blocks(n))
    blocks, at = first[-1], c["offset"]
    total = 128 * blocks
    there = torch.zeros(total, dtype=torch.bool, device="cuda")
    for b, n in zip(first, sizes):
        there[128 * b : 128 * b + n] = True
    st = {"c": c, "blocks": blocks, "seed": int(torch.randint(1 << 40, (1,), device="cuda", generator=g))}
    part = 1 << 26
    st["p"] = torch.zeros(at + total, dtype=TYPES[c["param"]], device="cuda")
    st["g"] = torch.zeros(at + total, dtype=TYPES[c["grad"]], device="cuda")
    T = F8 if c["bits"] == 8 else torch.float32
    st["m"], st["v"] = (torch.zeros(at + total, dtype=torch.uint8 if c["bits"] == 8 else T, device="cuda") for _ in range(2))
    scales = []
    for b in range(0, total, part):  # in parts: random numbers in fp32 take more room than what is kept of them
        e = min(total, b + part)
        here = there[b:e].float()
        size = torch.exp(_normal(g, (e - b) // 128, 1)).expand(-1, 128).reshape(-1)  # gradients of different magnitudes
        st["p"][at + b : at + e] = 0.02 * _normal(g, e - b) * here
        st["g"][at + b : at + e] = 1e-3 * size * _normal(g, e - b) * here
        m, r = 3e-4 * size * _normal(g, e - b) * here, 1e-3 * size * (0.5 + _normal(g, e - b).abs()) * here
        if c["bits"] == 8:
            (qm, sm), (qr, sr) = _quantise(m.view(-1, 128), 1), _quantise(r.view(-1, 128), 1)
            st["m"][at + b : at + e], st["v"][at + b : at + e] = qm.view(-1).view(torch.uint8), qr.view(-1).view(torch.uint8)
            scales.append((sm.view(-1).view(torch.uint8), sr.view(-1).view(torch.uint8)))
        else:
            st["m"][at + b : at + e], st["v"][at + b : at + e] = m, r * r
    if c["bits"] == 8:
        st["m"], st["v"] = st["m"].view(F8), st["v"].view(F8)
        st["sm"], st["sv"] = (torch.cat(s).view(E8) for s in zip(*scales))
    st["gs"] = torch.full((1,), 0.7, device="cuda") if c["scaled"] else None
    split = lambda x: [x[at + 128 * b : at + 128 * b + n] for b, n in zip(first, sizes)]  # noqa: E731
    st["lists"] = [split(st[x]) for x in "pgmv"]
    st["lists"] += [[st[x][b : b + _blocks(n)] for b, n in zip(first, sizes)] for x in ("sm", "sv")] if c["bits"] == 8 else [None, None]
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"gemm": _prepare_gemm, "act": _prepare_act, "adamw": _prepare_adamw}[case["op"]](dict(case), g)


# ---- one pass -------------------------------------------------------------------------------------------------------
def _b2():
    from paper_1611_08035_b200 import binding
    return binding


def _workspace(st, nbytes):
    """A program keeps its workspace; it is asked for once per state."""
    if "ws" not in st:
        n = nbytes()
        st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return st["ws"]


def _gemm_outputs(st):
    c, m = st["c"], st["c"]["m"]
    out = {"c": st["out"][:, :m]} if c["c"] else {}
    if c["q"]:
        out |= {"q": st["q"][:, :m], "s": st["s"]}
    return out | {"z": st["z"][:, :m]} if c["z"] else out


def _own_gemm(st):
    c, b2 = st["c"], _b2()
    m, n, k, ld = c["m"], c["n"], c["k"], st["ld"]
    ws = _workspace(st, lambda: b2.b2_gemm_f8_workspace_bytes(c["ta"], "N", m, n, k, st["A"], st["lda"], st["B"], st["ldb"]))
    act = getattr(b2, "ACT_" + c["act"].upper()) | (b2.ACT_GRADIENT if c["grad"] else 0)
    b2.b2_gemm_f8_act(c["ta"], "N", m, n, k, 1.0, st["A"], st["lda"], st["sa"], st["sa"].shape[1], c["ba"], st["B"], st["ldb"], st["sb"], st["sb"].shape[1], c["bb"],
                      act, st["bias"], st["z"], ld, st["r"], ld, st["out"], ld, st["q"], ld, st["s"], _blocks(m), ws)
    return _gemm_outputs(st)


def _act_outputs(st):
    c, d = st["c"], st["c"]["d"]
    out = {"dz": st["dz"][:, :d]} if c["dz"] else {}
    if c["q"]:
        out |= {"q": st["q"][:, :d], "s": st["s"]}
    return out | {"db": st["db"]} if c["db"] else out


def _own_act(st):
    c, b2, ld = st["c"], _b2(), st["ld"]
    ws = _workspace(st, lambda: b2.b2_act_backward_workspace_bytes(c["d"], c["t"]))
    b2.b2_act_backward(c["d"], c["t"], getattr(b2, "ACT_" + c["act"].upper()), st["dy"], ld, st["z"], ld, st["dz"], ld, st["q"], ld, st["s"], _blocks(c["d"]), st["db"], ws)
    return _act_outputs(st)


def _adamw_outputs(st):
    at = st["c"]["offset"]
    out = {x: st[x][at:] for x in "pmv"}
    return out | {"sm": st["sm"], "sv": st["sv"]} if st["c"]["bits"] == 8 else out


def _own_adamw(st):
    a = ADAMW
    _b2().b2_adamw(*st["lists"], a["lr"], a["beta1"], a["beta2"], a["eps"], a["wd"], a["step"], st["seed"], st["gs"])
    return _adamw_outputs(st)


_OWN = {"gemm": _own_gemm, "act": _own_act, "adamw": _own_adamw}


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(z * -(0.5**0.5))
    return z * torch.sigmoid(z if act == "silu" else 2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z**3))


def _act_gradient(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.special.erfc(z * -(0.5**0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "silu":
        s, du = torch.sigmoid(z), 1.0
    else:
        a = 2 * (2 / math.pi) ** 0.5
        s, du = torch.sigmoid(a * (z + 0.044715 * z**3)), a * (1 + 3 * 0.044715 * z * z)
    return s + z * s * (1 - s) * du


def _plain_gemm(st):
    c = st["c"]
    m, n, k, T = c["m"], c["n"], c["k"], TYPES[c["out"]]
    a, b = st["A"].float(), st["B"].float()
    a = a[:, :k] * _spread(st["sa"].float(), (m, k), c["ba"]) if c["ta"] == "T" else a[:, :m].t() * _spread(st["sa"].float().t(), (m, k), c["ba"])
    v = (b[:, :k] * _spread(st["sb"].float(), (n, k), c["bb"])) @ a.t()
    out = {}
    if c["grad"]:
        v = v * _act_gradient(st["z"][:, :m].float(), c["act"])
    else:
        v = v + st["bias"] if c["bias"] else v
        if c["z"]:
            out["z"] = v.to(T)
        v = _act(v, c["act"])
    if c["res"]:
        v = v + st["r"][:, :m].float()
    if c["c"]:
        out["c"] = v.to(T)
    if c["q"]:
        out["q"], out["s"] = _quantise(v, 1)
    return out


def _plain_act(st):
    c, d, out = st["c"], st["c"]["d"], {}
    v = st["dy"][:, :d].float()
    if c["act"] != "none":
        v = v * _act_gradient(st["z"][:, :d].float(), c["act"])
    if c["dz"]:
        out["dz"] = v.to(TYPES[c["type"]])
    if c["q"]:
        out["q"], out["s"] = _quantise(v, 1)
    if c["db"]:
        out["db"] = v.sum(0)
    return out


LOW = 0xFFFFFFFF


def _mix(x):
    """The finaliser of MurmurHash3 (A. Appleby) on 32-bit numbers, Python's or a tensor's."""
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & LOW
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & LOW
    return x ^ (x >> 16)


def _key(seed, step):
    return _mix(_mix(_mix(seed & LOW) ^ (seed >> 32 & LOW)) ^ (step & LOW))


STEP = 0x9E3779B9


def _random(e, key):
    """Two lists of 20 random bits for the elements with the numbers e: a hash for every eight of them, and for each of the eight a step further."""
    h = _mix(((e >> 3 & LOW) + _mix((e >> 35) + key & LOW)) & LOW)
    return [((x + (e & 7) * STEP) & LOW) >> 12 for x in (h, _mix(h + STEP & LOW))]


def _at_random(x, u):
    """|x| <= 448 to a neighbouring e4m3 number: the mantissa is cut after u, in [0, 2^20) of 2^20 of its last place, was added."""
    small = x < 2.0**-6  # numbers of one step, as in the binade above
    t = torch.where(small, x + 2.0**-6, x)
    t = ((t.view(torch.int32) + u.to(torch.int32)) & -(1 << 20)).view(torch.float32)
    return torch.where(small, t - 2.0**-6, t)


def _plain_adamw(st):
    c, a, at, nb = st["c"], ADAMW, st["c"]["offset"], st["blocks"]
    view = lambda x: st[x][at:].view(nb, 128)  # noqa: E731
    g = view("g").float()
    if c["scaled"]:
        g = g * st["gs"]
    m, v = view("m").float(), view("v").float()
    if c["bits"] == 8:
        m, r = m * st["sm"].float()[:, None], v * st["sv"].float()[:, None]
        v = r * r
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    m = m * f32(a["beta1"]) + g * f32(1 - a["beta1"])
    v = v * f32(a["beta2"]) + (g * g) * f32(1 - a["beta2"])
    r = torch.sqrt(v)
    size, root = a["lr"] / (1 - a["beta1"] ** a["step"]), (1 - a["beta2"] ** a["step"]) ** -0.5
    p = view("p").float() * (1 - a["lr"] * a["wd"]) - size * m / (r * root + a["eps"])
    if c["bits"] == 8:
        for name, x, u in zip("mv", (m, r), _random(torch.arange(nb * 128, device="cuda").view(nb, 128), _key(st["seed"], a["step"]))):
            s = _scale_e8m0(x.abs().amax(1))
            y = x.abs() / s.float()[:, None]
            q = _at_random(y, u)
            if name == "v":
                q = torch.where(y > 0, q.clamp(min=2.0**-9), q)  # a second moment that is not zero is not held as zero
            st[name][at:] = torch.copysign(q, x).to(F8).view(-1)
            st["s" + name].copy_(s)
    else:
        st["m"][at:], st["v"][at:] = m.view(-1), v.view(-1)
    st["p"][at:] = p.to(st["p"].dtype).view(-1)
    return _adamw_outputs(st)


_PLAIN = {"gemm": _plain_gemm, "act": _plain_act, "adamw": _plain_adamw}


def run(state):
    return (_OWN if own else _PLAIN)[state["c"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "adamw":
        n = sum(_sizes(c))
        state = 4 * n + 4 * sum(map(_blocks, _sizes(c))) if c["bits"] == 8 else 16 * n
        return {"bytes": n * (2 * TYPES[c["param"]].itemsize + TYPES[c["grad"]].itemsize) + state, "flops": (40 if c["bits"] == 8 else 16) * n}
    if c["op"] == "act":
        d, t, e = c["d"], c["t"], TYPES[c["type"]].itemsize
        moved = t * d * e * (1 + (c["act"] != "none") + c["dz"]) + (t * (d + _blocks(d)) if c["q"] else 0) + (4 * d if c["db"] else 0)
        return {"bytes": moved, "flops": (3 if c["act"] == "none" else 20) * t * d}
    m, n, k, e = c["m"], c["n"], c["k"], TYPES[c["out"]].itemsize
    es = 1 if c["scale"] == "e8m0" else 4
    moved = k * (m + n) + es * _blocks(k) * (_blocks(m, c["ba"]) + _blocks(n, c["bb"])) + (4 * m if c["bias"] else 0)
    moved += m * n * e * (c["res"] + c["z"] + c["grad"] + c["c"]) + (n * (m + _blocks(m)) if c["q"] else 0)
    return {"bytes": moved, "flops": 2 * m * n * k}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
def _power_of_two(amax):
    """The scale from the logarithm's definition; the powers of two come from a table."""
    powers = torch.tensor([2.0**i for i in range(-300, 301)], dtype=torch.float64, device=amax.device)
    pow2 = lambda e: powers[e.clamp(-300, 300).long() + 300]  # noqa: E731
    e = torch.floor(torch.log2(amax / E4M3_MAX))  # at most one off the wanted power, mended by comparison
    for _ in range(2):
        e = torch.where(amax > E4M3_MAX * pow2(e), e + 1, e)
    e = torch.where(amax <= E4M3_MAX * pow2(e - 1), e - 1, e)
    return pow2(torch.where(amax > 0, e.clamp(-127, 127), torch.zeros_like(e)))


def _spacing(v):
    """Distance of neighbouring e4m3 numbers at v."""
    return 2.0 ** (torch.floor(torch.log2(v.abs().clamp(min=2.0**-6))) - 3)


def _exact_quantised(y):
    t, d = y.shape
    q, s = torch.empty_like(y), torch.empty(t, _blocks(d), dtype=torch.float64, device=y.device)
    for j in range(_blocks(d)):
        part = y[:, 128 * j : 128 * j + 128]
        s[:, j] = _power_of_two(part.abs().amax(1))
        v = part / s[:, j, None]
        q[:, 128 * j : 128 * j + 128] = torch.round(v / _spacing(v)) * _spacing(v)
    return q, s


def _exact_act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.relu(z), torch.heaviside(z, torch.zeros_like(z))
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        e = torch.exp(-z)
        return z / (1 + e), 1 / (1 + e) + z * e / (1 + e) ** 2
    th = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z**3))
    return 0.5 * z * (1 + th), 0.5 * (1 + th) + 0.5 * z * (1 - th**2) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z**2)


def _exact_gemm(c, st):
    m, n, k = c["m"], c["n"], c["k"]
    z = torch.zeros(n, m, dtype=torch.float64, device="cuda")
    for p in range(_blocks(k)):  # one block of the summed index at a time: its scales factor out
        at = slice(128 * p, min(k, 128 * p + 128))
        a = st["A"][:, at].double() if c["ta"] == "T" else st["A"][at, :m].double().t()
        fa = (st["sa"][:, p] if c["ta"] == "T" else st["sa"][p]).double().repeat_interleave(c["ba"])[:m]
        fb = st["sb"][:, p].double().repeat_interleave(c["bb"])[:n]
        z.addmm_(st["B"][:, at].double() * fb[:, None], (a * fa[:, None]).t())
    out = {}
    if c["grad"]:
        v = z * _exact_act(st["z"][:, :m].double(), c["act"])[1]
    else:
        if c["bias"]:
            z += st["bias"].double()
        if c["z"]:
            out["z"] = z
        v = _exact_act(z, c["act"])[0]
    if c["res"]:
        v = v + st["r"][:, :m].double()
    if c["q"]:
        out["q"], out["s"] = _exact_quantised(v)
    return out | {"c": v} if c["c"] else out


def _exact_act_backward(c, st):
    d, out = c["d"], {}
    v = st["dy"][:, :d].double()
    if c["act"] != "none":
        v = v * _exact_act(st["z"][:, :d].double(), c["act"])[1]
    if c["q"]:
        out["q"], out["s"] = _exact_quantised(v)
    if c["dz"]:
        out["dz"] = v
    return out | {"db": torch.einsum("td->d", v)} if c["db"] else out


def _exact_adamw(c, st):
    """Part by part, for the room that what lies between takes."""
    a, at, nb = ADAMW, c["offset"], st["blocks"]
    names = ("p", "m", "v", "sm", "sv") if c["bits"] == 8 else ("p", "m", "v")
    parts = {x: [] for x in names}
    for b in range(0, nb, 1 << 18):
        k = slice(b, min(nb, b + (1 << 18)))
        p, g, m, v = (st[x][at + 128 * k.start : at + 128 * k.stop].double().view(-1, 128) for x in "pgmv")
        if c["scaled"]:
            g = g * st["gs"].double()
        if c["bits"] == 8:
            m, v = m * st["sm"][k].double()[:, None], (v * st["sv"][k].double()[:, None]) ** 2
        m, v = torch.lerp(g, m, a["beta1"]), torch.lerp(g**2, v, a["beta2"])
        mh, vh = m / (1 - a["beta1"] ** a["step"]), v / (1 - a["beta2"] ** a["step"])
        parts["p"].append((p - a["lr"] * (mh / (vh**0.5 + a["eps"]) + a["wd"] * p)))
        if c["bits"] == 32:
            parts["m"].append(m), parts["v"].append(v)
            continue
        e = torch.arange(128 * k.start, 128 * k.stop, device="cuda").view(-1, 128)
        for x, y, u in zip("mv", (m, v**0.5), _random(e, _key(st["seed"], a["step"]))):
            s = _power_of_two(y.abs().amax(1))
            w = y.abs() / s[:, None]
            step = _spacing(w)
            q = torch.floor(w / step + u.double() / 2**20) * step
            if x == "v":
                q = torch.where(w > 0, q.clamp(min=2.0**-9), q)
            parts[x].append(torch.sign(y) * q), parts["s" + x].append(s)
    return {x: torch.cat(y).view(-1) for x, y in parts.items()}


def exact(case, seed):
    st = prepare(case, seed)
    return {"gemm": _exact_gemm, "act": _exact_act_backward, "adamw": _exact_adamw}[case["op"]](dict(case), st)
