"""The AdamW step on the GPU against its definition in 64 bits (oracle/ffn.py).

Tolerances, u = 2^-24, derived before the first run.  m and v: beta and 1 - beta are rounded to fp32 (u each), products and the sum once each, the scaled gradient
once: |m - ref| <= 4 u (|b1 m| + |a1 g|), v likewise with one rounding more in g^2 and two for a given root: 6 u.  The step: sqrt halves v's error and rounds, root,
size, eps are rounded constants, a multiply-add, an approximate division (2 ulp, 4 u): 16 u of its size; p's decay and difference 3 u |p|; stored in bf16 2^-8
|p| more.  8-bit states: the scale is a comparison, where a largest magnitude may fall to the other side of a power of two; q s is within a step of e4m3 (2^-3
relative, the step that is chosen is that of the same random bits), and all but a few are the oracle's number exactly: one whose fraction is within its
error of the random bits' border falls to the other side, 2^-20 * 8 of them at most in the mean; 20 of a million are allowed beside three."""
import numpy as np
import pytest
import torch

from oracle import f8, ffn

pytestmark = pytest.mark.gpu
U = 2.0**-24
BF, F32 = torch.bfloat16, torch.float32
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
LR, B1, B2_, EPS, WD = 1e-3, 0.9, 0.95, 1e-8, 0.1


def np64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def placed(x, offset):
    """x on the GPU, `offset` elements into an allocation."""
    flat = torch.empty(offset + x.numel(), dtype=torch.uint8 if x.element_size() == 1 else x.dtype, device="cuda")
    flat[offset:] = x.view(torch.uint8).cuda() if x.element_size() == 1 else x.cuda()
    return flat[offset:].view(x.dtype)


def quantised(x):
    q, s = f8.quantise(np64(x)[None], 1)
    return torch.from_numpy(q[0]).view(F8), torch.from_numpy(s[0]).view(E8)


def tensors(sizes, bits, tp, tg, seed=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for n in sizes:
        size = torch.exp(torch.randn(n, generator=g))
        p, gr = 0.1 * torch.randn(n, generator=g), 1e-3 * size * torch.randn(n, generator=g)
        m, r = 3e-4 * size * torch.randn(n, generator=g), 1e-3 * size * (0.5 + torch.randn(n, generator=g).abs())
        t = {"p": placed(p.to(tp), offset), "g": placed(gr.to(tg), offset)}
        if bits == 8:
            (qm, sm), (qr, sr) = quantised(m), quantised(r)
            t |= {"m": placed(qm, offset), "v": placed(qr, offset), "sm": sm.cuda(), "sv": sr.cuda()}
        else:
            t |= {"m": placed(m, offset), "v": placed(r * r, offset), "sm": None, "sv": None}
        out.append(t)
    return out


def call(b2, ts, step=10, seed=12345678901, **kw):
    lists = [[t[x] for t in ts] for x in ("p", "g", "m", "v", "sm", "sv")]
    b2.b2_adamw(*lists, kw.pop("lr", LR), kw.pop("beta1", B1), kw.pop("beta2", B2_), EPS, kw.pop("wd", WD), step, seed, kw.pop("scale", None))


def values(t, key):
    x = np64(t[key].float())
    return x * np.repeat(f8.e8m0(t["s" + key].view(torch.uint8).cpu().numpy()), 128)[: x.size] if t["s" + key] is not None else x


def check(before, after, first, step, seed, scale=1.0, lr=LR, beta1=B1, beta2=B2_, wd=WD, flips=None):
    """One tensor; `before`: a copy of it, `first`: the number of its first element."""
    bits = 8 if before["sm"] is not None else 32
    p, g, m, v = np64(before["p"]), np64(before["g"]) * scale, values(before, "m"), values(before, "v")
    v = v * v if bits == 8 else v
    wp, wm, wv = ffn.adamw(p, g, m, v, lr, beta1, beta2, EPS, wd, step)
    em = 5 * U * (beta1 * np.abs(m) + (1 - beta1) * np.abs(g))
    ev = 7 * U * wv
    move = np.abs(lr / (1 - beta1**step) / (np.sqrt(wv / (1 - beta2**step)) + EPS))
    ep = 16 * U * move * np.abs(wm) + move * em + 3 * U * (np.abs(p) + move * np.abs(wm))
    got = np64(after["p"])
    assert np.all(np.abs(got - wp) <= ep + (2.0**-8 if after["p"].dtype is BF else U) * (np.abs(wp) + ep))
    if bits == 32:
        assert np.all(np.abs(values(after, "m") - wm) <= em) and np.all(np.abs(values(after, "v") - wv) <= ev)
        return
    u = ffn.random_bits(first + np.arange(p.size), seed, step)
    for key, x, bits_, e in (("m", wm, u[0], em), ("v", np.sqrt(wv), u[1], 5 * U * np.sqrt(wv))):
        q, s = ffn.quantise_at_random(x, bits_, key == "v")
        got_s = f8.e8m0(after["s" + key].view(torch.uint8).cpu().numpy())
        for j in np.flatnonzero(got_s != s):  # the largest is at a power of two times 448, on the other side of it
            a = np.max(np.abs(x[128 * j : 128 * j + 128]))
            assert abs(a / (448 * min(s[j], got_s[j])) - 1) <= 8 * U
            at = slice(128 * j, 128 * j + 128)
            q[at] = np.copysign(ffn.at_random(np.abs(x[at]) / got_s[j], bits_[at]), x[at])
        got_q = np64(after[key].float())
        sv = np.repeat(got_s, 128)[: x.size]
        assert np.all(np.abs(got_q * sv - x) <= np.maximum(np.abs(x) * 2.0**-3, sv * 2.0**-9) + e)
        flips.append((int((got_q != q).sum()), x.size))


def run(b2, sizes, bits, tp=F32, tg=F32, offset=0, seed=0, **kw):
    ts = tensors(sizes, bits, tp, tg, seed, offset)
    before = [{k: None if x is None else x.clone() for k, x in t.items()} for t in ts]
    step, rnd, scale = kw.get("step", 10), kw.get("seed_", 12345678901), kw.pop("scale", 1.0)
    call(b2, ts, step, rnd, scale=None if scale == 1.0 else torch.tensor([scale], device="cuda"), **{k: v for k, v in kw.items() if k in ("lr", "beta1", "beta2", "wd")})
    flips, first = [], 0
    for t, b, n in zip(ts, before, sizes):
        check(b, t, first, step, rnd, float(np.float32(scale)), flips=flips, **{k: v for k, v in kw.items() if k in ("lr", "beta1", "beta2", "wd")})
        assert torch.equal(t["g"], b["g"])
        first += -(-n // 128) * 128
    if flips:
        off, total = (sum(x) for x in zip(*flips))
        assert off <= 3 + 20e-6 * total, (off, total)


SIZES = [[1], [7], [128], [129, 1, 255, 4096], [1000, 3, 4097, 128, 12289, 5, 100003], [384, 512 * 384, 512, 384 * 512, 384], list(range(1, 700, 2))]


@pytest.mark.parametrize("offset", [0, 1, 8])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_step(b2, sizes, bits, offset):
    run(b2, sizes, bits, offset=offset)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("tp,tg", [(F32, BF), (BF, F32), (BF, BF)])
def test_types(b2, tp, tg, bits):
    run(b2, [1000, 130, 9001], bits, tp, tg, scale=0.37)
    run(b2, [1000, 130, 9001], bits, tp, tg, offset=3)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("kw", [{"step": 1}, {"step": 2**33 + 5}, {"beta1": 0.0}, {"beta2": 0.0}, {"lr": 0.0}, {"wd": 0.0}, {"beta2": 0.999, "step": 3}, {"lr": 1.0, "wd": 1.0}, {"seed_": 0},
                                {"seed_": 2**64 - 1}])
def test_numbers(b2, kw, bits):
    if kw.get("seed_") == 2**64 - 1:
        kw = {"seed_": -1}
        ts = tensors([300], bits, F32, F32)
        other = [{k: None if x is None else x.clone() for k, x in t.items()} for t in ts]
        call(b2, ts, seed=-1), call(b2, other, seed=2**64 - 1)  # the same 64 bits
        assert all(torch.equal(ts[0][k].view(torch.uint8), other[0][k].view(torch.uint8)) for k in "pmv")
        return
    run(b2, [1000, 4200], bits, **kw)


def test_kinds_in_one_list(b2):
    """Every combination of types and states in one call, empty tensors among them; element numbers go on through the list."""
    sizes, ts = [], []
    for i, (bits, tp, tg) in enumerate([(b, p, g) for b in (8, 32) for p in (F32, BF) for g in (F32, BF)] * 2):
        n = [300, 0, 5001, 129][i % 4]
        sizes.append(n)
        ts += tensors([n], bits, tp, tg, i, offset=i % 3)
    before = [{k: None if x is None else x.clone() for k, x in t.items()} for t in ts]
    call(b2, ts)
    flips, first = [], 0
    for t, b, n in zip(ts, before, sizes):
        if n:
            check(b, t, first, 10, 12345678901, flips=flips)
        first += -(-n // 128) * 128
    assert sum(f for f, _ in flips) <= 3


def test_zero_states_and_first_steps(b2):
    """From nothing: zeros stay zeros where the gradient is 0, a root that is not 0 is never held as 0 beside one 2^20 times as large."""
    n = 256
    zero8 = lambda: torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8)  # noqa: E731
    ones = lambda: torch.full((2,), 127, dtype=torch.uint8, device="cuda").view(E8)  # noqa: E731
    g = torch.zeros(n, device="cuda")
    g[0], g[1], g[2] = 1.0, 2.0**-20, -(2.0**-20)
    t = {"p": torch.zeros(n, device="cuda"), "g": g, "m": zero8(), "v": zero8(), "sm": ones(), "sv": ones()}
    call(b2, [t], step=1)
    r = values(t, "v")
    assert r[1] > 0 and r[2] > 0 and bool((t["v"].float()[3:] == 0).all()) and bool((t["p"][3:] == 0).all())
    assert bool((t["v"].float()[1:3] == 2.0**-9).all())
    # At step 1 m / (1 - b1) = g and sqrt(v / (1 - b2)) = |g|: the step is lr g / (|g| + eps), here lr 2^-20 / (2^-20 + 1e-8) = 0.98962 lr.
    assert abs(float(t["p"][1]) + LR / (1 + EPS * 2.0**20)) < (16 + 5 + 3) * U * LR


def test_gradients_that_are_not_finite(b2):
    """A NaN or an infinity takes its block of an 8-bit state with it, and nothing else."""
    n = 1000
    for bad in (float("nan"), float("inf")):
        t = tensors([n], 8, F32, F32)[0]
        t["g"][300] = bad
        call(b2, [t])
        m, v = t["m"].view(torch.uint8).cpu(), t["v"].view(torch.uint8).cpu()
        hit = torch.zeros(n, dtype=torch.bool)
        hit[256:384] = True
        assert torch.equal(m == 0x7F, hit) and torch.equal(v == 0x7F, hit) and int(torch.isnan(t["p"]).sum()) == 1
        assert (t["sm"].view(torch.uint8).cpu() == 255).nonzero().view(-1).tolist() == [2]


def test_the_mean_over_random_roundings_is_right(b2):
    """4096 seeds of one block: the mean of m and of the root within five standard errors (a rounding's deviation is at most half a step, 2^-4 relative)."""
    n, seeds = 128, 4096
    t0 = tensors([n], 8, F32, F32, seed=3)[0]
    sums = {k: np.zeros(n) for k in "mv"}
    many = [{k: x.clone() for k, x in t0.items()} for _ in range(seeds)]
    for i in range(seeds):
        call(b2, [many[i]], seed=i * 7919)
    for t in many:
        for k in "mv":
            sums[k] += values(t, k)
    _, wm, wv = ffn.adamw(np64(t0["p"]), np64(t0["g"]), values(t0, "m"), values(t0, "v") ** 2, LR, B1, B2_, EPS, WD, 10)
    for k, x in (("m", wm), ("v", np.sqrt(wv))):
        s = np.repeat(f8.e8m0(many[0]["s" + k].view(torch.uint8).cpu().numpy()), 128)[:n]
        # rootless: 2^-20 of a step is the bits' own resolution; roots below 2^-9 of the scale are held there
        step = np.maximum(np.abs(x) * 2.0**-3, s * 2.0**-9)
        fine = np.abs(x) > s * 2.0**-9
        assert np.all(np.abs(sums[k] / seeds - x)[fine] <= (5 * 0.5 * step / np.sqrt(seeds) + 2.0**-19 * step)[fine])


def test_device_numbers_and_graphs(b2):
    """lr, step and the gradient's scale in device memory: a replayed graph follows them, with the bits of direct calls."""
    ts, direct = tensors([1000, 384], 8, F32, BF), tensors([1000, 384], 8, F32, BF)
    lr, step, scale = torch.tensor(LR, device="cuda"), torch.tensor([10], device="cuda"), torch.tensor([0.5], device="cuda")
    lists = [[t[x] for t in ts] for x in ("p", "g", "m", "v", "sm", "sv")]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b2.b2_adamw(*lists, lr, B1, B2_, EPS, WD, step, 99, scale)
        step += 1
    for i in range(4):
        lr.fill_(LR / (i + 1)), scale.fill_(0.5 + i)
        graph.replay()
        call(b2, direct, 10 + i, 99, lr=float(np.float32(LR / (i + 1))), scale=torch.tensor([0.5 + i], device="cuda"))
    torch.cuda.synchronize()
    for a, b in zip(ts, direct):
        assert all(torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)) for k in ("m", "v", "sm", "sv"))
        # the factors are computed on the device in fp64 and rounded to fp32: at most a last place apart, four times
        assert float((a["p"] - b["p"]).abs().max()) <= 4 * 4 * U * float(b["p"].abs().max())


def test_other_stream_and_ctypes(b2):
    """On another stream, and through the call without the extension, the same bits."""
    a, b, c = (tensors([1000, 4097], 8, F32, F32) for _ in range(3))
    call(b2, a)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call(b2, b)
    full = b2._connected.get("b2_adamw", (None, b2.b2_adamw))[1]
    full(*[[t[x] for t in c] for x in ("p", "g", "m", "v", "sm", "sv")], LR, B1, B2_, EPS, WD, 10, 12345678901)
    torch.cuda.synchronize()
    for x, y, z in zip(a, b, c):
        assert all(torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)) and torch.equal(x[k].view(torch.uint8), z[k].view(torch.uint8)) for k in ("p", "m", "v", "sm", "sv"))


def test_more_than_32_bits_of_elements(b2):
    """One tensor of 2^32 + 300 elements: its end is as the end of nothing else, element numbers past 32 bits among it."""
    n = 2**32 + 300
    tail = 5000
    p, g = torch.zeros(n, dtype=BF, device="cuda"), torch.zeros(n, dtype=BF, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8), torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8)
    sm, sv = (torch.full(((n + 127) // 128,), 127, dtype=torch.uint8, device="cuda").view(E8) for _ in range(2))
    g[-tail:] = torch.randn(tail, device="cuda").to(BF)
    b2.b2_adamw([p], [g], [m], [v], [sm], [sv], LR, B1, B2_, EPS, WD, 1, 5)
    first = (n - tail + 127) // 128 * 128  # a block's beginning
    want_g = np64(g[first:])
    _, wm, wv = ffn.adamw(np.zeros(want_g.size), want_g, 0.0, 0.0, LR, B1, B2_, EPS, WD, 1)
    u = ffn.random_bits(np.arange(first, n), 5, 1)
    for x, s, w, bits in ((m, sm, wm, u[0]), (v, sv, np.sqrt(wv), u[1])):
        q, want_s = ffn.quantise_at_random(w, bits, w is not wm)
        assert np.array_equal(f8.e8m0(s[first // 128 :].view(torch.uint8).cpu().numpy()), want_s)
        assert int((np64(x[first:].float()) != q).sum()) <= 3
    assert bool((p[: n - tail] == 0).all()) and bool((p[n - tail :] != 0).any())


def test_aligned_and_other_tensors_agree(b2):
    """The fast way of aligned tensors and the other one hold the same bits: m and v are computed by the same single roundings."""
    n = 1 << 24
    g = torch.Generator(device="cuda").manual_seed(0)
    gr = 1e-3 * torch.randn(n, device="cuda", generator=g)
    qm, qr = (torch.randint(0, 256, (n,), device="cuda", generator=g).to(torch.uint8) for _ in range(2))
    qm[(qm & 0x7F) == 0x7F] = 0
    qr = qr.clamp(1, 0x7E)
    results = []
    for offset in (0, 1):
        t = {k: torch.empty(n + offset, dtype=x.dtype, device="cuda") for k, x in (("p", gr), ("g", gr), ("m", qm), ("v", qr))}
        for k, x in (("p", gr), ("g", gr), ("m", qm), ("v", qr)):
            t[k][offset:] = x
        t = {k: x[offset:] if k in "pg" else x[offset:].view(F8) for k, x in t.items()}
        t |= {k: torch.full((n // 128,), b, dtype=torch.uint8, device="cuda").view(E8) for k, b in (("sm", 106), ("sv", 109))}
        call(b2, [t])
        results.append([t[k].view(torch.uint8).clone() for k in ("m", "v", "sm", "sv")])
    assert all(torch.equal(a, b) for a, b in zip(*results))
