"""GPU: the AdamW step.  Its definition fixes every operation and rounding, so a numpy emulation in fp32 has to agree bit for bit; the
emulation is held to the formula in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2312_08583_amd as P
from adapters_ref import normal

pytestmark = pytest.mark.gpu
F = np.float32
E4M3 = torch.float8_e4m3fn


def _power(b, t):
    r = 1.0
    while t:
        if t & 1:
            r *= b
        b *= b
        t >>= 1
    return r


def _hash(ids, t, seed):
    x = (ids * 0x9E3779B1 + t * 0x3C6EF373 + seed) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _decode(codes, scales, count):
    c = codes.astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (8 + m) * 2.0 ** (e - 10), m * 2.0 ** -9) * np.where(c & 128, -1.0, 1.0)
    return (v * 2.0 ** (np.repeat(scales.astype(np.int64), 256)[:count] - 127)).astype(F)


def _encode(x, noise, least):
    n = x.size
    pad = np.zeros(-(-n // 256) * 256, F)
    pad[:n] = np.abs(x)
    top = pad.reshape(-1, 256).max(1)
    f, e = np.frexp(top)
    e = np.where(top > 0, np.maximum(e - 9 + (f > 0.875), -126), -127)
    y = np.ldexp(pad, -np.repeat(e, 256))[:n].astype(F)
    ey = np.maximum(np.frexp(y)[1] - 1, -6)
    ey = np.where(y == 0, -6, ey)
    k = np.floor(np.ldexp(y, 3 - ey).astype(F) + noise.astype(F) * F(2.0 ** -16)).astype(np.int64)
    k = np.where((x != 0) & (k < least), least, k)
    return (((ey + 6) << 3) + k | np.signbit(x).astype(np.int64) << 7).astype(np.uint8), (e + 127).astype(np.uint8)


def _emulate(p, g, m, v, t, lr, b1, b2, eps, wd, gs, eight, first_id=0, seed=0):
    """One step in fp32; m and v as numbers (8 bits: (codes, scales) pairs)."""
    n = p.size
    first, second = F(lr / (1 - _power(b1, t))), F(1 / np.sqrt(1 - _power(b2, t)))
    if eight:
        m, v = _decode(*m, n), _decode(*v, n)
        v = v * v
    g = g.astype(F) * F(gs)
    m = m * F(b1) + g * F(1 - b1)
    v = v * F(b2) + g * g * F(1 - b2)
    u = np.sqrt(v)
    p = p * F(1 - lr * wd) - m / (u * second + F(eps)) * first
    if eight:
        noise = _hash((np.arange(n, dtype=np.int64) + first_id) & 0xFFFFFFFF, t, seed)
        m, v = _encode(m, noise >> 16, 0), _encode(u, noise & 0xFFFF, 1)
    return p, m, v


def _bits(t):
    return t.detach().cpu().contiguous().view(torch.uint8).numpy()


def _tensors(sizes, eight, grad, copy, seed):
    T = {"p": [], "g": [], "m": [], "v": [], "ms": [], "vs": [], "w": []}
    for i, n in enumerate(sizes):
        spread = torch.exp(2 * normal((n,), seed + i))
        p = normal((n,), seed + 100 + i, sigma=0.02)
        T["p"].append(p)
        T["g"].append((normal((n,), seed + 200 + i, sigma=1e-2) * spread).to(grad))
        T["w"].append(torch.zeros(n, dtype=copy or torch.float16, device="cuda"))
        blocks = -(-n // 256)
        if eight:
            for key in ("m", "v"):
                codes = torch.randint(0, 127, (n,), device="cuda", dtype=torch.uint8)
                if key == "m":
                    codes |= torch.randint(0, 2, (n,), device="cuda", dtype=torch.uint8) << 7
                T[key].append(codes.view(E4M3))
            T["ms"].append(torch.randint(105, 112, (blocks,), device="cuda", dtype=torch.uint8))
            T["vs"].append(torch.randint(105, 112, (blocks,), device="cuda", dtype=torch.uint8))
        else:
            T["m"].append(normal((n,), seed + 300 + i, sigma=1e-3) * spread)
            T["v"].append((1e-2 * spread) ** 2)
    return T


def _plan(T, eight, copy):
    return P.fp6_adamw_plan(T["p"], T["g"], T["m"], T["v"], T["ms"] if eight else None, T["vs"] if eight else None, T["w"] if copy else None)


def _numpy(t, kind):
    return t.detach().cpu().view(torch.uint8).numpy().copy() if kind == "codes" else t.detach().float().cpu().numpy().copy()


def _check(T, start, eight, copy, t, opts, seed=0):
    first_id = 0
    for i in range(len(T["p"])):
        n = T["p"][i].numel()
        p, m, v = _emulate(*[start[k][i] for k in ("p", "g", "m", "v")], t, *opts, eight, first_id, seed)
        first_id += -(-n // 256) * 256
        assert np.array_equal(_numpy(T["p"][i], "").view(np.uint32), p.view(np.uint32)), ("param", i)
        if copy:
            assert torch.equal(T["w"][i].cpu(), torch.from_numpy(p).to(copy)), ("copy", i)
        if eight:
            for key, (codes, scales) in (("m", m), ("v", v)):
                assert np.array_equal(T[key + "s"][i].cpu().numpy(), scales), (key, "scales", i)
                assert np.array_equal(_numpy(T[key][i], "codes"), codes), (key, i)
        else:
            assert np.array_equal(_numpy(T["m"][i], ""), m) and np.array_equal(_numpy(T["v"][i], ""), v), i


def _snapshot(T, eight):
    s = {k: [_numpy(t, "") for t in T[k]] for k in ("p", "g")}
    for k in ("m", "v"):
        s[k] = [(_numpy(c, "codes"), sc.cpu().numpy().copy()) for c, sc in zip(T[k], T[k + "s"])] if eight else [_numpy(t, "") for t in T[k]]
    return s


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("grad,copy", [(torch.float32, torch.float16), (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16),
                                       (torch.float32, None)])
@pytest.mark.parametrize("sizes", [(1,), (255, 256, 257), (4095, 4096, 4097, 3, 64 * 16), (0, 5, 0), (123457, 8, 70000)])
def test_bit_for_bit(sizes, grad, copy, eight):
    T = _tensors(sizes, eight, grad, copy, 7)
    plan, step = _plan(T, eight, copy), torch.tensor([41], dtype=torch.int32, device="cuda")
    opts = (3e-4, 0.9, 0.999, 1e-8, 0.1, 0.37)
    scale = torch.tensor([0.37], device="cuda")
    for turn in range(3):
        start = _snapshot(T, eight)
        P.fp6_adamw(plan, step, *opts[:5], grad_scale=scale, seed=99)
        torch.cuda.synchronize()
        assert step.item() == 42 + turn
        _check(T, start, eight, copy, 42 + turn, opts, 99)


def test_the_emulation_is_the_formula():
    """64 bits against the emulation of one tensor: each value passes through at most twelve roundings of 2^-24 relative to terms no larger
    than those bounded here; eight bits: the neighbours on either side."""
    rng = np.random.default_rng(1)
    n, t, lr, b1, b2, eps, wd, gs = 5000, 17, 1e-3, 0.9, 0.99, 1e-8, 0.01, 0.5
    p, g, m = (rng.normal(size=n).astype(F) * F(s) for s in (0.02, 1e-2, 1e-3))
    v = (rng.normal(size=n) ** 2 * 1e-4).astype(F)
    P1, M1, V1 = _emulate(p, g, m, v, t, lr, b1, b2, eps, wd, gs, False)
    d = [a.astype(np.float64) for a in (p, g, m, v)]
    gg = d[1] * gs
    M = b1 * d[2] + (1 - b1) * gg
    V = b2 * d[3] + (1 - b2) * gg * gg
    update = lr * (M / (1 - b1 ** t)) / (np.sqrt(V / (1 - b2 ** t)) + eps)
    R = 12 * 2.0 ** -24
    assert (np.abs(M1 - M) <= R * (np.abs(d[2]) + np.abs(gg))).all() and (np.abs(V1 - V) <= R * V).all()
    slack = lr / (1 - b1 ** t) * (np.abs(d[2]) + np.abs(gg)) / (np.sqrt(V / (1 - b2 ** t)) + eps)
    assert (np.abs(P1 - (d[0] * (1 - lr * wd) - update)) <= R * (np.abs(d[0]) + slack)).all()
    for x, least in ((M, 0), (np.sqrt(V), 1)):
        x = x.astype(F)
        codes, scales = _encode(x, rng.integers(0, 65536, n), least)
        back = _decode(codes, scales, n).astype(np.float64)
        unit = np.maximum(2.0 ** (np.floor(np.log2(np.abs(x.astype(np.float64)) + 1e-300))), 2.0 ** (np.repeat(scales.astype(int), 256)[:n] - 127 - 6)) / 8
        assert (np.abs(back - x) <= unit).all() and (np.sign(back) * np.sign(x) >= 0).all() and (least == 0 or (back[x > 0] > 0).all())


def test_rounding_to_eight_bits_is_unbiased():
    """One value many times: the mean of what is kept lies within five standard errors (a rounding between neighbours one unit apart
    has a deviation of at most half a unit), and both neighbours occur; a number of the format stays itself."""
    n = 1 << 16
    for value in (0.3, 0.00123, 1.0):
        p, g, m, v = (torch.zeros(n, device="cuda") for _ in range(4))
        g.fill_(value * 10)                                           # m = 0.1 g
        g[::256] = 2.2 * value * 10                                   # the block's largest, elsewhere on the grid
        codes = [torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
        scales = [torch.zeros(n // 256, dtype=torch.uint8, device="cuda") for _ in range(2)]
        plan = P.fp6_adamw_plan([p], [g], [codes[0]], [codes[1]], [scales[0]], [scales[1]])
        P.fp6_adamw(plan, torch.zeros(1, dtype=torch.int32, device="cuda"), seed=3)
        got = _decode(_numpy(codes[0], "codes"), scales[0].cpu().numpy(), n).reshape(-1, 256)[:, 1:].astype(np.float64)
        want = float(F(F(value * 10) * F(1 - 0.9)))
        unit = 2.0 ** (np.floor(np.log2(want)) - 3)
        # (1.0 is a number of the format: floor(k + r) = k for every r below 1, so it has no second neighbour)
        assert len(np.unique(got)) == (1 if want / unit == np.floor(want / unit) else 2) and abs(got.mean() - want) <= 5 * unit / 2 / np.sqrt(got.size)


def test_fresh_state_is_zero_bytes_and_empty_blocks_stay_empty():
    n = 700
    p, g = normal((n,), 1), torch.zeros(n, device="cuda")
    g[:256] = normal((256,), 2)
    codes = [torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
    scales = [torch.zeros(3, dtype=torch.uint8, device="cuda") for _ in range(2)]
    before = p.clone()
    plan = P.fp6_adamw_plan([p], [g], [codes[0]], [codes[1]], [scales[0]], [scales[1]])
    P.fp6_adamw(plan, torch.zeros(1, dtype=torch.int32, device="cuda"), weight_decay=0.0)
    assert torch.equal(p[256:], before[256:]) and not torch.equal(p[:256], before[:256])
    for c, s in zip(codes, scales):
        assert not c[256:].view(torch.uint8).any() and s[1:].tolist() == [0, 0] and s[0] > 0
    assert torch.isfinite(p).all()


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_found_inf_changes_nothing(eight):
    T = _tensors((1000, 300), eight, torch.float32, torch.float16, 17)
    plan, step = _plan(T, eight, torch.float16), torch.tensor([7], dtype=torch.int32, device="cuda")
    before = {k: [_bits(t).copy() for t in T[k]] for k in T}
    found = torch.tensor([1.0], device="cuda")
    P.fp6_adamw(plan, step, found_inf=found)
    assert step.item() == 7 and all(np.array_equal(a, _bits(b)) for k in T for a, b in zip(before[k], T[k]))
    found.zero_()
    P.fp6_adamw(plan, step, found_inf=found)
    assert step.item() == 8 and not np.array_equal(before["p"][0], _bits(T["p"][0]))


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_captured_and_replayed_as_step_rate_and_scale_move(eight):
    T = _tensors((5000, 257, 64), eight, torch.bfloat16, torch.bfloat16, 27)
    plan, step = _plan(T, eight, torch.bfloat16), torch.zeros(1, dtype=torch.int32, device="cuda")
    lr, scale, found = (torch.tensor([x], device="cuda") for x in (1e-3, 1.0, 0.0))
    call = lambda: P.fp6_adamw(plan, step, lr, 0.9, 0.95, 1e-6, 0.02, grad_scale=scale, found_inf=found, seed=5)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    t = 1
    for turn, (rate, gs, skip) in enumerate([(1e-3, 1.0, 0.0), (5e-4, 0.25, 0.0), (2e-4, 0.5, 1.0), (1e-4, 2.0, 0.0)]):
        lr.fill_(rate), scale.fill_(gs), found.fill_(skip)
        for g in T["g"]:
            g.copy_(normal(g.shape, 300 + turn, sigma=1e-2))
        start = _snapshot(T, eight)
        graph.replay()
        torch.cuda.synchronize()
        if not skip:
            t += 1
            _check(T, start, eight, torch.bfloat16, t, (float(F(rate)), 0.9, 0.95, 1e-6, 0.02, gs), 5)
        assert step.item() == t


def test_nothing_beside_the_tensors_is_touched():
    for eight in (False, True):
        n, pad = 1003, 13
        guard = 0xA5
        T, raw = {}, []

        def carve(nbytes):
            buf = torch.full((nbytes + 64,), guard, dtype=torch.uint8, device="cuda")
            raw.append((buf, nbytes))
            return buf[:nbytes]

        p = carve(4 * n).view(torch.float32)
        p.copy_(normal((n,), 1))
        g = normal((n,), 2)
        if eight:
            m, v = carve(n).view(E4M3), carve(n).view(E4M3)
            m.view(torch.uint8).zero_(), v.view(torch.uint8).zero_()
            ms, vs = carve(4), carve(4)
            ms.zero_(), vs.zero_()
            plan = P.fp6_adamw_plan([p], [g], [m], [v], [ms], [vs], [carve(2 * n).view(torch.float16)])
        else:
            m, v = carve(4 * n).view(torch.float32), carve(4 * n).view(torch.float32)
            m.zero_(), v.zero_()
            plan = P.fp6_adamw_plan([p], [g], [m], [v], copies=[carve(2 * n).view(torch.float16)])
        P.fp6_adamw(plan, torch.zeros(1, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        for buf, nbytes in raw:
            assert (buf[nbytes:] == guard).all() and not (buf[:nbytes] == guard).all()


def test_infinite_and_nan_gradients_spoil_their_element_only():
    for eight in (False, True):
        T = _tensors((600,), eight, torch.float32, None, 37)
        T["g"][0][5], T["g"][0][300] = float("inf"), float("nan")
        plan = _plan(T, eight, None)
        P.fp6_adamw(plan, torch.zeros(1, dtype=torch.int32, device="cuda"))
        bad = ~torch.isfinite(T["p"][0])
        assert bad.nonzero()[:, 0].tolist() == [5, 300]
        m = T["m"][0].float()
        assert (~torch.isfinite(m)).nonzero()[:, 0].tolist() == [5, 300]


def test_refusals_of_the_binding():
    z = lambda n=8, dtype=torch.float32: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    for call in [lambda: P.fp6_adamw_plan([z()], [z(9)], [z()], [z()]), lambda: P.fp6_adamw_plan([z().half()], [z()], [z()], [z()]),
                 lambda: P.fp6_adamw_plan([z(16)[::2]], [z()], [z()], [z()]), lambda: P.fp6_adamw_plan([z(16)[1:9]], [z()], [z()], [z()]),
                 lambda: P.fp6_adamw_plan([z()], [z().double()], [z()], [z()]), lambda: P.fp6_adamw_plan([z()], [z()], [z()], [z()], copies=[z()]),
                 lambda: P.fp6_adamw_plan([z(), z()], [z()], [z(), z()], [z(), z()]), lambda: P.fp6_adamw_plan([z()], [z()], [z()], [z(8, E4M3)]),
                 lambda: P.fp6_adamw_plan([z()], [z()], [z(8, E4M3)], [z(8, E4M3)]), lambda: P.fp6_adamw_plan([z()], [z().cpu()], [z()], [z()])]:
        with pytest.raises(P.Fp6Error):
            call()
    p = z()
    with pytest.raises(P.Fp6Error, match="overlaps"):
        P.fp6_adamw_plan([p], [z()], [p], [z()])
    plan, step = P.fp6_adamw_plan([z()], [z()], [z()], [z()]), torch.zeros(1, dtype=torch.int32, device="cuda")
    for call in [lambda: P.fp6_adamw(plan, step.long()), lambda: P.fp6_adamw(plan, step, lr=torch.zeros(1)), lambda: P.fp6_adamw(plan, step, beta1=1.0),
                 lambda: P.fp6_adamw(plan, step, lr=-1.0), lambda: P.fp6_adamw(plan, step, grad_scale=torch.zeros(2, device="cuda")),
                 lambda: P.fp6_adamw(plan, torch.zeros(1, dtype=torch.int32))]:
        with pytest.raises(P.Fp6Error):
            call()
    assert step.item() == 0
