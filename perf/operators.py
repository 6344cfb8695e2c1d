"""What the operators around the frozen linear layer are timed on: low-rank adapters beside it, its gradient, the adapters' update.

Sizes are those of the repository's configurations (LLaMA-shaped linear layers, the 34B-class decoder block) or generic (a
ragged batch, a small layer); `draw` spreads over the same ranges.  A case is one of
  lora    Y + s (X A^T) B^T, the adapter of each row given by an index; `group`: q, k and v of a decoder block in one call;
          `hidden`: X A^T is kept for the backward pass
  bwd     the gradients of that: dX added to, dA and dB
  grad    dX = dY W of a frozen layer whose weight is held in six or five bits (formats as in perf/cases.py)
  adamw   one optimiser step over the adapters of `layers` decoder blocks, states in 32 or 8 bits
`run` computes the plain form where `own` is false: elementary operations in 32 bits.
"""
import math

import torch

own = False

BLOCK = 256                                                     # 8-bit states: elements that share a scale
LR, BETA1, BETA2, EPS, DECAY, STEP, SEED = 1e-4, 0.9, 0.999, 1e-8, 0.01, 100, 12345


def _lora_case(name, dtype, M, N, K, rank, adapters, order="runs", hidden=False):
    return {"name": name, "op": "lora", "dtype": dtype, "M": M, "N": N, "K": K, "kv": 0, "rank": rank, "adapters": adapters,
            "order": order, "hidden": hidden}


def _bwd_case(name, dtype, M, N, K, rank, adapters, order="runs"):
    return {"name": name, "op": "bwd", "dtype": dtype, "M": M, "N": N, "K": K, "rank": rank, "adapters": adapters, "order": order}


def _grad_case(name, fmt, M, N, K):
    return {"name": name, "op": "grad", "fmt": fmt, "M": M, "N": N, "K": K}


def _adamw_case(name, bits, layers, hidden, kv, mlp, rank, grad):
    return {"name": name, "op": "adamw", "bits": bits, "layers": layers, "hidden": hidden, "kv": kv, "mlp": mlp, "rank": rank,
            "grad": grad}


def listed():
    qkv = _lora_case("lora_qkv_34b_m16", "fp16", 16, 8192, 8192, 16, 16, "mixed")
    qkv["kv"] = 1024
    return [
        # one token, one adapter, a 7B-shaped projection: launch and latency
        _lora_case("lora_4096x4096_m1", "fp16", 1, 4096, 4096, 16, 1),
        # sixteen requests with adapters of their own (some without one) on q, k and v of the 34B-class block
        qkv,
        # a ragged batch of prompts of five requests
        _lora_case("lora_13824x5120_m333", "bf16", 333, 13824, 5120, 32, 5),
        # training: the forward pass of a down projection, which keeps X A^T
        _lora_case("lora_8192x22016_m2048", "fp16", 2048, 8192, 22016, 64, 1, hidden=True),
        # the gradients of a small layer on a short sequence
        _bwd_case("bwd_1024x1024_m40", "fp16", 40, 1024, 1024, 8, 1),
        # three adapters trained in one ragged batch
        _bwd_case("bwd_5120x13824_m1000", "bf16", 1000, 5120, 13824, 32, 3),
        # one adapter, a long batch: the gradients of an up projection
        _bwd_case("bwd_22016x8192_m4096", "fp16", 4096, 22016, 8192, 16, 1),
        # few rows through a small frozen layer
        _grad_case("grad_4096x4096_m16", "fp6", 16, 4096, 4096),
        # a ragged batch, bf16
        _grad_case("grad_13824x5120_m333", "bf16", 333, 13824, 5120),
        # a training batch through the up projection of the 34B-class block
        _grad_case("grad_22016x8192_m2048", "fp6", 2048, 22016, 8192),
        # the adapters of one 7B-shaped block, states in 32 bits: fourteen small tensors
        _adamw_case("adamw32_7b_layer", 32, 1, 4096, 4096, 11008, 8, "fp32"),
        # the adapters of the whole 34B-class stack, states in 8 bits: 672 tensors
        _adamw_case("adamw8_34b_stack", 8, 48, 8192, 1024, 22016, 16, "fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _log_size(rng, lo, hi):
    return max(1, _log_int(rng, lo, hi) // 64) * 64


def _layer(rng):
    """N and K of one layer: no more weights than 22016 x 8192."""
    N = _log_size(rng, 1024, 22016)
    return N, _log_size(rng, 1024, min(22016, 22016 * 8192 // N))


def draw(rng):
    kind = rng.random()
    if kind < 0.75:
        N, K = _layer(rng)
    rank, dtype = rng.choice([8, 16, 24, 32, 64]), rng.choice(["fp16", "bf16"])
    if kind < 0.3:
        M = _log_int(rng, 1, 4096)
        adapters = rng.choice([1, _log_int(rng, 2, 16)])
        if M <= 32 and rng.random() < 0.4:
            case = _lora_case("", dtype, M, N, N, rank, adapters, "mixed")
            case["kv"] = max(64, N // 8 // 64 * 64)
        else:
            case = _lora_case("", dtype, M, N, K, rank, adapters, "mixed" if M <= 64 else "runs", M > 64 and rng.random() < 0.5)
    elif kind < 0.55:
        case = _bwd_case("", dtype, _log_int(rng, 16, 4096), N, K, rank, rng.choice([1, _log_int(rng, 2, 6)]))
    elif kind < 0.75:
        case = _grad_case("", rng.choice(["fp6", "fp6", "fp5", "v2", "bf16"]), _log_int(rng, 1, 2048), N, K)
    else:
        hidden = _log_size(rng, 1024, 8192)
        case = _adamw_case("", rng.choice([8, 32]), _log_int(rng, 1, 32), hidden, rng.choice([hidden, 1024]),
                           _log_size(rng, 2 * hidden, 2.6 * hidden), rng.choice([8, 16]), rng.choice(["fp32", "fp16", "bf16"]))
    del case["name"]
    return case


# ---- a user's program: what it has in hand before the call

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
_MANTISSA = {"fp6": 2, "fp5": 1, "v2": 2, "bf16": 2}            # of the formats of a frozen weight
_SCALED = 0.0078125                                             # gradients' magnitude under a loss scale


def _normal(gen, shape, dtype, sigma=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * sigma).to(dtype)


def _index(case, gen):
    """The adapter of each row: requests of random lengths one after another, or any mix with rows that have none."""
    M, L = case["M"], case["adapters"]
    if L == 1 and case["order"] == "runs":
        return None
    if case["order"] == "mixed":
        return torch.randint(-1, L, (M,), generator=gen, device="cuda").to(torch.int32)
    cuts = torch.randint(0, M + 1, (L - 1,), generator=gen, device="cuda").sort().values
    return torch.searchsorted(cuts, torch.arange(M, device="cuda"), right=True).to(torch.int32)


def _adapter(case, gen, N, K, dtype):
    L, r = case["adapters"], case["rank"]
    return _normal(gen, (L, r, K), dtype, K ** -0.5), _normal(gen, (L, N, r), dtype, 0.05)


def _small_float(w, mantissa):
    """w (double, within the format) to the nearest number with three exponent bits, bias 3, and `mantissa` bits."""
    step = torch.exp2(torch.frexp(w).exponent.clamp(min=-1).double() - 1 - mantissa)
    return torch.round(w / step) * step


def _frozen(case, gen):
    """An fp16 weight, the same weight rounded (values of the small format, as fp16) and its row scales."""
    mantissa = _MANTISSA[case["fmt"]]
    W = torch.randn((case["N"], case["K"]), generator=gen, device="cuda") * 0.02
    W = torch.where(torch.rand(W.shape, generator=gen, device="cuda") < 0.001, W * 10, W).half()
    top = 28.0 if mantissa == 2 else 24.0
    scales = (W.abs().amax(1).double() / top).half()
    values = torch.cat([_small_float((w.double() / s[:, None].double()).clamp(-top, top), mantissa).half()
                        for w, s in zip(W.split(2048), scales.split(2048))])
    return W, values, scales


def _shapes(case):
    """The adapters of a decoder block: [rank, in] and [out, rank] for q, k, v, o, gate, up and down."""
    h, kv, mlp, r = case["hidden"], case["kv"], case["mlp"], case["rank"]
    pairs = [(h, h), (kv, h), (kv, h), (h, h), (mlp, h), (mlp, h), (h, mlp)] * case["layers"]
    return [s for N, K in pairs for s in ((r, K), (N, r))]


def _decoded(codes, scales):
    """8-bit states as values: codes times the power of two of their block (exact in bf16)."""
    return codes.float() * torch.exp2(scales.float() - 127).repeat_interleave(BLOCK)


def _encoded(x):
    """x to e4m3 (nearest) with one power of two per block, the smallest that brings the block under 448."""
    top = x.abs().view(-1, BLOCK).amax(1)
    mantissa, exponent = torch.frexp(top)
    exponent = torch.where(top > 0, (exponent - 9 + (mantissa > 0.875).int()).clamp(min=-126), -127)
    scaled = x.view(-1, BLOCK) * torch.exp2(-exponent.float())[:, None]
    return scaled.reshape(-1).to(torch.float8_e4m3fn), (exponent + 127).to(torch.uint8)


def _prepare_adamw(case, gen):
    shapes = _shapes(case)
    starts, total = [], 0
    for a, b in shapes:                                         # every tensor starts a block
        starts.append(total)
        total += -(-a * b // BLOCK) * BLOCK
    inside = torch.zeros(total, device="cuda")
    for (a, b), at in zip(shapes, starts):
        inside[at:at + a * b] = 1
    p = _normal(gen, (total,), torch.float32, 0.02) * inside
    spread = torch.exp(_normal(gen, (total,), torch.float32)) * inside
    g = (_normal(gen, (total,), torch.float32, 1e-2) * spread).to(_TYPES[case["grad"]])
    m = _normal(gen, (total,), torch.float32, 3e-3) * spread
    v = (spread * 1e-2) ** 2
    flat = {"p": p, "g": g, "w": p.half()}
    if case["bits"] == 32:
        flat.update(m=m, v=v)
    else:
        flat["m"], flat["ms"] = _encoded(m)
        flat["v"], flat["vs"] = _encoded(v.sqrt())
    state = {"case": case, "flat": flat, "step": torch.tensor([STEP], dtype=torch.int32, device="cuda"),
             "grad_scale": torch.tensor([0.5], device="cuda")}
    if own:                                                     # the plan of the tensors, made once
        import paper_2312_08583_amd as P

        def views(key):
            return [flat[key][at:at + a * b].view(a, b) for (a, b), at in zip(shapes, starts)]

        def scales(key):
            return [flat[key][at // BLOCK:at // BLOCK + -(-a * b // BLOCK)] for (a, b), at in zip(shapes, starts)] if key in flat else None

        state["plan"] = P.fp6_adamw_plan(views("p"), views("g"), views("m"), views("v"), scales("ms"), scales("vs"), views("w"))
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000 + seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, gen)
    M, N, K = case["M"], case["N"], case["K"]
    if case["op"] == "grad":
        dtype = _TYPES["bf16" if case["fmt"] == "bf16" else "fp16"]
        W, values, scales = _frozen(case, gen)
        state = {"case": case, "values": values, "scales": scales, "dY": _normal(gen, (M, N), dtype, _SCALED),
                 "out": torch.empty((M, K), dtype=dtype, device="cuda")}
        if own:                                                 # the packed weight and its transpose, made once
            import paper_2312_08583_amd as P
            pack = {"fp6": P.fp6_quantize_pack, "fp5": P.fp5_quantize_pack}.get(case["fmt"], P.fp6_quantize_pack_v2)
            form = _format(P, case["fmt"])
            state["planes"] = P.fp6_transpose_pack(*pack(W), N, K, format=form)
            state["workspace"] = P.new_workspace(P.fp6_linear_grad_workspace_bytes(M, N, K, format=form), "cuda")
        return state
    dtype, L, r = _TYPES[case["dtype"]], case["adapters"], case["rank"]
    state = {"case": case, "index": _index(case, gen), "scaling": torch.rand((L,), generator=gen, device="cuda") + 0.5}
    X = _normal(gen, (M, K), dtype)
    if case["op"] == "lora":
        heights = [N, case["kv"], case["kv"]] if case["kv"] else [N]
        state["layers"] = [(X,) + _adapter(case, gen, n, K, dtype) + (_normal(gen, (M, n), dtype),) for n in heights]
        state["outs"] = [torch.empty_like(layer[3]) for layer in state["layers"]]
        state["hidden"] = torch.empty((M, r), device="cuda") if case["hidden"] else None
    else:
        A, B = _adapter(case, gen, N, K, dtype)
        at = torch.zeros((M,), dtype=torch.long, device="cuda") if state["index"] is None else state["index"].long()
        hidden = torch.zeros((M, r), device="cuda")
        for a in range(L):                                      # X A^T as the forward pass keeps it
            hidden = torch.where((at == a)[:, None], X.float() @ A[a].float().T, hidden)
        state.update(dY=_normal(gen, (M, N), dtype, _SCALED), X=X, hidden=hidden, A=A, B=B,
                     dX=_normal(gen, (M, K), dtype, _SCALED), out=torch.empty_like(X),
                     dA=torch.empty((L, r, K), device="cuda"), dB=torch.empty((L, N, r), device="cuda"))
    if own:                                                     # the workspace that the program keeps
        import paper_2312_08583_amd as P
        if case["op"] == "bwd":
            need = P.fp6_lora_backward_workspace_bytes(M, N, K, r, L)
        else:
            need = P.fp6_lora_group_workspace_bytes(M, [(n, K, r) for n in heights], L)
        state["workspace"] = P.new_workspace(need, "cuda")
    return state


def _format(P, fmt):
    return {"fp6": P.FP6_FORMAT_E3M2, "fp5": P.FP6_FORMAT_E3M1, "v2": P.FP6_FORMAT_E3M2_V2, "bf16": P.FP6_FORMAT_E3M2_V2_BF16}[fmt]


# ---- one pass

def _run_own(state):
    import paper_2312_08583_amd as P
    case = state["case"]
    if case["op"] == "adamw":
        P.fp6_adamw(state["plan"], state["step"], LR, BETA1, BETA2, EPS, DECAY, grad_scale=state["grad_scale"], seed=SEED)
        return _adamw_outputs(state)
    if case["op"] == "grad":
        return P.fp6_linear_grad(state["dY"], *state["planes"], case["N"], case["K"], format=_format(P, case["fmt"]),
                                 out=state["out"], workspace=state["workspace"])
    if case["op"] == "bwd":
        return P.fp6_lora_backward(state["dY"], state["X"], state["hidden"], state["A"], state["B"], state["dX"], state["index"],
                                   state["scaling"], dA=state["dA"], dB=state["dB"], out=state["out"],
                                   workspace=state["workspace"])
    if case["kv"]:
        return P.fp6_lora_group(state["layers"], state["index"], state["scaling"], outs=state["outs"],
                                workspace=state["workspace"])
    Y = P.fp6_lora(*state["layers"][0], state["index"], state["scaling"], hidden=state["hidden"], out=state["outs"][0],
                   workspace=state["workspace"])
    return [Y, state["hidden"]] if case["hidden"] else [Y]


def _adamw_outputs(state):
    flat = state["flat"]
    if state["case"]["bits"] == 32:
        return {**flat, "step": state["step"]}
    # (a code's value has four significant bits: bf16 holds it)
    return {"p": flat["p"], "w": flat["w"], "step": state["step"], "m": _decoded(flat["m"], flat["ms"]).bfloat16(),
            "v": _decoded(flat["v"], flat["vs"]).bfloat16()}


def _rows_of(state, dtype):
    """[M, L]: the scale of the row's adapter in its column, 0 elsewhere; and which entries those are."""
    case = state["case"]
    at = torch.zeros((case["M"],), dtype=torch.int32, device="cuda") if state["index"] is None else state["index"]
    mine = at[:, None] == torch.arange(case["adapters"], device="cuda", dtype=torch.int32)
    return mine.to(dtype) * state["scaling"].to(dtype), mine


def _plain_lora(layer, state):
    X, A, B, Y = layer
    L, r, K = A.shape
    scaled, mine = _rows_of(state, torch.float32)
    H = (X.float() @ A.float().view(L * r, K).T).view(-1, L, r)          # against every adapter, those of others dropped
    weighted = (H * scaled[:, :, None]).view(-1, L * r)
    out = Y.float() + weighted @ B.float().permute(0, 2, 1).reshape(L * r, -1)
    return out.to(Y.dtype), (H * mine[:, :, None]).sum(1)


def _plain_backward(state):
    dY, X, A, B = state["dY"].float(), state["X"].float(), state["A"].float(), state["B"].float()
    L, r, K = A.shape
    scaled, _ = _rows_of(state, torch.float32)
    dH = ((dY @ B.permute(1, 0, 2).reshape(-1, L * r)).view(-1, L, r) * scaled[:, :, None]).view(-1, L * r)
    H = (state["hidden"][:, None, :] * scaled[:, :, None]).view(-1, L * r)
    dX = (state["dX"].float() + dH @ A.view(L * r, K)).to(state["X"].dtype)
    dA = (dH.T @ X).view(L, r, K)
    dB = (H.T @ dY).view(L, r, -1).permute(0, 2, 1).contiguous()
    return dX, dA, dB


def _hash(ids, step):
    """32 bits of a counter hash per element, in the low half of int64."""
    x = (ids * 0x9E3779B1 + step * 0x3C6EF373 + SEED) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _rounded(x, noise, floor):
    """x to e4m3 values with a power of two per block; up or down by 16 bits of noise, never below `floor` of the smallest."""
    top = x.abs().view(-1, BLOCK).amax(1)
    mantissa, exponent = torch.frexp(top)
    exponent = torch.where(top > 0, (exponent - 9 + (mantissa > 0.875).int()).clamp(min=-126), -127)
    y = (x.view(-1, BLOCK) * torch.exp2(-exponent.to(x.dtype))[:, None]).view(-1)
    quantum = torch.exp2((torch.frexp(y).exponent - 1).clamp(min=-6).to(x.dtype) - 3)
    k = torch.floor(y.abs() / quantum + noise.to(x.dtype) * 2.0 ** -16)
    k = torch.where(x != 0, torch.maximum(k, torch.full_like(k, floor)), k)
    return (torch.copysign(k * quantum, x)).to(torch.float8_e4m3fn), (exponent + 127).to(torch.uint8)


def _plain_adamw(state):
    case, flat, step = state["case"], state["flat"], state["step"]
    step += 1
    t = step.double()
    first, second = (LR / (1 - BETA1 ** t)).float(), (1 / (1 - BETA2 ** t).sqrt()).float()
    g = flat["g"].float() * state["grad_scale"]
    eight = case["bits"] == 8
    m = _decoded(flat["m"], flat["ms"]) if eight else flat["m"]
    v = _decoded(flat["v"], flat["vs"]).square() if eight else flat["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g.square() * (1 - BETA2)
    u = v.sqrt()
    p = flat["p"] * (1 - LR * DECAY) - m / (u * second + EPS) * first
    flat["p"].copy_(p)
    flat["w"].copy_(p)
    if eight:
        noise = _hash(torch.arange(p.numel(), device="cuda"), step.long())
        (mc, ms), (vc, vs) = _rounded(m, noise >> 16, 0), _rounded(u, noise & 0xFFFF, 1)
        flat["m"].copy_(mc), flat["ms"].copy_(ms), flat["v"].copy_(vc), flat["vs"].copy_(vs)
    else:
        flat["m"].copy_(m), flat["v"].copy_(v)
    return _adamw_outputs(state)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "adamw":
        return _plain_adamw(state)
    if case["op"] == "grad":
        return ((state["dY"].float() * state["scales"].float()) @ state["values"].float()).to(state["dY"].dtype)
    if case["op"] == "bwd":
        return _plain_backward(state)
    if case["kv"]:
        return [_plain_lora(layer, state)[0] for layer in state["layers"]]
    Y, hidden = _plain_lora(state["layers"][0], state)
    return [Y, hidden] if case["hidden"] else [Y]


# ---- what a pass cannot do without

def work(case):
    if case["op"] == "adamw":
        n = sum(a * b for a, b in _shapes(case))
        state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK               # m and v, read and written
        return {"bytes": n * (8 + 2 + {"fp32": 4}.get(case["grad"], 2) + state), "flops": 16 * n}
    M, N, K = case["M"], case["N"], case["K"]
    if case["op"] == "grad":
        return {"bytes": (0.625 if case["fmt"] == "fp5" else 0.75) * N * K + 2 * N + 2 * M * (N + K), "flops": 2 * M * N * K}
    L, r = case["adapters"], case["rank"]
    used = min(L, M)
    if case["op"] == "bwd":
        return {"bytes": 2 * M * (N + 3 * K) + 4 * M * r + 2 * used * r * (N + K) + 4 * L * r * (N + K),
                "flops": 8 * M * r * (N + K)}
    heights = [N, case["kv"], case["kv"]] if case["kv"] else [N]
    return {"bytes": 2 * M * K + sum(4 * M * n + 2 * used * r * (n + K) for n in heights) + (4 * M * r if case["hidden"] else 0),
            "flops": sum(2 * M * r * (n + K) for n in heights)}


# ---- the definition in 64 bits

def _exact_rounding(x, noise, least):
    """The 8-bit state of x: per block the scale 2^e with max |x| in (224, 448] 2^e, then sign and four bits, cut at `noise`."""
    out = torch.zeros_like(x)
    for lo in range(0, x.numel(), BLOCK << 14):
        y = x[lo:lo + (BLOCK << 14)].view(-1, BLOCK)
        e = torch.ceil(torch.log2(y.abs().amax(1, keepdim=True).clamp(min=1e-300) / 448)).clamp(min=-126)
        z = y.abs() / 2 ** e
        unit = 2 ** (torch.floor(torch.log2(z.clamp(min=2.0 ** -6))) - 3)
        count = torch.floor(z / unit + noise[lo:lo + (BLOCK << 14)].view(-1, BLOCK).double() / 65536)
        count[(z > 0) & (count < least)] = least
        out[lo:lo + (BLOCK << 14)] = (y.sign() * count * unit * 2 ** e).reshape(-1)
    return out


def _exact_adamw(case, state):
    flat = {k: x.double() for k, x in state["flat"].items()}
    t, eight = STEP + 1, case["bits"] == 8
    m, v = flat["m"], flat["v"]
    if eight:
        m = (m.view(-1, BLOCK) * 2 ** (flat["ms"][:, None] - 127)).reshape(-1)
        v = ((v.view(-1, BLOCK) * 2 ** (flat["vs"][:, None] - 127)) ** 2).reshape(-1)
    g = flat["g"] * 0.5
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
    p = flat["p"] - LR * DECAY * flat["p"] - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    if not eight:
        return {"p": p, "g": None, "w": p, "m": m, "v": v, "step": None}
    x = torch.arange(p.numel(), device="cuda") * 0x9E3779B1 + (t * 0x3C6EF373 + SEED)
    for shift, factor in ((16, 0x6A09E667), (15, 0xBB67AE85)):
        x = x % 2 ** 32
        x = (x ^ (x >> shift)) * factor
    x = x % 2 ** 32
    x = x ^ (x >> 16)
    return {"p": p, "w": p, "step": None, "m": _exact_rounding(m, x // 65536, 0), "v": _exact_rounding(v.sqrt(), x % 65536, 1)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(case, state)
    if case["op"] == "grad":
        W = state["values"].double() * state["scales"].double()[:, None]
        return torch.mm(state["dY"].double(), W)
    M, L = case["M"], case["adapters"]
    rows = [torch.arange(M, device="cuda")] if state["index"] is None else [(state["index"] == a).nonzero()[:, 0] for a in range(L)]
    s = state["scaling"].double()
    if case["op"] == "lora":
        outs, H = [], torch.zeros((M, case["rank"]), dtype=torch.float64, device="cuda")
        for X, A, B, Y in state["layers"]:
            Z = Y.double()
            for a, at in enumerate(rows):
                H[at] = X[at].double() @ A[a].double().T
                Z[at] += s[a] * (H[at] @ B[a].double().T)
            outs.append(Z)
        return outs + [H] if case["hidden"] else outs
    dX, dA, dB = state["dX"].double(), [], []
    for a, at in enumerate(rows):
        up = s[a] * state["dY"][at].double()
        down = up @ state["B"][a].double()
        dX[at] += down @ state["A"][a].double()
        dA.append(down.T @ state["X"][at].double())
        dB.append(up.T @ state["hidden"][at].double())
    return dX, torch.stack(dA), torch.stack(dB)
