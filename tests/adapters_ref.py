"""Low-rank adapters in 64 bits, with the magnitudes that error bounds are made of (test infrastructure)."""
import torch

STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}            # half a step of the type, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}          # half a step of its smallest numbers
SPLIT = {torch.float16: 2.0 ** -21, torch.bfloat16: 2.0 ** -17}          # an fp32 operand as two 16-bit terms


def depth(contraction):
    """Roundings that an fp32 sum of this many products passes through at most, in units of 2^-24, doubled: matrix instructions of 32
    products one after another (32 inside one), then wavefronts, slices and splits."""
    return 2 * (contraction / 32 + 32 + 64) * 2.0 ** -24


def rows_of(index, M, L):
    at = torch.zeros(M, dtype=torch.long) if index is None else index.cpu().long()
    return [(at == a).nonzero()[:, 0] for a in range(L)]


def forward(X, A, B, Y, index, scaling):
    """out, H and the largest error of out and H that rounding can cause."""
    dtype, (M, K), (L, N, r) = Y.dtype, X.shape, B.shape
    X, A, B, Y = (t.cpu().double() for t in (X, A, B, Y))
    s = torch.ones(L, dtype=torch.float64) if scaling is None else scaling.cpu().double()
    out, H, err, herr = Y.clone(), torch.zeros(M, r, dtype=torch.float64), torch.zeros(M, N, dtype=torch.float64), torch.zeros(M, r, dtype=torch.float64)
    for a, at in enumerate(rows_of(index, M, L)):
        x = X[at]
        H[at] = x @ A[a].T
        herr[at] = depth(K) * (x.abs() @ A[a].abs().T)
        out[at] += s[a] * (H[at] @ B[a].T)
        top = H[at].abs().amax(1, keepdim=True) if len(at) else H[at][:, :1]
        spread = H[at].abs() * (SPLIT[dtype] + depth(r)) + top * 2.0 ** -36
        err[at] = s[a].abs() * ((herr[at] + spread) @ B[a].abs().T) + 2.0 ** -22 * (out[at] - Y[at]).abs()
    err = err * (1 + 2 * STEP[dtype]) + out.abs() * STEP[dtype] + TINY[dtype]
    return out, H, err, herr


def backward(dY, X, hidden, A, B, dX, index, scaling):
    """(dX', dA, dB) and their largest errors."""
    dtype, (M, K), (L, N, r) = X.dtype, X.shape, B.shape
    dY, X, H, A, B, dX = (t.cpu().double() for t in (dY, X, hidden, A, B, dX))
    s = torch.ones(L, dtype=torch.float64) if scaling is None else scaling.cpu().double()
    out, err = dX.clone(), torch.zeros(M, K, dtype=torch.float64)
    dA, dB = torch.zeros(L, r, K, dtype=torch.float64), torch.zeros(L, N, r, dtype=torch.float64)
    ea, eb = torch.zeros_like(dA), torch.zeros_like(dB)
    for a, at in enumerate(rows_of(index, M, L)):
        if not len(at):
            continue
        up = s[a] * dY[at]
        dH = up @ B[a]
        herr = (depth(N) + 2.0 ** -23) * (up.abs() @ B[a].abs())
        top = dH.abs().amax(1, keepdim=True)
        out[at] += dH @ A[a]
        err[at] = (herr + dH.abs() * (SPLIT[dtype] + depth(r)) + top * 2.0 ** -36) @ A[a].abs() + 2.0 ** -22 * (dH @ A[a]).abs()
        # (the outer products split to 22 bits of the column's largest in 64 rows, or to 24)
        each = herr + dH.abs() * (2.0 ** -21 + depth(len(at))) + dH.abs().amax(0, keepdim=True) * 2.0 ** -36
        dA[a], ea[a] = dH.T @ X[at], each.T @ X[at].abs()
        spread = H[at].abs() * (2.0 ** -21 + depth(len(at))) + H[at].abs().amax(0, keepdim=True) * 2.0 ** -36
        dB[a], eb[a] = up.T @ H[at], up.abs().T @ spread + 2.0 ** -23 * (up.T @ H[at]).abs()
    err = err * (1 + 2 * STEP[dtype]) + out.abs() * STEP[dtype] + TINY[dtype]
    return (out, dA, dB), (err, ea, eb)


def assert_within(got, want, err, what):
    d = (got.cpu().double() - want).abs()
    assert torch.isfinite(got).all(), what
    worst = (d - err).max().item() if d.numel() else -1.0
    assert worst <= 0, (what, worst, d.max().item())


def normal(shape, seed, dtype=torch.float32, sigma=1.0, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=device) * sigma).to(dtype)


def adapters(L, r, N, K, seed, dtype, device="cuda"):
    return normal((L, r, K), seed, dtype, K ** -0.5, device), normal((L, N, r), seed + 1, dtype, 0.05, device)


def index_of(order, M, L, seed, device="cuda"):
    """None; runs of one adapter after another; any order with rows that have none."""
    if order == "none":
        return None
    g = torch.Generator()
    g.manual_seed(seed)
    if order == "runs":
        return torch.sort(torch.randint(0, L, (M,), generator=g))[0].to(torch.int32).to(device)
    return torch.randint(-1, L, (M,), generator=g).to(torch.int32).to(device)
