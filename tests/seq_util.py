"""Plain 64-bit forms of the sequence operators on the host, with bounds on the
rounding errors of an evaluation in the accumulation type; helpers of their
GPU tests."""
import torch

UNIT = {torch.float64: 2.0 ** -53, torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11,
        torch.bfloat16: 2.0 ** -8}  # largest relative error of rounding to the type
LEAST = {torch.float64: 0.0, torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25,
         torch.bfloat16: 2.0 ** -134}  # largest absolute error among its subnormals
TYPES = [torch.float64, torch.float32, torch.bfloat16, torch.float16]


def acc_of(dtype):
    return torch.float64 if dtype == torch.float64 else torch.float32


def within(got, want, bound, dtype):
    """Every |got - want| <= bound + the error of rounding want to dtype; NaN where NaN."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    # the rounding is of a value up to `bound` from want
    slack = bound + UNIT[dtype] * (want.abs() + bound) + LEAST[dtype]
    bad = ((got - want).abs() > slack) & ~nan
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / slack)[~nan].max()))


def recurrence(a, u, h0, lens, sigmoid, dh=None, dhT=None):
    """{name: (value, bound)} by the definition, step after step, in float64. A bound follows the
    loop: what an earlier error has become, and K roundings of this step's terms, each at most
    as large as the sum S of the magnitudes of everything that was added up."""
    dtype = a.dtype
    unit = UNIT[acc_of(dtype)]
    a, u = a.cpu().double(), u.cpu().double()
    B, T, D = a.shape
    lens = torch.full((B,), T) if lens is None else lens.cpu().clamp(0, T)
    live = (torch.arange(T)[None, :] < lens[:, None]).unsqueeze(2)
    a, u = (torch.where(live, v, torch.zeros_like(v)) for v in (a, u))
    if sigmoid:
        # exp's argument is rounded, which moves its value by |a| units; from 104 on exp(-|a|)
        # is beyond the 32-bit range
        K = 16 + 4 * min(104.0, float(a.nan_to_num(0, 0, 0).abs().max() if a.numel() else 0))
        c, q = torch.sigmoid(a), torch.sigmoid(-a)
        d = q * u
    else:
        K = 8
        c, d, q = a, u, torch.ones_like(a)
    x = torch.zeros(B, D, dtype=torch.float64) if h0 is None else h0.cpu().double()
    S, E = x.abs(), torch.zeros_like(x)
    h, hE, old, oldE, oldS = (torch.zeros(B, T, D, dtype=torch.float64) for _ in range(5))
    for t in range(T):
        on = live[:, t]
        old[:, t], oldE[:, t], oldS[:, t] = x, E, S
        x = torch.where(on, c[:, t] * x + d[:, t], x)
        S = torch.where(on, c[:, t].abs() * S + d[:, t].abs(), S)
        E = torch.where(on, c[:, t].abs() * E + K * unit * S, E)
        h[:, t], hE[:, t] = torch.where(on, x, 0.0), torch.where(on, E, 0.0)
    out = {"h": (h, hE), "hT": (x, E)}
    if dh is None:
        return out
    dh = torch.where(live, dh.cpu().double(), 0.0)
    G = torch.zeros(B, D, dtype=torch.float64) if dhT is None else dhT.cpu().double()
    S, E = G.abs(), torch.zeros_like(G)
    da, daE, du, duE = (torch.zeros(B, T, D, dtype=torch.float64) for _ in range(4))
    for t in reversed(range(T)):
        on = live[:, t]
        G1, S1 = G + dh[:, t], S + dh[:, t].abs()
        E1 = E + K * unit * S1
        f = c[:, t] * q[:, t] if sigmoid else torch.ones_like(G)
        y = old[:, t] - u[:, t] if sigmoid else old[:, t]
        yS = oldS[:, t] + (u[:, t].abs() if sigmoid else 0.0)
        f_abs = f.abs()
        da[:, t] = torch.where(on, G1 * y * f, 0.0)
        daE[:, t] = torch.where(
            on, f_abs * (E1 * yS + S1 * oldE[:, t] + K * unit * S1 * yS), 0.0)
        du[:, t] = torch.where(on, G1 * q[:, t], 0.0)
        duE[:, t] = torch.where(on, q[:, t].abs() * (E1 + K * unit * S1), 0.0)
        G = torch.where(on, c[:, t] * G1, G)
        S = torch.where(on, c[:, t].abs() * S1, S)
        E = torch.where(on, c[:, t].abs() * E1 + K * unit * S, E)
    out.update(da=(da, daE), du=(du, duE), dh0=(G, E))
    return out


def layer_norm(x, w, b, eps, dy=None):
    """{name: (value, bound)} in float64. A sum of n terms in any order is within n units of the
    sum of their magnitudes."""
    unit = UNIT[acc_of(x.dtype)]
    x = x.cpu().double()
    rows, n = x.shape
    w = torch.ones(n, dtype=torch.float64) if w is None else w.cpu().double()
    b = torch.zeros(n, dtype=torch.float64) if b is None else b.cpu().double()
    mean = x.mean(1, keepdim=True)
    mid = x - mean
    var = (mid * mid).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    N = (n + 8) * unit
    size = x.abs().mean(1, keepdim=True)
    meanE = N * size
    midE = meanE + unit * (x.abs() + size)
    # the centred values' errors move the variance to first order by twice their product,
    # to second order by their square
    varE = 2 * (mid.abs() * midE).mean(1, keepdim=True) + (midE * midE).mean(1, keepdim=True) \
        + N * var
    rstdE = rstd * (0.5 * varE * rstd * rstd + 4 * unit)
    hat = mid * rstd
    hatE = midE * rstd + (mid.abs() + midE) * rstdE + unit * hat.abs()
    out = {"y": (hat * w + b, hatE * w.abs() + 4 * unit * (hat * w).abs() + 2 * unit * b.abs()),
           "mean": (mean[:, 0], meanE[:, 0]), "rstd": (rstd[:, 0], rstdE[:, 0])}
    if dy is None:
        return out
    dy = dy.cpu().double()
    e = dy * w
    s1, s2 = e.mean(1, keepdim=True), (e * hat).mean(1, keepdim=True)
    eE = unit * e.abs()
    s1E = N * e.abs().mean(1, keepdim=True) + eE.mean(1, keepdim=True)
    s2E = N * (e * hat).abs().mean(1, keepdim=True) + \
        (eE * hat.abs() + e.abs() * hatE).mean(1, keepdim=True)
    inner = e - s1 - hat * s2
    innerE = eE + s1E + hat.abs() * s2E + hatE * s2.abs() + \
        4 * unit * (e.abs() + s1.abs() + (hat * s2).abs())
    R = (rows + 8) * unit
    out.update(
        dx=(inner * rstd, innerE * rstd + (inner.abs() + innerE) * rstdE + unit * inner.abs() * rstd),
        dw=((dy * hat).sum(0), R * (dy * hat).abs().sum(0) + (dy.abs() * hatE).sum(0)),
        db=(dy.sum(0), R * dy.abs().sum(0)))
    return out
