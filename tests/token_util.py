"""Plain 64-bit forms of the token operators on the host, with bounds on the rounding errors of an
evaluation in the accumulation type; helpers of their GPU tests.

A bound follows the evaluation (running error analysis): a Num is a value and how far a computed
one may be from it. An operation adds the errors of what it is given, to first order and their
product, and a rounding of its result, at most one unit of the sum of the magnitudes that it
adds up; a sum of n terms in any order is within n units of the sum of their magnitudes."""
import torch

from tests.seq_util import UNIT, acc_of, within  # noqa: F401


class Num:
    def __init__(self, v, e, unit):
        self.v, self.e, self.unit = v, e, unit

    def make(self, v, e):
        return Num(v, e, self.unit)

    def __getitem__(self, at):
        return self.make(self.v[at], self.e[at])

    def __add__(self, o):
        return self.make(self.v + o.v, self.e + o.e + self.unit * (self.v.abs() + o.v.abs()
                                                                  + self.e + o.e))

    def __mul__(self, o):
        a, b = self.v.abs(), o.v.abs()
        far = a * o.e + b * self.e + self.e * o.e
        return self.make(self.v * o.v, far + self.unit * (a * b + far))

    def exp(self):
        """The argument is rounded, twice where it is taken to another base, which moves the
        value by twice its size in units; the exponential itself is within 4."""
        v = torch.exp(self.v)
        k = 4 + 2 * self.v.abs().clamp(max=800)
        # results below the normal range may be 0
        least = 2.0 ** (-1022 if self.unit < 2.0 ** -40 else -126)
        return self.make(v, v * torch.expm1(self.e.clamp(max=1)) + k * self.unit * v + least)

    def sigmoid(self):
        """1 / (1 + exp(-v)), with an exponential as above."""
        v, q = torch.sigmoid(self.v), torch.sigmoid(-self.v)
        k = 10 + 2 * self.v.abs().clamp(max=104)
        least = 2.0 ** (-1022 if self.unit < 2.0 ** -40 else -126)
        return self.make(v, v * q * self.e * (1 + self.e) + 0.5 * self.e ** 2
                         + k * self.unit * v + least)

    def other(self):
        """1 - sigmoid, to its own precision."""
        return self.make(-self.v, self.e).sigmoid()

    def softplus(self):
        """max(v, 0) + log(1 + exp(-|v|)): the exponential as above, then 16 roundings at most of
        a quotient and a series."""
        v = torch.logaddexp(self.v, torch.zeros_like(self.v))
        k = 24 + 2 * self.v.abs().clamp(max=104)
        least = 2.0 ** (-1022 if self.unit < 2.0 ** -40 else -126)
        return self.make(v, torch.sigmoid(self.v) * self.e * (1 + self.e) + 0.5 * self.e ** 2
                         + k * self.unit * v + least)

    def sum(self, dims):
        dims = (dims,) if isinstance(dims, int) else dims
        n = 1
        for d in dims:
            n *= self.v.shape[d]
        size = (self.v.abs() + self.e).sum(dims)
        return self.make(self.v.sum(dims), self.e.sum(dims) + (n + 2) * self.unit * size)

    def where(self, on):
        return self.make(torch.where(on, self.v, 0.0), torch.where(on, self.e, 0.0))

    def pair(self):
        return self.v, self.e


def num(t, dtype):
    v = t.detach().cpu().double()
    return Num(v, torch.zeros_like(v), UNIT[acc_of(dtype)])


def stack(nums, dim):
    return Num(torch.stack([n.v for n in nums], dim), torch.stack([n.e for n in nums], dim),
               nums[0].unit)


def live_of(lens, B, T):
    lens = torch.full((B,), T) if lens is None else lens.cpu().clamp(0, T).long()
    return lens, (torch.arange(T)[None, :] < lens[:, None]).unsqueeze(2)


def clean(t, live):
    """t without what is not to be read."""
    return torch.where(live, t.detach().cpu().double(), 0.0)


# -------------------------------------------------------------- convolution
def conv(x, w, b, x0, lens, silu, dy=None, dxT=None):
    """{name: (value, bound)}."""
    dtype = x.dtype
    B, T, D = x.shape
    K = w.shape[0]
    lens, live = live_of(lens, B, T)
    x0 = torch.zeros(B, K - 1, D, dtype=torch.float64) if x0 is None else x0.cpu().double()
    seen = num(torch.cat([x0, clean(x, live)], 1), dtype)
    wn = num(w, dtype)
    pre = num(torch.zeros(B, T, D, dtype=torch.float64) if b is None
              else b.cpu().double().expand(B, T, D), dtype)
    for k in range(K):
        pre = pre + seen[:, k:k + T] * wn[k]
    s, q = pre.sigmoid(), pre.other()
    y = pre * s if silu else pre
    at = lens[:, None] + torch.arange(K - 1)[None]
    out = {"y": y.where(live).pair(),
           "xT": (torch.gather(seen.v, 1, at[..., None].expand(B, K - 1, D)),
                  torch.zeros(B, K - 1, D, dtype=torch.float64))}
    if dy is None:
        return out
    g = num(clean(dy, live), dtype)
    if silu:
        one = num(torch.ones_like(pre.v), dtype)
        g = g * (s * (one + pre * q))
    g = g.where(live)
    dseen = num(torch.zeros(B, T + K - 1, D, dtype=torch.float64), dtype)
    if dxT is not None:
        dseen.v.scatter_(1, at[..., None].expand(B, K - 1, D), dxT.cpu().double())
    for k in range(K):
        t = g * wn[k]
        pad = [torch.zeros(B, k, D, dtype=torch.float64),
               torch.zeros(B, K - 1 - k, D, dtype=torch.float64)]
        dseen = dseen + t.make(torch.cat([pad[0], t.v, pad[1]], 1),
                               torch.cat([pad[0], t.e, pad[1]], 1))
    out["dx0"], out["dx"] = dseen[:, :K - 1].pair(), dseen[:, K - 1:].where(live).pair()
    out["dw"] = stack([(g * seen[:, k:k + T]).sum((0, 1)) for k in range(K)], 0).pair()
    out["db"] = g.sum((0, 1)).pair()
    return out


# ------------------------------------------------------------ selective scan
def scan(x, delta, A, B, C, D=None, z=None, delta_bias=None, h0=None, lens=None, softplus=True,
         dy=None, dhT=None):
    """{name: (value, bound)}. Where the time axis may be cut into segments a state goes through
    exp(A sum s), whose sum of at most T terms is within T units: that moves the state by at most
    T units of |A sum s| exp(A sum s) <= 0.37 of an earlier one."""
    dtype = x.dtype
    Bt, T, Dn = x.shape
    N = A.shape[1]
    B, C = (v.unsqueeze(2) if v.dim() == 3 else v for v in (B, C))
    G = B.shape[2]
    lens_, live = live_of(lens, Bt, T)
    x_, raw = num(clean(x, live), dtype), num(clean(delta, live), dtype)
    if delta_bias is not None:
        raw = raw + num(delta_bias.expand(Bt, T, Dn), dtype)
    s = raw.softplus() if softplus else raw
    Bc, Cc = (num(clean(v.reshape(Bt, T, G * N), live), dtype) for v in (B, C))

    def spread(n):  # to each channel of a group
        f = lambda v: v.view(Bt, T, G, 1, N).expand(Bt, T, G, Dn // G, N).reshape(Bt, T, Dn, N)
        return n.make(f(n.v), f(n.e))

    Bc, Cc = spread(Bc), spread(Cc)
    An = num(A, dtype)
    h = num(torch.zeros(Bt, Dn, N, dtype=torch.float64) if h0 is None else h0, dtype)
    sx = s * x_
    arg = s[..., None] * An
    a = arg.exp()
    drive = sx[..., None] * Bc
    cut = 0.4 * T * h.unit if T >= 200 else 0.0
    top = h.v.abs()
    hs = [h]
    for t in range(T):
        on = live[:, t, :, None]
        new = a[:, t] * h + drive[:, t]
        top = torch.maximum(top, new.v.abs())
        h = h.make(torch.where(on, new.v, h.v), torch.where(on, new.e, h.e))
        hs.append(h.make(h.v, h.e + cut * top))
    all_h = stack(hs, 1)
    now, before = all_h[:, 1:], all_h[:, :-1]
    pre = (now * Cc).sum(3)
    skip = num(torch.zeros(Dn, dtype=torch.float64) if D is None else D, dtype)
    if D is not None:
        pre = pre + x_ * skip
    y = pre
    if z is not None:
        zn = num(clean(z, live), dtype)
        f, q = zn.sigmoid(), zn.other()
        y = pre * (zn * f)
    out = {"y": y.where(live).pair(), "hT": hs[-1].pair()}
    if dy is None:
        return out
    d = num(clean(dy, live), dtype)
    one = num(torch.ones_like(d.v), dtype)
    if z is not None:
        out["dz"] = (d * pre * (f * (one + zn * q))).where(live).pair()
        d = d * (zn * f)
    Gr = num(torch.zeros(Bt, Dn, N, dtype=torch.float64) if dhT is None else dhT, dtype)
    top = Gr.v.abs()
    totals, downs = [None] * T, [None] * T
    for t in reversed(range(T)):
        on = live[:, t, :, None]
        total = Gr + d[:, t, :, None] * Cc[:, t]
        top = torch.maximum(top, total.v.abs())
        total = total.make(total.v, total.e + cut * top)
        down = total * a[:, t]
        totals[t], downs[t] = total.where(on), down.where(on)
        Gr = Gr.make(torch.where(on, down.v, Gr.v), torch.where(on, down.e, Gr.e))
    out["dh0"] = Gr.make(Gr.v, Gr.e + cut * top).pair()
    if T == 0:
        return out
    total, down = stack(totals, 1), stack(downs, 1)
    per = lambda n: n.make(n.v.view(Bt, T, G, Dn // G, N), n.e.view(Bt, T, G, Dn // G, N)).sum(3)
    out["dC"] = per(d[..., None] * now).pair()
    out["dB"] = per(total * sx[..., None]).pair()
    q_ = (down * before).where(live[..., None])
    u = (total * Bc).sum(3)
    out["dA"] = (q_ * s[..., None]).sum((0, 1)).pair()
    dx = s * u
    if D is not None:
        dx = dx + d * skip
        out["dD"] = (d * x_).where(live).sum((0, 1)).pair()
    out["dx"] = dx.where(live).pair()
    ds = (q_ * An).sum(3) + x_ * u
    if softplus:
        ds = ds * raw.sigmoid()
    ds = ds.where(live)
    out["ddelta"] = ds.pair()
    if delta_bias is not None:
        out["ddelta_bias"] = ds.sum((0, 1)).pair()
    return out


# ------------------------------------------------------------- cross entropy
def xent(x, w, labels, dloss=None, train=True):
    """{name: (value, bound)}. Beside 16-bit types g is rounded to the type, to which its scaling
    adds two roundings of the accumulation type; below the type's normal range it is off by at
    most the least value times the scale's inverse, 2^-24 / 2^14 of the largest |dloss| in F16."""
    dtype = x.dtype
    V = w.shape[0]
    labels = labels.cpu().long()
    valid = (labels >= 0) & (labels < V)
    x_ = x.detach().cpu().double()
    dl = torch.ones(x.shape[0], dtype=torch.float64) if dloss is None else dloss.cpu().double()
    dl = torch.where(valid, dl, 0.0)
    xn, wn = num(x_, dtype), num(w, dtype)
    unit, K = xn.unit, x.shape[1]
    logits = x_ @ wn.v.T
    off = (K + 2) * unit * (x_.abs() @ wn.v.abs().T)
    l = xn.make(logits, off)
    top = logits.max(1, keepdim=True).values
    shifted = l.make(logits - top, off + unit * (logits.abs() + top.abs()) + off.max(1, keepdim=True)
                     .values)
    total = shifted.exp().sum(1)
    lse = torch.logsumexp(logits, 1)
    lseE = total.e / total.v + 4 * unit * (lse.abs() + top[:, 0].abs() + 1)
    # the largest logit's own error cancels in the exact value: only roundings are left of it
    rows = torch.arange(x.shape[0])
    target, targetE = logits[rows, labels.clamp(0, V - 1)], off[rows, labels.clamp(0, V - 1)]
    out = {"lse": (lse, lseE),
           "loss": (torch.where(valid, lse - target, 0.0),
                    torch.where(valid, lseE + targetE + unit * (lse.abs() + target.abs()), 0.0))}
    if not train:
        return out
    p = l.make(logits - lse[:, None],
               off + lseE[:, None] + unit * (logits.abs() + lse.abs()[:, None])).exp()
    hot = torch.zeros_like(logits)
    hot[rows[valid], labels[valid]] = 1.0
    g = (p.v - hot) * dl[:, None]
    gE = (p.e + 4 * unit * (p.v + hot)) * dl.abs()[:, None]
    if dtype in (torch.bfloat16, torch.float16):
        most = dl.abs().max() if dl.numel() else 0.0
        gE = gE + (UNIT[dtype] + 4 * unit) * (g.abs() + gE)
        if dtype == torch.float16:
            gE = gE + 2.0 ** -38 * most
    on = (dl != 0)[:, None]
    g, gE = torch.where(on, g, 0.0), torch.where(on, gE, 0.0)
    xk = torch.where(on, x_, 0.0)
    far = lambda n: (n + 8) * unit
    out["dx"] = (g @ wn.v, gE @ wn.v.abs() + far(V) * ((g.abs() + gE) @ wn.v.abs()))
    out["dw"] = (g.T @ xk, gE.T @ xk.abs() + far(x.shape[0]) * ((g.abs() + gE).T @ xk.abs()))
    return out


def check(got, want, dtype, of_type):
    """of_type: the outputs in the element type; the others are in the accumulation type."""
    for name, (value, bound) in want.items():
        kind = of_type.get(name, acc_of(dtype)) if isinstance(of_type, dict) else \
            (dtype if name in of_type else acc_of(dtype))
        assert got[name].dtype == kind, name
        try:
            within(got[name], value, bound, kind)
        except AssertionError as e:
            raise AssertionError(f"{name}: {e}") from None
