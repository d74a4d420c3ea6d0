"""The operators around the KAN blocks of a language model in 64 bits, with elementwise bounds of what fp32 arithmetic and
one rounding to the result's type may do (not collected by pytest)."""
import torch

U = 2.0 ** -24                                     # half a step of fp32
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}


def rows_of(ids, V):
    """Row of every id (0 where it names none), and whether it names one."""
    t = ids.long() & 0xFFFF if ids.dtype == torch.int16 else ids.long() & 0xFFFFFFFF if ids.dtype == torch.int32 else ids
    ok = (t >= 0) & (t < V)
    return torch.where(ok, t, torch.zeros_like(t)), ok


def check(got, ref, bound):
    """|got - ref| <= bound (of the arithmetic in fp32) + the rounding to got's type."""
    assert got.shape == ref.shape
    g = got.double()
    assert bool(torch.isfinite(g).all())
    limit = bound * (1 + HALF[got.dtype]) + HALF[got.dtype] * ref.abs() + TINY[got.dtype]
    bad = (g - ref).abs() > limit
    if bool(bad.any()):
        k = int(((g - ref).abs() / limit).argmax())
        raise AssertionError((int(bad.sum()), k, float(g.reshape(-1)[k]), float(ref.reshape(-1)[k]), float(limit.reshape(-1)[k])))


def lookup(table, ids, scale):
    t, ok = rows_of(ids, table.shape[0])
    return torch.where(ok[..., None], table.double()[t] * scale, 0.0)


def segment_sums(d, t, V):
    """Sums of the rows of d by t, without atomics (a million additions to one row in 64 bits take minutes): differences
    of running sums, off by 2^-53 of the sum of all magnitudes a step."""
    order = torch.argsort(t, stable=True)
    run = torch.cat([torch.zeros_like(d[:1]), d[order].cumsum(0)])
    ends = torch.searchsorted(t[order].contiguous(), torch.arange(V, device=d.device), right=True)
    return run[ends] - run[torch.cat([ends.new_zeros(1), ends[:-1]])]


def lookup_grad(dy, ids, V, scale):
    """The gradient, and the bound of fp32 sums of the terms in any order."""
    t, ok = rows_of(ids.reshape(-1), V)
    d = torch.where(ok[:, None], dy.reshape(len(t), -1).double(), 0.0)
    count = segment_sums(torch.ones_like(d[:, :1]), t, V)
    size = segment_sums(d.abs(), t, V).clamp(min=0.0)
    exact = len(t) * 2.0 ** -53 * d.abs().sum(0)
    return segment_sums(d, t, V) * scale, abs(scale) * ((count + 4) * U * size + 2 * exact)


def rms(a, eps):
    return (a.pow(2).mean(-1, keepdim=True) + eps).sqrt()


def norms(x, v, gate, wa, wb, scale, eps):
    """(y, its bound, u, its bound): sums of positive terms over a row in fp32 (under 40 roundings one behind the other,
    half of that in the root), the sigmoid's argument times log2(e) rounded: 128 half steps of each term."""
    c = 128 * U
    y, ey = x.double(), torch.zeros_like(x, dtype=torch.float64)
    if v is not None:
        s = torch.sigmoid(gate.double()) if gate is not None else 1.0
        b = scale * s * (1.0 if wa is None else wa.double()) * v.double() / rms(v.double(), eps)
        y, ey = y + b, c * b.abs() + U * (y + b).abs()
    r = rms(y, eps)
    w = torch.ones_like(y[0]) if wb is None else wb.double()
    # a relative change of the rms is at most that of y in the rms norm
    return y, ey, w * y / r, (w.abs() / r) * (ey + (c + rms(ey, 0.0) / r) * y.abs())


def norms_grad(y, dy, du, v, gate, wa, wb, scale, eps):
    """[(gradient, bound)] of dx, dv, dgate, dw_before, dw_after; None where there is none."""
    c, N, out = 128 * U, y.shape[0], {}
    sums = (N / 512 + 200) * U + c                 # rows of a group one by one, then the groups
    yd = y.double()
    one = torch.ones(y.shape[-1], dtype=torch.float64, device=y.device)
    g = torch.zeros_like(yd) if dy is None else dy.double()
    G = g.abs()
    if du is not None:
        w, r = one if wb is None else wb.double(), 1.0 / rms(yd, eps)
        hat, t = yd * r, du.double() * w
        g = g + r * (t - hat * (t * hat).mean(-1, keepdim=True))
        G = G + r * (t.abs() + hat.abs() * (t * hat).abs().mean(-1, keepdim=True))
        if wb is not None:
            out["dw_before"] = ((du.double() * hat).sum(0), sums * (du.double() * hat).abs().sum(0))
    out["dx"] = (g, c * G)
    if v is not None:
        vd, w = v.double(), one if wa is None else wa.double()
        r = 1.0 / rms(vd, eps)
        m = vd * r
        s = torch.sigmoid(gate.double()) if gate is not None else torch.ones_like(vd)
        q, Q = scale * s * g * w, abs(scale) * s * G * w.abs()
        out["dv"] = (r * (q - m * (q * m).mean(-1, keepdim=True)), 3 * c * r * (Q + m.abs() * (Q * m.abs()).mean(-1, keepdim=True)))
        if wa is not None:
            out["dw_after"] = ((scale * s * g * m).sum(0), (sums + 2 * c) * (abs(scale) * s * G * m.abs()).sum(0))
        if gate is not None:
            out["dgate"] = (scale * g * w * m * s * (1 - s), 3 * c * abs(scale) * G * (w * m).abs() * s)
    return [out.get(k) for k in ("dx", "dv", "dgate", "dw_before", "dw_after")]


class Loss:
    """Softmax cross entropy and its gradients in 64 bits, with bounds.

    A logit: products of 16-bit numbers are exact, a matrix instruction adds at least four of them a rounding: D / 4 + 16
    roundings of the sum of magnitudes; fp32 rows: six products of parts and what is left out of them, three steps of 2^-24."""

    def __init__(self, h, table, targets, scale):
        self.h, self.w, self.scale, self.type = h.reshape(-1, h.shape[-1]).double(), table.double(), scale, h.dtype
        V, D = table.shape
        self.t, self.ok = rows_of(targets.reshape(-1), V)
        self.h = torch.where(self.ok[:, None], self.h, 0.0) if not bool(torch.isfinite(self.h).all()) else self.h
        z = scale * (self.h @ self.w.t())
        size = abs(scale) * (self.h.abs() @ self.w.abs().t())
        steps = D / 4 + 16 if h.dtype != torch.float32 else 6 * D / 4 + 20
        self.ez = (steps * U * size).amax(1) + U * z.abs().amax(1)
        self.lse = torch.logsumexp(z, 1)
        self.elog = self.ez + (self.lse.abs() + 64) * U            # logarithm, exponentials and V sums in a tree
        zt = z.gather(1, self.t[:, None])[:, 0]
        self.loss = torch.where(self.ok, self.lse - zt, 0.0)
        self.eloss = torch.where(self.ok, self.elog + self.ez + U * zt.abs(), 0.0)
        self.p = torch.exp(z - self.lse[:, None])
        self.far = (z - self.lse[:, None]).abs()

    def grads(self, dloss):
        """(dh, bound, rms bound), (dtable, bound, rms bound).  An entry of dS: the exponential of an argument that is off by
        the logit's and lse's bounds and by 2 half steps of itself; then the rounding to the operands' type (fp32: three bf16
        parts, 2^-24).  The rounding errors are independent: their sum's deviation is at most that of its terms."""
        weight = torch.where(self.ok, dloss.reshape(-1).double(), 0.0)[:, None] * self.scale
        d = self.p.clone()
        d[torch.arange(len(self.t), device=d.device), self.t] -= 1.0
        d = torch.where(self.ok[:, None], d, 0.0) * weight
        off = torch.expm1((self.ez + self.elog)[:, None] + 3 * U * self.far)
        half = HALF[self.type] if self.type != torch.float32 else 2 * U
        # (below 2^-126 the exponential, and the matrix instructions' operands and products, are 0)
        e = weight.abs() * self.p * off + 4 * U * d.abs() + 2.0 ** -126
        if self.type == torch.float16:
            e = e + 2.0 ** -25 / 16384 * weight.abs().max()
        out = []
        for a, other in ((lambda m: m, self.w), (lambda m: m.t(), self.h)):
            ref = a(d) @ other
            n = other.shape[0]
            size = a(d.abs()) @ other.abs()
            base = a(e) @ other.abs() + n * 2.0 ** -126 + (n / 4 * (6 if self.type == torch.float32 else 1) + 64) * U * size
            spread = half * torch.sqrt(a(d * d) @ (other * other))
            out.append((ref, base + half * size, float((base.square().mean()).sqrt() + spread.square().mean().sqrt())))
        return out


def check_rms(got, ref, bound):
    err = (got.double() - ref).square().mean().sqrt()
    assert float(err) <= bound + HALF[got.dtype] * float(ref.square().mean().sqrt()) + TINY[got.dtype], (float(err), bound)
