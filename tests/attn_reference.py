"""Attention over visible pairs in 64 bits, its gradients, and bounds on what
float arithmetic with bf16 operands may be off (test aid)."""
import torch

HALF = 2.0 ** -8      # half a bf16 step
U = 2.0 ** -24        # half a float step


def visible(p, j, window, sinks):
    """[queries, keys]: which keys at places j the queries at places p see."""
    p, j = p[:, None], j[None]
    see = j <= p
    return see & ((p - j < window) | (j < sinks)) if window else see


class Attention:
    """One head: q [n, D], k, v [m, D], see [n, m], in float64.

    `o`, `lse`, and their bounds: a score is a float sum of D exact products (each
    addition is off by at most U of the sum of magnitudes, and so are scale and
    exponent), so P, relative, by 2 U (D + 8) of the largest such sum, and by the
    exponential's own 2^-22; sums of n terms of P by n U; its rounding for the
    product by HALF; the output's by HALF."""

    def __init__(self, q, k, v, see, scale):
        self.q, self.k, self.v, self.see, self.scale = q, k, v, see, scale
        n = k.shape[0]
        x = (q @ k.t() * scale).masked_fill(~see, -torch.inf)
        self.any = see.any(1)
        m = x.amax(1, keepdim=True) if n else x.new_full((q.shape[0], 1), -torch.inf)
        m = torch.where(self.any[:, None], m, torch.zeros_like(m))
        e = torch.exp(x - m).masked_fill(~see, 0)
        total = e.sum(1, keepdim=True)
        self.p = torch.where(self.any[:, None], e / total, torch.zeros_like(e))
        self.o = self.p @ v
        self.lse = torch.where(self.any, (m + total.log())[:, 0], torch.full_like(m[:, 0], -torch.inf))
        mag = (q.abs() @ k.abs().t() * scale).masked_fill(~see, 0)
        self.big = mag.amax(1, keepdim=True) if n else mag.sum(1, keepdim=True)
        self.ep = 2 * U * (q.shape[1] + 8) * (1 + self.big) + 2.0 ** -21 + 2 * n * U
        self.o_bound = HALF * self.o.abs() + (HALF + 2 * self.ep) * (self.p @ v.abs()) + 1e-30
        self.lse_bound = self.ep[:, 0] + 2.0 ** -22 * self.lse.abs().nan_to_num(posinf=0)

    def gradients(self, go, D):
        """(grad_q, grad_k, grad_v) and their bounds.  P is off by ep, dP by 2 U D
        of its sum of magnitudes, delta by HALF of that of grad_out . o (o is
        rounded); P and dS are rounded for the products, the sums off by their
        length times U, the gradients rounded."""
        n, m = self.see.shape
        dp = go @ self.v.t()
        delta = (go * self.o).sum(1, keepdim=True)
        ds = self.p * (dp - delta)
        off = self.p * (2 * U * D * (go.abs() @ self.v.abs().t()) + (HALF + 4 * self.ep) * (go.abs() * (self.o.abs() + self.o_bound)).sum(1, keepdim=True))
        off = off + (HALF + 2 * self.ep) * ds.abs()
        gq, gk, gv = ds @ self.k * self.scale, ds.t() @ self.q * self.scale, self.p.t() @ go
        bq = HALF * gq.abs() + (off + U * m * ds.abs()) @ self.k.abs() * self.scale
        bk = (off + U * n * ds.abs()).t() @ self.q.abs() * self.scale
        bv = ((HALF + 2 * self.ep + U * n) * self.p).t() @ go.abs()
        return (gq, gk, gv), (bq + 1e-30, bk, bv)


def packed(q, k, v, q_start, k_start, window, sinks, scale, go=None, offset=True):
    """The whole call on the GPU in float64: dict of values and of bounds, rows of
    no sequence zero.  q [T, Hq, D], k and v [S, Hk, D]; starts as lists."""
    q, k, v = q.double(), k.double(), v.double()
    (T, Hq, D), Hk = q.shape, k.shape[1]
    out = {"o": torch.zeros_like(q), "lse": torch.zeros(Hq, T, dtype=torch.float64, device=q.device)}
    grads = {"gq": torch.zeros_like(q), "gk": torch.zeros_like(k), "gv": torch.zeros_like(v)}
    bound = {n: torch.zeros_like(t) for n, t in list(out.items()) + list(grads.items())}
    for a, b, c, d in zip(q_start, q_start[1:], k_start, k_start[1:]):
        p = torch.arange(b - a, device=q.device) + (d - c) - (b - a)
        see = visible(p, torch.arange(d - c, device=q.device), window, sinks)
        for h in range(Hq):
            g = h * Hk // Hq
            x = Attention(q[a:b, h], k[c:d, g], v[c:d, g], see, scale)
            out["o"][a:b, h], out["lse"][h, a:b] = x.o, x.lse
            bound["o"][a:b, h], bound["lse"][h, a:b] = x.o_bound, x.lse_bound
            if go is not None:
                val, bnd = x.gradients(go[a:b, h].double(), D)
                for n, i, y, z in (("gq", h, val[0], bnd[0]), ("gk", g, val[1], bnd[1]), ("gv", g, val[2], bnd[2])):
                    rows = slice(a, b) if n == "gq" else slice(c, d)
                    grads[n][rows, i] += y
                    bound[n][rows, i] += z
    if go is not None:
        for n in ("gk", "gv"):
            bound[n] += HALF * grads[n].abs() + 1e-30
        out.update(grads)
    return out, bound


def off(got, want, bound):
    """How many bounds the worst element is off; NaN and infinities have to agree."""
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), "NaN in other places"
    fine = want.isfinite()
    same = got[~fine] == want[~fine]
    assert (same | want[~fine].isnan()).all(), "infinities in other places"
    assert got[fine].isfinite().all()
    return ((got - want).abs() / bound)[fine].max().item() if fine.any() else 0.0
