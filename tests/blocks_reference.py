"""The operators around the layers in 64 bits, written from their definitions, and how far the kernels' outputs may be from that.

u = 2^-24 is half a step of float.  A bound counts the roundings of the library's steps, each relative to the numbers that the step
works on; the last one, to the output's type, is half a step of that type.
"""
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def inside(lengths, N, L):
    at = torch.arange(L, device="cuda")
    n = torch.full((N,), L, device="cuda") if lengths is None else lengths.clamp(0, L)
    return (at < n[:, None])[:, None]


# ---- embedding ---------------------------------------------------------------------------------------------------------------
def embed(table, tokens, scale, lengths):
    N, L = tokens.shape
    V = table.shape[0]
    t = tokens.long()
    fine = (t >= 0) & (t < V) & inside(lengths, N, L)[:, 0]
    y = torch.where(fine[:, :, None], table.double()[t.clamp(0, V - 1)] * scale, 0.0)
    return y.transpose(1, 2)


def embed_grad(dy, tokens, V, scale, lengths):
    """(dtable, the sum of magnitudes behind each of its numbers)."""
    N, D, L = dy.shape
    t = tokens.long()
    fine = ((t >= 0) & (t < V) & inside(lengths, N, L)[:, 0]).view(-1)
    rows = dy.double().transpose(1, 2).reshape(-1, D)[fine].cpu()
    at = t.reshape(-1)[fine].cpu()
    sums = [torch.zeros(V, D, dtype=torch.float64).index_add_(0, at, r) * scale for r in (rows, rows.abs())]
    return [s.cuda() for s in sums]


# ---- group norm ---------------------------------------------------------------------------------------------------------------
def norm(x, dy, groups, weight, bias, act, eps, lengths):
    """{name: (value, bound before the rounding to its type)} of y, dx, dweight, dbias, and of stats (values alone)."""
    N, C, L = x.shape
    m = inside(lengths, N, L)
    x, dy = (torch.where(m, v.double(), 0.0).contiguous() for v in (x, dy))
    count = (m.sum(2).double() * (C // groups)).clamp(min=1).view(N, 1, 1)
    w = torch.ones(C, 1, device="cuda").double() if weight is None else weight.double()[:, None]
    b = torch.zeros(C, 1, device="cuda").double() if bias is None else bias.double()[:, None]

    def mean(v):
        """The mean over a group, on each of its values' places."""
        s = torch.where(m, v, 0.0).view(N, groups, -1).sum(2, keepdim=True) / count
        return s.expand(N, groups, C // groups).reshape(N, C, 1)

    mu = mean(x)
    off = torch.where(m, x - mu, 0.0)
    rstd = (mean(off * off) + eps) ** -0.5
    h = off * rstd
    p = h * w + b
    sig = 1 / (1 + torch.exp(-p))
    # h: a difference, rstd, a product and a sum; p: a product and sum more
    big = (h * w).abs() + b.abs()
    ep, eh = 5 * U * big, 4 * U * h.abs()
    if act == "silu":
        # the exponential is off by 2 u |p| for its argument and 2 u, 1 + exp by u, the reciprocal by 2 u, the product by u
        y, slope = p * sig, sig * (1 + p * (1 - sig))
        ey = 1.1 * ep + U * (6 + 2 * p.abs()) * y.abs()
        # |second derivative| <= 1/2; sig as above in both its places, and three roundings
        edp = dy.abs() * (0.5 * ep + U * (20 + 8 * p.abs()))
    elif act == "relu":
        y, slope = p.clamp(min=0), (p > 0).double()
        ey, edp = ep, torch.zeros_like(p)
    else:
        y, slope, ey, edp = p, torch.ones_like(p), ep, torch.zeros_like(p)
    dp = dy * slope
    g = dp * w
    s1, q1 = mean(g), mean(g * h)
    dx = rstd * (g - s1 - h * q1)
    # sums of eight in float (8 u of the magnitudes), then in 64 bits, and rounded to float
    es = mean(edp * w.abs() + 10 * U * g.abs())
    eq = mean(edp * (w * h).abs() + g.abs() * eh + 10 * U * (g * h).abs())
    edx = rstd * (edp * w.abs() + es + h.abs() * eq + q1.abs() * eh + 5 * U * (g.abs() + s1.abs() + (h * q1).abs()))
    total = lambda v: torch.where(m, v, 0.0).sum((0, 2))  # noqa: E731
    stats = torch.stack((mu, rstd), 3)[:, ::C // groups, 0]
    zero = lambda v: torch.where(m, v, 0.0)  # noqa: E731
    return {"y": (zero(y), zero(ey)), "dx": (zero(dx), zero(edx)), "dweight": (total(dp * h), total(edp * h.abs() + dp.abs() * eh + 10 * U * (dp * h).abs())),
            "dbias": (total(dp), total(edp + 10 * U * dp.abs())), "stats": stats}


# ---- dropout ------------------------------------------------------------------------------------------------------------------
def words(rows, L, key, call):
    """The generator's words [rows, L], by Python's whole numbers."""
    out, mask = [], 2 ** 32 - 1
    for row in range(rows):
        line = []
        for block in range(row * -(-L // 4), (row + 1) * -(-L // 4)):
            c, k = [block & mask, block >> 32, call & mask, call >> 32], [key & mask, key >> 32]
            for _ in range(7):
                a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
                c = [b >> 32 ^ c[1] ^ k[0], b & mask, a >> 32 ^ c[3] ^ k[1], a & mask]
                k = [k[0] + 0x9E3779B9 & mask, k[1] + 0xBB67AE85 & mask]
            line += c
        out.append(line[:L])
    return out


def dropout(x, kept, p, residual, lengths):
    """(y, bound before the rounding to its type)."""
    N, C, L = x.shape
    v = torch.where(kept, x.double() / (1 - p) if p < 1 else torch.zeros_like(x).double(), 0.0)
    y = v if residual is None else v + residual.double()
    m = inside(lengths, N, L)
    y, v = torch.where(m, y, 0.0), torch.where(m, v, 0.0)
    # 1 / (1 - p) and the product are rounded, then the sum
    return y, 2 * U * v.abs() + (0.0 if residual is None else U * y.abs())


def near(got, want, bound, name=""):
    """Every element of `got` within bound and its own last rounding of `want`."""
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs()
    # (the rounding is of a number that is itself off by the bound; 1e-37: floats below the smallest normal one are lost)
    most = bound + half_step(got.dtype) * (want.abs() + bound) + 1e-37
    bad = ~(off <= most)
    assert not bad.any(), (name, int(bad.sum()), float(off[bad].max()), float((off / most)[bad].max()), bad.nonzero()[:3].tolist())
