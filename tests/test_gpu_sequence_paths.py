"""Paths of the sequence operators that the sizes of test_gpu_sequence.py do not reach, and bounds of the scan that are counted, on
the GPU."""
import math

import pytest
import torch

from test_gpu_sequence import U32, _causal_ref, _check_scan, _close, _gen, _lengths, _normal, _scan_case, _u, seq  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


# ---- states: 17 to 32 are four a lane on eight lanes, 5 to 8 two a lane, whole and cut -----------------------------------------
@TYPES
@pytest.mark.parametrize("N,Dg,L,S,G", [(1, 1, 1, 17, 1), (2, 5, 2, 32, 1), (1, 9, 15, 24, 2), (2, 8, 64, 32, 2), (3, 7, 17, 20, 3), (2, 33, 65, 32, 1),
                                        (1, 70, 100, 25, 1), (1, 3, 40, 31, 4), (2, 5, 130, 48, 1), (1, 6, 90, 7, 1)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
def test_scan_of_other_states(seq, dtype, N, Dg, L, S, G, kind):  # noqa: F811
    gen = _gen(N + Dg + L + S + G)
    c = _scan_case(gen, dtype, N, Dg, L, S, G)
    lengths = _lengths(kind, N, L, gen)
    _check_scan(seq, c, lengths, _normal(gen, N, G * Dg, L).to(dtype), _normal(gen, N, G * Dg, S))


@TYPES
@pytest.mark.parametrize("N,Dg,L,S,G", [(1, 3, 1999, 8, 1), (2, 20, 1024, 6, 1), (1, 5, 1500, 17, 2), (1, 9, 1300, 32, 1), (2, 3, 777, 24, 2), (1, 2, 1500, 48, 1)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
def test_cut_scan_of_other_states(seq, dtype, N, Dg, L, S, G, kind):  # noqa: F811
    from paper_2104_08002_amd import binding

    assert binding.load().conv1d_scan_fwd_workspace_bytes(N, G * Dg, L, S, G) > 0
    gen = _gen(L + S)
    c = _scan_case(gen, dtype, N, Dg, L, S, G)
    lengths = None if kind == "all" else torch.tensor([L - 333, 0][:N], dtype=torch.int32, device="cuda")
    _check_scan(seq, c, lengths, _normal(gen, N, G * Dg, L).to(dtype), _normal(gen, N, G * Dg, S))


@TYPES
@pytest.mark.parametrize("S,G", [(17, 1), (24, 3), (32, 1), (48, 1), (7, 2)])
def test_steps_of_other_states(seq, dtype, S, G):  # noqa: F811
    gen = _gen(S + G)
    c = _scan_case(gen, dtype, 3, 13, 9, S, G)
    ref = _bounds(c, None)
    head = {k: v[..., :4] if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    state = seq.conv1d_scan_fwd(**head, want_final=True)[1]
    for t in range(4, 9):
        one = {k: v[..., t].contiguous() if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items() if k != "init"}
        y = seq.conv1d_scan_step(one.pop("x"), one.pop("dt"), one.pop("A"), one.pop("B"), one.pop("C"), state, **one)
        _held("y", y, *(v[:, :, t] for v in ref["y"]))
    _held("state", state, *ref["final"])


# ---- counted bounds of the scan ------------------------------------------------------------------------------------------------
def _held(name, got, ref, err):
    bound = _u(got.dtype) * (1 + 2.0 ** -7) * ref.abs() + 1.1 * U32 * err + 1e-37
    bad = ~((got.double() - ref).abs() <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(((got.double() - ref).abs() / bound).nan_to_num(nan=math.inf).max()))


def _bounds(c, lengths, dy=None, dfinal=None, per_step=0.0):
    """Every result of the scan in 64 bits with a bound on its error in units of 2^-24, to first order (1.1 for the rest).

    A quantity q has its value, the sum of the magnitudes of what it is made of (|.|), and the error E: a rounding is 1 of the value,
    the exponential and reciprocal instructions 2.
      v = dt + bias: 1 of |v|.  softplus: u = exp(-|v|) is off by 2 |v| + 2, r = u / (2 + u) by 4 more, the polynomial and its product
      by 6, and |v| comes in with a slope over the softplus of at most 1: E_e = (3 |v| + 12) e.
      decay a = exp2(e rate): rate = A log2(e) by 2, its product with e by 1, the exponential by 2: a ((E_e / e + 3) |e A| + 2).
      Where the sequence is cut, a state comes in over decays exp(A sum e) in their place: the sum's roundings (`per_step`: those of
      a segment, shared by its steps) are added to the 3.
      h = a h + (e x) B: E_h = a E_h' + E_a |h'| + |e x B| (E_e / e + 3) + |h|
      y = sum C h + skip x: sum |C| E_h + (S + 2) sum |C h| + 2 |skip x|; the gate z sigmoid(z) is off by 2 |z| + 7, its slope by
      2 |z| + 9 of sigmoid + |z| sigmoid.
      g = C dy + a g' and what is made of g and h: products of both have E_g |h| + |g| E_h, and roundings counted beside each."""
    N, D, L = c["x"].shape
    G, S = c["B"].shape[1:3]
    f = {k: v.double() for k, v in c.items() if isinstance(v, torch.Tensor)}
    inside = torch.ones(N, L, dtype=torch.bool, device="cuda")
    if lengths is not None:
        inside = torch.arange(L, device="cuda") < lengths[:, None]
    m = inside[:, None].double()
    raw = f["dt"] + f["dt_bias"][:, None]
    e = torch.logaddexp(raw, torch.zeros_like(raw)) * m
    re = 3 * raw.abs() + 12                                      # E_e / e
    x, skip = f["x"] * m, f["skip"][:, None]
    B, C = ((f[k] * inside[:, None, None]).repeat_interleave(D // G, 1) for k in "BC")
    A = f["A"]
    eA = e[..., None] * A[:, None]                               # [N, D, L, S]
    a = torch.exp(eA)
    ra = (re[..., None] + 3 + per_step) * eA.abs() + 2           # E_a / a
    h, hm = f["init"], f["init"].abs()
    eh = torch.zeros_like(h)
    hs, hms, ehs = [h], [hm], [eh]
    for t in range(L):
        b = (e * x)[:, :, t, None] * B[:, :, :, t]
        h = a[:, :, t] * h + b
        eh = a[:, :, t] * (eh + ra[:, :, t] * hm) + b.abs() * (re[:, :, t, None] + 3)
        hm = a[:, :, t] * hm + b.abs()
        eh = eh + hm
        hs.append(h), hms.append(hm), ehs.append(eh)
    hs, hms, ehs = (torch.stack(v, 2) for v in (hs, hms, ehs))   # [N, D, L + 1, S]
    Ct, Bt = C.transpose(2, 3), B.transpose(2, 3)                # [N, D, L, S]
    now, nowm, nowe = hs[:, :, 1:], hms[:, :, 1:], ehs[:, :, 1:]
    s, sm = (Ct * now).sum(3) + skip * x, (Ct.abs() * nowm).sum(3) + (skip * x).abs()
    es = (Ct.abs() * nowe).sum(3) + (S + 3) * sm
    z = f["z"] * m if "z" in f else None
    sig = torch.sigmoid(z) if z is not None else None
    zs, rz = (z * sig, 2 * z.abs() + 8) if z is not None else (torch.ones_like(s), torch.zeros_like(s))
    out = {"y": (s * zs * m, (es + sm * rz) * zs.abs() * m), "final": (hs[:, :, -1], ehs[:, :, -1])}
    if dy is None:
        return out
    do = dy.double() * m
    d, rd = do * zs, rz + 1                                      # dy of the sums, and its error
    g = f["init"] * 0 if dfinal is None else dfinal.double()
    gm, eg = g.abs(), torch.zeros_like(g)
    gs, gms, egs = [], [], []
    for t in reversed(range(L)):
        p = Ct[:, :, t] * d[:, :, t, None]
        g, gm, eg = g + p, gm + p.abs(), eg + p.abs() * (rd[:, :, t, None] + 1)
        eg = eg + gm
        gs.append(g), gms.append(gm), egs.append(eg)
        g, eg, gm = g * a[:, :, t], a[:, :, t] * (eg + (ra[:, :, t] + 1) * gm), gm * a[:, :, t]
    out["dinit"] = (g, eg + gm)
    gs, gms, egs = (torch.stack(v[::-1], 2) for v in (gs, gms, egs))
    group = lambda v: v.view(N, G, D // G, L, S).sum(2).transpose(2, 3)  # noqa: E731
    ex = (e * x)[..., None]
    adds = D // G + 4                                            # channels are added one behind the other at most
    out["dC"] = (group(now * d[..., None]), group(d.abs()[..., None] * (nowe + nowm * (rd[..., None] + adds))))
    out["dB"] = (group(gs * ex), group(ex.abs() * (egs + gms * (re[..., None] + 2 + adds))))
    gb, gbm, egb = (gs * Bt).sum(3), (gms * Bt.abs()).sum(3), (egs * Bt.abs()).sum(3)
    egb = egb + (S + 2) * gbm
    out["dx"] = ((gb * e + skip * d) * m, (egb * e + gbm * e * (re + 2) + (skip * d).abs() * (rd + 2)) * m)
    q, qm = gs * a * hs[:, :, :-1], gms * a * hms[:, :, :-1]
    eq = a * (egs * hms[:, :, :-1] + gms * ehs[:, :, :-1]) + (ra + 3) * qm
    de = gb * x + (q * A[:, None]).sum(3)
    dem = (gbm * x.abs()) + (qm * A[:, None].abs()).sum(3)
    ede = egb * x.abs() + (eq * A[:, None].abs()).sum(3) + (S + 6) * dem
    slope = torch.sigmoid(raw)
    rs = 3 * raw.abs() + 8
    out["ddt"] = (de * slope * m, (ede + dem * rs) * slope * m)
    terms = L + 8                                                # one behind the other within a segment; 64 bits beyond
    eL = e[..., None]
    out["dA"] = ((q * eL).sum((0, 2)), ((eq + qm * (re[..., None] + 2 + terms)) * eL).sum((0, 2)))
    out["dskip"] = ((d * x).sum((0, 2)), ((d * x).abs() * (rd + 2 + terms)).sum((0, 2)))
    out["ddt_bias"] = (out["ddt"][0].sum((0, 2)), (out["ddt"][1] + (terms + 2) * out["ddt"][0].abs()).sum((0, 2)))
    if z is not None:
        dz, sl = do * s, sig + z * sig * (1 - sig)
        slm = sig + z.abs() * sig
        out["dz"] = (dz * sl * m, (do.abs() * (es * sl.abs() + sm * slm * (2 * z.abs() + 11))) * m)
    return out


@TYPES
@pytest.mark.parametrize("N,Dg,L,S,G", [(2, 9, 70, 16, 2), (1, 17, 200, 8, 1), (2, 5, 90, 4, 1), (1, 9, 130, 32, 1), (2, 3, 65, 17, 2), (1, 5, 100, 64, 1), (1, 130, 40, 2, 1)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
def test_scan_within_its_roundings(seq, dtype, N, Dg, L, S, G, kind):  # noqa: F811
    gen = _gen(N + Dg + L + S + G + 1)
    c = _scan_case(gen, dtype, N, Dg, L, S, G)
    lengths = _lengths(kind, N, L, gen)
    _within(seq, c, lengths, _normal(gen, N, G * Dg, L).to(dtype), _normal(gen, N, G * Dg, S), 0.0)


@TYPES
@pytest.mark.parametrize("N,Dg,L,S,G", [(1, 3, 700, 16, 1), (2, 5, 333, 8, 1), (1, 4, 600, 3, 2), (1, 5, 700, 32, 1), (1, 2, 600, 64, 1)])
def test_cut_scan_within_its_roundings(seq, dtype, N, Dg, L, S, G):  # noqa: F811
    """Segments of one tile, 32 or 64 steps: a sum of them has 16 roundings of at most the sum, one more in its product with the rate,
    and joining has three a segment."""
    from paper_2104_08002_amd import binding

    assert binding.load().conv1d_scan_fwd_workspace_bytes(N, G * Dg, L, S, G) > 0
    gen = _gen(L + S + 2)
    c = _scan_case(gen, dtype, N, Dg, L, S, G)
    _within(seq, c, None, _normal(gen, N, G * Dg, L).to(dtype), _normal(gen, N, G * Dg, S), 17.0)


def _within(seq, c, lengths, dy, dfinal, per_step):  # noqa: F811
    ref = _bounds(c, lengths, dy, dfinal, per_step)
    y, final, saved = seq.conv1d_scan_fwd(**c, lengths=lengths, want_final=True, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c, lengths=lengths, dfinal=dfinal, want_init=True)
    _held("y", y, *ref["y"])
    _held("final", final, *ref["final"])
    for k, v in g._asdict().items():
        _held(k, v, *ref[k])


# ---- more segments than are joined at once -----------------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("N,D,L,S", [(1, 3, 40000, 16), (2, 2, 20000, 64), (1, 3, 36000, 24)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
def test_scan_joined_in_several_passes(seq, dtype, N, D, L, S, kind):  # noqa: F811
    """1250, 313 and 563 segments, of which 1024, 256 and 512 are joined at once; lengths that end in the first and the second pass.
    Steps of one sign and slow rates: what is joined first reaches the end."""
    gen = _gen(L)
    slow = 20.0 / L
    c = {"x": _normal(gen, N, D, L).to(dtype), "dt": (0.5 + torch.rand(N, D, L, generator=gen, device="cuda")).to(dtype),
         "A": -slow * (0.1 + torch.rand(D, S, generator=gen, device="cuda")), "B": _normal(gen, N, 1, S, L).to(dtype), "C": _normal(gen, N, 1, S, L).to(dtype),
         "init": _normal(gen, N, D, S) * L ** 0.5}
    lengths = None if kind == "all" else torch.tensor([L - 11, 1500][-N:], dtype=torch.int32, device="cuda")
    dy, dfinal = _normal(gen, N, D, L).to(dtype), _normal(gen, N, D, S) * L ** 0.5
    y, final, saved = seq.conv1d_scan_fwd(**c, lengths=lengths, want_final=True, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c, lengths=lengths, dfinal=dfinal, want_init=True)
    m = torch.ones(N, 1, L, device="cuda", dtype=torch.float64) if lengths is None else (torch.arange(L, device="cuda") < lengths[:, None])[:, None].double()
    f = {k: v.double() for k, v in c.items()}
    e, x, do = f["dt"] * m, f["x"] * m, dy.double() * m
    B, C = (f[k] * m[:, :, None] for k in "BC")                   # [N, 1, S, L]
    # in 64 bits as sums: h[t] = P[t] (h0 + sum b[s] / P[s]), P the decays up to t, which span exp(33)
    log = (e[:, :, None] * f["A"][:, :, None]).cumsum(3)          # [N, D, S, L]
    P = torch.exp(log)
    b = (e * x)[:, :, None] * B
    h = P * (f["init"][..., None] + (b / P).cumsum(3))
    later = (P * C * do[:, :, None]).flip(3).cumsum(3).flip(3)
    a = (later + (P[..., -1] * dfinal.double())[..., None]) / P   # the adjoint, the output's part in it
    q = a * (h - b)
    gb = (a * B).sum(2)
    want = {"y": (C * h).sum(2), "final": h[..., -1], "dx": gb * e, "ddt": (gb * x + (q * f["A"][:, :, None]).sum(2)) * m,
            "dA": (q * e[:, :, None]).sum((0, 3)), "dinit": a[..., 0] * P[..., 0]}
    # Roundings of a state: three a step within a tile of up to 64, three a segment behind it, and those of exponents of at most 33,
    # 20 each; sums of gradients and over states.  They do not know the signs of the terms, which cancel alike in the values: of the
    # root mean square
    held = 3 * 64 + 3 * 1250 + 33 * 20 + 400
    for k, got in {"y": y, "final": final, "dx": g.dx, "ddt": g.ddt, "dA": g.dA, "dinit": g.dinit}.items():
        ref, scale = want[k], want[k].square().mean().sqrt()
        bound = _u(got.dtype) * (1 + 2.0 ** -7) * ref.abs() + held * U32 * torch.maximum(ref.abs(), scale) + 1e-37
        bad = ~((got.double() - ref).abs() <= bound)
        assert not bad.any(), (k, int(bad.sum()), float(((got.double() - ref).abs() / bound).max()))


# ---- causal convolution: four steps a lane backwards, and eight with other taps -----------------------------------------------
@TYPES
@pytest.mark.parametrize("N,C,L,S", [(2, 1100, 2049, 2), (2, 1100, 2049, 4), (1, 2100, 2500, 3), (2, 1030, 2060, 8), (2, 1100, 4099, 2), (2, 1100, 4099, 3),
                                     (1, 1400, 8200, 8), (1, 4096, 600, 5)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
@pytest.mark.parametrize("silu", [True, False])
def test_causal_of_many_rows(seq, dtype, N, C, L, S, kind, silu):  # noqa: F811
    gen = _gen(N * 1000 + C * 100 + L + S)
    x = _normal(gen, N, 2 * C, L).to(dtype)[:, C:]
    w, bias = _normal(gen, C, S).to(dtype), _normal(gen, C)
    dy = _normal(gen, N, 2 * C, L).to(dtype)[:, :C]
    init, dfinal = (_normal(gen, N, C, S - 1).to(dtype) for _ in range(2))
    lengths = None if kind == "all" else torch.tensor([L - 3, 513][-N:], dtype=torch.int32, device="cuda")
    ref = _causal_ref(x, w, bias, silu, init, lengths, dy, dfinal)
    dx, dw, db, dinit = seq.conv1d_causal_bwd(dy, x, w, bias=bias, silu=silu, init=init, lengths=lengths, dfinal=dfinal, want_init=True)
    _close("dx", dx, *ref["dx"], 4 * S + 12)
    _close("dinit", dinit, *ref["dinit"], 4 * S + 12)
    _close("dw", dw, *ref["dw"], 2 * S + 84)   # (a lane adds 8 R <= 64 products, 6 more over the wave)
    _close("db", db, *ref["db"], 2 * S + 84)


def test_outputs_into_the_halves_of_a_projection(seq):  # noqa: F811
    """The gate lies in one half, what is written in the other; a position's rows likewise."""
    gen = _gen(31)
    N, D, L, S = 3, 6, 50, 16
    c = _scan_case(gen, torch.float32, N, D, L, S, 1)
    want, state, _ = seq.conv1d_scan_fwd(**c, want_final=True)
    xz = torch.cat((torch.full_like(c["x"], 7.0), c["z"]), 1)
    gate = c["z"].clone()
    got = seq.conv1d_scan_fwd(**{**c, "x": c["x"].contiguous(), "z": xz[:, D:]}, out=xz[:, :D])[0]
    assert torch.equal(got, want) and torch.equal(xz[:, :D], want) and torch.equal(xz[:, D:], gate)
    w, one = _normal(gen, D, 4), _normal(gen, N, 2 * D)
    before, states = one.clone(), [_normal(gen, N, D, 3)] * 2
    want = seq.conv1d_causal_step(before[:, D:], w, states[0].clone(), silu=True)
    seq.conv1d_causal_step(one[:, D:], w, states[1].clone(), silu=True, out=one[:, :D])
    assert torch.equal(one[:, :D], want) and torch.equal(one[:, D:], before[:, D:])


def test_forward_mode_and_transforms_are_refused(seq):  # noqa: F811
    """Not answered with a wrong tangent, nor with none."""
    from torch.autograd import forward_ad

    from paper_2104_08002_amd import autograd

    gen = _gen(32)
    c = _scan_case(gen, torch.float32, 2, 3, 9, 4, 1)
    w, x = _normal(gen, 3, 4), c["x"].contiguous()
    scan = lambda v: autograd.conv1d_scan(v, c["dt"], c["A"], c["B"], c["C"])  # noqa: E731
    for call in (lambda v: autograd.conv1d_causal(v, w), scan):
        with pytest.raises(RuntimeError), forward_ad.dual_level():
            call(forward_ad.make_dual(x, torch.ones_like(x)))
        with pytest.raises(RuntimeError):
            torch.func.grad(lambda v: call(v).sum())(x)
        with pytest.raises(RuntimeError):
            torch.func.vmap(call)(torch.stack((x, x)))


def test_more_parameters_than_a_launch_sums(seq):  # noqa: F811
    """6 million channels: 36 million sums over samples, 16 a workgroup, in more than one launch; against 64 bits."""
    gen = _gen(33)
    N, D = 2, 6000001
    x, dt, dy, A = (0.5 + torch.rand(s, generator=gen, device="cuda") for s in ((N, D, 1), (N, D, 1), (N, D, 1), (D, 1)))
    skip, h0 = _normal(gen, D), _normal(gen, N, D, 1)
    B, C = (_normal(gen, N, 1, 1, 1) for _ in range(2))
    y, _, saved = seq.conv1d_scan_fwd(x, dt, -A, B, C, skip=skip, init=h0, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, x, dt, -A, B, C, skip=skip, init=h0)
    left = torch.exp(-dt.double() * A.double()) * h0.double()
    h = left + dt.double() * x.double() * B[:, 0].double()
    want = C[:, 0].double() * h + skip.double()[:, None] * x.double()
    mag = C[:, 0].abs() * (left.abs() + (dt * x * B[:, 0]).abs()) + (skip[:, None] * x).abs()
    assert ((y.double() - want).abs() <= 16 * U32 * mag).all()           # a decay by 2 + 3 |e A| <= 9, products and sums by 7
    dA = (dt.double() * C[:, 0].double() * dy.double() * left).sum(0)
    mag = (dt.double() * C[:, 0].double() * dy.double() * left).abs().sum(0)
    assert ((g.dA.double() - dA).abs() <= 20 * U32 * mag + 1e-37).all()  # the decay, 6 products, one rounding behind 64 bits
    dskip = (dy.double() * x.double()).sum((0, 2))
    assert ((g.dskip.double() - dskip).abs() <= 4 * U32 * dskip.abs()).all()


@TYPES
def test_gradients_that_are_not_wanted(seq, dtype):  # noqa: F811
    """Null pointers in their places: the others are the same."""
    from paper_2104_08002_amd import binding

    lib, gen = binding.load(), _gen(34)
    stream = torch.cuda.current_stream().cuda_stream
    for N, C, L, S in ((2, 5, 700, 4), (2, 1100, 2049, 3)):
        x, dy, w, bias = _normal(gen, N, C, L).to(dtype), _normal(gen, N, C, L).to(dtype), _normal(gen, C, S).to(dtype), _normal(gen, C)
        want = seq.conv1d_causal_bwd(dy, x, w, bias=bias, silu=True)
        p = seq._causal(x, w, bias, True, None, None)[0]
        dx, dw = torch.empty_like(x), torch.empty(C, S, device="cuda")
        n = lib.conv1d_causal_bwd_workspace_bytes(N, C, L, S)
        room = torch.empty(n, dtype=torch.uint8, device="cuda")
        assert lib.conv1d_causal_bwd(p, dy.data_ptr(), C * L, L, None, dx.data_ptr(), None, None, None, None, 0, stream) == 0
        assert torch.equal(dx, want[0])
        dx.zero_()
        assert lib.conv1d_causal_bwd(p, dy.data_ptr(), C * L, L, None, dx.data_ptr(), dw.data_ptr(), None, None, room.data_ptr(), n, stream) == 0
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    for N, Dg, L, S, G in ((2, 9, 130, 16, 2), (1, 3, 900, 5, 1)):
        c = _scan_case(gen, dtype, N, Dg, L, S, G)
        D, dy = G * Dg, _normal(gen, N, G * Dg, L).to(dtype)
        saved = seq.conv1d_scan_fwd(**c, save=True)[2]
        want = seq.conv1d_scan_bwd(dy, saved, **c)
        p = seq._scan(c["x"], c["dt"], c["A"], c["B"], c["C"], c["skip"], c["z"], c["dt_bias"], True, c["init"], None)[0]
        n = lib.conv1d_scan_bwd_workspace_bytes(N, D, L, S, G)
        room = torch.empty(n, dtype=torch.uint8, device="cuda")
        dx, ddt, dz = (torch.empty(N, D, L, dtype=dtype, device="cuda") for _ in range(3))
        dB, dC = (torch.empty(N, G, S, L, dtype=dtype, device="cuda") for _ in range(2))
        dA = torch.empty(D, S, device="cuda")
        assert lib.conv1d_scan_bwd(p, dy.data_ptr(), D * L, L, None, saved.data_ptr(), dx.data_ptr(), ddt.data_ptr(), dA.data_ptr(), dB.data_ptr(), dC.data_ptr(),
                                   None, dz.data_ptr(), None, None, room.data_ptr(), n, stream) == 0
        for a, b in ((dx, want.dx), (ddt, want.ddt), (dz, want.dz), (dB, want.dB), (dC, want.dC), (dA, want.dA)):
            assert torch.equal(a, b)
