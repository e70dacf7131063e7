"""The sequence operators against plain implementations in 64 bits, on the GPU.

Bounds.  A result rounded to type t is off by u(t) = eps(t) / 2 of its value (2^-8 bfloat16, 2^-24 float); a sum of n products
in float by n + 1 roundings, each of at most 2^-24 of the sum of the magnitudes, so |got - ref| <= u |ref| + c 2^-24 mag with
`mag` the same formula over absolute values, and c counted for each output below.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def _u(t):
    return torch.finfo(t).eps / 2


@pytest.fixture(scope="module")
def seq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2104_08002_amd import binding, sequence

    binding.load()
    return sequence


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _close(name, got, ref, mag, c):
    """Within one rounding to got's type and c roundings in float of sums of magnitude mag; NaN nowhere."""
    bound = _u(got.dtype) * (1 + 2.0 ** -7) * ref.abs() + c * U32 * mag + 1e-37
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (name, int(bad.sum()), float((err / bound).nan_to_num(nan=math.inf).max()))


def _lengths(kind, N, L, gen):
    if kind == "all":
        return None
    v = torch.randint(0, L + 1, (N,), generator=gen, device="cuda").to(torch.int32)
    v[0] = 0
    if N > 1:
        v[1] = L
    return v


# ---- depthwise causal convolution --------------------------------------------------------------------------------------
def _causal_ref(x, w, bias, silu, init, lengths, dy=None, dfinal=None):
    """Position by position of the definition, in 64 bits, with the same over magnitudes."""
    x, w = x.double(), w.double()
    N, C, L = x.shape
    S = w.shape[1]
    init = x.new_zeros(N, C, S - 1) if init is None else init.double()
    inside = torch.ones(N, 1, L, dtype=torch.bool, device=x.device)
    if lengths is not None:
        inside = (torch.arange(L, device=x.device) < lengths[:, None])[:, None]
    x = torch.where(inside, x, 0.0)
    xe = torch.cat((init, x), 2).requires_grad_(True)
    wl = w.clone().requires_grad_(True)
    b = (x.new_zeros(C) if bias is None else bias.double()).requires_grad_(True)
    p = b[:, None] + sum(wl[:, s, None] * xe[:, :, s:s + L] for s in range(S))
    y = torch.where(inside, p * torch.sigmoid(p) if silu else p, 0.0)
    at = inside.sum(2).expand(N, C)[:, :, None] + torch.arange(S - 1, device=x.device)
    final = xe.gather(2, at)
    pmag = b.detach().abs()[:, None] + sum(w[:, s, None].abs() * xe.detach()[:, :, s:s + L].abs() for s in range(S))
    out = {"y": (y.detach(), pmag * inside), "final": final.detach()}
    if dy is not None:
        loss = (y * dy.double()).sum() + (0 if dfinal is None else (final * dfinal.double()).sum())
        gx, gw, gb = torch.autograd.grad(loss, (xe, wl, b), allow_unused=True)
        # dp = dy act'(p): its error is that of p times |act''| <= 1/2, and of the slope itself
        dmag = torch.where(inside, dy.double().abs(), 0.0) * (1.2 + pmag if silu else 1.0)
        after = torch.cat((dmag, dmag.new_zeros(N, C, S - 1)), 2)
        xmag = torch.cat((dmag.new_zeros(N, C, S - 1), dmag), 2) * 0
        for s in range(S):
            xmag[:, :, s:s + L] += w[:, s, None].abs() * after[:, :, :L]
        if dfinal is not None:
            xmag.scatter_add_(2, at, dfinal.double().abs())
        xa = xe.detach().abs()
        out.update(dx=(torch.where(inside, gx[:, :, S - 1:], 0.0), xmag[:, :, S - 1:]), dinit=(gx[:, :, :S - 1], xmag[:, :, :S - 1]),
                   dw=(gw, torch.stack([(dmag * xa[:, :, s:s + L]).sum((0, 2)) for s in range(S)], 1)), db=(gb, dmag.sum((0, 2))))
    return out


# c: S + 1 products for p, three roundings and two units of the exponential and reciprocal for its sigmoid and slope, S products
# for dx; a lane adds 32 products, 6 more over the wave, the rest in 64 bits
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,C,L,S", [(1, 1, 1, 1), (2, 3, 1, 4), (3, 5, 2, 8), (2, 4, 7, 3), (2, 3, 8, 4), (1, 3, 9, 2), (4, 6, 100, 4), (2, 3, 511, 5),
                                     (2, 3, 513, 8), (1, 2, 2049, 4), (2, 1100, 4099, 4), (1, 7, 20011, 6)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
@pytest.mark.parametrize("silu", [True, False])
def test_causal(seq, dtype, N, C, L, S, kind, silu):
    gen = _gen(N * 1000 + C * 100 + L + S)
    x = _normal(gen, N, 2 * C, L).to(dtype)[:, C:]
    w, bias = _normal(gen, C, S).to(dtype), _normal(gen, C)
    dy = _normal(gen, N, 2 * C, L).to(dtype)[:, :C]
    init, dfinal = (_normal(gen, N, C, S - 1).to(dtype) for _ in range(2))
    lengths = _lengths(kind, N, L, gen)
    for b, i, f in ((bias, init, dfinal), (None, None, None)):
        ref = _causal_ref(x, w, b, silu, i, lengths, dy, f)
        y, final = seq.conv1d_causal_fwd(x, w, bias=b, silu=silu, init=i, lengths=lengths, want_final=True)
        _close("y", y, *ref["y"], 2 * S + 8)
        assert torch.equal(final, ref["final"].to(dtype))
        dx, dw, db, dinit = seq.conv1d_causal_bwd(dy, x, w, bias=b, silu=silu, init=i, lengths=lengths, dfinal=f, want_init=True)
        assert (db is None) == (b is None)
        _close("dx", dx, *ref["dx"], 4 * S + 12)
        if S > 1:
            _close("dinit", dinit, *ref["dinit"], 4 * S + 12)
        _close("dw", dw, *ref["dw"], 2 * S + 52)
        if b is not None:
            _close("db", db, *ref["db"], 2 * S + 52)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("S", [1, 2, 4, 8])
def test_causal_steps_continue_a_prompt(seq, dtype, S):
    gen = _gen(S)
    N, C, L = 3, 37, 20
    x, w, bias = _normal(gen, N, C, L).to(dtype), _normal(gen, C, S).to(dtype), _normal(gen, C)
    whole, last = seq.conv1d_causal_fwd(x, w, bias=bias, silu=True, want_final=True)
    y, state = seq.conv1d_causal_fwd(x[:, :, :13], w, bias=bias, silu=True, want_final=True)
    assert torch.equal(y, whole[:, :, :13])
    for t in range(13, L):
        xt = torch.stack((x[:, :, t], x[:, :, t]), 1).view(N, 2 * C)[:, :C]  # rows that are 2 C apart
        y = seq.conv1d_causal_step(xt, w, state, bias=bias, silu=True)
        assert torch.equal(y, whole[:, :, t]), t
    assert torch.equal(state, last)


# ---- selective scan ----------------------------------------------------------------------------------------------------
def _scan_case(gen, dtype, N, Dg, L, S, G, gate=True):
    D = G * Dg
    xz, bc = _normal(gen, N, 2 * D, L).to(dtype), _normal(gen, N, 2 * G, S, L).to(dtype)
    return {"x": xz[:, :D], "dt": (0.5 * _normal(gen, N, D, L) - 2).to(dtype), "A": -torch.exp(0.5 * _normal(gen, D, S)) * 2, "B": bc[:, :G], "C": bc[:, G:],
            "skip": _normal(gen, D), "z": xz[:, D:] if gate else None, "dt_bias": _normal(gen, D), "softplus": True, "init": _normal(gen, N, D, S)}


def _scan_ref(c, lengths, dy=None, dfinal=None):
    """The recurrence one position after the other in 64 bits, gradients by autograd through it."""
    N, D, L = c["x"].shape
    G, S = c["B"].shape[1:3]
    leaf = {k: v.detach().double().clone().requires_grad_(True) for k, v in c.items() if isinstance(v, torch.Tensor)}
    inside = torch.ones(N, L, dtype=torch.bool, device="cuda")
    if lengths is not None:
        inside = torch.arange(L, device="cuda") < lengths[:, None]
    raw = leaf["dt"] + (leaf["dt_bias"][:, None] if "dt_bias" in leaf else 0)
    e = torch.where(inside[:, None], torch.logaddexp(raw, torch.zeros_like(raw)) if c["softplus"] else raw, 0.0)
    x = torch.where(inside[:, None], leaf["x"], 0.0)
    B, C = (torch.where(inside[:, None, None], leaf[k], 0.0).repeat_interleave(D // G, 1) for k in "BC")
    h = leaf["init"] if "init" in leaf else x.new_zeros(N, D, S)
    ys = []
    for t in range(L):
        h = torch.exp(e[:, :, t, None] * leaf["A"]) * h + (e[:, :, t] * x[:, :, t])[:, :, None] * B[:, :, :, t]
        ys.append((C[:, :, :, t] * h).sum(2))
    y = torch.stack(ys, 2) + (leaf["skip"][:, None] * x if "skip" in leaf else 0)
    out = torch.where(inside[:, None], y * leaf["z"] * torch.sigmoid(leaf["z"]) if "z" in leaf else y, 0.0)
    ref = {"y": out.detach(), "final": h.detach()}
    if dy is not None:
        loss = (out * torch.where(inside[:, None], dy.double(), 0.0)).sum() + (0 if dfinal is None else (h * dfinal.double()).sum())
        names = list(leaf)
        for k, g in zip(names, torch.autograd.grad(loss, [leaf[k] for k in names])):
            ref["d" + k] = g
    return ref


def _near(name, got, ref, c, dims):
    """A recurrence mixes all it sums, so errors are held to the root mean square of the values that share its sums (`dims`), which
    bounds them from below: one rounding to the type, and c roundings in float."""
    scale = ref.square().mean(dims, keepdim=True).sqrt()
    bound = _u(got.dtype) * (1 + 2.0 ** -7) * ref.abs() + c * U32 * torch.maximum(ref.abs(), scale) + 1e-37
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (name, int(bad.sum()), float((err / bound).nan_to_num(nan=math.inf).max()))


# Roundings: a decay exp(e A) carries those of e (some 8 of softplus), of e A and of the exponential, about 12, and an ordinary
# state has forgotten all but the last 1 / (e |A|) of them; sums over up to 64 states and the gate add their own.  Terms of both
# signs cancel to within a tenth or so of the root mean square of their magnitudes: 2000 roundings of what is left.
SCAN_C = 2000.0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,Dg,L,S,G", [(1, 1, 1, 1, 1), (2, 3, 1, 16, 2), (2, 5, 2, 4, 1), (1, 17, 15, 16, 1), (2, 16, 16, 8, 2), (3, 7, 17, 5, 3),
                                        (2, 65, 33, 16, 1), (1, 70, 64, 64, 1), (2, 9, 65, 33, 1), (1, 130, 100, 3, 1), (1, 300, 40, 4, 2), (2, 6, 300, 16, 1), (1, 5, 700, 2, 1)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
def test_scan(seq, dtype, N, Dg, L, S, G, kind):
    gen = _gen(N + Dg + L + S + G)
    c = _scan_case(gen, dtype, N, Dg, L, S, G)
    lengths = _lengths(kind, N, L, gen)
    dy, dfinal = _normal(gen, N, G * Dg, L).to(dtype), _normal(gen, N, G * Dg, S)
    _check_scan(seq, c, lengths, dy, dfinal)


def _check_scan(seq, c, lengths, dy, dfinal):
    ref = _scan_ref(c, lengths, dy, dfinal)
    y, final, saved = seq.conv1d_scan_fwd(**c, lengths=lengths, want_final=True, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c, lengths=lengths, dfinal=dfinal, want_init=c["init"] is not None)
    _near("y", y, ref["y"], SCAN_C, (0, 1, 2))
    _near("final", final, ref["final"], SCAN_C, (0, 1, 2))
    for k, v in g._asdict().items():
        assert (v is None) == (k not in ref), k
        if v is not None:
            _near(k, v, ref[k], SCAN_C, tuple(range(v.dim())))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("without", ["z", "skip", "dt_bias", "init", "softplus", "all"])
def test_scan_without_its_options(seq, dtype, without):
    gen = _gen(11)
    c = _scan_case(gen, dtype, 2, 9, 83, 16, 2)
    for k in ("z", "skip", "dt_bias", "init") if without == "all" else (without,):
        if k != "softplus":
            c[k] = None
    if without in ("softplus", "all"):
        c.update(softplus=False, dt=(0.1 * torch.rand(2, 18, 83, generator=gen, device="cuda")).to(dtype), dt_bias=None)
    dy = _normal(gen, 2, 18, 83).to(dtype)
    _check_scan(seq, c, None, dy, None)


# few rows: the sequence is cut, forwards and backwards, at lengths that end within a segment
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,Dg,L,S,G", [(1, 3, 1999, 16, 1), (2, 20, 1024, 16, 1), (1, 5, 1500, 3, 2), (1, 4, 1300, 40, 1)])
@pytest.mark.parametrize("kind", ["all", "ragged"])
def test_cut_scan(seq, dtype, N, Dg, L, S, G, kind):
    from paper_2104_08002_amd import binding

    assert binding.load().conv1d_scan_fwd_workspace_bytes(N, G * Dg, L, S, G) > 0
    gen = _gen(L)
    c = _scan_case(gen, dtype, N, Dg, L, S, G)
    lengths = None if kind == "all" else torch.tensor([L - 333, 0][:N], dtype=torch.int32, device="cuda")
    dy, dfinal = _normal(gen, N, G * Dg, L).to(dtype), _normal(gen, N, G * Dg, S)
    _check_scan(seq, c, lengths, dy, dfinal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("S,G", [(1, 1), (3, 1), (8, 2), (16, 1), (16, 3), (40, 1), (64, 2)])
def test_scan_steps_continue_a_prompt(seq, dtype, S, G):
    gen = _gen(S + G)
    N, L = 3, 24
    c = _scan_case(gen, dtype, N, 13, L, S, G)
    ref = _scan_ref(c, None)
    head = {k: v[..., :17] if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    y, state, saved = seq.conv1d_scan_fwd(**head, want_final=True)
    assert saved is None
    _near("y", y, ref["y"][:, :, :17], SCAN_C, (0, 1, 2))
    for t in range(17, L):
        one = {k: v[..., t].contiguous() if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items() if k != "init"}
        yt = seq.conv1d_scan_step(one.pop("x"), one.pop("dt"), one.pop("A"), one.pop("B"), one.pop("C"), state, **one)
        _near("y", yt, ref["y"][:, :, t], SCAN_C, (0, 1))
    _near("state", state, ref["final"], SCAN_C, (0, 1, 2))


def test_gradients_against_differences(seq):
    """Central differences of the float32 operators along random directions: what is left is the third derivative, h^2 / 6 of it, and
    the rounding of the two sums, 2^-24 of their magnitude over 2 h."""
    gen = _gen(3)
    c = _scan_case(gen, torch.float32, 2, 5, 40, 6, 2)
    dy = _normal(gen, 2, 10, 40)
    _, _, saved = seq.conv1d_scan_fwd(**c, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c, want_init=True)._asdict()
    for k in ("x", "dt", "A", "B", "C", "skip", "z", "dt_bias", "init"):
        way = _normal(gen, *c[k].shape)
        h = 2.0 ** -8
        up, down = (seq.conv1d_scan_fwd(**{**c, k: c[k] + s * h * way})[0].double() for s in (1, -1))
        found = ((up - down) * dy.double()).sum() / (2 * h)
        told = (g["d" + k].double() * way.double()).sum()
        noise = 100 * U32 * ((up.abs() + down.abs()) * dy.double().abs()).sum() / (2 * h)
        scale = g["d" + k].double().norm() * way.double().norm() / way.numel() ** 0.5
        assert (found - told).abs() <= noise + 0.02 * scale + 0.02 * told.abs(), (k, float(found), float(told), float(noise), float(scale))


# ---- what stands behind the end of a sequence ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("L", [37, 1300])
def test_padding_is_not_read(seq, dtype, L):
    gen = _gen(L)
    N, D, S = 3, 6, 16
    c = _scan_case(gen, dtype, N, D, L, S, 1)
    lengths = torch.tensor([0, L // 2, L - 1], dtype=torch.int32, device="cuda")
    behind = (torch.arange(L, device="cuda") >= lengths[:, None])[:, None]
    dy = _normal(gen, N, D, L).to(dtype)
    bad = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(dtype).min], dtype=dtype, device="cuda")[torch.arange(L, device="cuda") % 4]

    def spoil(v):
        return torch.where(behind if v.dim() == 3 else behind[:, :, None], bad, v)

    spoilt = {k: spoil(v) if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    results = []
    for case, g in ((c, dy), (spoilt, spoil(dy))):
        y, final, saved = seq.conv1d_scan_fwd(**case, lengths=lengths, want_final=True, save=True)
        results.append([y, final] + list(seq.conv1d_scan_bwd(g, saved, **case, lengths=lengths, want_init=True)))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert torch.equal(results[0][1][0], c["init"][0])
    assert not torch.where(behind, results[0][0], 0).any()
    w, bias = _normal(gen, D, 4).to(dtype), _normal(gen, D)
    results = []
    for x, g in ((c["x"], dy), (spoil(c["x"]), spoil(dy))):
        y, final = seq.conv1d_causal_fwd(x, w, bias=bias, silu=True, lengths=lengths, want_final=True)
        results.append([y, final] + list(seq.conv1d_causal_bwd(g, x, w, bias=bias, silu=True, lengths=lengths, want_init=True)))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_rates_without_bound(seq):
    """A rate of the type's lowest value, or minus infinity: the state is forgotten by a step above 0 and kept by one of 0, also where
    the padding has its steps of 0."""
    gen = _gen(21)
    for lowest in (torch.finfo(torch.float32).min, -math.inf):
        for L in (40, 1500):
            c = _scan_case(gen, torch.float32, 2, 3, L, 4, 1)
            c.update(softplus=False, dt=torch.ones(2, 3, L, device="cuda"), dt_bias=None, z=None, skip=None)
            c["A"][:, 1] = lowest
            lengths = torch.tensor([L - 7, 0], dtype=torch.int32, device="cuda")
            y, final, saved = seq.conv1d_scan_fwd(**c, lengths=lengths, want_final=True, save=True)
            assert y.isfinite().all() and torch.equal(final[1], c["init"][1])
            assert torch.equal(final[0, :, 1], c["x"][0, :, L - 8] * c["B"][0, 0, 1, L - 8])
            g = seq.conv1d_scan_bwd(torch.ones_like(y), saved, **c, lengths=lengths, want_init=True)
            assert g.dx.isfinite().all() and g.dinit.isfinite().all() and not g.dinit[:, :, 1].any()
            state = c["init"].clone()
            seq.conv1d_scan_step(c["x"][:, :, 0].contiguous(), torch.zeros(2, 3, device="cuda"), c["A"], c["B"][..., 0].contiguous(),
                                 c["C"][..., 0].contiguous(), state)
            assert torch.equal(state, c["init"])


def test_lengths_outside_the_tensor_are_brought_into_it(seq):
    gen = _gen(8)
    c = _scan_case(gen, torch.float32, 2, 3, 50, 16, 1)
    out = [seq.conv1d_scan_fwd(**c, lengths=torch.tensor(v, dtype=torch.int32, device="cuda"), want_final=True)[:2] for v in ([-7, 1000], [0, 50])]
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_a_bad_sample_stays_alone(seq):
    """NaN and infinity in one sample reach no other."""
    gen = _gen(9)
    c = _scan_case(gen, torch.float32, 3, 5, 90, 16, 1)
    dy = _normal(gen, 3, 5, 90)
    clean = seq.conv1d_scan_fwd(**c, save=True)
    grads = seq.conv1d_scan_bwd(dy, clean[2], **c)
    c["x"] = c["x"].clone()
    c["x"][1, 2, 40], c["x"][1, 3, 7] = math.nan, math.inf
    y, _, saved = seq.conv1d_scan_fwd(**c, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c)
    assert y[1, 2, 40:].isnan().all()
    for n in (0, 2):
        assert torch.equal(y[n], clean[0][n])
        for k in ("dx", "ddt", "dB", "dC", "dz"):
            assert torch.equal(getattr(g, k)[n], getattr(grads, k)[n]), k
    assert torch.equal(y[1, :2], clean[0][1, :2])


@pytest.mark.parametrize("L", [90, 700])
@pytest.mark.parametrize("G", [1, 2])
def test_a_bad_channel_stays_alone(seq, L, G):
    """NaN in the first channel of a group that does not fill a wave: of the group, dB and dC alone have it."""
    gen = _gen(25)
    c = _scan_case(gen, torch.float32, 2, 5, L, 16, G)
    dy = _normal(gen, 2, 5 * G, L)
    y0, _, saved = seq.conv1d_scan_fwd(**c, save=True)
    g0 = seq.conv1d_scan_bwd(dy, saved, **c)
    c["x"] = c["x"].clone()
    c["x"][:, 0, L // 2] = math.nan
    y, _, saved = seq.conv1d_scan_fwd(**c, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c)
    assert torch.equal(y[:, 1:], y0[:, 1:]) and y[:, 0, L // 2:].isnan().all()
    for k in ("dx", "ddt", "dz"):
        assert torch.equal(getattr(g, k)[:, 1:], getattr(g0, k)[:, 1:]), k
    for k in ("dA", "dskip", "ddt_bias"):
        assert torch.equal(getattr(g, k)[1:], getattr(g0, k)[1:]), k
    assert torch.equal(g.dB[:, 1:], g0.dB[:, 1:]) and torch.equal(g.dC[:, 1:], g0.dC[:, 1:]) and g.dC[:, 0].isnan().any()


# ---- streams, graphs, order ------------------------------------------------------------------------------------------------
def test_same_bits_again_and_on_another_stream(seq):
    gen = _gen(12)
    for shape in ((2, 130, 500, 16, 1), (1, 6, 3000, 16, 1)):
        c = _scan_case(gen, torch.bfloat16, *shape)
        dy = _normal(gen, *c["x"].shape).bfloat16()
        w = _normal(gen, c["x"].shape[1], 4).bfloat16()

        def run(stream=None):
            y, final, saved = seq.conv1d_scan_fwd(**c, want_final=True, save=True, stream=stream)
            causal = seq.conv1d_causal_bwd(dy, c["x"], w, silu=True, stream=stream)
            return [y, final, *seq.conv1d_scan_bwd(dy, saved, **c, stream=stream), *causal[:2]]

        first = run()
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        second = run(other)
        torch.cuda.current_stream().wait_stream(other)
        for a, b in zip(first, second):
            assert a is None and b is None or torch.equal(a, b)


def test_two_calls_at_once(seq):
    """On two streams, each with its own outputs and workspaces."""
    gen = _gen(22)
    cases = [_scan_case(gen, torch.bfloat16, *shape) for shape in ((2, 70, 700, 16, 1), (1, 9, 2500, 8, 1))]
    dys = [_normal(gen, *c["x"].shape).bfloat16() for c in cases]

    def run(c, dy, stream=None):
        y, final, saved = seq.conv1d_scan_fwd(**c, want_final=True, save=True, stream=stream)
        return [y, final, *seq.conv1d_scan_bwd(dy, saved, **c, stream=stream)]

    want = [run(c, dy) for c, dy in zip(cases, dys)]
    streams = [torch.cuda.Stream() for _ in cases]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    got = [[run(c, dy, st) for c, dy, st in zip(cases, dys, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for turn in got:
        for a, b in zip(turn, want):
            assert all(u is None and v is None or torch.equal(u, v) for u, v in zip(a, b))


def test_more_sums_than_a_launch_has_waves(seq):
    """8.4 million channels: 42 million sums over samples, one wave each."""
    gen = _gen(23)
    N, C, L, S = 2, 8400001, 2, 4
    x, dy = _normal(gen, N, C, L), _normal(gen, N, C, L)
    w, bias = _normal(gen, C, S), _normal(gen, C)
    dx, dw, db, _ = seq.conv1d_causal_bwd(dy, x, w, bias=bias)
    ref = dy.double().sum((0, 2))
    assert ((db.double() - ref).abs() <= 4 * U32 * dy.double().abs().sum((0, 2))).all()
    ref = (dy.double() * x.double()).sum((0, 2))
    assert ((dw[:, 3].double() - ref).abs() <= 6 * U32 * (dy * x).double().abs().sum((0, 2))).all() and not dw[:, :2].any()


def test_expanded_inputs(seq):
    """One sequence read by every sample, one B by every group: strides of 0."""
    gen = _gen(24)
    c = _scan_case(gen, torch.float32, 3, 4, 90, 16, 2)
    x1, B1 = c["x"][:1], c["B"][:, :1]
    dy = _normal(gen, 1, 8, 1).expand(3, 8, 90)
    wide = {**c, "x": x1.expand(3, 8, 90), "B": B1.expand(3, 2, 16, 90)}
    full = {**c, "x": wide["x"].contiguous(), "B": wide["B"].contiguous()}
    a, b = (seq.conv1d_scan_fwd(**v, want_final=True, save=True) for v in (wide, full))
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    with pytest.raises(ValueError):
        seq.conv1d_scan_bwd(dy, a[2], **wide)  # (a gradient is contiguous along the sequence)
    ga, gb = (seq.conv1d_scan_bwd(dy.contiguous(), a[2], **v) for v in (wide, full))
    assert all(u is None and v is None or torch.equal(u, v) for u, v in zip(ga, gb))


def test_captured_and_replayed(seq):
    """Two graphs, of a cut sequence and of another, replayed in turn with eager work between them."""
    gen = _gen(13)
    graphs = []
    for shape in ((1, 6, 3000, 16, 1), (2, 70, 300, 16, 2)):
        c = _scan_case(gen, torch.bfloat16, *shape)
        dy, w = _normal(gen, *c["x"].shape).bfloat16(), _normal(gen, c["x"].shape[1], 4).bfloat16()

        def run(c=c, dy=dy, w=w):
            u = seq.conv1d_causal_fwd(c["x"], w, silu=True)
            y, _, saved = seq.conv1d_scan_fwd(**{**c, "x": u}, save=True)
            g = seq.conv1d_scan_bwd(dy, saved, **{**c, "x": u})
            return [y, *g[:8], *seq.conv1d_causal_bwd(g.dx, c["x"], w, silu=True)[:2]]

        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = run()
        graphs.append((graph, outs, run, c))
    for turn in range(3):
        for graph, outs, run, c in graphs:
            c["x"].copy_(_normal(gen, *c["x"].shape))
            graph.replay()
            got = [o.clone() for o in outs]
            torch.cuda.synchronize()
            for a, b in zip(got, run()):
                assert torch.equal(a, b), turn


def test_outputs_by_the_caller(seq):
    gen = _gen(14)
    c = _scan_case(gen, torch.float32, 2, 4, 50, 16, 1)
    both = torch.full((2, 8, 50), 7.0, device="cuda")
    y, _, _ = seq.conv1d_scan_fwd(**c, out=both[:, 4:])
    assert torch.equal(y, seq.conv1d_scan_fwd(**c)[0]) and (both[:, :4] == 7).all()
    w = _normal(gen, 4, 4)
    seq.conv1d_causal_fwd(c["x"], w, out=both[:, :4])
    assert torch.equal(both[:, :4], seq.conv1d_causal_fwd(c["x"], w)) and torch.equal(both[:, 4:], y)


def test_elements_behind_32_bit_offsets(seq):
    """A tensor of more than 2^32 bytes: the last rows of it, against the same rows alone."""
    gen = _gen(15)
    N, D, L = 5, 1100, 400000
    x = torch.empty(N, D, L, dtype=torch.bfloat16, device="cuda")
    x[-1, -70:] = _normal(gen, 70, L).bfloat16()
    x[:-1] = 0.5
    x[-1, :-70] = 0.25
    w = _normal(gen, D, 4).bfloat16()
    y = seq.conv1d_causal_fwd(x, w, silu=True)
    assert torch.equal(y[-1:, -70:], seq.conv1d_causal_fwd(x[-1:, -70:], w[-70:], silu=True))
    A, dt = -torch.ones(D, 2, device="cuda"), torch.full_like(x, 0.1)
    B = _normal(gen, N, 1, 2, L).bfloat16()
    out = seq.conv1d_scan_fwd(x, dt, A, B, B, want_final=True)
    one = seq.conv1d_scan_fwd(x[-1:, -70:], dt[-1:, -70:], A[-70:], B[-1:], B[-1:], want_final=True)
    # another cut of the sequence, and so another order of its products
    _near("y", out[0][-1:, -70:].float(), one[0].double(), 2.0 ** 17, (0, 1, 2))  # (one rounding to bfloat16 either way: 2^-7)
    _near("final", out[1][-1:, -70:], one[1].double(), SCAN_C, (0, 1, 2))


# ---- refusals ----------------------------------------------------------------------------------------------------------------
def test_refusals(seq):
    from paper_2104_08002_amd.binding import Conv1dError

    gen = _gen(16)
    c = _scan_case(gen, torch.float32, 2, 4, 20, 16, 1)
    x, w = c["x"].contiguous(), _normal(gen, 4, 4)
    with pytest.raises(ValueError):
        seq.conv1d_causal_fwd(x.transpose(1, 2), w)
    with pytest.raises(ValueError):
        seq.conv1d_causal_fwd(x, w[:3])
    with pytest.raises(ValueError):
        seq.conv1d_causal_fwd(x, w.bfloat16())
    with pytest.raises(ValueError):
        seq.conv1d_causal_fwd(x, w, init=torch.zeros(2, 4, 4, device="cuda"))
    with pytest.raises(ValueError):
        seq.conv1d_causal_fwd(x, w, lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        seq.conv1d_causal_fwd(x, w, out=x)
    with pytest.raises(ValueError):
        seq.conv1d_causal_fwd(x, w, out=torch.empty(1, 1, 20, device="cuda").expand(2, 4, 20))
    with pytest.raises(Conv1dError) as e:
        seq.conv1d_causal_fwd(x, _normal(gen, 4, 9))
    assert e.value.status == -2
    with pytest.raises(TypeError):
        seq.conv1d_causal_fwd(x.half(), w.half())
    with pytest.raises(ValueError):
        seq.conv1d_scan_fwd(**{**c, "B": c["B"][:, :, :15]})
    with pytest.raises(ValueError):
        seq.conv1d_scan_fwd(**{**c, "A": c["A"].bfloat16()})
    with pytest.raises(ValueError):
        seq.conv1d_scan_fwd(**{**c, "z": c["z"].cpu()})
    with pytest.raises(Conv1dError) as e:
        big = torch.zeros(2, 1, 65, 20, device="cuda")
        seq.conv1d_scan_fwd(**{**c, "A": torch.zeros(4, 65, device="cuda"), "B": big, "C": big, "init": None})
    assert e.value.status == -2
    _, _, saved = seq.conv1d_scan_fwd(**c, save=True)
    with pytest.raises(ValueError):
        seq.conv1d_scan_bwd(x, saved[:-1], **c)
    with pytest.raises(Conv1dError) as e:
        seq.conv1d_scan_bwd(x, saved, **c, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -3
