"""Selective scans whose state grows, on the GPU: decays above 1, whose product over a part of a long sequence is beyond FP32's range.

Every case has summands of one sign, so that nothing cancels: a state is a sum of products of decays, each with a relative error that
adds up over the steps it spans.  |e A| is 1/2 or 1/4 here, whose sums over a segment are exact: a step carries the roundings of the
rate and of e times it (1 of 2^-24 each, times |e A|), of the exponential (2) and of two products, a segment less.  At most 6 a step, 64
for the sums over states, and twice that for what is left out here (products of errors): 12 steps + 64.
"""
import pytest
import torch

from test_gpu_sequence import U32, _gen, seq  # noqa: F401

pytestmark = pytest.mark.gpu


def _pos(gen, *shape):
    return 0.5 + torch.rand(shape, generator=gen, device="cuda")


def _recurrence(c, lengths=None):
    """Outputs and all states in 64 bits, [N, D, L] and [L + 1, N, D, S]."""
    x, dt, A, B, C = (c[k].double() for k in ("x", "dt", "A", "B", "C"))
    N, D, L = x.shape
    h = c["init"].double() if c.get("init") is not None else x.new_zeros(N, D, A.shape[1])
    ys, hs = [], [h]
    for t in range(L):
        h = torch.exp(dt[:, :, t, None] * A) * h + (dt[:, :, t] * x[:, :, t])[:, :, None] * B[:, 0, None, :, t]
        ys.append((C[:, 0, None, :, t] * h).sum(2))
        hs.append(h)
    return torch.stack(ys, 2), torch.stack(hs)


def _relative(name, got, ref, c):
    assert got.isfinite().all(), (name, int((~got.isfinite()).sum()))
    bad = (got.double() - ref).abs() > c * U32 * ref.abs() + 1e-37
    assert not bad.any(), (name, int(bad.sum()), float(((got.double() - ref).abs() / (c * U32 * ref.abs() + 1e-37)).max()))


def _case(gen, sign, L, S, N=1, D=3):
    """Decays exp(1/2) a step: a rate above 0 with a step above 0, or both below."""
    return {"x": torch.zeros(N, D, L, device="cuda"), "dt": torch.full((N, D, L), 0.5 * sign, device="cuda"),
            "A": torch.full((D, S), 1.0 * sign, device="cuda"), "B": _pos(gen, N, 1, S, L), "C": _pos(gen, N, 1, S, L)}


SHAPES = [(2048, 16), (1999, 3), (1999, 8), (4100, 24), (4100, 64)]


def _cut(c):
    from paper_2104_08002_amd import binding

    N, D, L = c["x"].shape
    assert binding.load().conv1d_scan_fwd_workspace_bytes(N, D, L, c["A"].shape[1], 1) > 0


@pytest.mark.parametrize("L,S", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_a_state_of_zero_before_a_growing_end(seq, L, S, sign):  # noqa: F811
    """Nothing but the last 50 inputs: the state before them is 0, whatever the decays of all that time multiply to."""
    gen = _gen(L + S)
    c = _case(gen, sign, L, S)
    _cut(c)
    c["x"][:, :, -50:] = sign * _pos(gen, 1, 3, 50)
    y, hs = _recurrence(c)
    got, final, _ = seq.conv1d_scan_fwd(**c, want_final=True)
    assert not got[:, :, :-50].any()
    _relative("y", got, y, 12 * 50 + 64)
    _relative("final", final, hs[-1], 12 * 50 + 64)


@pytest.mark.parametrize("L,S", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_no_gradient_behind_a_growing_start(seq, L, S, sign):  # noqa: F811
    """Gradients reach the first 50 outputs alone: what comes from all that time behind them is 0."""
    gen = _gen(L + S + 1)
    c = _case(gen, sign, L, S)
    dy = torch.zeros_like(c["x"])
    dy[:, :, :50] = _pos(gen, 1, 3, 50)
    _, _, saved = seq.conv1d_scan_fwd(**c, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c, want_init=True)
    carry = torch.zeros(1, 3, S, dtype=torch.float64, device="cuda")
    dx = torch.zeros_like(dy, dtype=torch.float64)
    decay = torch.exp(c["dt"].double()[:, :, 0, None] * c["A"].double())
    for t in reversed(range(50)):
        carry = carry + c["C"][:, 0, None, :, t].double() * dy[:, :, t, None].double()
        dx[:, :, t] = (carry * c["B"][:, 0, None, :, t].double()).sum(2) * 0.5 * sign
        carry = carry * decay
    _relative("dx", g.dx, dx, 12 * 50 + 64)
    _relative("dinit", g.dinit, carry, 12 * 50 + 64)
    for name in ("ddt", "dA", "dB", "dC"):  # (x and all states are 0)
        assert torch.equal(getattr(g, name), torch.zeros_like(getattr(g, name))), name


@pytest.mark.parametrize("L,S", [(2048, 16), (1999, 8)])
def test_a_small_state_that_grows_past_the_range_of_a_decay(seq, L, S):  # noqa: F811
    """From 1e-30 by exp(150) over 600 steps: the state stays in range, the decay over them does not."""
    gen = _gen(L)
    c = _case(gen, 1, L, S)
    c["dt"][:] = 0.0
    c["dt"][:, :, 512:1112] = 0.25
    c["init"] = 1e-30 * _pos(gen, 1, 3, S)
    y, hs = _recurrence(c)
    got, final, _ = seq.conv1d_scan_fwd(**c, want_final=True)
    _relative("y", got, y, 12 * 600 + 64)
    _relative("final", final, hs[-1], 12 * 600 + 64)


@pytest.mark.parametrize("first,last", [(1, -1), (-1, 1)])
def test_growth_and_decline_in_turn(seq, first, last):  # noqa: F811
    """exp(100) up and down again, several times within what is joined at once: 0 stays 0, and what comes in at the end counts."""
    gen = _gen(7)
    L, S = 4000, 16
    c = _case(gen, 1, L, S)
    turn = torch.arange(L, device="cuda") // 200 % 2
    c["dt"][:] = torch.where(turn == 0, 0.5 * first, 0.5 * last)
    c["x"][:, :, -50:] = c["dt"][:, :, -50:].sign() * _pos(gen, 1, 3, 50)
    y, hs = _recurrence(c)
    got, final, _ = seq.conv1d_scan_fwd(**c, want_final=True)
    assert not got[:, :, :-50].any()
    _relative("y", got, y, 12 * 50 + 64)
    _relative("final", final, hs[-1], 12 * 50 + 64)


def test_growth_is_the_same_cut_and_whole(seq):  # noqa: F811
    """A batch large enough is not cut; a padded one ends within the first, a later and the last part."""
    from paper_2104_08002_amd import binding

    gen = _gen(11)
    N, D, L, S = 5, 3, 1500, 16
    c = _case(gen, 1, L, S, N)
    lengths = torch.tensor([0, 3, 700, 1499, 1500], dtype=torch.int32, device="cuda")
    for n, m in enumerate(lengths.tolist()):
        if m:
            c["x"][n, :, max(0, m - 50):m] = _pos(gen, D, m - max(0, m - 50))
    _cut(c)
    wide = 16384
    assert binding.load().conv1d_scan_fwd_workspace_bytes(N, wide, L, S, 1) == 0
    y, final, _ = seq.conv1d_scan_fwd(**c, lengths=lengths, want_final=True)
    whole = {k: v if k in "BC" else v.repeat_interleave(wide // D + 1, 0 if k == "A" else 1)[tuple([slice(None)] * (k != "A") + [slice(wide)])]
             for k, v in c.items()}
    y1, final1, _ = seq.conv1d_scan_fwd(**whole, lengths=lengths, want_final=True)
    per = wide // D + 1
    _relative("y", y, y1[:, ::per].double(), 2 * (12 * 50 + 64))
    _relative("final", final, final1[:, ::per].double(), 2 * (12 * 50 + 64))


@pytest.mark.parametrize("lowest", [torch.finfo(torch.float32).min, -float("inf")])
def test_a_rate_without_bound_beside_a_growing_state(seq, lowest):  # noqa: F811
    """Forgotten by every step, in a wave whose other states grow; also over 16 segments and more at once, and kept by steps of 0."""
    gen = _gen(12)
    L, S = 2048, 4
    c = _case(gen, 1, L, S, N=2)
    c["dt"][:] = 0.0078125
    c["x"][:] = _pos(gen, 2, 3, L)
    c["A"][:, 1] = lowest
    c["init"] = _pos(gen, 2, 3, S)
    _cut(c)
    lengths = torch.tensor([L - 7, 0], dtype=torch.int32, device="cuda")
    y, final, saved = seq.conv1d_scan_fwd(**c, lengths=lengths, want_final=True, save=True)
    ex = c["dt"][0, :, L - 8] * c["x"][0, :, L - 8]
    assert y.isfinite().all() and torch.equal(final[0, :, 1], ex * c["B"][0, 0, 1, L - 8])
    assert torch.equal(final[1], c["init"][1])
    g = seq.conv1d_scan_bwd(torch.ones_like(y), saved, **c, lengths=lengths, want_init=True)
    assert g.dx.isfinite().all() and g.dinit.isfinite().all() and not g.dinit[:, :, 1].any()
    assert (g.dinit[0, :, [0, 2, 3]] > 1e6).all()
