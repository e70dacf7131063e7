"""The operators around the layers on the GPU against their definitions in 64 bits (blocks_reference)."""
import math

import pytest
import torch

import blocks_reference as ref

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
ORDER = pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])


@pytest.fixture(scope="module")
def blocks():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2104_08002_amd import binding, blocks

    binding.load()
    return blocks


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _lengths(kind, N, L):
    if kind == "whole":
        return None
    return torch.tensor([(L, 0, L // 2, 1, -3, L + 5, max(0, L - 1))[i % 7] for i in range(N)], dtype=torch.int32, device="cuda")


def _put(v, last, padded=False):
    """v in the wanted order; with `padded` as the second half of a wider tensor full of NaN."""
    N, C, L = v.shape
    if last:
        whole = torch.full((N, L, 2 * C if padded else C), float("nan"), device="cuda", dtype=v.dtype)
        view = whole[:, :, whole.shape[2] - C:].transpose(1, 2)
    else:
        whole = torch.full((N, 2 * C if padded else C, L), float("nan"), device="cuda", dtype=v.dtype)
        view = whole[:, whole.shape[1] - C:]
    view.copy_(v)
    return view


# ---- embedding -----------------------------------------------------------------------------------------------------------------
def _tokens(gen, N, L, V, kind, wide=True):
    if kind == "one":
        t = torch.full((N, L), V - 1, device="cuda")
    else:
        t = torch.randint(0, V, (N, L), generator=gen, device="cuda")
        if kind == "skewed":
            t = t * t // max(1, V) * t // max(1, V)
    if kind == "outside":
        t = torch.where(torch.rand(N, L, generator=gen, device="cuda") < 0.3, torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1], device="cuda")[t % 4], t)
    return t.to(torch.int64 if wide else torch.int32)


# Many tokens: 31 sums of up to 32 numbers in float and the product with the scale, 34 u.  Few: an instruction adds 32 products, each
# addition cut off by less than 2 u of the magnitudes; up to 8 steps are added in float by each of four waves, and these; the scale: 75 u.
GRAD = 75 * ref.U

EMBED = [(1, 1, 1, 1), (2, 3, 7, 5), (3, 15, 1000, 5), (2, 64, 129, 255), (2, 65, 128, 256), (4, 16, 513, 257), (1, 17, 2049, 4000), (2, 130, 300, 70000), (5, 8, 64, 2),
         (2, 2100, 40, 30), (1, 1, 40000, 3), (2, 512, 200, 1000), (70, 20, 9, 300), (9, 40, 1000, 1024),
         (3, 33, 700, 1025), (2, 5, 40, 30000), (1, 48, 100, 65520)]


@TYPES
@ORDER
@pytest.mark.parametrize("kind,lengths", [("plain", "whole"), ("skewed", "ragged"), ("outside", "ragged"), ("one", "whole")])
@pytest.mark.parametrize("N,D,L,V", EMBED)
def test_embedding(blocks, dtype, last, kind, lengths, N, D, L, V):
    gen = _gen(N * D + L)
    table, tokens, lengths = _normal(gen, V, D).to(dtype), _tokens(gen, N, L, V, kind, wide=D % 2 == 0), _lengths(lengths, N, L)
    scale = 1.375
    y = blocks.conv1d_embed_fwd(table, tokens, scale=scale, lengths=lengths, channels_last=last)
    assert y.dtype == dtype and y.shape == (N, D, L)
    want = ref.embed(table, tokens, scale, lengths)
    ref.near(y, want, ref.U * want.abs(), "y")
    dy = _normal(gen, N, D, L).to(dtype)
    # what is behind a sequence's end, and where there is no token, is used for nothing
    t = tokens.long()
    there = ((t >= 0) & (t < V))[:, None] & ref.inside(lengths, N, L)
    dy = torch.where(there, dy, float("nan"))
    dy_in = _put(dy, last, padded=True)
    got = blocks.conv1d_embed_bwd(dy_in, tokens, V, scale=scale, lengths=lengths)
    want, size = ref.embed_grad(torch.where(there, dy, 0.0), tokens, V, scale, lengths)
    ref.near(got, want, GRAD * size, "dtable")
    # the same call again; one channel is in either order, so that another stride may take another way
    assert torch.equal(got, blocks.conv1d_embed_bwd(dy_in, tokens, V, scale=scale, lengths=lengths))


@pytest.mark.parametrize("V", [255, 256, 65535, 65536, 1 << 20])
def test_embedding_of_as_many_tokens_as_digits_hold(blocks, V):
    gen = _gen(V)
    N, D, L = 2, 2, 6000
    tokens = torch.cat((torch.randint(0, V, (N, L - 3), generator=gen, device="cuda"), torch.tensor([[0, V - 1, V], [V - 1, 0, -1]], device="cuda")), 1)
    dy = _normal(gen, N, D, L)
    want, size = ref.embed_grad(dy, tokens, V, 1.0, None)
    ref.near(blocks.conv1d_embed_bwd(dy, tokens, V), want, GRAD * size)


def test_embedding_of_long_runs(blocks):
    """One token on nearly all of 400000 positions: its sum crosses thousands of chunks."""
    gen = _gen(3)
    N, D, L, V = 4, 24, 100000, 9
    tokens = torch.full((N, L), 4, device="cuda")
    tokens[:, ::997] = torch.randint(0, V - 1, tokens[:, ::997].shape, generator=gen, device="cuda")
    dy = _normal(gen, N, D, L)
    want, size = ref.embed_grad(dy, tokens, V, 0.5, None)
    ref.near(blocks.conv1d_embed_bwd(dy, tokens, V, scale=0.5), want, GRAD * size)


@TYPES
@ORDER
@pytest.mark.parametrize("V", [3, 40, 2000])
def test_embedding_gradients_that_are_not_finite(blocks, dtype, last, V):
    """They reach the rows of their own tokens alone, in their own channels."""
    gen = _gen(V)
    N, D, L = 2, 37, 600
    tokens, dy = torch.randint(0, V, (N, L), generator=gen, device="cuda"), _normal(gen, N, D, L).to(dtype)
    fine = blocks.conv1d_embed_bwd(_put(dy, last), tokens, V)
    inf = float("inf")
    for bad in ((float("nan"),), (inf,), (-inf,), (inf, inf), (inf, -inf), (torch.finfo(dtype).max,) * 2):
        z, t, want = dy.clone(), tokens.clone(), fine.clone()
        places = [(0, 5, 17), (1, 5, 599)][:len(bad)]
        for (n, d, l), v in zip(places, bad):
            z[n, d, l] = v
            t[n, l] = 1
        want = blocks.conv1d_embed_bwd(_put(dy, last), t, V)
        want[1, 5] = sum(bad) if sum(bad) != sum(bad) or abs(sum(bad)) == inf else inf
        got = blocks.conv1d_embed_bwd(_put(z, last), t, V)
        assert torch.equal(got.nan_to_num(1e30, 2e30, 3e30), want.nan_to_num(1e30, 2e30, 3e30)), bad


@TYPES
@pytest.mark.parametrize("N,D,V", [(1, 1, 1), (4, 128, 4096), (33, 77, 10), (1000, 2050, 50)])
def test_embedding_step(blocks, dtype, N, D, V):
    gen = _gen(N)
    table, tokens = _normal(gen, V, D).to(dtype), torch.randint(-1, V + 1, (N,), generator=gen, device="cuda")
    want = ref.embed(table, tokens[:, None], 3.0, None)[:, :, 0]
    ref.near(blocks.conv1d_embed_step(table, tokens, scale=3.0), want, ref.U * want.abs())
    out = torch.full((N, 2 * D), 7.0, device="cuda", dtype=dtype)
    blocks.conv1d_embed_step(table, tokens.repeat(2, 1).T.contiguous().view(N, 2)[:, 0], scale=3.0, out=out[:, D:])
    ref.near(out[:, D:], want, ref.U * want.abs())
    assert (out[:, :D] == 7).all()


# ---- group norm ------------------------------------------------------------------------------------------------------------------
NORM = [(1, 1, 1, 1), (2, 6, 1, 3), (3, 12, 7, 4), (2, 15, 2051, 3), (1, 8, 40001, 2), (2, 64, 300, 8), (3, 45, 129, 5), (2, 96, 33, 1), (1, 2100, 5, 7), (40, 32, 16, 32),
        (2, 3, 5000, 3), (1, 512, 70, 16), (300, 10, 3, 2), (1100, 12, 9, 1), (2, 1000, 3, 1), (40, 64, 200, 8), (3, 27, 60, 3), (130, 40, 100, 1)]


def _norm_inputs(gen, N, C, L, dtype, at=1.0):
    x = (at * _normal(gen, N, C, 1) + (0.5 + torch.rand(1, C, 1, generator=gen, device="cuda")) * _normal(gen, N, C, L)).to(dtype)
    return x, _normal(gen, N, C, L).to(dtype), 1 + 0.3 * _normal(gen, C), 0.3 * _normal(gen, C)


def _check_norm(blocks, x, dy, groups, weight, bias, act, lengths, last, eps=1e-5):
    N, C, L = x.shape
    how = {"weight": weight, "bias": bias, "relu": act == "relu", "silu": act == "silu", "eps": eps, "lengths": lengths}
    m = ref.inside(lengths, N, L)
    x, dy = (_put(torch.where(m, v, float("nan")), last, padded) for v, padded in ((x, True), (dy, True)))
    want = ref.norm(x, dy, groups, weight, bias, act, eps, lengths)
    y, stats = blocks.conv1d_norm_fwd(x, groups, **how, want_stats=True)
    assert y.dtype == x.dtype and (L == 1 or C == 1 or y.stride(1 if last else 2) == 1)
    ref.near(y, *want["y"], "y")
    assert torch.equal(y, blocks.conv1d_norm_fwd(x, groups, **how))
    some = m.any(2)[:, 0]
    # sums of 64 bits of differences: far below half a step of float of the spread
    assert ((stats[:, :, 0] - want["stats"][:, :, 0]).abs() * stats[:, :, 1])[some].max().nan_to_num() <= 1e-9 if some.any() else True
    assert ((stats[:, :, 1] / want["stats"][:, :, 1] - 1).abs()[some].max() <= 1e-9) if some.any() else True
    got = blocks.conv1d_norm_bwd(dy, stats, x, groups, **how)
    for name, g in zip(("dx", "dweight", "dbias"), got):
        if g is None:
            assert (weight if name == "dweight" else bias) is None
        else:
            ref.near(g, *want[name], name)
    for a, b in zip(got, blocks.conv1d_norm_bwd(dy, stats, x, groups, **how)):
        assert a is None or torch.equal(a, b)


@TYPES
@ORDER
@pytest.mark.parametrize("act,affine,lengths", [("none", True, "whole"), ("relu", True, "ragged"), ("silu", True, "ragged"), ("silu", False, "whole")])
@pytest.mark.parametrize("N,C,L,G", NORM)
def test_norm(blocks, dtype, last, act, affine, lengths, N, C, L, G):
    x, dy, weight, bias = _norm_inputs(_gen(C + L), N, C, L, dtype)
    _check_norm(blocks, x, dy, G, weight if affine else None, bias if affine else None, act, _lengths(lengths, N, L), last)


@ORDER
@pytest.mark.parametrize("L", [40, 5000])
def test_norm_of_one_parameter(blocks, last, L):
    x, dy, weight, bias = _norm_inputs(_gen(L), 3, 24, L, torch.bfloat16)
    _check_norm(blocks, x, dy, 3, weight, None, "relu", None, last)
    _check_norm(blocks, x, dy, 3, None, bias, "silu", _lengths("ragged", 3, L), last)


@ORDER
def test_relu_of_values_next_to_zero(blocks, last):
    """A bias that brings many values of p to within some roundings of 0: which side they lie on is the definition's."""
    gen = _gen(31)
    x = torch.randn(2, 16, 3000, generator=gen, device="cuda")
    x[:, 8:] = x[:, 8:].round()              # few values, so that
    h = ref.norm(x, x, 2, None, None, "none", 1e-5, None)["y"][0]
    bias = -h[0, :, 7].float()               # one value a channel lies next to 0
    _check_norm(blocks, x, torch.randn(2, 16, 3000, generator=gen, device="cuda"), 2, None, bias, "relu", None, last)


@ORDER
@pytest.mark.parametrize("at", [1e3, 1e6])
def test_norm_of_values_far_from_zero(blocks, last, at):
    """A mean of thousands and millions of spreads; a first value far from the others."""
    x, dy, weight, bias = _norm_inputs(_gen(1), 2, 8, 3001, torch.float32)
    _check_norm(blocks, x + at, dy, 2, weight, bias, "silu", None, last)
    x[:, :, 0] += at
    _check_norm(blocks, x, dy, 2, weight, bias, "relu", None, last)


@ORDER
def test_norm_of_equal_values(blocks, last):
    """No spread at all: h is 0, y the bias."""
    x = torch.full((2, 6, 100), 123456.7, device="cuda")
    bias = torch.arange(6.0, device="cuda")
    y, stats = blocks.conv1d_norm_fwd(_put(x, last), 3, bias=bias, want_stats=True)
    assert torch.equal(y, bias[:, None].expand(2, 6, 100)) and (stats[:, :, 1] == 1e-5 ** -0.5).all()


@ORDER
def test_norm_of_values_that_are_not_finite(blocks, last):
    """They reach their own sample and group alone."""
    gen = _gen(2)
    x = _normal(gen, 3, 8, 700)
    fine = blocks.conv1d_norm_fwd(_put(x, last), 4, silu=True)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for c, l in ((2, 0), (3, 699)):
            z = x.clone()
            z[1, c, l] = bad
            y, stats = blocks.conv1d_norm_fwd(_put(z, last), 4, silu=True, want_stats=True)
            assert y[1, 2:4].isnan().all()
            y[1, 2:4] = fine[1, 2:4]
            assert torch.equal(y, fine)
            dx, _, _ = blocks.conv1d_norm_bwd(_put(x, last), stats, _put(z, last), 4, silu=True)
            assert dx[1, 2:4].isnan().all() and dx.isfinite().sum() == dx.numel() - 2 * 700


# ---- dropout ---------------------------------------------------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("N,C,L,residual,lengths", [(1, 1, 1, False, "whole"), (2, 3, 7, True, "ragged"), (3, 5, 130, True, "whole"), (7, 2, 33, False, "ragged"), (1, 2, 1031, True, "whole")])
def test_dropout(blocks, dtype, p, N, C, L, residual, lengths):
    gen = _gen(L)
    key, call = 0x9876543210fedcba, 0xfedcba9876543210
    x, r = (_put(_normal(gen, N, C, L).to(dtype), False, padded=True) for _ in range(2))
    r, lengths = r if residual else None, _lengths(lengths, N, L)
    kept = torch.tensor([[w >= math.floor(p * 2 ** 32) for w in line] for line in ref.words(N * C, L, key, call)], device="cuda").view(N, C, L)
    y = blocks.conv1d_dropout(x, p, key, call, residual=r, lengths=lengths)
    ref.near(y, *ref.dropout(x, kept, p, r, lengths))
    counter = torch.tensor(5, device="cuda")
    assert torch.equal(y, blocks.conv1d_dropout(x, p, key, call - 5, counter=counter, residual=r, lengths=lengths))


def test_what_is_dropped_reaches_nothing(blocks):
    x = torch.full((2, 4, 500), float("nan"), device="cuda")
    x[1] = float("inf")
    y = blocks.conv1d_dropout(x, 0.5, 1)
    kept = torch.tensor(ref.words(8, 500, 1, 0), device="cuda").view(2, 4, 500) >= 2 ** 31
    assert torch.equal(y == 0, ~kept) and y[0][kept[0]].isnan().all() and (y[1][kept[1]] == float("inf")).all()
    assert (blocks.conv1d_dropout(x, 1.0, 1) == 0).all()


def test_dropout_drops_its_share(blocks):
    """Over 2^24 elements the share is within five deviations of p, for neighbours alike or not as often as chance has it, and other
    calls and keys drop others."""
    n = 1 << 24
    x = torch.ones(4, 4, n // 16, device="cuda")
    for p in (0.1, 0.5):
        first, second, third = (blocks.conv1d_dropout(x, p, key, call) == 0 for key, call in ((7, 0), (7, 1), (8, 0)))
        for share, of in ((first, p), (first & second, p * p), (first & third, p * p), (first[:, :, 1:] & first[:, :, :-1], p * p), (first[:, 1:] & first[:, :-1], p * p)):
            assert abs(share.double().mean().item() - of) < 5 * (of * (1 - of) / share.numel()) ** 0.5 * 1.5
