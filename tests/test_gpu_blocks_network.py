"""The operators around the layers together, as a network uses them: tokens, embedding, dropout, a layer, group norm with its activation,
dropout with the residual, and a layer of logits; gradients by autograd; captured; on streams; with offsets beyond 32 bits.

The plain form is the same network of elementary operations in 64 bits on the same (rounded) inputs and weights, with the masks that
the generator's definition gives.  In float32 every product and sum is off by some roundings of 2^-24 of the values around it; a
tensor's error is held to 2e-5 of its norm, a few hundred of them.  In bfloat16 each of the eight tensors between the operators
is rounded once forward and once backward, to 2^-8 of its values, and errors of one place meet those of others at random: 16 * 2^-8 = 6 % of the norm.
"""
import math

import pytest
import torch

import blocks_reference as ref

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 2e-5, torch.bfloat16: 16 * 2.0 ** -8}


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2104_08002_amd import autograd, binding, blocks

    binding.load()
    return autograd, blocks


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _network(dtype, gen, V=11, D=24, S=3, G=4):
    def normal(*shape, std=1.0):
        return std * torch.randn(shape, generator=gen, device="cuda")
    p = {"table": normal(V, D).to(dtype), "w": normal(D, D, S, std=(D * S) ** -0.5).to(dtype), "out": normal(V, D, 1, std=D ** -0.5).to(dtype),
         "weight": 1 + normal(D, std=0.1), "bias": normal(D, std=0.1)}
    return {k: v.requires_grad_(True) for k, v in p.items()}, G


DROP, SCALE = 0.25, 1.5


def _block(ops, p, G, tokens, dtype, lengths=None, counter=None):
    autograd, _ = ops
    low = dtype == torch.bfloat16
    x = autograd.conv1d_embed(p["table"], tokens, SCALE, lengths)
    x = autograd.conv1d_dropout(x, DROP, 5, 0, counter=counter, lengths=lengths)
    u = autograd.conv1d(x, p["w"], padding=1, bf16_out=low)
    u = autograd.conv1d_norm(u, G, p["weight"], p["bias"], silu=True, lengths=lengths)
    x = autograd.conv1d_dropout(u, DROP, 6, 0, counter=counter, residual=x, lengths=lengths)
    return autograd.conv1d(x, p["out"], bf16_out=low)


def _kept(N, C, L, key, call):
    return torch.tensor(ref.words(N * C, L, key, call), device="cuda").view(N, C, L) >= math.floor(DROP * 2 ** 32)


def _plain(p, G, tokens, lengths=None, call=0):
    p = {k: v.detach().double().requires_grad_(True) for k, v in p.items()}
    N, L = tokens.shape
    D = p["table"].shape[1]
    m = ref.inside(lengths, N, L)
    drop = lambda v, key: torch.where(_kept(N, D, L, key, call), v / (1 - DROP), 0.0)  # noqa: E731
    x = torch.where(m, drop(SCALE * p["table"][tokens.long()].transpose(1, 2), 5), 0.0)
    xe = torch.nn.functional.pad(x, (1, 1))
    u = sum(p["w"][:, :, s][None] @ xe[:, :, s:s + L].contiguous() for s in range(3))
    count = (m.sum(2).double() * (D // G)).clamp(min=1).view(N, 1, 1)
    u = torch.where(m, u, 0.0).view(N, G, D // G, L)
    off = torch.where(m[:, None], u - (u.sum((2, 3)) / count[:, :, 0]).view(N, G, 1, 1), 0.0)
    h = (off / ((off * off).sum((2, 3)) / count[:, :, 0] + 1e-5).sqrt().view(N, G, 1, 1)).view(N, D, L)
    v = h * p["weight"][:, None] + p["bias"][:, None]
    x = torch.where(m, x + drop(v * torch.sigmoid(v), 6), 0.0)
    return p["out"][:, :, 0][None] @ x, p


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,L,ragged", [(2, 70, False), (3, 133, True), (1, 1, False)])
def test_training_step(ops, dtype, N, L, ragged):
    gen = _gen(L)
    p, G = _network(dtype, gen)
    tokens = torch.randint(0, 11, (N, L), generator=gen, device="cuda")
    lengths = torch.tensor([L, 0, L // 2], dtype=torch.int32, device="cuda") if ragged else None
    out = _block(ops, p, G, tokens, dtype, lengths)
    gy = torch.randn(out.shape, generator=gen, device="cuda").to(dtype)
    out.backward(gy)
    want, q = _plain(p, G, tokens, lengths)
    want.backward(gy.double())

    def near(name, got, want):
        assert (got.double() - want).norm() <= TOL[dtype] * want.norm() + 1e-30, (name, float((got.double() - want).norm() / want.norm()))

    near("out", out, want.detach())
    for k in p:
        near(k, p[k].grad, q[k].grad)


def test_training_step_captured(ops):
    """The whole step in a graph, replayed on new tokens with a counter that the step moves on, with eager work between: each replay
    drops others, and the same as the eager step with that counter."""
    gen = _gen(8)
    p, G = _network(torch.bfloat16, gen)
    tokens, counter = torch.randint(0, 11, (2, 90), generator=gen, device="cuda"), torch.zeros((), dtype=torch.int64, device="cuda")
    gy = torch.randn(2, 11, 90, generator=gen, device="cuda").bfloat16()

    def step():
        at = counter.clone()
        out = _block(ops, p, G, tokens, torch.bfloat16, counter=at)
        grads = [g.clone() for g in torch.autograd.grad(out, list(p.values()), gy)]
        counter.add_(1)
        return [out.detach()] + grads

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    last = None
    for turn in range(4):
        if turn % 2 == 0:
            tokens.copy_(torch.randint(0, 11, tokens.shape, generator=gen, device="cuda"))
        before = counter.clone()
        graph.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        assert counter == before + 1
        counter.copy_(before)
        for a, b in zip(got, step()):
            assert torch.equal(a, b), turn
        assert turn % 2 == 0 or not torch.equal(last, got[0])  # the same tokens, another mask
        last = got[0]


@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
def test_calls_captured(ops, last):
    """Every way that a call can take, in a graph, replayed on new inputs with eager calls between: sorted and few tokens, groups of one
    workgroup and of many."""
    _, blocks = ops
    gen = _gen(21)
    order = (lambda v: v.transpose(1, 2).contiguous().transpose(1, 2)) if last else (lambda v: v)
    sizes = ((3, 16, 4000, 2), (2, 64, 50, 8), (40, 32, 64, 32))
    xs = [order(torch.randn(N, C, L, generator=gen, device="cuda")) for N, C, L, _ in sizes]
    tokens = [torch.randint(0, 5000, (N, L), generator=gen, device="cuda") for N, _, L, _ in sizes]
    table = torch.randn(5000, 16, generator=gen, device="cuda")

    def calls():
        out = []
        for x, t, (_, C, _, G) in zip(xs, tokens, sizes):
            y, stats = blocks.conv1d_norm_fwd(x, G, silu=True, want_stats=True)
            out += [y, blocks.conv1d_norm_bwd(y, stats, x, G, silu=True)[0], blocks.conv1d_embed_bwd(x, t, 5000), blocks.conv1d_embed_bwd(x, t % 40, 40),
                    blocks.conv1d_embed_fwd(table, t, channels_last=last), blocks.conv1d_embed_fwd(table, t % 40, channels_last=last)]
        return out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = calls()
    for turn in range(3):
        for x, t in zip(xs, tokens):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            t.copy_(torch.randint(0, 5000, t.shape, generator=gen, device="cuda") ** (turn + 1) % 5000)
        graph.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, calls())):
            assert torch.equal(a, b), (turn, i)


@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_norm_gradients_against_differences(ops, act, last):
    """(f(v + s d) - f(v - s d)) / 2 s against <gradient, d>, f the sum of y dy, taken in 64 bits, s = 1/64 and d of about 1 an element.
    12000 third derivatives of about 1 add s^2 / 6 each, at random 110 times that, 0.0045; 12000 roundings of u |y dy|, 110 u / s = 0.0004;
    along the gradient's own direction s^2 / 6 of the slope."""
    _, blocks = ops
    gen = _gen(11)
    new = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    N, C, L, G = 2, 12, 500, 3
    order = (lambda v: v.transpose(1, 2).contiguous().transpose(1, 2)) if last else (lambda v: v)
    v = {"x": new(N, C, L) + 0.5, "weight": 1 + 0.2 * new(C), "bias": 0.2 * new(C)}
    dy, how = order(new(N, C, L)), {"silu": act == "silu"}
    f = lambda x, weight, bias: (blocks.conv1d_norm_fwd(order(x), G, weight=weight, bias=bias, **how).double() * dy.double()).sum()  # noqa: E731
    _, stats = blocks.conv1d_norm_fwd(order(v["x"]), G, weight=v["weight"], bias=v["bias"], **how, want_stats=True)
    grads = dict(zip(v, blocks.conv1d_norm_bwd(dy, stats, order(v["x"]), G, weight=v["weight"], bias=v["bias"], **how)))
    for k in v:
        d = new(*v[k].shape) + grads[k].float() / grads[k].float().norm() * 3
        s = 1 / 64
        slope = (f(**{**v, k: v[k] + s * d}) - f(**{**v, k: v[k] - s * d})) / (2 * s)
        want = (grads[k].double() * d.double()).sum()
        assert abs(slope - want) <= 0.03 + 1e-3 * abs(want), (k, float(slope), float(want))


def test_streams(ops):
    """On a stream of the caller's, and two calls beside each other on two streams, with workspaces of their own."""
    _, blocks = ops
    gen = _gen(12)
    x = torch.randn(4, 64, 30011, generator=gen, device="cuda").bfloat16()
    tokens = torch.randint(0, 3000, (4, 30011), generator=gen, device="cuda")
    y, stats = blocks.conv1d_norm_fwd(x, 4, silu=True, want_stats=True)
    want = [y, blocks.conv1d_norm_bwd(x, stats, x, 4, silu=True)[0], blocks.conv1d_embed_bwd(x, tokens, 3000), blocks.conv1d_embed_bwd(x, tokens % 7, 7),
            blocks.conv1d_dropout(x, 0.3, 1)]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for s in (a, b, a, b):
        got.append([blocks.conv1d_norm_fwd(x, 4, silu=True, stream=s), blocks.conv1d_norm_bwd(x, stats, x, 4, silu=True, stream=s)[0],
                    blocks.conv1d_embed_bwd(x, tokens, 3000, stream=s), blocks.conv1d_embed_bwd(x, tokens % 7, 7, stream=s), blocks.conv1d_dropout(x, 0.3, 1, stream=s)])
    torch.cuda.synchronize()
    for outs in got:
        for g, w in zip(outs, want):
            assert torch.equal(g, w)


def test_workspaces_and_outputs_of_the_caller(ops):
    _, blocks = ops
    gen = _gen(13)
    x = torch.randn(2, 16, 9000, generator=gen, device="cuda")
    tokens = torch.randint(0, 2000, (2, 9000), generator=gen, device="cuda")
    room = torch.full((1 << 26,), 0xff, dtype=torch.uint8, device="cuda")
    wide = torch.full((2, 32, 9000), 7.0, device="cuda")
    y, stats = blocks.conv1d_norm_fwd(x, 2, want_stats=True)
    assert torch.equal(blocks.conv1d_norm_fwd(x, 2, out=wide[:, 16:], workspace=room), y)
    room.fill_(0xff)
    assert torch.equal(blocks.conv1d_norm_bwd(x, stats, x, 2, workspace=room)[0], blocks.conv1d_norm_bwd(x, stats, x, 2)[0])
    for last in (False, True):
        dy = x.transpose(1, 2).contiguous().transpose(1, 2) if last else x
        for V in (20, 2000):
            room.fill_(0xff)  # NaN, and keys and positions of -1
            assert torch.equal(blocks.conv1d_embed_bwd(dy, tokens % V, V, workspace=room), blocks.conv1d_embed_bwd(dy, tokens % V, V))
    table = torch.randn(2000, 16, generator=gen, device="cuda")
    assert torch.equal(blocks.conv1d_embed_fwd(table, tokens, out=wide[:, 16:]), blocks.conv1d_embed_fwd(table, tokens))
    assert torch.equal(blocks.conv1d_dropout(x, 0.5, 3, out=wide[:, 16:]), blocks.conv1d_dropout(x, 0.5, 3))
    assert (wide[:, :16] == 7).all()
    for call in (lambda: blocks.conv1d_norm_fwd(x, 2, out=x), lambda: blocks.conv1d_dropout(x, 0.5, 3, out=x), lambda: blocks.conv1d_norm_fwd(x, 2, workspace=room.cpu()),
                 lambda: blocks.conv1d_norm_fwd(x, 2, out=wide.transpose(1, 2).contiguous().transpose(1, 2)[:, 16:]), lambda: blocks.conv1d_norm_fwd(x, 5),
                 lambda: blocks.conv1d_norm_fwd(x[:, :, ::2], 2), lambda: blocks.conv1d_norm_bwd(x.transpose(1, 2).contiguous().transpose(1, 2), stats, x, 2),
                 lambda: blocks.conv1d_norm_fwd(x, 2, relu=True, silu=True), lambda: blocks.conv1d_embed_bwd(x, tokens[:1], 2000),
                 lambda: blocks.conv1d_embed_bwd(x, tokens.double(), 2000), lambda: blocks.conv1d_dropout(x, 1.5, 3), lambda: blocks.conv1d_dropout(x, 0.5, -1),
                 lambda: blocks.conv1d_dropout(x, 0.5, 1 << 64), lambda: blocks.conv1d_dropout(x, 0.5, 1, counter=torch.zeros((), device="cuda")),
                 lambda: blocks.conv1d_dropout(x, 0.5, 1, residual=x[:1]), lambda: blocks.conv1d_embed_fwd(table, tokens, out=x[:, :, :10])):
        with pytest.raises((ValueError, TypeError)):
            call()


def _row_kept(row, L):
    """The first 20 elements of a row at key 9, call 4, p = 1/2."""
    kept = []
    for block in range(row * -(-L // 4), row * -(-L // 4) + 5):
        c, k = [block & 0xffffffff, block >> 32, 4, 0], [9, 0]
        for _ in range(7):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [b >> 32 ^ c[1] ^ k[0], b & 0xffffffff, a >> 32 ^ c[3] ^ k[1], a & 0xffffffff]
            k = [k[0] + 0x9E3779B9 & 0xffffffff, k[1] + 0xBB67AE85 & 0xffffffff]
        kept += [w >= 2 ** 31 for w in c]
    return torch.tensor(kept, device="cuda")


def test_dropout_of_blocks_beyond_32_bits(ops):
    """One row, read for each of 18 (43 GB are written): the last ones' blocks have numbers of 33 bits."""
    _, blocks = ops
    L = 1 << 30
    x = torch.ones(1, 1, L, dtype=torch.bfloat16, device="cuda").expand(1, 18, L)
    y = blocks.conv1d_dropout(x, 0.5, 9, 4)
    for row in (0, 15, 16, 17):
        assert torch.equal(y[0, row, :20], 2.0 * _row_kept(row, L)), row


def test_offsets_beyond_32_bits(ops):
    """Tensors of more than 2^31 elements: their ends are what calls on the ends alone give."""
    _, blocks = ops
    N, C, L = 3, 1024, 700000                       # the last row begins behind element 2^31; 4.3 GB
    x = torch.empty(N, C, L, dtype=torch.bfloat16, device="cuda")
    for n in range(N):
        x[n].normal_(generator=_gen(n))
    y, stats = blocks.conv1d_norm_fwd(x, 4, silu=True, want_stats=True)
    assert torch.equal(y[2:], blocks.conv1d_norm_fwd(x[2:], 4, silu=True)) or (y[2:].float() - blocks.conv1d_norm_fwd(x[2:], 4, silu=True).float()).abs().max() <= 2.0 ** -6
    y = blocks.conv1d_dropout(x, 0.5, 9, 4)
    assert torch.equal(y[2, -1, :20], torch.where(_row_kept(N * C - 1, L), 2 * x[2, -1, :20], 0.0))
    del y
    # one token for each position of the last sample's end: its gradient is dy there
    V = 2000
    tokens = torch.zeros(N, L, dtype=torch.int64, device="cuda")
    tokens[2, -100:] = torch.arange(1900, 2000, device="cuda")
    lengths = torch.tensor([5, 0, L], dtype=torch.int32, device="cuda")
    lengths[2] = L
    dtable = blocks.conv1d_embed_bwd(x, tokens, V, lengths=lengths)
    assert torch.equal(dtable[1900:], x[2, :, -100:].float().T) and (dtable[1:1900] == 0).all()
    del dtable, x
    table = torch.randn(V, C, generator=_gen(5), device="cuda").bfloat16()
    y = blocks.conv1d_embed_fwd(table, tokens)
    assert torch.equal(y[2, :, -100:], table[1900:].T) and torch.equal(y[1, :, 7], table[0])


def test_autograd_of_broadcast_and_unusual_inputs(ops):
    """An input expanded over the batch, gradients that are expanded or transposed, parameters in other types, only some inputs that want
    a gradient, the modules."""
    autograd, blocks = ops
    gen = _gen(6)
    new = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    N, C, L = 3, 8, 37
    one = new(1, C, L).requires_grad_(True)
    weight = (1 + 0.1 * new(C)).bfloat16().requires_grad_(True)
    y = autograd.conv1d_norm(one.expand(N, C, L), 2, weight)
    g = new(N, L, C).transpose(1, 2)
    y.backward(g)
    full, weight2 = one.detach().expand(N, C, L).contiguous().requires_grad_(True), weight.detach().clone().requires_grad_(True)
    autograd.conv1d_norm(full, 2, weight2).backward(g.contiguous())
    assert torch.equal(one.grad, full.grad.sum(0, keepdim=True)) and torch.equal(weight.grad, weight2.grad) and weight.grad.dtype == torch.bfloat16
    table, tokens = new(5, C).requires_grad_(True), torch.randint(0, 5, (N, L), generator=gen, device="cuda")
    autograd.conv1d_embed(table, tokens).sum().backward()
    assert torch.equal(table.grad, torch.bincount(tokens.flatten(), minlength=5)[:, None].float().expand(5, C))
    x, r = new(N, C, L).requires_grad_(True), new(N, C, L).requires_grad_(True)
    lengths = torch.tensor([L, 0, 9], dtype=torch.int32, device="cuda")
    autograd.conv1d_dropout(x, 0.5, 1, residual=r, lengths=lengths).sum().backward()
    m = ref.inside(lengths, N, L).expand(N, C, L)
    kept = torch.tensor(ref.words(N * C, L, 1, 0), device="cuda").view(N, C, L) >= 2 ** 31
    assert torch.equal(r.grad, m.float()) and torch.equal(x.grad, 2.0 * (m & kept))
    counter = torch.zeros((), dtype=torch.int64, device="cuda")
    y = autograd.conv1d_dropout(x, 0.5, 1, counter=counter)
    counter.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    layer = autograd.Dropout(0.5, key=3)
    a, b = layer(x.detach()), layer(x.detach())
    assert not torch.equal(a, b) and torch.equal(b, blocks.conv1d_dropout(x.detach(), 0.5, 3, 1))
    again = autograd.Dropout(0.5, key=9)
    again.load_state_dict(layer.state_dict())
    assert torch.equal(again(x.detach()), layer(x.detach()))
    layer.eval()
    assert torch.equal(layer(x.detach(), residual=r.detach()), x.detach() + r.detach())
    norm, embed = autograd.GroupNorm(2, C, relu=True), autograd.Embedding(5, C, scale=2.0, dtype=torch.bfloat16)
    for last in (False, True):
        y = norm(embed(tokens, channels_last=last).float())
        assert (y >= 0).all()
        y.square().sum().backward()
    assert embed.weight.grad.dtype == torch.bfloat16 and norm.weight.grad.isfinite().all()
    assert torch.equal(embed.step(tokens[:, 0]), 2 * embed.weight.detach()[tokens[:, 0]])
    with torch.no_grad():
        assert not autograd.conv1d_norm(x, 2).requires_grad
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(autograd.conv1d_norm(x, 2).sum(), x, create_graph=True)
        g.sum().backward()
