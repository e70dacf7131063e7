"""The sequence operators together, as a network uses them: 1 x 1 layers, the causal convolution, the scan, gradients by autograd,
clipping; a prompt, then one position at a time.

The plain form is the same network of elementary operations in 64 bits on the same (rounded) inputs and weights.  In float32 every
product and sum is off by some roundings of 2^-24 of the values around it; a tensor's error is held to 2e-5 of its norm, a few
hundred of them.  In bfloat16 each of the ten tensors between the operators is rounded once, to 2^-8 of its values, and errors of
one place meet those of others at random: 10 * 2^-8 = 4 % of the norm.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 2e-5, torch.bfloat16: 10 * 2.0 ** -8}


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2104_08002_amd import autograd, binding, gradients, sequence

    binding.load()
    return autograd, sequence, gradients


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _network(dtype, gen, M=10, D=24, R=3, S=16, taps=4):
    """Weights of one block: M features in and out, D channels inside, R ranks of the steps."""
    def normal(*shape, std=1.0):
        return (std * torch.randn(shape, generator=gen, device="cuda"))
    p = {"w_in": normal(2 * D, M, 1, std=M ** -0.5).to(dtype), "taps": normal(D, taps, std=0.5).to(dtype), "w_x": normal(R + 2 * S, D, 1, std=D ** -0.5).to(dtype),
         "w_dt": normal(D, R, 1, std=R ** -0.5).to(dtype), "w_out": normal(M, D, 1, std=D ** -0.5).to(dtype), "bias": normal(D, std=0.1),
         "dt_bias": normal(D) - 2, "A_log": torch.log(torch.arange(1, S + 1, device="cuda").float()).repeat(D, 1) + normal(D, S, std=0.1), "skip": normal(D)}
    return {k: v.requires_grad_(True) for k, v in p.items()}, D, R, S


def _block(ops, p, sizes, x, dtype, lengths=None, states=None):
    autograd, _, _ = ops
    D, R, S = sizes
    low = dtype == torch.bfloat16
    xz = autograd.conv1d(x, p["w_in"], bf16_out=low)
    u, conv = autograd.conv1d_causal(xz[:, :D], p["taps"], p["bias"], silu=True, init=None if states is None else states[0], lengths=lengths, want_final=True)
    proj = autograd.conv1d(u, p["w_x"], bf16_out=low)
    dt = autograd.conv1d(proj[:, :R], p["w_dt"], bf16_out=low)
    y, ssm = autograd.conv1d_scan(u, dt, -torch.exp(p["A_log"]), proj[:, None, R:R + S], proj[:, None, R + S:], p["skip"], xz[:, D:], p["dt_bias"],
                                  softplus=True, init=None if states is None else states[1], lengths=lengths, want_final=True)
    return autograd.conv1d(y, p["w_out"], bf16_out=low), conv, ssm


def _plain(p, sizes, x, lengths=None):
    D, R, S = sizes
    p, x = {k: v.detach().double().requires_grad_(True) for k, v in p.items()}, x.double()
    N, _, L = x.shape
    inside = torch.arange(L, device="cuda") < (torch.full((N,), L, device="cuda") if lengths is None else lengths)[:, None]
    inside = inside[:, None].double()
    mix = lambda w, v: (w[:, :, 0][None] @ v)  # noqa: E731
    xz = mix(p["w_in"], x) * inside
    taps = p["taps"].shape[1]
    xe = torch.cat((xz.new_zeros(N, D, taps - 1), xz[:, :D]), 2)
    u = p["bias"][:, None] + sum(p["taps"][:, s, None] * xe[:, :, s:s + L] for s in range(taps))
    u = u * torch.sigmoid(u) * inside
    proj = mix(p["w_x"], u)
    e = torch.nn.functional.softplus(mix(p["w_dt"], proj[:, :R]) + p["dt_bias"][:, None], threshold=200) * inside
    A, h, ys = -torch.exp(p["A_log"]), x.new_zeros(N, D, S), []
    for t in range(L):
        h = torch.exp(e[:, :, t, None] * A) * h + (e[:, :, t] * u[:, :, t])[:, :, None] * proj[:, None, R:R + S, t]
        ys.append((proj[:, None, R + S:, t] * h).sum(2))
    z = xz[:, D:]
    y = (torch.stack(ys, 2) + p["skip"][:, None] * u) * z * torch.sigmoid(z) * inside
    return mix(p["w_out"], y), p


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,L,ragged", [(2, 70, False), (3, 133, True), (1, 1, False)])
def test_training_step(ops, dtype, N, L, ragged):
    gen = _gen(L)
    p, *sizes = _network(dtype, gen)
    x, gy = (torch.randn(N, 10, L, generator=gen, device="cuda").to(dtype) for _ in range(2))
    lengths = torch.tensor([L, 0, L // 2], dtype=torch.int32, device="cuda") if ragged else None
    out, _, _ = _block(ops, p, sizes, x, dtype, lengths)
    out.backward(gy)
    ref, q = _plain(p, sizes, x, lengths)
    ref.backward(gy.double())

    def near(name, got, want):
        assert (got.double() - want).norm() <= TOL[dtype] * want.norm() + 1e-30, (name, float((got.double() - want).norm() / want.norm()))

    near("out", out, ref.detach())
    for k in p:
        near(k, p[k].grad, q[k].grad)
    norm = torch.stack([v.grad.double().square().sum() for v in p.values()]).sum().sqrt()
    before = {k: v.grad.clone() for k, v in p.items()}
    got = ops[2].conv1d_grad_clip([v.grad for v in p.values()], 0.25)
    assert abs(float(got) - float(norm)) <= 2.0 ** -23 * float(norm)
    # the norm is rounded to float (2^-24), so is the factor, and the product to the gradient's type (eps / 2): in float 3 2^-24,
    # more than the eps of 2 2^-24 that stood here
    bound = lambda t: 1.01 * (torch.finfo(t).eps / 2 + 2 * 2.0 ** -24)  # noqa: E731
    for k, v in p.items():
        want = before[k].double() * min(1.0, 0.25 / (float(norm) + 1e-6))
        assert ((v.grad.double() - want).abs() <= bound(v.dtype) * want.abs() + 1e-37).all(), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_prompt_then_positions(ops, dtype):
    """A prompt in two parts of a batch whose sequences end at different places, then one position at a time: the same as each
    sequence whole."""
    autograd, sequence, _ = ops
    gen = _gen(4)
    p, *sizes = _network(dtype, gen)
    D, R, S = sizes
    N, L = 3, 40
    x = torch.randn(N, 10, L, generator=gen, device="cuda").to(dtype)
    low = dtype == torch.bfloat16
    with torch.no_grad():
        whole, _, _ = _block(ops, p, sizes, x, dtype)
        first, conv, ssm = _block(ops, p, sizes, x[:, :, :16].contiguous(), dtype)
        lengths = torch.tensor([5, 0, 14], dtype=torch.int32, device="cuda")
        second, conv, ssm = _block(ops, p, sizes, x[:, :, 16:30].contiguous(), dtype, lengths, (conv, ssm))
        scale = whole.float().abs().max()
        near = lambda a, b: bool(((a.float() - b.float()).abs() <= TOL[dtype] * scale).all())  # noqa: E731
        assert near(first, whole[:, :, :16])
        at = 16 + lengths.long()
        for n in range(N):
            assert near(second[n, :, :lengths[n]], whole[n, :, 16:at[n]])
        for _ in range(6):
            xt = x[torch.arange(N, device="cuda"), :, at][:, :, None].contiguous()
            xz = autograd.conv1d(xt, p["w_in"], bf16_out=low)
            u = sequence.conv1d_causal_step(xz[:, :D, 0], p["taps"], conv, bias=p["bias"], silu=True)
            proj = autograd.conv1d(u[:, :, None], p["w_x"], bf16_out=low)
            dt = autograd.conv1d(proj[:, :R], p["w_dt"], bf16_out=low)[:, :, 0]
            y = sequence.conv1d_scan_step(u, dt, -torch.exp(p["A_log"]), proj[:, None, R:R + S, 0], proj[:, None, R + S:, 0], ssm, skip=p["skip"],
                                          z=xz[:, D:, 0], dt_bias=p["dt_bias"], softplus=True)
            out = autograd.conv1d(y[:, :, None], p["w_out"], bf16_out=low)[:, :, 0]
            assert near(out, whole[torch.arange(N, device="cuda"), :, at])
            at += 1


def test_states_are_kept_for_a_graph_alone(ops):
    autograd, sequence, _ = ops
    gen = _gen(9)
    N, D, L, S = 2, 64, 4096, 16
    new = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    x, A, B = new(N, D, L), (-torch.rand(D, S, generator=gen, device="cuda")).requires_grad_(True), new(N, 1, S, L)
    saved = sequence.conv1d_scan_fwd(x, x, A.detach(), B, B, softplus=True, save=True)[2].numel()

    def most(fn):
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        out = fn()
        return torch.cuda.max_memory_allocated() - before, out

    with_graph, y = most(lambda: autograd.conv1d_scan(x, x, A, B, B, softplus=True))
    with torch.no_grad():
        without, y0 = most(lambda: autograd.conv1d_scan(x, x, A, B, B, softplus=True))
    assert y.requires_grad and not y0.requires_grad and torch.equal(y, y0)
    assert with_graph - without >= saved - 4096


def test_what_is_written_in_place_is_known_to_autograd(ops):
    """A state that a graph keeps and that is then moved on, a gradient that a graph keeps and that is then clipped: refused, not wrong."""
    autograd, sequence, gradients = ops
    gen = _gen(8)
    N, D, L, S = 2, 3, 5, 4
    new = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    x, A, B, w = new(N, D, L).requires_grad_(True), -torch.rand(D, S, generator=gen, device="cuda"), new(N, 1, S, L), new(D, S)
    state, before = new(N, D, S), new(N, D, S - 1)
    y = autograd.conv1d_scan(x, x, A, B, B, init=state)
    sequence.conv1d_scan_step(x[:, :, 0].detach().contiguous(), x[:, :, 0].detach().contiguous(), A, B[..., 0].contiguous(), B[..., 0].contiguous(), state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y = autograd.conv1d_causal(x, w, init=before)
    sequence.conv1d_causal_step(x[:, :, 0].detach().contiguous(), w, before)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    g = new(4)
    y = (x[0, 0, :4] * g).sum()
    gradients.conv1d_grad_clip([g], 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    out, seen = new(N, D, L), new(N, D, L).requires_grad_(True)
    y = (seen * out).sum()
    sequence.conv1d_causal_fwd(x.detach(), w, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():
        sequence.conv1d_causal_step(new(N, D), w, new(N, D, S - 1))
        gradients.conv1d_grad_clip([new(4)], 0.1)


def test_autograd_of_broadcast_and_unusual_inputs(ops):
    """An input expanded over the batch, a transposed one, a gradient that is expanded, parameters in other types, only some inputs
    that want a gradient."""
    autograd, _, _ = ops
    gen = _gen(6)
    N, D, L, S = 3, 5, 37, 4
    one = torch.randn(1, D, L, generator=gen, device="cuda", requires_grad=True)
    dt = torch.rand(N, L, D, generator=gen, device="cuda").transpose(1, 2)
    A = (-torch.rand(D, S, generator=gen, device="cuda").bfloat16()).requires_grad_(True)
    B, C = (torch.randn(N, 1, S, L, generator=gen, device="cuda") for _ in range(2))
    init = torch.randn(N, D, S, generator=gen, device="cuda").requires_grad_(True)
    y = autograd.conv1d_scan(one.expand(N, D, L), dt, A, B, C, init=init)
    y.sum().backward()
    assert one.grad.shape == one.shape and A.grad.dtype == torch.bfloat16 and dt.grad is None
    full = one.detach().expand(N, D, L).contiguous().requires_grad_(True)
    A2, init2 = A.detach().clone().requires_grad_(True), init.detach().clone().requires_grad_(True)
    autograd.conv1d_scan(full, dt.contiguous(), A2, B, C, init=init2).backward(torch.ones(N, D, L, device="cuda"))
    assert torch.equal(one.grad, full.grad.sum(0, keepdim=True)) and torch.equal(A.grad, A2.grad) and torch.equal(init.grad, init2.grad)
    layer = autograd.CausalConv1d(D, 4, silu=True)
    whole, state = layer(full.detach(), want_final=True)
    part, state1 = layer(full.detach()[:, :, :-1], want_final=True)
    assert torch.equal(layer.step(full.detach()[:, :, -1].contiguous(), state1), whole[:, :, -1]) and torch.equal(state, state1)
    x = full.detach().clone().requires_grad_(True)
    y, final = layer(x, init=torch.zeros(N, D, 3, device="cuda"), want_final=True)
    g, = torch.autograd.grad(final.sum(), x)
    want = torch.zeros_like(x)
    want[:, :, -3:] = 1
    assert torch.equal(g, want)
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(layer(x).sum(), x, create_graph=True)
        g.sum().backward()
    with torch.no_grad():
        assert not autograd.conv1d_scan(one.expand(N, D, L), dt, A, B, C, init=init).requires_grad


def test_training_step_captured(ops):
    """The whole step in a graph, replayed on new inputs with eager work between: gradients by torch.autograd.grad, with no eager graph
    of the same leaves alive."""
    autograd, _, gradients = ops
    gen = _gen(8)
    p, *sizes = _network(torch.bfloat16, gen)
    x, gy = (torch.randn(2, 10, 90, generator=gen, device="cuda").bfloat16() for _ in range(2))

    def step():
        out, _, _ = _block(ops, p, sizes, x, torch.bfloat16)
        grads = [g.clone() for g in torch.autograd.grad(out, list(p.values()), gy)]
        return [gradients.conv1d_grad_clip(grads, 0.5), out.detach()] + grads

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for turn in range(3):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        graph.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b), turn
