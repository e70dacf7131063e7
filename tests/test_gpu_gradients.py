"""The norm over many gradient tensors and clipping by it, against 64 bits, on the GPU.

Squares and their sums are in 64 bits, so the norm is off by its one rounding to float (and n 2^-53).  The factor is a float:
one rounding of the norm, one of the factor, one of the product to the tensor's type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def grad():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2104_08002_amd import binding, gradients

    binding.load()
    return gradients


def _tensors(sizes, types, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(scale * torch.randn(n, generator=gen, device="cuda")).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def _norm64(grads, kind):
    if kind == 2.0:
        return sum(float(g.double().square().sum()) for g in grads) ** 0.5
    return max([float(g.double().abs().max()) for g in grads if g.numel()] or [0.0])


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("types", [(F32,), (BF16,), (F32, BF16)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", [(1,), (7, 0, 9), (16384, 16385, 1, 16383), (3,) * 161, tuple(range(1, 500)), (1000003, 5, 70000)],
                         ids=["one", "empty", "pieces", "tables", "many", "large"])
@pytest.mark.parametrize("kind", [2.0, math.inf])
def test_norm_and_clip(grad, types, sizes, kind):
    grads = _tensors(sizes, types, len(sizes))
    ref = _norm64(grads, kind)
    norm = grad.conv1d_grad_norm(grads, kind)
    assert norm.dtype == F32 and norm.dim() == 0 and abs(float(norm) - ref) <= (U32 + 1e-12) * ref
    before = [g.clone() for g in grads]
    assert float(grad.conv1d_grad_clip(grads, 2 * ref + 1, kind)) == float(norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    limit = 0.3 * ref
    grad.conv1d_grad_clip(grads, limit, kind)
    factor = limit / (ref + 1e-6)
    for a, b in zip(grads, before):
        want = b.double() * factor
        u = torch.finfo(a.dtype).eps / 2
        assert ((a.double() - want).abs() <= (u + 4 * U32) * 1.01 * want.abs() + torch.finfo(a.dtype).tiny * u).all()


def test_values_whose_squares_are_no_floats(grad):
    big, small = torch.full((1000,), 2.0 ** 100, device="cuda"), torch.full((1000,), 2.0 ** -100, device="cuda")
    for t, v in ((big, 2.0 ** 100), (small, 2.0 ** -100)):
        want = v * 1000 ** 0.5
        assert abs(float(grad.conv1d_grad_norm([t])) - want) <= U32 * want
        assert float(grad.conv1d_grad_norm([t], math.inf)) == v


@pytest.mark.parametrize("kind", [2.0, math.inf])
@pytest.mark.parametrize("where", [0, 4097, 29999])
def test_nan_and_infinity(grad, kind, where):
    t = torch.ones(30000, device="cuda")
    t[where] = -math.inf
    assert float(grad.conv1d_grad_norm([t], kind)) == math.inf
    t[where] = math.nan
    t[(where + 1) % 30000] = math.inf
    assert math.isnan(float(grad.conv1d_grad_norm([torch.ones(5, device="cuda"), t, torch.ones(5, device="cuda")], kind)))
    ones = torch.ones(9, device="cuda")
    grad.conv1d_grad_clip([ones], 1.0, norm=torch.tensor(math.inf, device="cuda"))
    assert not ones.any()
    grad.conv1d_grad_clip([ones], 1.0, norm=torch.tensor(math.nan, device="cuda"))
    assert ones.isnan().all()


def test_unaligned_views_leave_their_neighbours(grad):
    for t in (F32, BF16):
        flat = _tensors((5000,), (t,), 3)[0]
        before = flat.clone()
        views = [flat[1:8], flat[9:2500], flat[2501:4999]]
        norm = _norm64(views, 2.0)
        got = grad.conv1d_grad_clip(views, 1.0)
        assert abs(float(got) - norm) <= (U32 + 1e-12) * norm
        keep = torch.tensor([0, 8, 2500, 4999], device="cuda")
        assert torch.equal(flat[keep], before[keep]) and not torch.equal(flat, before)


def test_any_dense_layout_and_none(grad):
    t = torch.randn(6, 5, 7, device="cuda")
    ref = _norm64([t], 2.0)
    assert abs(float(grad.conv1d_grad_norm([None, t.permute(2, 0, 1)])) - ref) <= (U32 + 1e-12) * ref
    assert float(grad.conv1d_grad_norm([])) == 0.0 and float(grad.conv1d_grad_norm([None])) == 0.0
    assert float(grad.conv1d_grad_clip([], 1.0)) == 0.0
    assert abs(float(grad.conv1d_grad_norm(t)) - ref) <= (U32 + 1e-12) * ref


def test_refusals(grad):
    from paper_2104_08002_amd.binding import Conv1dError

    t = torch.ones(10, device="cuda")
    for twice in ([t, t], [t[:6], t[5:]]):
        with pytest.raises(Conv1dError) as e:
            grad.conv1d_grad_clip(twice, 1.0)
        assert e.value.status == -1
    assert (t == 1).all()
    with pytest.raises(ValueError):
        grad.conv1d_grad_norm([t[::2]])
    with pytest.raises(ValueError):
        grad.conv1d_grad_norm([t.expand(3, 10)])
    with pytest.raises(ValueError):
        grad.conv1d_grad_norm([t.cpu()])
    with pytest.raises(TypeError):
        grad.conv1d_grad_norm([t.half()])
    with pytest.raises(ValueError):
        grad.conv1d_grad_norm([t], 1.0)
    with pytest.raises(ValueError):
        grad.conv1d_grad_clip([t], -1.0)
    with pytest.raises(ValueError):
        grad.conv1d_grad_clip([t], math.nan)
    with pytest.raises(ValueError):
        grad.conv1d_grad_clip([t], 1.0, norm=torch.ones(2, device="cuda"))


def test_captured_and_replayed(grad):
    grads = _tensors((70000, 3, 1001), (F32, BF16), 1)
    source = [g.clone() for g in grads]
    grad.conv1d_grad_clip(grads, 1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = grad.conv1d_grad_clip(grads, 1.0)
    for turn in range(3):
        for g, s in zip(grads, source):
            g.copy_(s * (turn + 1))
        graph.replay()
        again = [(s * (turn + 1)).to(s.dtype) for s in source]
        want = grad.conv1d_grad_clip(again, 1.0)
        assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(grads, again))
