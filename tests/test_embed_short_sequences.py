"""The embedding's gradient of many short sequences, whose every sample is a block of its own to the product, and of many tokens on few positions, whose
sums are many to join: sorted where that is much faster."""
import pytest
import torch

from test_embed_long_sums import _chunks

SORTED = [(20000, 8, 16, 600), (20000, 16, 16, 256), (20000, 64, 16, 64), (100000, 64, 4, 64), (20000, 128, 16, 20), (4000, 300, 16, 30), (20000, 8, 64, 600), (4000, 64, 4, 64),
          (2, 110, 2, 31203), (1, 55, 26, 23921), (3, 56, 5, 23834)]
PRODUCT = [(1000, 64, 200, 64), (16, 64, 100, 64), (2000, 16, 100, 64), (100000, 16, 4, 16), (300, 16, 60, 5)]


@pytest.mark.parametrize("sizes", SORTED)
def test_many_short_sequences_are_sorted(sizes):
    assert _chunks(*sizes, torch.bfloat16) is None


@pytest.mark.parametrize("sizes", PRODUCT + [(16, 15, 60000, 5), (8, 512, 8192, 128), (12, 49, 4999, 257), (160, 16, 1 << 20, 64)])
def test_others_are_a_product(sizes):
    assert _chunks(*sizes, torch.bfloat16) is not None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,L,V", [(20000, 8, 16, 600), (4000, 64, 4, 64), (4000, 64, 3, 64), (2000, 16, 100, 64), (30001, 16, 2, 16), (700, 70, 33, 40), (2, 110, 2, 31203), (300, 16, 1500, 5), (900, 16, 513, 16)])
def test_values(dtype, N, D, L, V):
    """Both ways, several samples a workgroup among them, some sequences empty.  (83 u: see test_embed_long_sums.)"""
    from paper_2104_08002_amd import blocks

    import blocks_reference as ref

    gen = torch.Generator(device="cuda").manual_seed(N + L)
    tokens = torch.randint(-1, V + 1, (N, L), generator=gen, device="cuda")
    lengths = torch.tensor([(L, 0, L // 2, 1, L + 5, -3, L)[n % 7] for n in range(N)], dtype=torch.int32, device="cuda")
    inside = ref.inside(lengths, N, L)
    dy = torch.where(inside, torch.randn(N, D, L, generator=gen, device="cuda"), float("nan")).to(dtype)
    want, size = ref.embed_grad(torch.where(inside, dy, 0.0), tokens, V, 1.25, lengths)
    ref.near(blocks.conv1d_embed_bwd(dy, tokens, V, scale=1.25, lengths=lengths), want, 83 * ref.U * size)
