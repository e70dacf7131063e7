"""The embedding's gradient by a product: how many sums a wave adds in float before 64 bits take over.  Without a GPU by the workspace that a
call asks for, which holds the partial sums; on the GPU by gradients whose float sums are all rounded to one side."""
import pytest
import torch

from paper_2104_08002_amd import binding

U = 2.0 ** -24
WAVES, STEP, MOST = 4, 32, 16          # waves of a workgroup, positions of an instruction, additions of a wave in float
BF16 = {torch.bfloat16: 1, torch.float32: 0}


def _up(n, to):
    return -(-n // to) * to


def _chunks(N, D, L, V, dtype):
    """Workgroups' shares of the positions in the product's plan; None where the positions are sorted: with positions contiguous that takes room for
    dy's rows more than with channels contiguous."""
    have, last = (binding.load().conv1d_embed_bwd_workspace_bytes(N, D, L, V, BF16[dtype], *s) for s in ((L, 1), (1, max(2, D))))
    if have - last == _up(N * L * _up(D, 8) * dtype.itemsize, 256):
        return None
    assert have % (4 * _up(V, 16) * _up(D, 16)) == 0
    return have // (4 * _up(V, 16) * _up(D, 16))


def _steps(L, U4):
    """Additions that a sample of L positions costs the first wave of a workgroup, which takes U4 of each block's steps."""
    block = WAVES * STEP * U4
    return L // block * U4 + min(U4, -(-(L % block) // STEP))


# (L2-sized and long sequences, few and many tokens and channels, sequences shorter than a block)
SIZES = [(64, 8, 60001, 600), (8, 128, 60001, 64), (1, 1, 1 << 28, 600), (1, 16, 1 << 28, 64), (8, 512, 8192, 128), (16, 15, 60000, 5), (12, 49, 4999, 257), (64, 16, 60001, 256),
         (100000, 64, 4, 64), (3000, 16, 100, 16), (1 << 20, 8, 2, 16), (700, 64, 513, 64), (1, 16, 5000, 60000), (160, 16, 1 << 20, 64)]


@pytest.mark.parametrize("dtype", BF16, ids=["bf16", "f32"])
@pytest.mark.parametrize("N,D,L,V", SIZES)
def test_float_sums_are_short(N, D, L, V, dtype):
    chunks = _chunks(N, D, L, V, dtype)
    if chunks is None:
        return  # sorted: 16 or 32 rows in float
    U4 = {(1, True): 4, (1, False): 2, (4, True): 2, (4, False): 1}[1 if D <= 16 else 4, dtype == torch.bfloat16]
    if chunks < N:
        samples = -(-N // chunks)
        assert samples * _steps(L, U4) <= MOST
    else:
        per_sample = chunks // N
        assert chunks == N * per_sample and -(-L // per_sample) <= MOST * WAVES * STEP


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,L,V", [(160, 16, 1 << 20, 64), (64, 1, 1 << 20, 600), (500, 3, 400000, 20)])
def test_sums_that_are_rounded_to_one_side(dtype, N, D, L, V):
    """Every 32 positions add up to v or 32 v, of which float sums lose a quarter of a step each time on average (640 of them: 160 u).
    An instruction's 31 additions are cut off by less than 2 u each, the parts of a float are added; 16 of a wave, four waves; the scale: 83 u."""
    from paper_2104_08002_amd import blocks

    v = float.fromhex("0x1.b39ap0")
    if dtype == torch.bfloat16:
        h = float(torch.tensor(v).bfloat16())
        row = torch.zeros(L, device="cuda")
        row[::32], row[1::32] = h, v - h
    else:
        row = torch.full((L,), v, device="cuda")
    row = row.to(dtype)
    token = torch.full((L,), V - 1, dtype=torch.int32, device="cuda")
    got = blocks.conv1d_embed_bwd(row.expand(N, D, L), token.expand(N, L), V)
    want = N * row.double().sum()
    assert ((got[V - 1].double() - want).abs() <= (83 + 1) * U * N * row.double().abs().sum()).all(), (got[V - 1].double() / want - 1) / U
    assert (got[:V - 1] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,L,V", [(3, 5, 1500003, 7), (20, 16, 300001, 3), (5, 20, 1000000, 40)])
def test_values_of_many_chunks(dtype, N, D, L, V):
    """Chunks that are joined in several slices: values, and numbers that are not finite in their own places alone."""
    from paper_2104_08002_amd import blocks

    import blocks_reference as ref

    assert _chunks(N, D, L, V, dtype) > 2048
    gen = torch.Generator(device="cuda").manual_seed(L)
    tokens = torch.randint(0, V, (N, L), generator=gen, device="cuda")
    lengths = torch.tensor([(L, L - 5, L // 3)[n % 3] for n in range(N)], dtype=torch.int32, device="cuda")
    dy = torch.randn(N, D, L, generator=gen, device="cuda").to(dtype)
    want, size = ref.embed_grad(dy, tokens, V, 0.75, lengths)
    got = blocks.conv1d_embed_bwd(dy, tokens, V, scale=0.75, lengths=lengths)
    ref.near(got, want, 83 * U * size)
    assert torch.equal(got, blocks.conv1d_embed_bwd(dy, tokens, V, scale=0.75, lengths=lengths))
    inf = float("inf")
    for bad in ((inf,), (inf, inf), (inf, -inf), (float("nan"),)):
        z, t = dy.clone(), tokens.clone()
        for at, v in zip(((0, 2, 77), (1, 2, L - 9)), bad):
            z[at], t[at[0], at[2]] = v, 1
        got, fine = blocks.conv1d_embed_bwd(z, t, V, lengths=lengths), blocks.conv1d_embed_bwd(dy, t, V, lengths=lengths)
        fine[1, 2] = sum(bad)
        assert torch.equal(got.nan_to_num(1e30, 2e30, 3e30), fine.nan_to_num(1e30, 2e30, 3e30)), bad
