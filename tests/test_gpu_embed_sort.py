"""The embedding's gradient by sorted tokens, whatever sizes the product is taken for: channels contiguous are always sorted, and so are more tokens
than 16 bits number.  Keys of four a lane and places by a launch of their own (many positions), runs over many workgroups, channels that
divide a workgroup's lanes unevenly or fill more than one."""
import pytest
import torch

import blocks_reference as ref
from test_gpu_blocks import _gen, _normal, _put, _tokens

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
# 31 sums of up to 32 rows in float, what of a run lies in a workgroup, the product with the scale, and one more
SORTED = 34 * ref.U
MOST_FEW, MANY_KEYS, MANY_TILES = 65520, 256 * 1024, 256 * 4 * 1024   # tokens of the product; positions of one key a lane, of summed counts


@pytest.fixture(scope="module")
def blocks():
    from paper_2104_08002_amd import binding, blocks

    binding.load()
    return blocks


def _check(blocks, dy, tokens, V, lengths=None, scale=0.5):
    from paper_2104_08002_amd import binding

    N, D, L = dy.shape
    bf16 = int(dy.dtype == torch.bfloat16)
    # sorted: four arrays of all positions, and dy's rows where they have to be made
    room = binding.load().conv1d_embed_bwd_workspace_bytes(N, D, L, V, bf16, *dy.stride()[1:])
    assert room >= 16 * N * L + (N * L * -(-D // 8) * 8 * dy.element_size() if dy.stride(2) == 1 else 0)
    if dy.stride(2) == 1:
        assert V > MOST_FEW
    want, size = ref.embed_grad(dy, tokens, V, scale, lengths)
    got = blocks.conv1d_embed_bwd(dy, tokens, V, scale=scale, lengths=lengths)
    ref.near(got, want, SORTED * size)
    assert torch.equal(got, blocks.conv1d_embed_bwd(dy, tokens, V, scale=scale, lengths=lengths))


def _dominant(gen, N, L, V, token):
    """One token on all but each 997th position."""
    t = torch.full((N, L), token, device="cuda")
    t[:, ::997] = torch.randint(0, V, t[:, ::997].shape, generator=gen, device="cuda")
    return t


# D: lane groups of 3, 5, 13 and 88 lanes leave some of 256 idle; 2100 channels take two workgroups and two turns of the join
WIDE = [(4, 24, 100000), (3, 40, 9000), (2, 100, 5001), (2, 700, 1500), (2, 2100, 700), (1, 9, 300000)]


@TYPES
@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
@pytest.mark.parametrize("N,D,L", WIDE)
def test_runs_over_many_workgroups(blocks, dtype, last, N, D, L):
    gen = _gen(D)
    V = 9 if last else MOST_FEW + 9
    for token in (0, V - 1):
        dy = _put(_normal(gen, N, D, L).to(dtype), last)
        _check(blocks, dy, _dominant(gen, N, L, V, token), V)


@TYPES
@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
@pytest.mark.parametrize("kind", ["plain", "skewed", "outside"])
@pytest.mark.parametrize("N,D,L", [(4, 24, 100000), (3, 5, 400001), (1, 17, MANY_KEYS), (1, 3, MANY_KEYS + 1), (1, 2, MANY_TILES), (1, 2, MANY_TILES + 1)])
def test_many_positions(blocks, dtype, last, kind, N, D, L):
    """Random tokens where a lane sorts four keys (above 2^18 positions) and where counts are made into places by a launch (above 2^20)."""
    gen = _gen(L)
    V = 5000 if last else 70000
    lengths = torch.tensor([(L, L - 3, L // 2, 0)[n % 4] for n in range(N)], dtype=torch.int32, device="cuda")
    _check(blocks, _put(_normal(gen, N, D, L).to(dtype), last, padded=True), _tokens(gen, N, L, V, kind, wide=D % 2 == 0), V, lengths)


@pytest.mark.parametrize("V", [1, 2, 254, 255, 256, 257, 65535, 65536, 1 << 20])
@pytest.mark.parametrize("L", [6000, MANY_KEYS // 2 + 100])
def test_as_many_tokens_as_digits_hold(blocks, V, L):
    """Keys 0 ... V fill 8 bits at V = 255 and begin a second pass at 256."""
    gen = _gen(V)
    tokens = torch.cat((torch.randint(0, V, (2, L - 3), generator=gen, device="cuda"), torch.tensor([[0, V - 1, V], [V - 1, 0, -1]], device="cuda")), 1)
    _check(blocks, _put(_normal(gen, 2, 3, L), True), tokens, V)


@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
def test_gradients_beyond_32_bits(blocks, last):
    """dy of more than 2^31 elements: the one long run, the rows of single positions at its end, and the rows that no token has."""
    N, D, L, V = 3, 1024, 700000, 2000
    dy = torch.empty((N, L, D) if last else (N, D, L), dtype=torch.bfloat16, device="cuda")
    for n in range(N):
        dy[n].normal_(generator=_gen(n))
    dy = dy.transpose(1, 2) if last else dy
    tokens = torch.zeros(N, L, dtype=torch.int32, device="cuda")
    tokens[2, -100:] = torch.arange(1900, 2000, device="cuda")
    lengths = torch.tensor([5, 0, L], dtype=torch.int32, device="cuda")
    dtable = blocks.conv1d_embed_bwd(dy, tokens, V, lengths=lengths)
    assert torch.equal(dtable[1900:], dy[2, :, -100:].float().T) and (dtable[1:1900] == 0).all()
    want, size = (sum(f(dy[n, :, a:b].double()).sum(1) for n, a, b in [(0, 0, 5)] + [(2, a, min(a + 100000, L - 100)) for a in range(0, L - 100, 100000)])
                  for f in (lambda v: v, torch.abs))
    ref.near(dtable[0], want, SORTED * size)
