"""Behind the end of a sequence gradients are 0, whatever became of the sequence itself."""
import math

import pytest
import torch

from test_gpu_sequence import _gen, _normal, _scan_case, seq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D,L,S", [(3, 37, 16), (3, 1300, 16), (70, 90, 16), (300, 40, 4), (9, 90, 40), (3, 41, 24)])  # (one workgroup a group, and several)
@pytest.mark.parametrize("what", ["nan", "inf", "overflow", "dfinal"])
def test_a_bad_sequence_ends_at_its_end(seq, dtype, D, L, S, what):  # noqa: F811
    """NaN or infinity in an input, a state that leaves FP32's range, a gradient of the final state that is NaN."""
    gen = _gen(D + L + S)
    N = 3
    c = _scan_case(gen, dtype, N, D, L, S, 1)
    lengths = torch.tensor([L - 9, L // 2, 0], dtype=torch.int32, device="cuda")
    dy, dfinal = _normal(gen, N, D, L).to(dtype), _normal(gen, N, D, S)
    c["x"] = c["x"].clone()
    if what == "nan":
        c["x"][0, 1, 5] = math.nan
    elif what == "inf":
        c["x"][0, 1, 5] = math.inf
    elif what == "overflow":
        c["x"][0, 1, 5] = 3e38
        c["dt"][0, 1, 5] = 100.0
    else:
        dfinal[0, 1, 0] = math.nan
    behind = torch.arange(L, device="cuda") >= lengths[:, None]
    y, _, saved = seq.conv1d_scan_fwd(**c, lengths=lengths, want_final=True, save=True)
    g = seq.conv1d_scan_bwd(dy, saved, **c, lengths=lengths, dfinal=dfinal, want_init=True)
    assert not (torch.isfinite(y).all() and torch.isfinite(g.dC).all() and torch.isfinite(g.dB).all())
    for name, v in (("y", y), ("dx", g.dx), ("ddt", g.ddt), ("dz", g.dz), ("dB", g.dB), ("dC", g.dC)):
        part = v.movedim(-1, 1)[behind]
        assert torch.equal(part, torch.zeros_like(part)), (name, int((part != 0).sum()))
    for name, v in (("y", y), ("dx", g.dx), ("ddt", g.ddt), ("dz", g.dz), ("dB", g.dB), ("dC", g.dC)):
        assert v[1:].isfinite().all(), name
