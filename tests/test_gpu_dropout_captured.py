"""A module that is used several times in a captured step: with a counter that moves by as many as its calls, every use of every replay drops
other elements, and those that the functional form drops at call + counter."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("uses", [1, 3])
@pytest.mark.parametrize("checkpointed", [False, True])
def test_uses_of_all_replays_differ(uses, checkpointed):
    from paper_2104_08002_amd import autograd, blocks

    layer = autograd.Dropout(0.5, key=11)
    counter = torch.zeros((), dtype=torch.int64, device="cuda")
    x = torch.ones(2, 5, 203, device="cuda").requires_grad_(True)
    calls = []

    def use(call):
        calls.append(call)
        if checkpointed:
            return torch.utils.checkpoint.checkpoint(lambda v: layer(v, counter=counter, call=call).sin(), x, use_reentrant=False, preserve_rng_state=False)
        return layer(x, counter=counter, call=call).sin()

    def step():
        calls.clear()
        ys = [use(layer.next_call()) for _ in range(uses)]
        grads = [torch.autograd.grad(y.sum(), x)[0] for y in ys]
        counter.add_(uses)
        return [y.detach() for y in ys], grads

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    counter.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys, grads = step()
    counter.zero_()
    seen = []
    for replay in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert counter == (replay + 1) * uses
        for y, g, call in zip(ys, grads, calls):
            want = blocks.conv1d_dropout(x.detach(), 0.5, 11, call + replay * uses)
            # (the sine and its slope by the same torch calls on the same numbers)
            assert torch.equal(y, want.sin()) and torch.equal(g, blocks.conv1d_dropout(want.cos(), 0.5, 11, call + replay * uses))
            seen.append(y.clone())
    for a, b in itertools.combinations(seen, 2):
        assert 0.3 < ((a == 0) == (b == 0)).float().mean() < 0.7   # 2030 elements, alike by chance: 1/2 and 18 deviations
