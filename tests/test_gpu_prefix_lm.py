"""The prefix language model of examples/prefix_lm.py: its operators together in training and in generation."""
import importlib.util
import os

import pytest

from tests.gpu_util import announce, torch_cuda

pytestmark = pytest.mark.gpu


def _example():
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "prefix_lm.py")
    spec = importlib.util.spec_from_file_location("prefix_lm", at)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_training_and_generation():
    """The loss falls below half of what guessing costs (log 32), generation against the cache gives the packed
    pass's logits (fp32 sums in another order through two layers: 1e-4 of their size), and most tokens continue the
    pattern."""
    torch = torch_cuda()
    announce("prefix language model, 200 steps")
    E = _example()
    model, losses = E.train(200, torch.float32)
    assert abs(losses[0] - 3.47) < 1.5 and sum(losses[-10:]) / 10 < 1.73
    prompts = torch.randint(0, E.VOCAB, (4, E.PERIOD), generator=torch.Generator().manual_seed(5)).cuda()
    got, logits = E.generate(model, prompts, 2 * E.PERIOD)
    assert (got == prompts.repeat(1, 2)).float().mean() > 0.5
    whole = torch.cat([prompts, got], 1)[:, :-1]
    with torch.no_grad():
        seq = E.Packed([whole.shape[1]] * 4, [E.PERIOD] * 4)
        full = model.packed(whole.flatten().contiguous(), seq).view(4, -1, E.VOCAB)[:, E.PERIOD - 1:]
    assert float((full - logits).abs().max()) <= 1e-4 * float(full.abs().max())


def test_same_run_again():
    """Twenty bf16 steps give the same losses twice where torch's own kernels do: the operators add no disorder."""
    torch = torch_cuda()
    announce("prefix language model, bf16, twice")
    E = _example()
    torch.use_deterministic_algorithms(True, warn_only=True)
    try:
        a, b = (E.train(20, torch.bfloat16)[1] for _ in range(2))
    finally:
        torch.use_deterministic_algorithms(False)
    assert all(x == x for x in a) and a == b
