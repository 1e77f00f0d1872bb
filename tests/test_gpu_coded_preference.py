"""examples/coded_preference.py: training a head with the operators under gradient coding."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    spec = importlib.util.spec_from_file_location("coded_preference", os.path.join(ROOT, "examples", "coded_preference.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("scheme,n,c", [("FR", 4, 2), ("CR", 6, 3)])
def test_training_ranks_the_pairs_and_raises_the_preferred_answers(example, scheme, n, c):
    print("\n[gpu case] coded preference", scheme, flush=True)
    out = example.train(scheme, n, c)
    first, last = out["preference"][0], sum(out["preference"][-5:]) / 5
    assert abs(first - 0.693) < 0.15          # nothing is learned yet: h is dropout's noise around 0
    assert last < 0.5 * first and out["accuracy"] > 0.9
    assert out["policy"][-1] < out["policy"][0]


def test_fr_training_is_the_same_for_every_set_of_stragglers(example):
    """FR decodes one word per group, and a group's workers send identical words: the parameters agree
    to the last bit, dropout included."""
    print("\n[gpu case] coded preference, stragglers", flush=True)
    runs = [example.train("FR", 4, 2, steps=8, policy_steps=4, mask_seed=s)["w"] for s in (3, 4)]
    assert torch.equal(runs[0], runs[1])


def test_a_partition_has_one_gradient_whoever_evaluates_it(example):
    """Alone, among other rows and in another order: the logits' gradients of the same tokens agree."""
    print("\n[gpu case] one gradient per partition", flush=True)
    from paper_2607_20739_amd import ops
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    h = torch.randn(50, 64, generator=g, device="cuda").to(torch.bfloat16)
    numbers = torch.randint(0, 1 << 40, (50,), generator=g, device="cuda")
    whole = ops.dropout(h, 0.2, 5, row_ids=numbers)
    part = ops.dropout(h[20:31], 0.2, 5, row_ids=numbers[20:31])
    assert torch.equal(whole[20:31], part)
    back = torch.arange(49, -1, -1, device="cuda")
    assert torch.equal(ops.dropout(h[back], 0.2, 5, row_ids=numbers[back]), whole[back])
