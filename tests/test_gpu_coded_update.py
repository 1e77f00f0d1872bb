"""examples/coded_preference.py with the scores' entropy, the gradients' norm and the AdamW step: what coding promises holds
for every update, and the gradient with the bonus is that of the formula."""

import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import ops as O

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    spec = importlib.util.spec_from_file_location("coded_preference_update", os.path.join(ROOT, "examples", "coded_preference.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("optimizer", ["sgd", "adamw", "adamw8"])
def test_every_set_of_stragglers_gives_the_same_parameters(example, optimizer):
    print("\n[gpu case] coded update", optimizer, flush=True)
    runs = [example.train("FR", 4, 2, steps=6, policy_steps=5, mask_seed=s, optimizer=optimizer, entropy=0.05) for s in (3, 4)]
    assert torch.equal(runs[0]["w"], runs[1]["w"]) and runs[0]["entropy"] == runs[1]["entropy"]
    assert np.isfinite(runs[0]["policy"]).all() and 0 < runs[0]["entropy"] < np.log(1000) + 1e-3 and 0 <= runs[0]["first"] <= 1
    one = example.train("FR", 4, 2, steps=6, policy_steps=5, optimizer=optimizer, entropy=0.05, each_worker=True)
    assert torch.equal(one["w"], runs[0]["w"])


@pytest.mark.parametrize("scheme,n,c", [("FR", 4, 2), ("CR", 6, 3)])
def test_workers_and_updates_run_under_both_codes(example, scheme, n, c):
    print("\n[gpu case] coded update", scheme, flush=True)
    out = example.train(scheme, n, c, steps=3, policy_steps=2, optimizer="adamw8", entropy=0.01)
    assert len(out["preference"]) == 3 and len(out["policy"]) == 2 and torch.isfinite(out["w"]).all()


def test_the_update_is_the_oracles(example):
    """The norm bounded, then the step: against 64 bits.  The gradient g is clipped by a factor of error 2 u; m', v' and the step
    carry some 30 u of the step, x' two roundings more."""
    print("\n[gpu case] coded update, one step", flush=True)
    u = 2.0 ** -24
    head = example.Head(16, 50, "cuda")
    for how in ("adamw", "adamw8"):
        update = example.Update(head, how, max_norm=0.5)
        w = head.w.clone()
        x, m, v = w.double().cpu().numpy(), 0.0, 0.0
        for step in (1, 2) if how == "adamw" else (1,):
            g = torch.randn(w.numel(), device="cuda", generator=torch.Generator("cuda").manual_seed(step))
            factor = O.grad_norm([g.double().cpu().numpy()], 0.5)[1]
            update(w, g, 0.1)
            x, m, v = O.adamw(x, g.double().cpu().numpy(), m, v, step, 0.01, weight_decay=0.01, factor=factor)
            off = np.abs(w.double().cpu().numpy() - x)
            assert (off <= step * (0.011 * 40 * u + 4 * u * np.abs(x))).all(), (how, step, off.max())


def test_the_gradient_with_a_bonus_is_that_of_differences(example):
    """Of the mean policy loss less the weighted entropy, along a direction, in 32-bit logits: differences of the oracle with a step
    of 1e-4 (truncation of order 1e-8, times third derivatives below 100 of 60 rows' means) and 32-bit sums."""
    print("\n[gpu case] entropy bonus gradient", flush=True)
    ops = example.ops
    rng = np.random.default_rng(4)
    rows, cols, weight, step = 60, 130, 0.3, 1e-4
    z = torch.from_numpy(rng.normal(size=(rows, cols))).float()
    y = rng.integers(-1, cols, rows).astype(np.int32)
    z64 = z.double().numpy()
    old = (O.token_logprobs(z64, y) - rng.choice([-0.5, -0.1, 0.1, 0.5], rows)).astype(np.float32)
    adv, d = rng.normal(size=rows).astype(np.float32), rng.normal(size=(rows, cols))
    zg, yg = z.cuda(), torch.from_numpy(y).cuda()
    _, _, dz = ops.policy_loss(zg, yg, torch.from_numpy(old).cuda(), torch.from_numpy(adv).cuda(), scale=1.0 / rows)
    _, h, _, _, stats = ops.token_scores(zg, yg)
    dz += ops.token_scores_backward(zg, yg, stats, h, grad_entropy=torch.full_like(h, -weight / rows))

    def value(x):
        return (O.policy(x, y, old, adv)[0].sum() - weight * O.entropy(x, y).sum()) / rows
    want = (value(z64 + step * d) - value(z64 - step * d)) / (2 * step)
    assert abs((dz.double().cpu().numpy() * d).sum() - want) < 1e-6
