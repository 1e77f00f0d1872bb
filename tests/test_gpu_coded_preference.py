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


class _Among:
    """The operators as a worker calls them that has the rows in an order of its own, among rows of other partitions;
    each call has another order.  Results come back in the caller's order."""

    def __init__(self, real):
        self.real, self.calls = real, 0

    def __getattr__(self, name):
        return getattr(self.real, name)

    def _order(self, count, extra):
        """Places in [rows, `extra` others] in an order by chance, and where the rows are in it."""
        self.calls += 1
        order = torch.randperm(count + extra, generator=torch.Generator().manual_seed(self.calls)).cuda()
        return order, torch.argsort(order)[:count]

    def dropout(self, x, p, seed, residual, row_ids):
        extra = 3 + self.calls % 40
        order, back = self._order(len(x), extra)
        other = torch.randn(extra, x.shape[1], device=x.device).to(x.dtype)
        ids = torch.cat([row_ids, -1 - torch.arange(extra, device=x.device)])
        return self.real.dropout(torch.cat([x, other])[order], p, seed, residual=torch.cat([residual, other])[order],
                                 row_ids=ids[order])[back]

    def preference_loss(self, z, targets, offsets, ref, **kw):
        pairs, o = (len(offsets) - 1) // 2, offsets.tolist()
        order, back = self._order(pairs, self.calls % 30)
        order = [int(i) if i < pairs else 0 for i in order]        # the others: copies of the first, in another row's place
        rows = torch.cat([torch.arange(o[2 * i], o[2 * i + 2]) for i in order]).cuda()
        lengths = [o[2 * i + k + 1] - o[2 * i + k] for i in order for k in (0, 1)]
        ends = torch.tensor([0] + lengths).cumsum(0)
        value, margins, lp, dz = self.real.preference_loss(z[rows], targets[rows], ends.to(torch.int32).cuda(), ref[rows], **kw)
        mine = torch.cat([torch.arange(int(ends[2 * b]), int(ends[2 * b + 2])) for b in back.tolist()]).cuda()
        return value[back], margins[back], lp[mine], None if dz is None else dz[mine]

    def policy_loss(self, z, targets, old, advantages, ref_logprobs, **kw):
        extra = 5 + self.calls % 50
        order, back = self._order(len(z), extra)

        def among(t):
            return torch.cat([t, t[:1].expand(extra, *t.shape[1:])])[order]
        value, lp, dz = self.real.policy_loss(among(z), among(targets), among(old), among(advantages),
                                              ref_logprobs=among(ref_logprobs), **kw)
        return value[back], lp[back], dz[back]


def test_every_worker_sends_the_same_word_whatever_rows_it_has_beside(example, monkeypatch):
    """Each worker evaluates its own copies, in an order of its own and among other rows: an FR group's words are equal
    bit for bit at every step, and the parameters are those of training with one evaluation for all."""
    print("\n[gpu case] coded preference, each worker", flush=True)
    kw = dict(steps=6, policy_steps=5)
    want = example.train("FR", 4, 2, **kw)["w"]
    among = _Among(example.ops)
    monkeypatch.setattr(example, "ops", among)
    out = example.train("FR", 4, 2, each_worker=True, **kw)
    assert among.calls > 100 and len(out["words"]) == 11
    for words in out["words"]:
        assert torch.equal(words[0], words[1]) and torch.equal(words[2], words[3]) and not torch.equal(words[0], words[2])
    assert torch.equal(out["w"], want)


def test_workers_that_evaluate_for_themselves_train_the_same_cyclic_code(example):
    print("\n[gpu case] coded preference, each worker, CR", flush=True)
    kw = dict(steps=5, policy_steps=4)
    a, b = (example.train("CR", 6, 3, each_worker=e, **kw)["w"] for e in (False, True))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [9, 1000, 9001])
def test_sequences_have_one_gradient_whoever_evaluates_them(example, dtype, vocab):
    """Both losses' values and logits' gradients of the same sequences, alone and among others."""
    print("\n[gpu case] one gradient", dtype, vocab, flush=True)
    ops = example.ops
    among = _Among(ops)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rows = 30
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 2).to(dtype)
    y = torch.randint(-1, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    ref, adv = torch.randn(rows, generator=g, device="cuda") - 5, torch.randn(rows, generator=g, device="cuda")
    offsets = torch.tensor([0, 4, 9, 9, 17, 24, 30], dtype=torch.int32, device="cuda")
    for _ in range(6):
        among.calls += 5
        for a, b in zip(among.preference_loss(z, y, offsets, ref, beta=0.3, scale=0.5), ops.preference_loss(z, y, offsets, ref, beta=0.3, scale=0.5)):
            assert torch.equal(a, b)
        for a, b in zip(among.policy_loss(z, y, ref, adv, ref, kl=0.1), ops.policy_loss(z, y, ref, adv, ref, kl=0.1)):
            assert torch.equal(a, b)
        h = torch.randn(rows, 33, generator=g, device="cuda").to(dtype)
        ids = torch.arange(rows, device="cuda") * 77
        assert torch.equal(among.dropout(h, 0.3, 9, h, ids), ops.dropout(h, 0.3, 9, residual=h, row_ids=ids))
