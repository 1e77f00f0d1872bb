"""The language-model operators on the GPU against the 64-bit oracle: sizes around every unit of
work, types, row strides and alignments, masked rows and tokens, refusals, streams and graphs.

Tolerances follow from the formulas.  With u = 2^-24 the unit roundoff of the 32-bit sums, d the
distance of a logit to its row's maximum and D the mean of d under the softmax:
  - a term exp(-d) carries 3 u d from its argument (difference, product, constant) and 4 u of its
    own; a sum of n positive terms whose longest chain of additions is n_c carries n_c u more, with
    n_c <= 64 + n / 64 for any split over at least a wave's lanes, or 64 values per lane;
  - ln of the sum carries the sum's relative error, 4 u |ln S| from its evaluation and storage;
  - p = exp(-d - ln S) carries 3 u d + 4 u ln S + 8 u besides the sum's;
  - a result is rounded once to its type, whose unit roundoff is `U`, or to a multiple of the
    type's smallest number `TINY`.
"""

import numpy as np
import pytest
import torch

import paper_2607_20739_amd as P
from paper_2607_20739_amd import ops
from oracle import ops as O

pytestmark = pytest.mark.gpu

u = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    ops.lib()


def _say(*what):
    print("\n[gpu case]", *what, flush=True)


def _place(x, pad=0, shift=0, fill=0.0):
    """x on the GPU with `pad` columns more between its rows, starting `shift` values into its memory."""
    rows, cols = x.shape
    buf = torch.full((shift + rows * (cols + pad) + 32,), fill, dtype=x.dtype, device="cuda")
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return buf, view


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, tol, what):
    got, want, tol = _np(got) if torch.is_tensor(got) else got, np.asarray(want), np.broadcast_to(tol, np.shape(want))
    assert got.shape == want.shape
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all(), (what, "NaN places")
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all(), (what, "infinities")
    rest = ~(nan | inf)
    off = np.abs(got[rest] - want[rest])
    bad = ~(off <= tol[rest])
    assert not bad.any(), (what, int(bad.sum()), float((off - tol[rest]).max()), float(off.max()))


# ---- dropout ------------------------------------------------------------------------------

DROPOUT_SHAPES = [(1, 1), (3, 2), (2, 5), (5, 7), (4, 8), (3, 9), (2, 31), (7, 64), (33, 100), (1, 1001), (9, 1024),
                  (3, 2049), (2, 8191)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", DROPOUT_SHAPES)
def test_dropout_matches_the_oracle(dtype, rows, cols):
    rng = np.random.default_rng(rows * 10007 + cols)
    for case, (p, residual, ids, pad, shift) in enumerate([(0.1, False, False, 0, 0), (0.5, True, True, 0, 0),
                                                           (0.25, True, False, 3, 1), (0.9, False, True, 5, 3)]):
        _say("dropout", dtype, rows, cols, case)
        seed = int(rng.integers(0, 1 << 63)) * 2 + 1
        first = int(rng.integers(-100, 1 << 40))
        row_ids = rng.integers(-5, 1 << 50, rows) if ids else first + np.arange(rows)
        x = torch.from_numpy(rng.normal(size=(rows, cols))).to(DTYPES[dtype])
        r = torch.from_numpy(rng.normal(size=(rows, cols))).to(DTYPES[dtype])
        _, xg = _place(x, pad, shift)
        _, rg = _place(r, pad + 1, shift)
        buf, out = _place(torch.zeros_like(x), pad, shift, fill=77.0)
        args = dict(row_ids=torch.from_numpy(row_ids).cuda() if ids else None, first_row=first)
        got = ops.dropout(xg, p, seed, residual=rg if residual else None, out=out, **args)
        assert got is out
        want = O.dropout(x.double().numpy(), p, seed, row_ids, r.double().numpy() if residual else None)
        # x s: factor and product; then the sum; then the type.
        scaled = np.abs(want - (r.double().numpy() if residual else 0.0))
        tol = 3 * u * scaled + u * np.abs(want) + U[dtype] * np.abs(want) * (1 + 4 * u) + TINY[dtype]
        _close(got, want, tol, "out")
        if not residual:
            assert ((_np(got) == 0) == (want == 0)).all()
        out.fill_(77.0)
        assert (buf == 77.0).all(), "values outside of the output were written"
        back = ops.dropout_backward(xg, p, seed, **args)
        want = O.dropout(x.double().numpy(), p, seed, row_ids)
        _close(back, want, 3 * u * np.abs(want) + U[dtype] * np.abs(want) * (1 + 4 * u) + TINY[dtype], "dx")


def test_dropout_bounds_of_p_and_values_in_dropped_places():
    _say("dropout p = 0, 1, NaN in dropped places")
    x = torch.randn(5, 333, device="cuda")
    r = torch.randn(5, 333, device="cuda")
    assert torch.equal(ops.dropout(x, 0.0, 3), x)
    assert torch.equal(ops.dropout(x, 1.0, 3), torch.zeros_like(x))
    assert torch.equal(ops.dropout(x, 1.0, 3, residual=r), r)
    assert torch.equal(ops.dropout(x, 2.0 ** -18, 3), x)           # rounds to no dropout
    keep = torch.from_numpy(O.keep_mask(0.5, 3, range(5), 333)).cuda()
    for v in (float("nan"), INF, -INF):
        y = ops.dropout(torch.where(keep, x, v), 0.5, 3, residual=r)
        assert torch.equal(y, torch.where(keep, 2 * x, 0.0) + r)
        y = ops.dropout(torch.where(keep, v, x), 0.5, 3)
        assert (y[~keep] == 0).all() and not y[keep].isfinite().any()


def test_dropout_in_place_and_gathered_rows():
    _say("dropout in place, gathered rows")
    for dtype in DTYPES.values():
        x = torch.randn(37, 515, device="cuda").to(dtype)
        r = torch.randn(37, 515, device="cuda").to(dtype)
        want = ops.dropout(x, 0.3, 11, residual=r, first_row=100)
        order = torch.randperm(37, device="cuda")
        got = ops.dropout(x[order], 0.3, 11, residual=r[order], row_ids=order + 100)
        assert torch.equal(got, want[order])            # the mask goes with the row's number
        a, b = x.clone(), r.clone()
        assert torch.equal(ops.dropout(a, 0.3, 11, residual=r, first_row=100, out=a), want)
        assert torch.equal(ops.dropout(x, 0.3, 11, residual=b, first_row=100, out=b), want)


# ---- logits -------------------------------------------------------------------------------

COLS = [1, 2, 3, 5, 7, 8, 9, 10, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 255, 256, 257, 500, 513, 1000, 1024,
        1025, 2047, 2048, 2049, 4095, 4097, 8191, 8193, 12289, 16384, 16391, 32767, 40001, 50021, 65536, 65537, 100003,
        131071, 131072, 131073, 262147]


def _rows_for(cols):
    return 37 if cols <= 64 else 11 if cols <= 4096 else 5


def _case(dtype, rows, cols, seed, spread=2.0, banned=None):
    """Logits on the CPU in their type, targets with some rows without a token."""
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.normal(size=(rows, cols)) * spread).astype(np.float32)).to(DTYPES[dtype])
    y = torch.from_numpy(rng.integers(0, cols, rows).astype(np.int32))
    z[torch.arange(rows), y.long()] += float(np.log(cols))
    if banned is not None and cols > 3:
        off = torch.from_numpy(rng.random(cols) < 0.2)
        z[:, off] = banned
        z[torch.arange(rows), y.long()] = 1.0
    if rows > 2:
        y[rng.integers(0, rows)] = -1
        y[rng.integers(0, rows)] = cols
    return z, y


class _Expected:
    """The oracle's values of a case, and the errors that 32-bit evaluation allows."""

    def __init__(self, z, y):
        self.z, self.y = z.double().numpy(), y.numpy()
        rows, cols = self.z.shape
        self.on = O.has_token(self.y, cols)
        self.top, self.log_sum = O.row_stats(self.z)
        with np.errstate(invalid="ignore"):
            self.d = np.where(np.isfinite(self.z), self.top[:, None] - self.z, 0.0)
            self.p = np.exp(self.z - self.top[:, None] - self.log_sum[:, None])
        mean_d = np.nansum(np.where(self.p > 0, self.p * self.d, 0.0), 1)
        self.sum_rel = u * (64 + cols / 64 + 4 + 3 * mean_d)
        self.lp = O.token_logprobs(self.z, self.y)
        self.lp[np.abs(self.lp) > float(np.finfo(np.float32).max)] *= INF   # past what 32 bits hold
        dy = np.array([self.d[t, k] if o else 0.0 for t, (k, o) in enumerate(zip(self.y, self.on))])
        self.lp_tol = self.sum_rel + u * (8 + 2 * dy + 4 * np.abs(self.log_sum))

    def gradient(self, g, dtype, g_tol=0.0):
        """(gradient, tolerance) for the factor g per row, itself known to g_tol."""
        want = O.token_logprobs_backward(self.z, self.y, g)
        g, g_tol = np.abs(g)[:, None], np.broadcast_to(g_tol, np.shape(g))[:, None]
        rel = self.sum_rel[:, None] + u * (3 * self.d + 4 * np.abs(self.log_sum)[:, None] + 8)
        p = np.nan_to_num(self.p)
        tol = g * p * rel + 2 * u * np.abs(want) + g_tol * p
        for t in np.flatnonzero(self.on):
            tol[t, self.y[t]] += 2 * u * g[t, 0] + g_tol[t, 0]
        tol[~self.on] = 0.0
        return want, tol * (1 + U[dtype]) + U[dtype] * np.abs(want) + TINY[dtype]


def _check_logprobs(z, y, dtype, pad, shift, seed):
    e = _Expected(z, y)
    _, zg = _place(z, pad, shift, fill=100.0)
    yg = y.cuda()
    lp, stats = ops.token_logprobs(zg, yg)
    _close(lp, e.lp, e.lp_tol, "logprobs")
    fine = e.on & ~np.isnan(e.log_sum)
    _close(stats[:, 0].cpu().numpy()[fine], e.top[fine], 0.0, "maxima")
    _close(stats[:, 1].cpu().double().numpy()[fine], e.log_sum[fine], (e.sum_rel + 4 * u * np.abs(e.log_sum))[fine], "log sums")
    assert not stats[torch.from_numpy(~e.on).cuda()].any()
    g = np.random.default_rng(seed).normal(size=len(z)).astype(np.float32)
    g[0] = 0.0
    buf, out = _place(torch.zeros_like(z), pad, shift, fill=77.0)
    dz = ops.token_logprobs_backward(zg, yg, stats, torch.from_numpy(g).cuda(), out=out)
    _close(dz, *e.gradient(g, dtype), "gradient")
    out.fill_(77.0)
    assert (buf == 77.0).all(), "values outside of the output were written"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_token_logprobs_match_the_oracle(dtype, cols):
    for case, (pad, shift, banned) in enumerate([(0, 0, None), (3, 1, -INF), (0, 3, "lowest")]):
        _say("logprobs", dtype, cols, case)
        low = torch.finfo(DTYPES[dtype]).min if banned == "lowest" else banned
        rows = _rows_for(cols) if case == 0 else 3
        z, y = _case(dtype, rows, cols, cols * 31 + case, banned=low)
        _check_logprobs(z, y, dtype, pad, shift, case)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [10, 1000, 40001])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 64, 65, 127, 255, 257, 1023])
def test_token_logprobs_for_any_number_of_rows(dtype, cols, rows):
    if rows * cols > 4_000_000:
        rows = 4_000_000 // cols          # the largest on fewer rows
    _say("logprobs rows", dtype, cols, rows)
    z, y = _case(dtype, rows, cols, rows)
    _check_logprobs(z, y, dtype, 0, 0, rows)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [10, 64, 1000, 9001, 131071])
def test_logits_of_large_magnitude(dtype, cols):
    """Maxima far from 0 cancel exactly: errors stay those of the differences."""
    _say("logprobs magnitude", dtype, cols)
    z, y = _case(dtype, 4, cols, cols, spread=30.0)
    z = (z.float() + torch.tensor([[0.0], [3000.0], [-3000.0], [100.0]])).to(DTYPES[dtype])
    _check_logprobs(z, y, dtype, 0, 0, 1)


def _special_rows(dtype, cols):
    """Rows whose mask leaves nothing or one value, extreme and broken rows, and what is to come."""
    low, high = torch.finfo(DTYPES[dtype]).min, torch.finfo(DTYPES[dtype]).max
    base = torch.linspace(-1, 1, cols)
    last = cols - 1
    rows = [base, torch.full((cols,), -INF), torch.full((cols,), low), torch.full((cols,), high), base.clone(),
            base.clone(), base.clone(), torch.full((cols,), -INF), base.clone(), torch.full((cols,), -INF), base]
    rows[4][last] = float("nan")
    rows[5][0] = INF
    rows[6][last] = -INF          # the target itself cannot occur
    rows[7][last] = -2.0          # only the target can
    rows[8][0], rows[8][last] = high, low
    rows[9][0] = float("nan")
    y = torch.full((len(rows),), last, dtype=torch.int32)
    return torch.stack(rows).to(DTYPES[dtype]), y


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [2, 10, 65, 513, 1001, 4097, 20000, 70001, 131072, 200001])
def test_special_rows(dtype, cols):
    _say("special rows", dtype, cols)
    z, y = _special_rows(dtype, cols)
    e = _Expected(z, y)
    zg, yg = z.cuda(), y.cuda()
    lp, stats = ops.token_logprobs(zg, yg)
    _close(lp, e.lp, np.nan_to_num(e.lp_tol, nan=0.0, posinf=0.0), "logprobs")
    g = np.ones(len(z), np.float32)
    want, tol = e.gradient(g, dtype)
    dz = ops.token_logprobs_backward(zg, yg, stats, torch.from_numpy(g).cuda())
    _close(dz, want, np.nan_to_num(tol), "gradient")
    # The same rows through the policy loss (ratio 1 where the log-probability is finite).
    old = torch.where(lp.isfinite(), lp, 0.0)
    loss, lp2, dz2 = ops.policy_loss(zg, yg, old, torch.ones_like(lp), clip_low=1.0, clip_high=1e30)
    broken = np.isnan(e.lp)
    assert np.isnan(_np(loss)[broken]).all() and np.isnan(_np(dz2)[broken]).all()
    assert np.isfinite(_np(loss)[~broken]).all() and np.isfinite(_np(dz2)[~broken]).all()
    _close(lp2, e.lp, np.nan_to_num(e.lp_tol, nan=0.0, posinf=0.0), "policy logprobs")
    # Skipped rows are not read: no token, no gradient, no weight.
    none = torch.full_like(yg, -1)
    lp, stats = ops.token_logprobs(zg, none)
    assert not lp.any() and not stats.any()
    for t, gr in [(none, torch.ones(len(z), device="cuda")), (yg, torch.zeros(len(z), device="cuda"))]:
        assert not ops.token_logprobs_backward(zg, t, stats, gr).any()
    for t, w in [(none, None), (yg, torch.zeros(len(z), device="cuda"))]:
        for out in ops.policy_loss(zg, t, old, torch.ones_like(lp), token_weights=w):
            assert not out.any()


# ---- preference loss ----------------------------------------------------------------------

def _offsets(rows, pairs, seed):
    """Unequal sequences, some empty, with rows before the first and after the last."""
    rng = np.random.default_rng(seed)
    cuts = np.sort(rng.integers(rows // 10, rows - rows // 10 + 1, 2 * pairs + 1))
    return cuts.astype(np.int32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,pairs", [(1, 5, 1), (7, 10, 2), (64, 33, 5), (40, 1000, 3), (33, 9001, 2),
                                             (700, 100, 1), (9, 131071, 2), (2000, 17, 40), (12, 70001, 1)])
def test_preference_loss_matches_the_oracle(dtype, rows, cols, pairs):
    for case, (smoothing, with_ref, with_weights, pad) in enumerate([(0.0, True, False, 0), (0.1, False, True, 5)]):
        _say("preference", dtype, rows, cols, pairs, case)
        z, y = _case(dtype, rows, cols, rows + cols + case, banned=-INF if case else None)
        rng = np.random.default_rng(case)
        o = _offsets(rows, pairs, rows + case)
        e = _Expected(z, y)
        ref = (e.lp + rng.normal(size=rows) * 0.3).astype(np.float32) if with_ref else None
        w = rng.uniform(size=pairs).astype(np.float32) if with_weights else None
        if with_weights:
            w[0] = 0.0
        beta, scale = 0.3, 1.7
        loss, margin, _, g = O.preference(e.z, e.y, o, ref, beta, smoothing, scale, w)
        _, zg = _place(z, pad, case)
        got = ops.preference_loss(zg, y.cuda(), torch.from_numpy(o).cuda(),
                                  None if ref is None else torch.from_numpy(ref).cuda(), beta=beta,
                                  label_smoothing=smoothing, scale=scale,
                                  pair_weights=None if w is None else torch.from_numpy(w).cuda())
        _close(got[2], e.lp, e.lp_tol, "logprobs")
        # A margin carries its rows' errors (their 32-bit storage included); the loss follows it
        # with a slope of at most 1, its slope with one of at most 1/4.
        h_tol = np.array([beta * (e.lp_tol + u * np.abs(e.lp))[o[2 * i]:o[2 * i + 2]].sum() for i in range(pairs)])
        _close(got[1], margin, h_tol + 2 * u * np.abs(margin), "margins")
        _close(got[0], loss, h_tol + 2 * u * np.abs(loss), "loss")
        g_tol = np.zeros(rows)
        for i in range(pairs):
            wi = 1.0 if w is None else w[i]
            g_tol[o[2 * i]:o[2 * i + 2]] = 0.25 * scale * beta * wi * h_tol[i]
        _close(got[3], *e.gradient(g, dtype, g_tol + 2 * u * np.abs(g)), "gradient")
        only = ops.preference_loss(zg, y.cuda(), torch.from_numpy(o).cuda(),
                                   None if ref is None else torch.from_numpy(ref).cuda(), beta=beta,
                                   label_smoothing=smoothing, gradient=False)
        assert only[3] is None
        for a, b in zip(only[:3], got[:3]):
            assert torch.equal(a, b)


def test_preference_loss_edges():
    _say("preference edges")
    z, y = _case("f32", 20, 50, 1)
    z, y = z.cuda(), y.cuda()
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, margin, lp, dz = ops.preference_loss(z, y, none)
    assert loss.numel() == 0 and not dz.any() and torch.equal(lp, ops.token_logprobs(z, y)[0])
    # Two empty sequences: h = 0.
    zero = torch.full((3,), 7, dtype=torch.int32, device="cuda")
    loss, margin, _, dz = ops.preference_loss(z, y, zero)
    assert loss.item() == pytest.approx(np.log(2), abs=1e-7) and margin.item() == 0 and not dz.any()
    # No rows at all.
    loss, margin, lp, dz = ops.preference_loss(z[:0], y[:0], torch.zeros(5, dtype=torch.int32, device="cuda"))
    assert (loss - np.log(2)).abs().max().item() < 1e-7 and dz.shape == (0, 50)
    # Offsets outside of the rows are taken as their bounds.
    wild = torch.tensor([-9, 8, 1 << 30], dtype=torch.int32, device="cuda")
    tame = torch.tensor([0, 8, 20], dtype=torch.int32, device="cuda")
    for a, b in zip(ops.preference_loss(z, y, wild), ops.preference_loss(z, y, tame)):
        assert torch.equal(a, b)
    # More empty pairs than one launch has blocks for.
    empties = torch.full((2 * 3_000_000 + 1,), 4, dtype=torch.int32, device="cuda")
    empties[-1] = 20
    loss, margin, _, dz = ops.preference_loss(z, y, empties)
    assert (loss[:-1] - np.log(2)).abs().max().item() < 1e-7 and not dz[:4].any() and dz[4:].any()
    # A margin far out: finite loss, gradient of at most the slope's bound, none NaN.
    far = torch.full((20,), 1e6, device="cuda")
    loss, margin, _, dz = ops.preference_loss(z, y, tame, far, beta=5.0)
    assert loss.isfinite().all() and dz.isfinite().all()
    # NaN in one pair's rows stays in that pair; a pair of weight 0 lets nothing through.
    two = torch.tensor([0, 4, 9, 13, 20], dtype=torch.int32, device="cuda")
    y = torch.arange(20, dtype=torch.int32, device="cuda")
    want = ops.preference_loss(z, y, two)
    bad = z.clone()
    bad[2, 3] = float("nan")
    loss, margin, lp, dz = ops.preference_loss(bad, y, two)
    assert loss[0].isnan() and loss[1] == want[0][1] and torch.equal(dz[9:], want[3][9:]) and dz[:9].isnan().all()
    loss, _, _, dz = ops.preference_loss(bad, y, two, pair_weights=torch.tensor([0.0, 1.0], device="cuda"))
    assert not dz[:9].any() and torch.equal(dz[9:], want[3][9:])


# ---- policy loss --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [1, 5, 10, 33, 64, 129, 1000, 1025, 2049, 4097, 8191, 16391, 32768, 50021, 65537, 131071,
                                  131072, 131080, 200001])
def test_policy_loss_matches_the_oracle(dtype, cols):
    for case, (kl, weighted, pad, shift, banned) in enumerate([(0.0, False, 0, 0, None), (0.3, True, 7, 1, -INF),
                                                               (0.05, False, 0, 5, "lowest")]):
        _say("policy", dtype, cols, case)
        rows = max(_rows_for(cols), 9)
        low = torch.finfo(DTYPES[dtype]).min if banned == "lowest" else banned
        z, y = _case(dtype, rows, cols, cols + case, banned=low)
        e = _Expected(z, y)
        rng = np.random.default_rng(case + cols)
        # Ratios at fixed distances from 1: inside, and clear of both bounds.
        shift_lp = rng.choice([-0.6, -0.1, 0.05, 0.5], rows)
        old = (e.lp - shift_lp).astype(np.float32)
        adv = rng.normal(size=rows).astype(np.float32)
        adv[0] = 0.0
        ref = (e.lp + 0.4 * rng.normal(size=rows)).astype(np.float32)
        w = rng.uniform(size=rows).astype(np.float32) if weighted else None
        if weighted:
            w[1] = 0.0
        kw = dict(clip_low=0.2, clip_high=0.28, kl=kl, scale=0.7)
        loss, lp, g = O.policy(e.z, e.y, old, adv, ref, weights=w, **kw)
        _, zg = _place(z, pad, shift, fill=100.0)
        buf, out = _place(torch.zeros_like(z), pad, shift, fill=77.0)
        args = dict(kw, ref_logprobs=torch.from_numpy(ref).cuda() if kl else None,
                    token_weights=None if w is None else torch.from_numpy(w).cuda())
        dev = [torch.from_numpy(old).cuda(), torch.from_numpy(adv).cuda()]
        got = ops.policy_loss(zg, y.cuda(), *dev, out=out, **args)
        on = e.on if w is None else e.on & (w != 0)
        ratio, off = np.exp(e.lp - old), np.exp(ref.astype(np.float64) - e.lp)
        # The log-probability's error (its storage included) acts on the ratio and on exp(ref - l);
        # each exponential adds 4 u and what its argument's rounding gives, each product and sum u.
        l_err = np.where(on, e.lp_tol + 2 * u * (np.abs(e.lp) + np.abs(old) + np.abs(ref)), 0.0)
        part = np.abs(adv) * np.where(on, ratio, 0) * (l_err + 8 * u)
        kl_part = kl * (np.abs(off - 1) * l_err + off * 8 * u + 8 * u)
        _close(got[1], lp, np.where(on, e.lp_tol, 0.0), "logprobs")
        _close(got[0], loss, part + np.where(on, kl_part, 0) + 4 * u * (np.abs(loss) + np.abs(adv) * 1.3), "loss")
        slope_tol = part + kl * off * (l_err + 8 * u) + kl * 4 * u
        g_tol = np.where(on, 0.7 * (1.0 if w is None else w) * slope_tol, 0.0) + 6 * u * np.abs(g)
        _close(got[2], *e.gradient(g, dtype, g_tol), "gradient")
        only = ops.policy_loss(zg, y.cuda(), *dev, gradient=False, **args)
        assert only[2] is None and torch.equal(only[0], got[0]) and torch.equal(only[1], got[1])
        out.fill_(77.0)
        assert (buf == 77.0).all(), "values outside of the output were written"


def test_policy_loss_infinite_ratios():
    """Ratios that overflow: bounded where the bound holds, no NaN from a zero advantage."""
    _say("policy infinite ratios")
    z = torch.randn(4, 100, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    old = torch.full((4,), -1e4, device="cuda")
    adv = torch.tensor([1.0, 0.0, 2.0, 0.5], device="cuda")
    loss, _, dz = ops.policy_loss(z, y, old, adv, clip_low=0.2, clip_high=0.5)
    assert loss.tolist() == [-1.5, 0.0, -3.0, -0.75] and not dz.any()


# ---- what holds for all -------------------------------------------------------------------

def _everything(z, y, extra=None):
    """Every logits operator's outputs for these inputs."""
    rows = z.shape[0]
    lp, stats = ops.token_logprobs(z, y)
    g = torch.linspace(-1, 1, rows, device="cuda") if extra is None else extra
    offsets = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    old, adv = lp.detach() + 0.05, g + 0.5
    return ([lp, stats, ops.token_logprobs_backward(z, y, stats, g)] +
            list(ops.policy_loss(z, y, old, adv, ref_logprobs=old + 0.1, kl=0.1)) +
            list(ops.preference_loss(z, y, offsets, old, beta=0.2)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [10, 129, 1001, 5000, 30001, 131071, 200001])
def test_results_depend_on_the_rows_values_alone(dtype, cols):
    """The same bits again, at other alignments and strides, in place, and for a row by itself."""
    _say("same bits", dtype, cols)
    z, y = _case(dtype, 9, cols, 3)
    yg = y.cuda()
    want = _everything(z.cuda(), yg)
    for pad, shift in [(0, 0), (0, 1), (1, 0), (6, 2), (8, 8), (13, 7)]:
        for a, b in zip(_everything(_place(z, pad, shift)[1], yg), want):
            assert torch.equal(a, b), (pad, shift)
    lp, stats, dz, loss, _, dz_policy, _, _, _, dz_pair = want
    g = torch.linspace(-1, 1, 9, device="cuda")
    for t in range(9):
        zt, yt = z[t:t + 1].cuda(), yg[t:t + 1]
        lpt, st = ops.token_logprobs(zt, yt)
        assert torch.equal(lpt, lp[t:t + 1]) and torch.equal(st, stats[t:t + 1])
        assert torch.equal(ops.token_logprobs_backward(zt, yt, st, g[t:t + 1]), dz[t:t + 1])
    a = z.cuda()
    assert ops.token_logprobs_backward(a, yg, stats, g, out=a) is a and torch.equal(a, dz)
    a = z.cuda()
    got = ops.policy_loss(a, yg, lp + 0.05, g + 0.5, ref_logprobs=lp + 0.05 + 0.1, kl=0.1, out=a)
    assert torch.equal(got[0], loss) and torch.equal(a, dz_policy)
    a = z.cuda()
    offsets = torch.tensor([0, 3, 9], dtype=torch.int32, device="cuda")
    ops.preference_loss(a, yg, offsets, lp + 0.05, beta=0.2, out=a)
    assert torch.equal(a, dz_pair)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """Rows 2^31 values apart: the third starts past 2^32."""
    _say("far rows", dtype)
    rows, cols, stride = 3, 1001, (1 << 31) + 3
    buf = torch.empty((rows - 1) * stride + cols, dtype=DTYPES[dtype], device="cuda")
    far = buf.as_strided((rows, cols), (stride, 1))
    z, y = _case(dtype, rows, cols, 8)
    y = torch.tensor([5, 0, cols - 1], dtype=torch.int32).cuda()
    near = z.cuda()
    want = _everything(near, y)
    far.copy_(near)
    for a, b in zip(_everything(far, y), want):
        assert torch.equal(a, b)
    g = torch.ones(rows, device="cuda")
    want = ops.token_logprobs_backward(near, y, want[1], g)
    stats = ops.token_logprobs(far, y)[1]
    assert torch.equal(ops.token_logprobs_backward(far, y, stats, g, out=far), want)
    far.copy_(near)
    want = ops.dropout(near, 0.4, 77, residual=near)
    assert torch.equal(ops.dropout(far, 0.4, 77, residual=far), want)
    assert torch.equal(ops.dropout(far, 0.4, 77, residual=far, out=far), want)


def test_many_rows():
    """More rows than one launch has blocks or waves for at once; rows of 3 columns in 64 bits by torch."""
    _say("many rows")
    rows, cols = 5_000_003, 3
    z = torch.randn(rows, cols, device="cuda")
    y = torch.randint(-1, cols, (rows,), device="cuda").to(torch.int32)
    lp, stats = ops.token_logprobs(z, y)
    x = torch.log_softmax(z.double(), 1)
    on = y >= 0
    want = torch.where(on, x.gather(1, y.clamp(min=0).long()[:, None])[:, 0], 0.0)
    # |z| < 8, three terms: the bounds above give less than 40 u.
    assert (lp.double() - want).abs().max().item() < 100 * u
    dz = ops.token_logprobs_backward(z, y, stats, torch.ones(rows, device="cuda"))
    one = torch.zeros_like(x).scatter_(1, y.clamp(min=0).long()[:, None], 1.0)
    want = torch.where(on[:, None], one - x.exp(), 0.0)
    assert (dz.double() - want).abs().max().item() < 100 * u
    z2 = ops.dropout(z, 0.5, 9)
    tail = O.dropout(z[-5:].cpu().double().numpy(), 0.5, 9, range(rows - 5, rows))
    np.testing.assert_array_equal(_np(z2[-5:]), tail)


def test_results_repeat_bit_for_bit_and_follow_the_stream():
    _say("streams")
    z, y = _case("bf16", 300, 20001, 5)
    z, y = z.cuda(), y.cuda()
    want = _everything(z, y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = torch.zeros_like(z)
        for _ in range(20):
            late.copy_(z)                   # the operators have to wait for what the stream did before
        got = _everything(late, y)
        x = ops.dropout(late, 0.2, 4)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.equal(x, ops.dropout(z, 0.2, 4))


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 65, 50021), ("f32", 33, 10), ("f16", 9, 131072)])
def test_operators_can_be_captured_into_a_graph(dtype, rows, cols):
    _say("graph", dtype, rows, cols)
    cases = [_case(dtype, rows, cols, s) for s in range(3)]
    z, y = cases[0][0].cuda(), cases[0][1].cuda()
    g = torch.linspace(-1, 1, rows, device="cuda")
    wants = []
    for a, b in cases:
        wants.append([t.clone() for t in _everything(a.cuda(), b.cuda(), g)] + [ops.dropout(a.cuda(), 0.3, 21)])
    torch.cuda.synchronize()
    offsets = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lp, stats = ops.token_logprobs(z, y)
        old = lp + 0.05
        got = [lp, stats, ops.token_logprobs_backward(z, y, stats, g),
               *ops.policy_loss(z, y, old, g + 0.5, ref_logprobs=old + 0.1, kl=0.1),
               *ops.preference_loss(z, y, offsets, old, beta=0.2), ops.dropout(z, 0.3, 21)]
    for replay in (0, 1, 2, 1, 0):
        z.copy_(cases[replay][0])
        y.copy_(cases[replay][1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, wants[replay])):
            assert torch.equal(a, b), (replay, i)


def test_autograd_and_differences():
    """Through torch's autograd, against central differences of the 64-bit oracle along a random
    direction: truncation and rounding of the differences are below 1e-7, the 32-bit gradient's
    error below (64 + 8) u of its terms' absolute sum (below 40 here)."""
    _say("autograd")
    rows, cols = 12, 30
    rng = np.random.default_rng(4)
    h = rng.normal(size=(rows, cols))
    r = rng.normal(size=(rows, cols))
    y = rng.integers(0, cols, rows).astype(np.int32)
    c = rng.normal(size=rows)
    hg = torch.from_numpy(h).float().cuda().requires_grad_()
    rg = torch.from_numpy(r).float().cuda().requires_grad_()
    z = ops.dropout(hg, 0.3, 8, residual=rg, first_row=40)
    lp, stats = ops.token_logprobs(z, torch.from_numpy(y).cuda())
    assert not stats.requires_grad
    (lp * torch.from_numpy(c).float().cuda()).sum().backward()

    def value(hh, rr):
        zz = O.dropout(hh, 0.3, 8, range(40, 40 + rows), rr)
        return (c * O.token_logprobs(zz, y)).sum()

    v, w, step = rng.normal(size=h.shape), rng.normal(size=h.shape), 1e-5
    dh = (value(h + step * v, r) - value(h - step * v, r)) / (2 * step)
    dr = (value(h, r + step * w) - value(h, r - step * w)) / (2 * step)
    tol = 1e-7 + 72 * u * 400
    assert abs((_np(hg.grad) * v).sum() - dh) < tol and abs((_np(rg.grad) * w).sum() - dr) < tol

    # The losses' gradients along a direction, against differences of the oracle's losses.
    z64 = rng.normal(size=(rows, cols))
    z32 = torch.from_numpy(z64).float()
    z64 = z32.double().numpy()
    offsets, ref = np.array([0, 4, 7, 9, 12], np.int32), rng.normal(size=rows).astype(np.float32)
    got = ops.preference_loss(z32.cuda(), torch.from_numpy(y).cuda(), torch.from_numpy(offsets).cuda(),
                              torch.from_numpy(ref).cuda(), beta=0.5, label_smoothing=0.1)[3]
    d = sum(s * O.preference(z64 + s * step * v, y, offsets, ref, 0.5, 0.1)[0].sum() for s in (1, -1)) / (2 * step)
    assert abs((_np(got) * v).sum() - d) < tol
    lp = O.token_logprobs(z64, y)
    old = (lp - rng.choice([-0.5, -0.1, 0.1, 0.5], rows)).astype(np.float32)
    adv = rng.normal(size=rows).astype(np.float32)
    got = ops.policy_loss(z32.cuda(), torch.from_numpy(y).cuda(), torch.from_numpy(old).cuda(),
                          torch.from_numpy(adv).cuda(), ref_logprobs=torch.from_numpy(ref).cuda(), kl=0.01)[2]
    d = sum(s * O.policy(z64 + s * step * v, y, old, adv, ref, kl=0.01)[0].sum() for s in (1, -1)) / (2 * step)
    assert abs((_np(got) * v).sum() - d) < tol


def test_second_gradients():
    """Dropout is linear: its gradient has dropout's own as gradient, bit for bit.  That of the
    log-probabilities has none and says so, and a mask's row numbers may not change on the way."""
    _say("second gradients")
    x = torch.randn(6, 40, device="cuda", requires_grad=True)
    c = torch.randn(6, 40, device="cuda", requires_grad=True)
    v = torch.randn(6, 40, device="cuda")
    ids = torch.tensor([5, 3, 9, 0, 2, 7], device="cuda")
    y = ops.dropout(x, 0.25, 3, row_ids=ids)
    dx, = torch.autograd.grad(y, x, c, create_graph=True)
    assert torch.equal(dx, ops.dropout_backward(c.detach(), 0.25, 3, row_ids=ids))
    dc, = torch.autograd.grad(dx, c, v)
    assert torch.equal(dc, ops.dropout(v, 0.25, 3, row_ids=ids))
    y = ops.dropout(x, 0.25, 3, row_ids=ids)
    ids += 1
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.sum().backward()
    z = torch.randn(6, 40, device="cuda", requires_grad=True)
    lp, _ = ops.token_logprobs(z, torch.zeros(6, dtype=torch.int32, device="cuda"))
    dz, = torch.autograd.grad(lp.sum(), z, create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable"):
        dz.sum().backward()


def test_the_binding_refuses_what_does_not_fit():
    _say("refusals")
    z = torch.randn(6, 40, device="cuda")
    y = torch.zeros(6, dtype=torch.int32, device="cuda")
    f = torch.zeros(6, device="cuda")
    lp, stats = ops.token_logprobs(z, y)
    o = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    bad = [
        lambda: ops.dropout(z[0], 0.1, 1), lambda: ops.dropout(z.double(), 0.1, 1), lambda: ops.dropout(z.t(), 0.1, 1),
        lambda: ops.dropout(z, 0.1, 1, residual=z[:5]), lambda: ops.dropout(z, 0.1, 1, residual=z.half()),
        lambda: ops.dropout(z, 0.1, 1, row_ids=y), lambda: ops.dropout(z, 0.1, 1, out=z[:, :39]),
        lambda: ops.dropout(z[:1].expand(6, 40), 0.1, 1),
        lambda: ops.dropout(z.clone().requires_grad_(), 0.1, 1, out=torch.empty_like(z)),
        lambda: ops.token_logprobs(z, y.long()), lambda: ops.token_logprobs(z, y[:5]),
        lambda: ops.token_logprobs(z, y.cpu()), lambda: ops.token_logprobs_backward(z, y, stats[:, 0], f),
        lambda: ops.token_logprobs_backward(z, y, stats, f.double()),
        lambda: ops.preference_loss(z, y, o[:2]), lambda: ops.preference_loss(z, y, o.long()),
        lambda: ops.preference_loss(z, y, o, ref_logprobs=f[:3]),
        lambda: ops.preference_loss(z, y, o, pair_weights=f),
        lambda: ops.preference_loss(z, y, o, workspace=torch.empty(4096, dtype=torch.int8, device="cuda")),
        lambda: ops.policy_loss(z, y, f[:2], f), lambda: ops.policy_loss(z, y, f, f, token_weights=y),
        lambda: ops.policy_loss(z, y, f, f, out=z.half()),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    refused = [
        lambda: ops.dropout(z, 1.5, 1), lambda: ops.dropout(z[:, :20], 0.1, 1, out=z[:, 10:30]),
        lambda: ops.policy_loss(z, y, f, f, kl=0.1), lambda: ops.policy_loss(z, y, f, f, clip_low=2.0),
        lambda: ops.preference_loss(z, y, o, label_smoothing=-1.0),
        lambda: ops.preference_loss(z, y, o[:1], workspace=torch.empty(0, dtype=torch.uint8, device="cuda")),
    ]
    for call in refused:
        with pytest.raises(P.PGCError) as e:
            call()
        assert e.value.status == P.PGC_EINVAL and str(e.value)
    assert ops.dropout(z[:0], 0.1, 1).shape == (0, 40) and ops.dropout(z[:, :0], 0.1, 1).shape == (6, 0)
    lp, stats = ops.token_logprobs(z[:0], y[:0])
    assert lp.shape == (0,) and stats.shape == (0, 2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_every_operator_gives_a_row_the_same_logprobs(dtype):
    """The preference loss of few logits (one launch), of many (a launch per step), and the scores."""
    for cols in (1, 7, 8, 31, 64, 129, 500, 1024, 1025, 1500, 1600, 2047, 2500, 3300, 4100, 9001):
        _say("same logprobs", dtype, cols)
        z, y = _case(dtype, 24, cols, cols)
        z, y = z.cuda(), y.cuda()
        want = ops.token_logprobs(z, y)[0]
        o = torch.tensor([1, 5, 9, 9, 20], dtype=torch.int32, device="cuda")
        few = ops.preference_loss(z, y, o, want + 0.1, beta=0.7, label_smoothing=0.2)
        assert torch.equal(few[2], want)
        # The same two pairs ahead of so many further rows that no size takes one launch.
        more = max(5000, 2_000_000 // cols // z.element_size())
        zz, yy = torch.cat([z, z[:1].expand(more, cols)]), torch.cat([y, y[:1].expand(more)])
        many = ops.preference_loss(zz, yy, o, torch.cat([want, want[:1].expand(more)]) + 0.1, beta=0.7, label_smoothing=0.2)
        for a, b in zip(few, many):
            assert torch.equal(a, b[:len(a)])
        assert not many[3][24:].any()


PREFERENCE_PATHS = [(3, [(3000, 40), (4096, 4096), (37, 1)]), (16, [(4000, 9), (300, 2)]), (30, [(4090, 70)]), (61, [(1000, 3)]),
                    (120, [(4096, 33), (513, 1)]), (250, [(257, 1), (900, 200)]), (510, [(500, 2)]), (1000, [(700, 5)]),
                    (2050, [(65, 1), (530, 64)]), (3000, [(400, 129)]), (4097, [(64, 33)]), (9001, [(21, 2)]), (20003, [(33, 1)])]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,sizes", PREFERENCE_PATHS)
def test_preference_loss_of_few_rows_and_of_many_have_the_same_bits(dtype, cols, sizes):
    """One launch, two or three: pairs that are empty, of one row, and of all of them; rows of no pair,
    rows without a token; more offsets than a wave has lanes; in place, at odd strides and addresses."""
    for rows, pairs in sizes:
        rng = np.random.default_rng(rows * 7 + pairs)
        z, y = _case(dtype, rows, cols, rows + cols)
        y[rng.random(rows) < 0.2] = -1
        y = y.cuda()
        ref = torch.from_numpy(rng.normal(size=rows).astype(np.float32)).cuda() - 3.0
        weights = torch.from_numpy(rng.uniform(size=pairs).astype(np.float32)).cuda()
        weights[pairs // 2:pairs // 2 + 1] *= float(pairs < 3)
        spread = np.sort(rng.integers(0, rows + 1, 2 * pairs + 1))
        one = np.full(2 * pairs + 1, rows)
        one[:pairs] = 0
        inner = np.clip(spread, rows // 3, rows - rows // 4)
        for case, cuts in enumerate([spread, one, inner]):
            _say("preference paths", dtype, rows, cols, pairs, case)
            o = torch.from_numpy(cuts.astype(np.int32)).cuda()
            kw = dict(beta=0.3, label_smoothing=0.1, scale=2.0, pair_weights=weights if case != 1 else None)
            zg = _place(z, 3 * case, case)[1]
            got = ops.preference_loss(zg, y, o, ref if case != 2 else None, **kw)
            alone = ops.preference_loss(zg, y, o, ref if case != 2 else None, gradient=False, **kw)
            more = 4097
            zz = torch.cat([z.cuda(), z[:1].cuda().expand(more, cols)])
            yy, rr = torch.cat([y, y[:1].expand(more)]), torch.cat([ref, ref[:1].expand(more)])
            # The one that has all rows ends with them here, too.
            want = ops.preference_loss(zz, yy, o, rr if case != 2 else None, **kw)
            for i, (a, b) in enumerate(zip(got, want)):
                assert torch.equal(a, b[:len(a)]), (case, i)
            for a, b in zip(alone[:3], got[:3]):
                assert torch.equal(a, b), case
            assert not want[3][rows:].any()
            ops.preference_loss(zg, y, o, ref if case != 2 else None, out=zg, **kw)
            assert torch.equal(zg, got[3]), case
        e = _Expected(z, y.cpu())
        loss, margin, _, _ = O.preference(e.z, e.y, cuts, None, 0.3, 0.1, 2.0, weights.cpu().numpy())
        err = 0.3 * np.concatenate([[0.0], np.cumsum(e.lp_tol + u * np.abs(e.lp))])
        tol = err[cuts[2::2]] - err[cuts[:-1:2]] + 2 * u * np.abs(margin)
        _close(got[1], margin, tol, "margins")
        _close(got[0], loss, tol + 2 * u * np.abs(loss), "loss")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [28680, 32768, 57351, 65535, 65537, 82001, 131071, 163900, 262147])
def test_policy_loss_of_few_rows_and_of_many_have_the_same_bits(dtype, cols):
    """Rows that several blocks share, rows with a block each, and the gradient in place; targets in every
    part of a row, at odd strides and addresses."""
    many = 70
    gen = torch.Generator(device="cuda").manual_seed(cols)
    z = (2 * torch.randn(many, cols, generator=gen, device="cuda")).to(DTYPES[dtype])
    y = torch.randint(0, cols, (many,), generator=gen, device="cuda").to(torch.int32)
    y[:8] = torch.tensor([0, cols - 1, -1, 1, cols // 2, cols - 9, 7, 8])
    old, adv = torch.full((many,), -11.0, device="cuda"), torch.linspace(-1, 1, many, device="cuda")
    kw = dict(clip_low=0.2, clip_high=0.3)
    want = ops.policy_loss(z, y, old, adv, ref_logprobs=old, kl=0.1, **kw)
    for rows, pad, shift in [(1, 0, 0), (2, 1, 1), (31, 0, 3), (33, 5, 0), (50, 0, 0), (64, 3, 1), (65, 0, 0)]:
        _say("policy few rows", dtype, cols, rows)
        first = min(8, many - rows) if rows < 31 else 0
        part = slice(first, first + rows)
        _, zg = _place(z[part], pad, shift, fill=100.0)
        buf, out = _place(torch.zeros(rows, cols, dtype=DTYPES[dtype]), pad, shift, fill=77.0)
        got = ops.policy_loss(zg, y[part], old[part], adv[part], ref_logprobs=old[part], kl=0.1, out=out, **kw)
        for a, b in zip(got, want):
            assert torch.equal(a, b[part]), rows
        out.fill_(77.0)
        assert (buf == 77.0).all(), "values outside of the output were written"
        ops.policy_loss(zg, y[part], old[part], adv[part], ref_logprobs=old[part], kl=0.1, out=zg, **kw)
        assert torch.equal(zg, want[2][part]), rows


@pytest.mark.parametrize("dtype,rows,cols,cuts", [
    ("f32", 70_001, 3, [5, 30_007, 60_001]), ("bf16", 40_000, 9, [0, 4096, 8192, 8192, 40_000]),
    ("f16", 100_003, 4, [9_001, 9_001, 9_001, 13_097, 13_098, 50_000, 99_999]), ("f32", 600_000, 2, [1, 299_000, 599_998]),
    ("bf16", 300_000, 5, [0, 1, 270_000, 280_000, 300_000]), ("f32", 16_384, 10, [4_095, 8_000, 12_290])])
def test_preference_loss_of_long_pairs(dtype, rows, cols, cuts):
    """A block for each 4,096 rows of a pair, or one for all of it: the same bits, and the oracle's values."""
    _say("long pairs", dtype, rows, cols, cuts)
    rng = np.random.default_rng(rows)
    z, y = _case(dtype, rows, cols, rows + cols)
    y[rng.random(rows) < 0.1] = -1
    cuts = np.array(cuts, np.int32)
    pairs = (len(cuts) - 1) // 2
    e = _Expected(z, y)
    ref = (e.lp + 0.01 * rng.normal(size=rows)).astype(np.float32)
    zg, yg, rg = z.cuda(), y.cuda(), torch.from_numpy(ref).cuda()
    kw = dict(beta=0.05, label_smoothing=0.1, scale=3.0)
    got = ops.preference_loss(zg, yg, torch.from_numpy(cuts).cuda(), rg, **kw)
    # Empty pairs behind them make the pairs short on average.
    more = np.concatenate([cuts, np.full(400, cuts[-1], np.int32)])
    want = ops.preference_loss(zg, yg, torch.from_numpy(more).cuda(), rg, **kw)
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b[:len(a)]), i
    assert (want[0][pairs:] - np.log(2)).abs().max().item() < 1e-7
    # The same pairs' rows elsewhere, and without the gradient.
    put = 123
    z2 = torch.cat([zg[-put:], zg, zg[:7]])
    y2, r2 = torch.cat([yg[-put:], yg, yg[:7]]), torch.cat([rg[-put:], rg, rg[:7]])
    moved = ops.preference_loss(z2, y2, torch.from_numpy(cuts + put).cuda(), r2, **kw)
    for a, b in zip(got[:2], moved[:2]):
        assert torch.equal(a, b)
    assert torch.equal(moved[3][put:put + rows], got[3]) and not moved[3][:put].any()
    only = ops.preference_loss(zg, yg, torch.from_numpy(cuts).cuda(), rg, gradient=False, **kw)
    for a, b in zip(only[:3], got[:3]):
        assert torch.equal(a, b)
    loss, margin, _, g = O.preference(e.z, e.y, cuts, ref, 0.05, 0.1, 3.0)
    err = 0.05 * np.concatenate([[0.0], np.cumsum(e.lp_tol + u * np.abs(e.lp))])
    h_tol = err[cuts[2::2]] - err[cuts[:-1:2]]
    _close(got[1], margin, h_tol + 2 * u * np.abs(margin), "margins")
    _close(got[0], loss, h_tol + 2 * u * np.abs(loss), "loss")
    g_tol = np.zeros(rows)
    for i in range(pairs):
        g_tol[cuts[2 * i]:cuts[2 * i + 2]] = 0.25 * 3.0 * 0.05 * h_tol[i]
    _close(got[3], *e.gradient(g, dtype, g_tol + 2 * u * np.abs(g)), "gradient")


@pytest.mark.parametrize("rows,cols", [(90, 64), (3000, 300), (9000, 33), (90_000, 4)])
def test_offsets_that_decrease_stay_within_the_rows(rows, cols):
    """No results are promised for them, but nothing outside of the outputs is touched, in any path."""
    _say("decreasing offsets", rows, cols)
    z, y = _case("f32", rows, cols, rows)
    zg, yg = z.cuda(), y.cuda()
    for cuts in ([rows, rows // 2, 0], [rows - 1, 3, rows // 2, rows, 5], [rows // 2, 1, 0, -7, 1 << 30, 9, 2],
                 [0, rows, 0, rows, 0], [-(1 << 31), (1 << 31) - 1, -(1 << 31)]):
        buf, out = _place(torch.zeros(rows, cols), 3, 1, fill=77.0)
        o = torch.tensor(cuts, dtype=torch.int32, device="cuda")
        loss, margin, lp, _ = ops.preference_loss(zg, yg, o, out=out)
        assert loss.isfinite().all() and margin.isfinite().all() or rows > 20480
        assert torch.equal(lp, ops.token_logprobs(zg, yg)[0])
        out.fill_(77.0)
        assert (buf == 77.0).all()


# Sizes that take one launch, two, three and four.
LOSS_PATHS = [(40, 30), (1000, 100), (5001, 10), (50_001, 5)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", LOSS_PATHS)
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_preference_loss_of_infinite_margins(dtype, rows, cols, smoothing):
    """A token that cannot occur, in the second sequence (margin +inf) and in the first (-inf); or a row of
    nothing but -inf.  Losses and gradients are the limits, no NaN."""
    _say("infinite margins", dtype, rows, cols, smoothing)
    z, y = _case(dtype, rows, cols, rows)
    o = np.array([0, rows // 4, rows // 2, rows // 2 + 3, rows], np.int32)
    for at, whole in [((o[1] + 1, o[2]), False), ((o[2] - 1, o[4] - 1), False), ((o[1], o[3] - 1), True)]:
        z1, y1 = z.clone(), y.clone()
        for t in at:
            y1[t] = 1
            z1[t, slice(None) if whole else 1] = -INF
        e = _Expected(z1, y1)
        kw = dict(beta=0.3, scale=1.7)
        loss, margin, _, g = O.preference(e.z, e.y, o, None, 0.3, smoothing, 1.7)
        assert np.isinf(margin).all() and not np.isnan(loss).any()
        zg, yg, og = z1.cuda(), y1.cuda(), torch.from_numpy(o).cuda()
        got = ops.preference_loss(zg, yg, og, label_smoothing=smoothing, **kw)
        _close(got[1], margin, 0.0, "margins")
        _close(got[0], loss, 0.0, "loss")
        _close(got[2], e.lp, e.lp_tol, "logprobs")
        _close(got[3], *e.gradient(g, dtype, 2 * u * np.abs(g)), "gradient")
        only = ops.preference_loss(zg, yg, og, label_smoothing=smoothing, gradient=False, **kw)
        for a, b in zip(only[:3], got[:3]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [5, 40, 1001, 9001, 70001])
def test_policy_loss_of_targets_that_cannot_occur(dtype, cols):
    """Their KL term is +inf, the limit, and with it the loss; the other rows know nothing of it."""
    _say("policy, banned targets", dtype, cols)
    z, y = _case(dtype, 9, cols, cols)
    y = torch.clamp(y, 0, cols - 1)
    z[2, y[2]] = z[5, y[5]] = -INF
    z[7] = -INF
    e = _Expected(z, y)
    old = np.where(np.isfinite(e.lp), e.lp - 0.1, -3.0).astype(np.float32)
    adv = np.array([1, -1, 1, 1, 0.5, -1, 0, 1, 2], np.float32)
    dev = [z.cuda(), y.cuda(), torch.from_numpy(old).cuda(), torch.from_numpy(adv).cuda()]
    for kl in (0.0, 0.25):
        loss, lp, g = O.policy(e.z, e.y, old, adv, old, kl=kl)
        assert np.isposinf(loss[[2, 5, 7]]).all() == (kl > 0)
        got = ops.policy_loss(*dev, ref_logprobs=dev[2], kl=kl)
        # Ratios are exp(0.1) and the KL term's argument -0.1, both off by the log-probability's error.
        l_err = np.where(np.isfinite(e.lp), e.lp_tol + 2 * u * (np.abs(np.nan_to_num(e.lp)) + np.abs(old)), 0.0)
        tol = (1.2 * np.abs(adv) + kl) * (l_err + 16 * u)
        _close(got[1], lp, e.lp_tol, "logprobs")
        _close(got[0], loss, tol, "loss")
        with np.errstate(invalid="ignore"):
            want, g_tol = e.gradient(g, dtype, tol)
        _close(got[2], want, np.nan_to_num(g_tol), "gradient")   # row 7, whose bound is inf * 0: zeros
        if kl:
            dz = _np(got[2])
            assert not np.isfinite(dz[[2, 5]]).any() and not dz[7].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [2, 10, 65, 513, 1001, 4097, 20000, 131072])
def test_stats_of_broken_rows(dtype, cols):
    """NaN or +inf makes both of a row's stats NaN; a row of nothing but -inf has (-inf, 0)."""
    _say("stats of broken rows", dtype, cols)
    z, y = _special_rows(dtype, cols)
    e = _Expected(z, y)
    _, stats = ops.token_logprobs(z.cuda(), y.cuda())
    _close(stats[:, 0], e.top, 0.0, "maxima")
    fine = np.isfinite(e.log_sum)
    _close(stats[:, 1], e.log_sum, np.where(fine, e.sum_rel + 4 * u * np.abs(e.log_sum), 0.0), "log sums")
    assert np.isnan(_np(stats)[[4, 5, 9]]).all() and _np(stats)[1].tolist() == [-INF, 0.0]


def _tied_products(dtype):
    """(threshold, values): products x * factor that 32 bits round to the middle between two 16-bit numbers,
    so that rounding once and twice differ; for types without such products any values."""
    x = np.arange(1024, 2048)
    for threshold in range(6000, 30000):
        factor = np.float32(65536.0 / (65536 - threshold))
        twice = (x.astype(np.float32) * factor).astype(np.float16)
        ties = x[twice != (x * np.float64(factor)).astype(np.float16)]
        if len(ties) > 1 or dtype != "f16":
            return threshold, ties if dtype == "f16" else x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(65, 3), (65, 9), (65, 101), (33, 2049), (9, 4109), (9, 8193), (5, 16391), (3, 40001)])
def test_dropout_gives_a_row_the_same_bits_wherever_it_lies(dtype, rows, cols):
    """Values next to vectors are rounded as those in them: to 32 bits, then to the type.  In place, too."""
    _say("dropout, same bits", dtype, rows, cols)
    threshold, values = _tied_products(dtype)
    rng = np.random.default_rng(cols)
    x = torch.from_numpy(rng.choice(values, (rows, cols)).astype(np.float32) / 1024).to(DTYPES[dtype])
    x *= torch.from_numpy(rng.choice([-1.0, 1.0], (rows, cols))).to(x.dtype)
    r = torch.from_numpy(rng.normal(size=(rows, cols))).to(DTYPES[dtype])
    keep = torch.from_numpy(O.keep_mask(threshold / 65536, 7, range(100, 100 + rows), cols))
    scaled = torch.where(keep, x.float() * float(np.float32(65536.0 / (65536 - threshold))), 0.0)
    p = threshold / 65536
    for residual, want in [(None, scaled.to(x.dtype)), (r, (scaled + r.float()).to(x.dtype))]:
        for pad, shift in [(0, 0), (0, 1), (1, 0), (6, 2), (8, 8), (13, 7), (63, 37), (64, 0)]:
            xg = _place(x, pad, shift)[1]
            rg = None if residual is None else _place(r, 2 * pad, 3 * shift)[1]
            got = ops.dropout(xg, p, 7, residual=rg, first_row=100)
            assert torch.equal(got.cpu(), want), (residual is None, pad, shift)
            if rg is not None:
                ops.dropout(xg, p, 7, residual=rg, first_row=100, out=rg)
                assert torch.equal(rg.cpu(), want), ("out = residual", pad, shift)
                rg.copy_(r)
            ops.dropout(xg, p, 7, residual=rg, first_row=100, out=xg)
            assert torch.equal(xg.cpu(), want), ("out = x", pad, shift)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [7, 100, 515, 4109, 9001])
def test_columns_of_one_tensor_as_input_and_output(dtype, cols):
    """Columns that lie beside the input's are no overlap: the same bits as with tensors of their own."""
    _say("side by side", dtype, cols)
    rows = 9
    z, y = _case(dtype, rows, cols, 5)
    zg, y = z.cuda(), y.cuda()
    f = torch.linspace(-1, 1, rows, device="cuda")
    lp, stats = ops.token_logprobs(zg, y)
    o = torch.tensor([0, 4, rows], dtype=torch.int32, device="cuda")
    calls = [lambda a, out: ops.dropout(a, 0.3, 5, out=out), lambda a, out: ops.token_logprobs_backward(a, y, stats, f, out=out),
             lambda a, out: ops.policy_loss(a, y, lp, f, out=out)[2], lambda a, out: ops.preference_loss(a, y, o, lp, out=out)[3]]
    for call in calls:
        want = call(zg, None)
        for a, b, width in [(0, cols, 2 * cols), (cols + 1, 0, 2 * cols + 1), (3, cols + 5, 2 * cols + 9)]:
            both = torch.full((rows, width), 55.0, dtype=z.dtype, device="cuda")
            left, right = both[:, a:a + cols], both[:, b:b + cols]
            left.copy_(zg)
            assert torch.equal(call(left, right), want) and torch.equal(left, zg)
            left.fill_(55.0)
            right.fill_(55.0)
            assert (both == 55.0).all()


def test_forward_mode_derivatives_are_refused():
    """A result without a tangent would count as one whose tangent is 0."""
    _say("forward mode")
    import torch.autograd.forward_ad as fw
    z, v = torch.randn(6, 40, device="cuda"), torch.randn(6, 40, device="cuda")
    y = torch.zeros(6, dtype=torch.int32, device="cuda")
    f = torch.zeros(6, device="cuda")
    o = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    stats = ops.token_logprobs(z, y)[1]
    with fw.dual_level():
        for primal in (z, z.clone().requires_grad_()):
            d = fw.make_dual(primal, v)
            for call in (lambda: ops.dropout(d, 0.1, 1), lambda: ops.dropout(z, 0.1, 1, residual=d),
                         lambda: ops.token_logprobs(d, y)):
                with pytest.raises(NotImplementedError):
                    call()
        d, df = fw.make_dual(z, v), fw.make_dual(f, f + 1)
        for call in (lambda: ops.dropout_backward(d, 0.1, 1), lambda: ops.token_logprobs_backward(d, y, stats, f),
                     lambda: ops.token_logprobs_backward(z, y, stats, df), lambda: ops.preference_loss(d, y, o),
                     lambda: ops.preference_loss(z, y, o, ref_logprobs=df), lambda: ops.policy_loss(d, y, f, f),
                     lambda: ops.policy_loss(z, y, f, df)):
            with pytest.raises(NotImplementedError, match="tangent"):
                call()
        primal = fw.unpack_dual(d).primal
        assert torch.equal(ops.dropout(primal, 0.1, 1), ops.dropout(z, 0.1, 1))   # without its tangent
    assert ops.dropout(z, 0.1, 1).shape == z.shape


@pytest.mark.parametrize("requires_grad", [False, True])
def test_traces_are_refused(requires_grad):
    """torch.jit.trace and make_fx would record a result as a constant and give it for other inputs, too."""
    _say("traces", requires_grad)
    from torch.fx.experimental.proxy_tensor import make_fx
    z = torch.randn(6, 40, device="cuda", requires_grad=requires_grad)
    y = torch.zeros(6, dtype=torch.int32, device="cuda")
    f = torch.zeros(6, device="cuda")
    o = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    stats = ops.token_logprobs(z.detach(), y)[1]
    for call in (lambda a: a + ops.dropout(a, 0.1, 1), lambda a: a + ops.dropout_backward(a, 0.1, 1),
                 lambda a: a.sum() + ops.token_logprobs(a, y)[0], lambda a: a + ops.token_logprobs_backward(a, y, stats, f),
                 lambda a: a.sum() + ops.preference_loss(a, y, o)[0], lambda a: a.sum() + ops.policy_loss(a, y, f, f)[0]):
        with pytest.raises(NotImplementedError, match="trace"):
            torch.jit.trace(call, (z,), check_trace=False)
        with pytest.raises(NotImplementedError, match="trace"):
            make_fx(call)(z.detach())
    assert ops.dropout(z.detach(), 0.1, 1).shape == z.shape


def test_views_that_negate_are_refused():
    """The imaginary part of a conjugate holds the values with the other sign, and a mark."""
    _say("negated views")
    z = torch.randn(6, 1, dtype=torch.complex64, device="cuda")
    neg, real = z.conj().imag, z.real.contiguous()
    y = torch.zeros(6, dtype=torch.int32, device="cuda")
    f, minus = torch.ones(6, device="cuda"), torch._neg_view(torch.ones(6, device="cuda"))
    assert neg.is_neg() and minus.is_neg()
    for call in (lambda: ops.dropout(neg, 0.0, 1), lambda: ops.dropout(real, 0.0, 1, residual=neg),
                 lambda: ops.dropout(real, 0.0, 1, out=neg), lambda: ops.token_logprobs(neg, y),
                 lambda: ops.policy_loss(real, y, f, minus), lambda: ops.policy_loss(real, y, f, f, token_weights=minus)):
        with pytest.raises(ValueError, match="resolve_neg"):
            call()
    assert torch.equal(ops.dropout(neg.resolve_neg(), 0.0, 1), -z.imag)


def test_outputs_that_ask_for_a_gradient_are_refused():
    """Parameters and a graph's tensors are not overwritten unnoticed; logits may be replaced by their gradient."""
    _say("out asks for a gradient")
    z = torch.randn(6, 40, device="cuda")
    y = torch.zeros(6, dtype=torch.int32, device="cuda")
    f = torch.linspace(-1, 1, 6, device="cuda")
    o = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    lp, stats = ops.token_logprobs(z, y)
    calls = [lambda a, out: ops.dropout(a, 0.1, 1, out=out), lambda a, out: ops.dropout_backward(a, 0.1, 1, out=out),
             lambda a, out: ops.token_logprobs_backward(a, y, stats, f, out=out),
             lambda a, out: ops.preference_loss(a, y, o, lp + f, out=out)[3], lambda a, out: ops.policy_loss(a, y, lp, f, out=out)[2]]
    leaf = torch.full((6, 40), 5.0, device="cuda", requires_grad=True)
    inner = leaf + 0
    for call in calls:
        for out in (leaf, inner, inner[:, :]):
            with pytest.raises(ValueError, match="out must not ask for a gradient"):
                call(z, out)
            with pytest.raises(ValueError):
                call(leaf, leaf)
        assert (leaf == 5.0).all() and (inner == 5.0).all()
        want = call(z, None)
        with torch.no_grad():
            assert torch.equal(call(z, torch.zeros(6, 40, device="cuda", requires_grad=True)), want)
    for call in calls[2:]:
        w = z.clone().requires_grad_()
        logits = w * 1
        want = call(z, None)
        assert call(logits, logits) is logits
        logits.backward(logits.detach())
        assert torch.equal(w.grad, want)


def test_losses_in_a_differentiated_sum_raise():
    """Without a graph they would be missing in the sum's gradient, without a word."""
    _say("losses without a graph")
    w = torch.randn(6, 40, device="cuda", requires_grad=True)
    y = torch.zeros(6, dtype=torch.int32, device="cuda")
    f = torch.linspace(-1, 1, 6, device="cuda")
    o = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    for call in (lambda a, **kw: ops.preference_loss(a, y, o, f, **kw), lambda a, **kw: ops.policy_loss(a, y, f, f, **kw)):
        z = w * 2
        got = call(z)
        for gradient in (True, False):
            for value in call(z, gradient=gradient)[:-1]:
                with pytest.raises(RuntimeError, match="dlogits"):
                    ((w * w).sum() + value.sum()).backward(retain_graph=True)
        assert w.grad is None
        want = call(z.detach())
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert not got[-1].requires_grad and call(z, gradient=False)[-1] is None
        z.backward(got[-1])
        assert torch.equal(w.grad, 2 * want[-1])
        w.grad = None
        with torch.no_grad():
            assert not any(t.requires_grad for t in call(z))
        assert not any(t.requires_grad for t in call(z.detach()))


# More rows than the grid's first dimensions hold: 2^20 blocks (x), 65,535 (y of the kernels whose x goes along a row).
GRID_ROWS = (1 << 20) + 3


def _ends(rows):
    """The first rows, those around either limit and the last, as slices."""
    return [slice(a, min(rows, a + 5)) for a in (0, 65_533, (1 << 20) - 2, rows - 5) if a < rows]


@pytest.mark.parametrize("dtype,cols", [("bf16", 4112), ("f16", 1031), ("f32", 300)])
def test_more_rows_than_one_grid_dimension(dtype, cols):
    """A block, half of one or a quarter per row: rows around the limits have the bits that they have alone."""
    rows = 8 * GRID_ROWS if cols == 300 else 4 * GRID_ROWS if cols == 1031 else GRID_ROWS
    _say("grid", dtype, rows, cols)
    z = torch.empty(rows, cols, dtype=DTYPES[dtype], device="cuda").fill_(0.25)
    y = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(cols)
    ends = _ends(rows)
    for part in ends:
        z[part].normal_(generator=gen)
        y[part] = torch.randint(0, cols, (len(y[part]),), generator=gen, device="cuda").to(torch.int32)
    alone = [z[part].clone() for part in ends]
    f = torch.linspace(-1, 1, rows, device="cuda")
    lp, stats = ops.token_logprobs(z, y)
    want = [ops.token_logprobs(a, y[part]) for a, part in zip(alone, ends)]
    for (l, s), part in zip(want, ends):
        assert torch.equal(lp[part], l) and torch.equal(stats[part], s) and l.isfinite().all()
    assert int((lp != 0).sum()) == int((y >= 0).sum())
    out = ops.token_logprobs_backward(z, y, stats, f)
    for a, (_, s), part in zip(alone, want, ends):
        assert torch.equal(out[part], ops.token_logprobs_backward(a, y[part], s, f[part]))
    loss, _, _ = ops.policy_loss(z, y, lp, f, out=out)
    for a, (l, _), part in zip(alone, want, ends):
        got = ops.policy_loss(a, y[part], l, f[part])
        assert torch.equal(loss[part], got[0]) and torch.equal(out[part], got[2])
    assert int((loss != 0).sum()) == int((y >= 0).sum())
    ops.dropout(z, 0.3, 5, first_row=7, out=out)
    for a, part in zip(alone, ends):
        assert torch.equal(out[part], ops.dropout(a, 0.3, 5, first_row=7 + part.start))
    # The untouched rows in between, by a second call over all but the first.
    z, first = z[1:], out[1:]
    assert torch.equal(ops.dropout(z, 0.3, 5, first_row=8), first)


def test_more_short_rows_than_one_grid_dimension():
    """256 rows to a block, one value each: 2^28 rows and some."""
    rows = (1 << 28) + 77
    _say("grid, short rows", rows)
    z = torch.zeros(rows, 1, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(rows, dtype=torch.int32, device="cuda")
    y[-80:-70] = -1
    lp, stats = ops.token_logprobs(z + 2, y)
    assert not lp.any() and int((stats[:, 0] == 2.0).sum()) == rows - 10 and not stats[-80:-70].any()
    out = ops.dropout(z + 1, 0.5, 3)
    want = ops.dropout(z[-300:] + 1, 0.5, 3, first_row=rows - 300)
    assert torch.equal(out[-300:], want)
    # Of so many fair draws the kept ones number half, to five standard deviations.
    assert abs(int((out != 0).sum()) - rows / 2) < 5 * (rows / 4) ** 0.5
    assert (out[: 1 << 20] == ops.dropout(z[: 1 << 20] + 1, 0.5, 3)).all()


def test_policy_loss_with_a_vanishing_kl_factor():
    """Below what 32 bits hold it is no factor: the results are those without the KL term, also where that is infinite."""
    _say("vanishing kl")
    z, y = _case("f32", 9, 40, 3)
    z, y = z.cuda(), y.clamp(0, 39).cuda()
    z[3, y[3]] = -INF
    old = torch.full((9,), -4.0, device="cuda")
    far = old + 200.0                     # exp(ref - l) overflows
    adv = torch.linspace(-1, 1, 9, device="cuda")
    want = ops.policy_loss(z, y, old, adv)
    assert want[0].isfinite().all() and want[2].isfinite().all()
    for kl in (1e-60, -1e-60):
        for a, b in zip(ops.policy_loss(z, y, old, adv, ref_logprobs=far, kl=kl), want):
            assert torch.equal(a, b)


def test_views_of_parameters_are_not_replaced_by_a_gradient():
    """A view of a parameter is no model's output, though it is no leaf itself; nor is its memory under another name."""
    _say("views of parameters")
    y = torch.zeros(6, dtype=torch.int32, device="cuda")
    f = torch.linspace(-1, 1, 6, device="cuda")
    o = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    leaf = torch.randn(6, 40, device="cuda", requires_grad=True)
    was = leaf.detach().clone()
    stats = ops.token_logprobs(was, y)[1]
    for call in (lambda a, out: ops.token_logprobs_backward(a, y, stats, f, out=out),
                 lambda a, out: ops.preference_loss(a, y, o, f, out=out), lambda a, out: ops.policy_loss(a, y, f, f, out=out)):
        view = leaf[:, :]
        for logits, out in [(view, view), (leaf.detach(), view), (leaf.detach(), leaf), (view, leaf)]:
            with pytest.raises(ValueError, match="out must not ask for a gradient"):
                call(logits, out)
        assert torch.equal(leaf.detach(), was)
        model = leaf * 2
        part = model[:, :]                   # of a model's output, which may go
        call(part, part)
