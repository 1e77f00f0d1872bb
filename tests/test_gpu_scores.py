"""Scores of tokens and their gradient on the GPU against the 64-bit oracle: sizes around every unit of
work, types, strides and alignments, equal logits, masked rows and tokens, refusals, autograd, graphs.

Tolerances follow from the formulas, with u = 2^-24 and d, D, the sums' n_c and `U`, `TINY` as for the
log-probabilities: a term e^-d has an error of u (3 d + 4), a sum n_c u more.  Further:
  - entropy: a term e^-d d has u (3 d + 6); beside it the sum that is rescaled whenever the maximum
    rises carries three roundings a step, n_c of them; the quotient has the sums' errors and 3 u;
  - gradient: p has the error of the log-probability, its factor those of g, e, ln p and H.
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
    assert got.shape == want.shape, what
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all(), (what, "NaN places")
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all(), (what, "infinities")
    rest = ~(nan | inf)
    off = np.abs(got[rest] - want[rest])
    bad = ~(off <= tol[rest])
    assert not bad.any(), (what, int(bad.sum()), float((off - tol[rest]).max()), float(off.max()))


def _case(dtype, rows, cols, seed, spread=2.0, levels=None, banned=False):
    """Logits on the CPU in their type (rounded to multiples of 1 / levels: many equal ones), targets with some
    rows without a token."""
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(rows, cols)) * spread
    if levels:
        z = np.round(z * levels) / levels
    if banned:
        z[:, rng.random(cols) < 0.3] = -INF
    y = rng.integers(0, cols, rows).astype(np.int32)
    if rows > 2:
        y[rng.integers(0, rows)] = -1
        y[rng.integers(0, rows)] = cols
    return torch.from_numpy(z.astype(np.float32)).to(DTYPES[dtype]), torch.from_numpy(y)


class _Expected:
    """The oracle's values, and the errors that evaluation in 32 bits allows."""

    def __init__(self, z, y, top):
        self.z, self.y = z.double().numpy(), None if y is None else y.numpy()
        rows, cols = self.z.shape
        self.on = O.read_rows(self.z, self.y)
        self.peak, self.log_sum = O.row_stats(self.z)
        with np.errstate(invalid="ignore", over="ignore"):
            self.d = np.where(np.isneginf(self.z), 0.0, self.peak[:, None] - self.z)
            self.p = np.nan_to_num(np.exp(self.z - self.peak[:, None] - self.log_sum[:, None]))
            pd = self.p * self.d
            chain = 64 + cols / 64 + 4
            self.sum_rel = u * (chain + 3 * pd.sum(1))
            self.h = O.entropy(self.z, self.y)
            quotient = pd.sum(1)
            self.ln_tol = self.sum_rel + 4 * u * np.abs(self.log_sum)
            self.h_tol = (self.ln_tol + u * (pd * (3 * self.d + 6 + 3 * chain)).sum(1) + quotient * (self.sum_rel + 3 * u) +
                          2 * u * np.abs(self.h))
            self.lp = None if y is None else O.token_logprobs(self.z, self.y)
            self.top_lp, self.tokens = O.top_tokens(self.z, top, self.y)
            self.lp_tol = self.lp_tols(self.lp) if y is not None else None
            self.top_tol = self.lp_tols(self.top_lp)

    def lp_tols(self, lp):
        """Of log-probabilities -d - ln S, whose d is at most |l| + |ln S|."""
        rows = (slice(None),) + (None,) * (lp.ndim - 1)
        d = np.abs(np.where(np.isfinite(lp), lp, 0.0)) + np.abs(self.log_sum[rows])
        return np.nan_to_num(self.sum_rel[rows] + u * (8 + 2 * d + 4 * np.abs(self.log_sum[rows])))

    def gradient(self, g, e, dtype):
        want = O.token_scores_backward(self.z, self.y, g, e)
        zero = np.zeros(len(self.z))
        g, e = (zero if a is None else np.abs(a.astype(np.float64)) for a in (g, e))
        with np.errstate(invalid="ignore"):
            ln = np.where(np.isneginf(self.z), 0.0, self.log_sum[:, None] + self.d)
            rel = self.sum_rel[:, None] + u * (3 * self.d + 4 * np.abs(self.log_sum)[:, None] + 8)
            size = g[:, None] + e[:, None] * np.abs(self.h[:, None] - ln)
            parts = self.d + np.abs(self.log_sum)[:, None] + np.abs(self.h)[:, None]
            factor = e[:, None] * ((self.h_tol + self.ln_tol)[:, None] + 4 * u * parts) + 3 * u * size
            tol = np.nan_to_num(self.p * (size * rel + factor) + 2 * u * np.abs(want))
        if self.y is not None:
            for t in np.flatnonzero(self.on):
                tol[t, self.y[t]] += 2 * u * g[t]
        tol[~self.on] = 0.0
        return want, np.nan_to_num(tol * (1 + U[dtype]) + U[dtype] * np.abs(want) + TINY[dtype])


def _check(z, y, top, dtype, pad=0, shift=0, gradient=True, seed=0):
    e = _Expected(z, y, top)
    zg, yg = _place(z, pad, shift, fill=100.0)[1], None if y is None else y.cuda()
    lp, h, top_lp, tokens, stats = ops.token_scores(zg, yg, top)
    assert tokens.dtype == torch.int32 and tokens.shape == (len(z), top)
    assert (tokens.cpu().numpy() == e.tokens).all(), "tokens"
    _close(top_lp, e.top_lp, e.top_tol, "top log-probabilities")
    if y is None:
        assert lp is None
    else:
        _close(lp, e.lp, e.lp_tol, "logprobs")
    _close(h, e.h, np.nan_to_num(e.h_tol), "entropy")
    fine = e.on & ~np.isnan(e.log_sum)
    _close(stats[:, 0].cpu().numpy()[fine], e.peak[fine], 0.0, "maxima")
    _close(stats[:, 1].cpu().double().numpy()[fine], e.log_sum[fine], e.ln_tol[fine], "log sums")
    assert not stats[torch.from_numpy(~e.on).cuda()].any() and torch.isnan(stats[torch.from_numpy(e.on & np.isnan(e.log_sum)).cuda()]).all()
    if not gradient:
        return
    rng = np.random.default_rng(seed)
    g, ge = (rng.normal(size=len(z)).astype(np.float32) for _ in range(2))
    g[0] = ge[-1] = 0.0
    for given, with_h in [(True, True), (True, False), (False, True)]:
        if given and y is None:
            continue
        gg, ee = torch.from_numpy(g).cuda() if given else None, torch.from_numpy(ge).cuda() if with_h else None
        buf, out = _place(torch.zeros_like(z), pad, shift, fill=77.0)
        dz = ops.token_scores_backward(zg, yg, stats, h, gg, ee, out=out)
        _close(dz, *e.gradient(g if given else None, ge if with_h else None, dtype), "gradient")
        out.fill_(77.0)
        assert (buf == 77.0).all(), "values outside of the output were written"


COLS = [1, 2, 3, 5, 7, 8, 9, 10, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 255, 256, 257, 500, 513, 1000, 1024,
        1025, 2047, 2048, 2049, 4095, 4097, 8191, 8193, 12289, 16384, 16391, 32767, 40001, 50021, 65536, 65537, 100003,
        131071, 131072, 131073, 262147]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_scores_match_the_oracle(dtype, cols):
    for case, (top, given, pad, shift, banned) in enumerate([(5, True, 0, 0, False), (20, False, 3, 1, True), (64, True, 0, 3, True),
                                                             (0, True, 0, 0, False), (1, False, 2, 7, False)]):
        _say("scores", dtype, cols, case)
        rows = (37 if cols <= 64 else 11 if cols <= 4096 else 5) if case == 0 else 3
        z, y = _case(dtype, rows, cols, cols * 31 + case, banned=banned)
        _check(z, y if given else None, top, dtype, pad, shift, seed=case)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [10, 100, 1000, 9001, 70001])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 15, 17, 31, 64, 65, 127, 257, 511])
def test_scores_of_any_number_of_rows(dtype, cols, rows):
    rows = min(rows, max(6, 2_000_000 // cols))
    _say("scores rows", dtype, cols, rows)
    z, y = _case(dtype, rows, cols, rows)
    _check(z, y, 7, dtype, seed=rows)


def _hard_rows(cols, seed):
    """Orders and repetitions that a search for the largest can stumble over."""
    rng = np.random.default_rng(seed)
    up = np.arange(cols, dtype=np.float64)
    every = [up / cols, -up / cols, np.zeros(cols), np.round(rng.normal(size=cols) * 2), (up % 7) / 7, (up // 64) / cols * 8,
             np.where(rng.random(cols) < 0.5, 1.0, 0.0), np.where(up % 512 == 3, 5.0 + up / cols, rng.normal(size=cols)),
             np.where(up >= cols - 70, 3.0, 0.0), np.where(up < 70, 3.0 - up / 100, rng.normal(size=cols) - 5),
             np.where(up == cols // 2, 1.0, -INF), np.where(up % 2 == 0, -0.0, 0.0), -np.abs(rng.normal(size=cols)) * 20,
             up % 1024 * 8 / 1024 + up / cols / 64]
    return torch.from_numpy(np.stack(every).astype(np.float32))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [1, 8, 33, 64])
@pytest.mark.parametrize("cols", [3, 10, 65, 100, 513, 1000, 2500, 4097, 9001, 20000, 70001, 131072, 200001])
def test_top_tokens_of_equal_and_ordered_logits(dtype, top, cols):
    _say("top of equal logits", dtype, top, cols)
    for case, shift in enumerate((0, 1)):
        z = _hard_rows(cols, cols + case).to(DTYPES[dtype])
        _check(z, None, top, dtype, shift, shift, gradient=False)


def _special_rows(dtype, cols):
    low, high = torch.finfo(DTYPES[dtype]).min, torch.finfo(DTYPES[dtype]).max
    base, last = torch.linspace(-1, 1, cols), cols - 1
    rows = [base, torch.full((cols,), -INF), torch.full((cols,), low), torch.full((cols,), high), base.clone(), base.clone(),
            base.clone(), torch.full((cols,), -INF), base.clone(), torch.full((cols,), -INF), base]
    rows[4][last] = float("nan")
    rows[5][0] = INF
    rows[6][last] = -INF          # the target itself cannot occur
    rows[7][last] = -2.0          # only the target can
    rows[8][0], rows[8][last] = high, low
    rows[9][0] = float("nan")
    return torch.stack(rows).to(DTYPES[dtype]), torch.full((len(rows),), last, dtype=torch.int32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [2, 10, 65, 513, 1001, 4097, 20000, 70001, 131072, 200001])
def test_special_rows(dtype, cols):
    """Masks that leave nothing or one token, lowest values, NaN and infinities in one row and not the next."""
    _say("special scores", dtype, cols)
    z, y = _special_rows(dtype, cols)
    for top in (0, 3, 64):
        e = _Expected(z, y, top)
        for targets in (y, None):
            lp, h, top_lp, tokens, stats = ops.token_scores(z.cuda(), None if targets is None else y.cuda(), top)
            assert (tokens.cpu().numpy() == e.tokens).all()
            # Distances past what 32 bits hold are infinite ones.
            far = np.abs(e.top_lp) > float(np.finfo(np.float32).max)
            _close(top_lp, np.where(far, -INF, e.top_lp), e.top_tol, "top")
            _close(h, e.h, np.nan_to_num(e.h_tol, posinf=0.0), "entropy")
            if targets is not None:
                _close(lp, np.where(np.abs(e.lp) > float(np.finfo(np.float32).max), -INF, e.lp), e.lp_tol, "logprobs")
    lp, h, _, _, stats = ops.token_scores(z.cuda(), y.cuda())
    one = np.ones(len(z), np.float32)
    with np.errstate(invalid="ignore"):
        want, tol = e.gradient(one, 0.5 * one, dtype)
    got = ops.token_scores_backward(z.cuda(), y.cuda(), stats, h, torch.ones(len(z), device="cuda"), torch.full((len(z),), 0.5, device="cuda"))
    _close(got, want, tol, "gradient")
    # Rows that are not read: no token, or no gradient.
    none, zero = torch.full_like(y, -1).cuda(), torch.zeros(len(z), device="cuda")
    lp, h, top_lp, tokens, st = ops.token_scores(z.cuda(), none, 4)
    assert not lp.any() and not h.any() and not top_lp.any() and not st.any() and (tokens == -1).all()
    assert not ops.token_scores_backward(z.cuda(), none, stats, h, zero + 1, zero + 1).any()
    assert not ops.token_scores_backward(z.cuda(), y.cuda(), stats, h, zero, zero).any()
    assert not ops.token_scores_backward(z.cuda(), None, stats, zero, None, zero).any()


def _spiked_rows(cols):
    """Values that the sums' reference points do not fit: the maximum far above or below the rest, at the front, in the
    middle, at the end; slopes over the whole row; parts of nothing but -inf."""
    rng = np.random.default_rng(cols)
    base, at = rng.normal(size=cols), np.arange(cols)
    rows = [base.copy() for _ in range(9)]
    rows[0][:8] += 300.0
    rows[1][-1] += 300.0
    rows[2][cols // 2] += 50.0
    rows[3][:cols // 2] -= 400.0
    rows[4][cols // 2:] -= 400.0
    rows[5] = at / cols * 200.0 - 100.0
    rows[6] = -at / cols * 200.0
    rows[7][:cols - cols // 3] = -INF
    rows[8] = np.where(at % 64 < 8, -INF, base + (at // 4096) * 13.0)
    return torch.from_numpy(np.stack(rows).astype(np.float32))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [9, 64, 513, 1000, 4100, 9001, 20000, 33000, 70001, 131073, 262147])
def test_maxima_far_from_the_rest(dtype, cols):
    _say("spikes", dtype, cols)
    for shift in (0, 1):
        z = _spiked_rows(cols).to(DTYPES[dtype])
        y = torch.from_numpy(np.random.default_rng(cols).integers(0, cols, len(z)).astype(np.int32))
        _check(z, y, 11, dtype, shift, shift)
        more = 70    # more rows than have blocks for their parts
        many = ops.token_scores(torch.cat([z, z[:1].expand(more, cols)]).cuda(), None, 11)
        few = ops.token_scores(z.cuda(), None, 11)
        for a, b in zip(many[1:], few[1:]):
            assert torch.equal(a[:len(z)], b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [7, 300, 1000, 4100, 20000, 70001, 140003, 300001])
def test_values_past_what_whole_numbers_reach(dtype, cols):
    """Logits past 2^20 in the whole row, in one stretch of it, or at its ends: there the sums take another way."""
    _say("large values", dtype, cols)
    rng = np.random.default_rng(cols)
    base = rng.normal(size=cols)
    rows = [base * 3.0 + 5e6, base * 2.0, base * 2.0, base * 2.0, base * 1e7, base - 4e8, base * 2.0, -np.abs(base) * 1e30]
    rows[1][cols // 2:cols // 2 + cols // 8 + 1] += 3e6
    rows[2][:1] = 1e9
    rows[3][-1:] = 2e6
    rows[6][cols // 3:cols // 2] -= 5e7
    z = torch.from_numpy(np.stack(rows).astype(np.float32)).to(DTYPES[dtype])
    y = torch.from_numpy(rng.integers(0, cols, len(z)).astype(np.int32))
    for shift in (0, 1):
        _check(z, y, 9, dtype, shift, shift)
    many = ops.token_scores(torch.cat([z, z[1:2].expand(70, cols)]).cuda(), None, 9)
    few = ops.token_scores(z.cuda(), None, 9)
    for a, b in zip(many[1:], few[1:]):
        assert torch.equal(a[:len(z)], b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [10, 64, 1000, 9001, 131071])
def test_logits_of_large_magnitude(dtype, cols):
    _say("scores magnitude", dtype, cols)
    z, y = _case(dtype, 4, cols, cols, spread=30.0)
    z = (z.float() + torch.tensor([[0.0], [3000.0], [-3000.0], [100.0]])).to(DTYPES[dtype])
    _check(z, y, 9, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [9, 100, 1000, 4099, 20011, 131072])
def test_a_row_has_the_same_bits_wherever_it_lies(dtype, cols):
    """Alone and among many, at any alignment and stride, with or without targets, top tokens or a gradient in
    place; and the stats of token_logprobs' meaning."""
    _say("same bits", dtype, cols)
    z, y = _case(dtype, 6, cols, cols, levels=16)
    y.clamp_(0, cols - 1)
    zg, yg = z.cuda(), y.cuda()
    want = ops.token_scores(zg, yg, 6)
    g, e = (torch.randn(6, device="cuda") for _ in range(2))
    dz = ops.token_scores_backward(zg, yg, want[4], want[1], g, e)
    for shift in (1, 2, 5):
        other = _place(z, 2 * shift + 1, shift)[1]
        for a, b in zip(ops.token_scores(other, yg, 6), want):
            assert torch.equal(a, b)
        assert torch.equal(ops.token_scores_backward(other, yg, want[4], want[1], g, e), dz)
    for t in range(6):
        for a, b in zip(ops.token_scores(zg[t:t + 1], yg[t:t + 1], 6), want):
            assert torch.equal(a, b[t:t + 1])
    more = max(700, min(5000, 20_000_000 // cols))
    many = ops.token_scores(torch.cat([zg, zg[:1].expand(more, cols)]), torch.cat([yg, yg[:1].expand(more)]), 6)
    for a, b in zip(many, want):
        assert torch.equal(a[:6], b) and torch.equal(a[6:], b[:1].expand_as(a[6:]))
    _, h, top_lp, tokens, stats = ops.token_scores(zg, None, 3)
    for a, b in [(h, want[1]), (top_lp, want[2][:, :3]), (tokens, want[3][:, :3]), (stats, want[4])]:
        assert torch.equal(a, b)
    assert torch.equal(ops.token_scores(zg, yg)[0], want[0])
    place = zg.clone()
    assert torch.equal(ops.token_scores_backward(place, yg, want[4], want[1], g, e, out=place), dz)


def test_scores_of_more_values_than_32_bits_count():
    _say("scores past 2^32 values")
    rows, cols = 33000, 131073
    z = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    y = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, rows // 2, rows - 1], device="cuda")
    z[at, cols - 1] = 3.0
    y[at] = cols - 1
    lp, h, top_lp, tokens, stats = ops.token_scores(z, y, 2)
    s = np.exp(-3.0) * (cols - 1) + 1.0
    assert (tokens[at].cpu() == torch.tensor([cols - 1, 0], dtype=torch.int32)).all() and (tokens[1] == -1).all()
    tol = u * (64 + cols / 64 + 40)
    assert (lp[at].double() + np.log(s)).abs().max() < tol * 2
    h64 = np.log(s) + 3.0 * np.exp(-3.0) * (cols - 1) / s
    assert (h[at].double() - h64).abs().max() < tol * 8
    dz = ops.token_scores_backward(z, y, stats, h, None, torch.ones(rows, device="cuda"), out=z)
    assert dz.data_ptr() == z.data_ptr() and not dz[1].any() and dz[at].float().sum(1).abs().max() < 0.05
    assert (dz[rows - 1, cols - 1] != 0) and (dz[rows - 1, 0] != 0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_a_row_of_the_most_columns(dtype):
    cols = 2 ** 31 - 1
    _say("longest row", dtype)
    z = torch.empty(1, cols, dtype=dtype, device="cuda").normal_(0.0, 0.1)
    at = [cols - 1, 0, cols // 2 + 3, 5, 2 ** 28 + 1, cols - 2]   # 0.1-sigma values stay far below
    for i, c in enumerate(at):
        z[0, c] = 3.0 - i / 16
    y = torch.tensor([cols - 1], dtype=torch.int32, device="cuda")
    lp, h, top_lp, tokens, stats = ops.token_scores(z, y, len(at))
    assert tokens[0].tolist() == at and stats[0, 0].item() == 3.0
    total = moved = 0.0
    for part in z[0].split(2 ** 27):
        d = part.double() - 3.0
        e = d.exp()
        total, moved = total + e.sum().item(), moved + (e * d).sum().item()
    # A lane adds cols / (4 parts of 512 lanes) values of a row one after the other, to W each by itself.
    n = cols / 2048
    assert abs(lp.item() + np.log(total)) < u * (n + 64) + u * 64
    assert abs(h.item() - (np.log(total) - moved / total)) < u * (2 * n + 128) * (1.0 - moved / total) + u * 64
    for i, c in enumerate(at):
        assert abs(top_lp[0, i].item() - (lp.item() + z[0, c].item() - 3.0)) <= u * 64
    g = torch.tensor([1.0], device="cuda")
    dz = ops.token_scores_backward(z, y, stats, h, g, None, out=z)
    # p is 2e-10 to 1e-8 (exp(3) of the largest): in fp16 less than half the smallest number.
    assert abs(dz[0, cols - 1].item() - 1.0) < 1e-6
    if dtype == torch.float16:
        assert sum(torch.count_nonzero(part).item() for part in dz[0].split(2 ** 27)) == 1
    else:
        for i, c in enumerate(at[1:], 1):
            p = np.exp(lp.item() - i / 16)
            assert abs(dz[0, c].item() + p) < p * u * 256
        assert all((part < 0).sum().item() >= part.numel() - 1 for part in dz[0].split(2 ** 27))


def test_more_rows_than_one_grid_dimension():
    _say("many rows")
    rows = (1 << 20) + 77
    z = torch.randn(rows, 3, device="cuda")
    y = torch.randint(0, 3, (rows,), device="cuda", dtype=torch.int32)
    lp, h, top_lp, tokens, stats = ops.token_scores(z, y, 2)
    p = torch.softmax(z.double(), 1)
    assert (lp.double() - p.gather(1, y.long()[:, None])[:, 0].log()).abs().max() < 64 * u
    assert (h.double() + (p * p.log()).sum(1)).abs().max() < 128 * u
    assert torch.equal(tokens.long(), z.topk(2, 1).indices)
    dz = ops.token_scores_backward(z, None, stats, h, None, torch.ones(rows, device="cuda"))
    want = -p * (p.log() + h.double()[:, None])
    assert (dz.double() - want).abs().max() < 256 * u


def test_autograd_gradients_and_differences():
    """Through logprobs, entropy and both, against the oracle's differences: truncation of order step^2 = 1e-8 of
    third derivatives below 10 and 32-bit errors."""
    _say("scores autograd")
    rng = np.random.default_rng(3)
    rows, cols, step = 9, 41, 1e-4
    z64 = torch.from_numpy(rng.normal(size=(rows, cols))).float()
    y = torch.from_numpy(rng.integers(-1, cols, rows).astype(np.int32))
    v, a, b = rng.normal(size=(rows, cols)), rng.normal(size=rows), rng.normal(size=rows)
    ag, bg = (torch.from_numpy(w).float().cuda() for w in (a, b))
    for with_lp, with_h in [(True, True), (True, False), (False, True)]:
        z = z64.cuda().requires_grad_()
        lp, h, top_lp, tokens, stats = ops.token_scores(z, y.cuda(), 3)
        assert lp.requires_grad and h.requires_grad and not top_lp.requires_grad and not stats.requires_grad
        ((lp * ag).sum() * with_lp + (h * bg).sum() * with_h if with_lp and with_h else (lp * ag).sum() if with_lp else (h * bg).sum()).backward()

        def value(x):
            return (O.token_logprobs(x, y) * a).sum() * with_lp + (O.entropy(x, y.numpy()) * b).sum() * with_h
        base = z64.double().numpy()
        d = (value(base + step * v) - value(base - step * v)) / (2 * step)
        assert abs((_np(z.grad) * v).sum() - d) < 1e-6 + 200 * u * np.abs(v).sum()
    z = z64.cuda().requires_grad_()
    lp, h, *_ = ops.token_scores(z)
    assert lp is None
    h.expand(3, rows).sum().backward()                     # a gradient that is broadcast
    e = _Expected(z64, None, 0)
    _close(z.grad, *e.gradient(None, np.full(rows, 3.0, np.float32), "f32"), "broadcast gradient")
    z = z64.cuda().requires_grad_()
    dz, = torch.autograd.grad(ops.token_scores(z)[1].sum(), z, create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable"):
        dz.sum().backward()
    with torch.no_grad():
        assert not ops.token_scores(z)[1].requires_grad


def test_scores_in_a_graph_and_on_a_side_stream():
    """Captured with its gradient, replayed on new logits between eager calls."""
    _say("scores graph")
    for rows, cols, top in [(1, 131072, 20), (40, 1000, 5), (3, 20001, 64)]:
        z, y = (t.cuda() for t in _case("bf16", rows, cols, 1))
        g = torch.randn(rows, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())

        def once():
            lp, h, top_lp, tokens, stats = ops.token_scores(z, y, top)
            return lp, h, top_lp, tokens, stats, ops.token_scores_backward(z, y, stats, h, g, g)
        with torch.cuda.stream(side):
            eager = once()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for a, b in zip(eager, once()):
            assert torch.equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = once()
        for replay in range(3):
            z.copy_(_case("bf16", rows, cols, 7 + replay)[0])
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(captured, once()):
                assert torch.equal(a, b), replay


def test_scores_refuse_what_does_not_fit():
    _say("scores refusals")
    z, y, f = torch.randn(6, 40, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, device="cuda")
    stats = torch.zeros(6, 2, device="cuda")
    for call in [lambda: ops.token_scores(z[0]), lambda: ops.token_scores(z.double()), lambda: ops.token_scores(z.t()),
                 lambda: ops.token_scores(z, y.long()), lambda: ops.token_scores(z, y[:5]), lambda: ops.token_scores(z, y.cpu()),
                 lambda: ops.token_scores_backward(z, y, stats[:, 0], f, f, f), lambda: ops.token_scores_backward(z, y, stats, f, f.double(), f),
                 lambda: ops.token_scores_backward(z, y, stats, f[:3], f, f),
                 lambda: ops.token_scores_backward(z, y, stats, f, f, f, out=z.half()),
                 lambda: ops.token_scores_backward(z, y, stats, f, f, f, out=z.clone().requires_grad_())]:
        with pytest.raises(ValueError):
            call()
    for call in [lambda: ops.token_scores(z, y, 65), lambda: ops.token_scores(z, y, -1), lambda: ops.token_scores(z[:, :0], y),
                 lambda: ops.token_scores_backward(z, y, stats, f), lambda: ops.token_scores_backward(z, None, stats, f, f, f),
                 lambda: ops.token_scores_backward(z, y, stats, None, f, f),
                 lambda: ops.token_scores_backward(z[:, :20], y, stats, f, f, f, out=z[:, 10:30])]:
        with pytest.raises(P.PGCError):
            call()
    with pytest.raises(TypeError):
        ops.token_scores(z, y, 2.5)
    with pytest.raises(NotImplementedError):
        torch.jit.trace(lambda x: ops.token_scores(x, y)[0], z, check_trace=False)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(NotImplementedError, match="tangent"):
            ops.token_scores(torch.autograd.forward_ad.make_dual(z, torch.ones_like(z)))
    for targets in (None, y[:0]):
        lp, h, top_lp, tokens, st = ops.token_scores(z[:0], targets, 3)
        assert h.shape == (0,) and top_lp.shape == tokens.shape == (0, 3) and st.shape == (0, 2)
        assert (lp is None) == (targets is None)
        assert ops.token_scores_backward(z[:0], targets, st, h, lp, h).shape == (0, 40)


def test_calls_on_several_streams_at_once():
    _say("calls at once")
    z = [torch.randn(rows, 131072, device="cuda").to(torch.bfloat16) for rows in (1, 3, 40)]
    want = [ops.token_scores(x, None, 20)[1:] for x in z]
    streams = [torch.cuda.Stream() for _ in z]
    torch.cuda.synchronize()
    got = [[] for _ in z]
    for _ in range(8):   # rows in parts have a workspace, and each call its own
        for x, s, results in zip(z, streams, got):
            with torch.cuda.stream(s):
                results.append(ops.token_scores(x, None, 20)[1:])
    torch.cuda.synchronize()
    for w, results in zip(want, got):
        assert all(torch.equal(a, b) for r in results for a, b in zip(r, w))


def test_two_graphs_of_one_pool_replayed_in_turn():
    _say("two graphs")
    z = [torch.randn(2, 131072, device="cuda") for _ in range(2)]
    for x in z:
        ops.token_scores(x, None, 9)
    torch.cuda.synchronize()
    pool = torch.cuda.graph_pool_handle()
    graphs, results = [], []
    for x in z:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            results.append(ops.token_scores(x, None, 9)[1:])
        graphs.append(graph)
    for turn in range(4):
        for x in z:
            x.normal_()
        for graph in graphs:   # one after the other, as graphs of one pool may be
            graph.replay()
        torch.cuda.synchronize()
        for x, r in zip(z, results):
            assert all(torch.equal(a, b) for a, b in zip(r, ops.token_scores(x, None, 9)[1:]))
