"""The norm of many gradients and the AdamW step on the GPU against the 64-bit oracle: numbers and sizes of
tensors around every unit of work, types, alignments, strides, 8-bit states, values that are not finite,
refusals, graphs.

Tolerances, with u = 2^-24 and `U` the unit roundoff of a type (`TINY` its smallest normal number):
  - the gradient times the factor has u; m' two products of two roundings (constant, product) and a sum;
    v' one product more and twice the gradient's error: relative, as all its terms are positive;
  - the step m' / (sqrt(v') spread + eps) rate: half of v's error, and two roundings for the root, the
    product, the sum, the quotient and each of rate, spread and eps as constants;
  - x' = x - (x decay + step): the decay's product three, the sum and the difference one each.
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
NAME = {t: n for n, t in DTYPES.items()}
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    ops.lib()


def _say(*what):
    print("\n[gpu case]", *what, flush=True)


def _np(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def _packed(values, dtype, gap=0, shift=0):
    """Tensors one after the other in one vector, `gap` values between them."""
    out, at = [], shift
    buf = torch.full((shift + sum(len(v) + gap for v in values) + 8,), 55.0 if dtype != torch.uint8 else 55, dtype=dtype, device="cuda")
    for v in values:
        buf[at:at + len(v)].copy_(v if torch.is_tensor(v) else torch.from_numpy(np.asarray(v)))
        out.append(buf[at:at + len(v)])
        at += len(v) + gap
    return buf, out


# ---- the norm -------------------------------------------------------------------------------

SIZES = [0, 1, 2, 3, 4, 5, 7, 255, 256, 257, 1023, 1024, 1025, 2049, 4095, 4096, 4097, 8193, 20000]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("count", [1, 2, 19, 63, 64, 65, 128, 200])
def test_grad_norm_matches_the_oracle(dtype, count):
    _say("norm", dtype, count)
    rng = np.random.default_rng(count)
    grads = [torch.from_numpy(rng.normal(size=SIZES[(i * 7 + count) % len(SIZES)])).to(DTYPES[dtype]) for i in range(count)]
    want = O.grad_norm([g.double().numpy() for g in grads])[0]
    alone = None
    for gap, shift in [(0, 0), (0, 1), (3, 5)]:
        on = _packed(grads, DTYPES[dtype], gap, shift)[1]
        for max_norm, scale in [(INF, 1.0), (0.5 * want + 1e-3, 1.0), (1.0, -0.25), (1e30, 2.0 ** -12)]:
            got = ops.grad_norm(on, max_norm, scale)
            norm, factor = O.grad_norm([g.double().numpy() for g in grads], max_norm, scale)
            # Sums in 64 bits; each result is rounded once.
            assert abs(_np(got[0])[0] - norm) <= 1.01 * u * norm and abs(_np(got[1])[0] - factor) <= 1.01 * u * abs(factor)
        norm = ops.grad_norm(on)[0]
        alone = norm if alone is None else alone
        assert torch.equal(norm, alone), "the order of the sum follows from the sizes"


def test_grad_norm_of_large_tensors_and_mixed_types():
    _say("norm large")
    big = torch.randn((1 << 24) + 4099, device="cuda")
    rest = [torch.randn(70001, device="cuda").to(t) for t in DTYPES.values()]
    total = sum(float((g.double() ** 2).sum()) for g in [big] + rest)
    got = ops.grad_norm([big] + rest, 3.0)
    assert abs(float(got[0]) - total ** 0.5) <= 2 * u * total ** 0.5 and abs(float(got[1]) - 3 / total ** 0.5) <= 2 * u * 3 / total ** 0.5
    long = torch.ones((1 << 31) + 9, dtype=torch.bfloat16, device="cuda")
    long[-1] = 2.0 ** 17
    want = ((1 << 31) + 8 + 2.0 ** 34) ** 0.5
    assert abs(float(ops.grad_norm([long])[0]) - want) <= 2 * u * want


def test_grad_norm_at_the_ends_of_the_range():
    """Squares that 32 bits do not hold; zeros; values that are not finite; layouts."""
    _say("norm range")
    for value in (3e38, 1e-38, 2.0 ** -149):
        x = torch.full((1000,), value, device="cuda")
        want = float(x[0].double()) * 1000 ** 0.5
        norm, factor = ops.grad_norm([x], max_norm=2.0)
        if want < 3.4e38:
            assert abs(float(norm) - want) <= 2 * u * want + 2.0 ** -150
        else:
            assert float(norm) == INF
        f = min(1.0, 2.0 / want)
        # 2 / (3e38 sqrt(1000)) = 2.1e-40 lies below 2^-126, where floats are multiples of 2^-149: half of that more.
        assert abs(float(factor) - f) <= 2 * u * f + 2.0 ** -150
    norm, factor = ops.grad_norm([torch.zeros(5, device="cuda"), torch.zeros(0, device="cuda")], 1.0, 0.5)
    assert float(norm) == 0 and float(factor) == 0.5
    norm, factor = ops.grad_norm([torch.zeros(0, device="cuda")])
    assert float(norm) == 0 and float(factor) == 1
    for value in (NAN, INF, -INF):
        x = torch.ones(5000, device="cuda")
        x[4321] = value
        norm, factor = ops.grad_norm([torch.ones(3, device="cuda"), x], 1.0)
        assert not np.isfinite(float(norm)) and np.isnan(float(factor))
    a = torch.randn(3, 5, 7, 2, device="cuda")
    for t in (a.to(memory_format=torch.channels_last), a.permute(3, 1, 0, 2), a[1], a[0, 0, 0, 0]):
        assert abs(float(ops.grad_norm([t])[0]) - float(t.double().norm())) <= 2 * u * float(t.double().norm())


# ---- states in 8 bits -------------------------------------------------------------------------

def test_state_values_match_the_oracle():
    """Every byte under ordinary, tiny, huge, zero and broken scales; short last blocks; both types, gaps and
    odd addresses."""
    _say("state values")
    rng = np.random.default_rng(5)
    scales = np.array([1.0, 1.875, 2.0 ** -126, 2.0 ** -140, 0.0, 1.5 * 2.0 ** 127, NAN, INF, 2.0 ** -100, 0.625], np.float32)
    for count in (1, 3, 255, 256, 257, 2305, 2560):
        blocks = -(-count // 256)
        m, v = (rng.permutation(np.resize(np.arange(256), 2560).astype(np.uint8))[:count] for _ in range(2))
        s = np.stack([scales[:blocks], np.roll(scales, 3)[:blocks]], 1)
        for shift in (0, 1, 3):
            mg, vg = _packed([m], torch.uint8, 0, shift)[1], _packed([v], torch.uint8, 0, shift)[1]
            for dtype in (torch.float32, torch.bfloat16):
                buf, out = _packed([np.zeros(count)], dtype, 0, shift)
                got = ops.adamw_state_values(mg, vg, [torch.from_numpy(s).cuda()], out=(out, [torch.empty(count, dtype=dtype, device="cuda")]))
                for x, codes, scale, signed in [(got[0][0], m, s[:, 0], True), (got[1][0], v, s[:, 1], False)]:
                    assert np.array_equal(_np(x), O.decode_states(codes, scale, signed), equal_nan=True), (count, shift, signed)
                out[0].fill_(55.0)
                assert (buf == 55.0).all()
    a, b, c = ops.adamw_states([torch.zeros(600, device="cuda"), torch.zeros(0, device="cuda")], 8)
    for x in sum(ops.adamw_state_values(a, b, c), []):
        assert not x.any() and x.dtype == torch.float32


def test_8_bit_states_are_rounded_as_the_oracle_rounds():
    """beta1 = beta2 = 1/2 from zero states and gradients of 11 bits: m' = g / 2 and v' = g^2 / 2 are exact, so
    that the bytes have to be the oracle's."""
    _say("8-bit rounding")
    rng = np.random.default_rng(6)
    for spread, low in [(1.0, 0), (8.0, 0), (25.0, -10), (40.0, 0)]:
        for count in (1, 2, 255, 256, 300, 5000, 70001):
            g = rng.normal(size=count) * np.exp2(-rng.uniform(0, spread, count) + low)
            mantissa, exponent = np.frexp(g)
            g = np.ldexp(np.rint(mantissa * 2048) / 2048, exponent).astype(np.float32)
            g[rng.random(count) < 0.1] = 0.0
            x = torch.zeros(count, device="cuda")
            m, v, s = ops.adamw_states([x], 8)
            ops.adamw([x], [torch.from_numpy(g).cuda()], m, v, 1, 1e-3, betas=(0.5, 0.5), scales=s)
            for codes, scale, value, signed in [(m[0], s[0][:, 0], g / 2, True), (v[0], s[0][:, 1], g * g / 2, False)]:
                want, want_scale = O.encode_states(value, signed)
                assert np.array_equal(scale.cpu().numpy(), want_scale), (count, spread, signed)
                assert np.array_equal(codes.cpu().numpy(), want), (count, spread, signed)


# ---- the step -----------------------------------------------------------------------------------

def _expected(x, g, m, v, step, lr, beta1, beta2, eps, decay, factor, dtype):
    """The oracle's (x', m', v') and what 32-bit evaluation may be off."""
    want = O.adamw(x, g, m, v, step, lr, beta1, beta2, eps, decay, factor)
    x, g, m, v = (np.asarray(a, np.float64) for a in (x, g, m, v))
    gf = np.abs(g * factor)
    m_tol = u * (3 * beta1 * np.abs(m) + 4 * (1 - beta1) * gf + np.abs(want[1])) + 2.0 ** -148
    v_rel = 7 * u
    rate, spread = lr / (1 - beta1 ** step), 1 / np.sqrt(1 - beta2 ** step)
    below = np.sqrt(want[2]) * spread + eps
    move = np.abs(want[1]) * rate / below
    tol = rate / below * m_tol + move * (v_rel / 2 + 14 * u) + 4 * u * np.abs(lr * decay * x) + 2 * u * np.abs(want[0]) + u * np.abs(x)
    return want, (tol * (1 + U[dtype]) + U[dtype] * np.abs(want[0]) + TINY[dtype], m_tol, v_rel * want[2] + 2.0 ** -146)


def _off(got, want, tol, what):
    off = np.abs(_np(got) - want)
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.max(off - tol)))


def _states(rng, count):
    m = rng.normal(size=count) * 1e-3
    return m.astype(np.float32), (m * m * rng.uniform(0.5, 3, count) + 1e-9).astype(np.float32)


TYPES = [("f32", "f32", None), ("f32", "bf16", "bf16"), ("bf16", "bf16", None), ("f16", "f16", None), ("f32", "f16", "f16"),
         ("bf16", "f32", "f32")]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("count", [1, 2, 19, 47, 48, 49, 100])
def test_adamw_matches_the_oracle(bits, types, count):
    pt, gt, ct = types
    rng = np.random.default_rng(count)
    sizes = [SIZES[(i * 5 + count) % len(SIZES)] for i in range(count)]
    step, lr, betas, eps = [(1, 1e-2, (0.9, 0.999), 1e-8), (77, 3e-4, (0.8, 0.95), 1e-6), (10 ** 6, 0.1, (0.0, 0.5), 1e-3)][count % 3]
    decay = [0.1 * (i % 3) for i in range(count)]
    xs = [torch.from_numpy(rng.normal(size=n) * 0.1).to(DTYPES[pt]) for n in sizes]
    gs = [torch.from_numpy(rng.normal(size=n) * 1e-3).to(DTYPES[gt]) for n in sizes]
    states = [_states(rng, n) for n in sizes]
    if bits == 8:
        coded = [(O.encode_states(m, True), O.encode_states(v, False)) for m, v in states]
        states = [tuple(O.decode_states(c, s, i == 0) for i, (c, s) in enumerate(pair)) for pair in coded]
    factor = torch.tensor([0.625], device="cuda") if count % 2 else None
    first = None
    for gap, shift in [(0, 0), (1, 3)]:
        _say("adamw", bits, types, count, gap, shift)
        bx, x = _packed(xs, DTYPES[pt], gap, shift)
        g = _packed(gs, DTYPES[gt], gap, shift)[1]
        kinds = torch.float32 if bits == 32 else torch.uint8
        m_in, v_in = ([s[k] for s in states] if bits == 32 else [c[k][0] for c in coded] for k in (0, 1))
        (bm, m), (bv, v) = _packed(m_in, kinds, gap, shift), _packed(v_in, kinds, gap, shift)
        s = None if bits == 32 else [torch.from_numpy(np.stack([a[1], b[1]], 1)).cuda() for a, b in coded]
        copies = None if ct is None else _packed([torch.zeros(n) for n in sizes], DTYPES[ct], gap, shift)[1]
        ops.adamw(x, g, m, v, step, lr, betas=betas, eps=eps, weight_decay=decay, scales=s, copies=copies, factor=factor)
        ms, vs = (m, v) if bits == 32 else ops.adamw_state_values(m, v, s)
        for i in range(count):
            args = (xs[i].double().numpy(), gs[i].double().numpy(), *states[i], step, lr, *betas, eps, decay[i], 0.625 if count % 2 else 1.0)
            want, tol = _expected(*args, pt)
            _off(x[i], want[0], tol[0], "param")
            if ct:
                tol32 = _expected(*args, "f32")[1][0]
                _off(copies[i], want[0], tol32 * (1 + U[ct]) + U[ct] * np.abs(want[0]) + TINY[ct], "copy")
            if bits == 32:
                _off(ms[i], want[1], tol[1], "m")
                _off(vs[i], want[2], tol[2], "v")
                continue
            # Rounded to 4 significant bits, or to the block's smallest number.
            for k, least in [(1, 2.0 ** -15), (2, 2.0 ** -31)]:
                top = np.repeat([np.abs(want[k][b:b + 256]).max() for b in range(0, sizes[i], 256)], 256)[:sizes[i]] if sizes[i] else 0.0
                _off((ms, vs)[k - 1][i], want[k], tol[k] * 1.1 + np.abs(want[k]) / 16 + top * least, "8-bit state")
        after = [_np(t) for t in (*x, *m, *v)]
        if first is None:
            first = after
        for a, b in zip(after, first):
            assert np.array_equal(a, b), "bits follow from the values alone"
        # What lies between the tensors stays.
        for t in (*x, *m, *v):
            t.fill_(55)
        assert (bx == 55).all() and (bm == 55).all() and (bv == 55).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_large_tensors_and_together_or_alone(bits):
    """Past the size from which blocks take more values; each tensor by itself ends with the same bits."""
    _say("adamw large", bits)
    sizes = [(1 << 24) + 777, 300001, 5, 65536]
    make = lambda seed, scale: [torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(seed + n)).mul_(scale) for n in sizes]  # noqa: E731
    x, g = make(1, 0.1), make(2, 1e-3)
    y = [t.clone() for t in x]
    a, b = ops.adamw_states(x, bits), ops.adamw_states(y, bits)
    for step in (1, 2, 3):
        ops.adamw(x, g, *a[:2], step, 1e-2, scales=a[2])
        for i in range(len(sizes)):
            ops.adamw([y[i]], [g[i]], [b[0][i]], [b[1][i]], step, 1e-2, scales=None if bits == 32 else [b[2][i]])
    for p, q in zip([*x, *a[0], *a[1], *(a[2] or [])], [*y, *b[0], *b[1], *(b[2] or [])]):
        assert torch.equal(p, q)
    if bits == 32:
        h = [t.double() for t in make(1, 0.1)]
        m, v = ([torch.zeros_like(t) for t in h] for _ in range(2))
        for step in (1, 2, 3):
            for i in range(len(sizes)):
                m[i] = 0.9 * m[i] + 0.1 * g[i].double()
                v[i] = 0.999 * v[i] + 0.001 * g[i].double() ** 2
                h[i] -= 1e-2 * (0.01 * h[i] + m[i] / (1 - 0.9 ** step) / ((v[i] / (1 - 0.999 ** step)).sqrt() + 1e-8))
        for p, q in zip(x, h):     # three steps of at most 0.01, some 25 u each, and the sums' roundings
            assert ((p.double() - q).abs() <= 3 * (0.01 * 30 * u + 4 * u * q.abs())).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_of_more_values_than_32_bits_count(bits):
    _say("adamw past 2^32 bytes and values", bits)
    n = (1 << 32) + 1000
    x, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, n // 2, n - 1], device="cuda")
    g[at] = 1.0
    a = ops.adamw_states([x], bits)
    ops.adamw([x], [g], *a[:2], 1, 0.5, scales=a[2])
    assert (x[at] == -0.5).all() and int((x != 0).sum()) == 3
    assert int((a[0][0] != 0).sum()) == 3 and (a[0][0][at] != 0).all()


def test_layouts_that_are_not_contiguous():
    _say("adamw strides")
    base = torch.randn(4, 6, 5, 3, device="cuda")
    for bits in (32, 8):
        for make in (lambda t: t.to(memory_format=torch.channels_last), lambda t: t.permute(2, 0, 3, 1), lambda t: t[1:2]):
            x = make(base.clone())
            g = torch.empty_like(x).copy_(make(base * 0.01))
            a = ops.adamw_states([x], bits)
            assert a[0][0].stride() == x.stride()
            want, g1 = x.contiguous().clone(), g.contiguous()
            b = ops.adamw_states([want], 32)
            ops.adamw([x], [g], *a[:2], 1, 0.1, scales=a[2])
            ops.adamw([want], [g1], *b[:2], 1, 0.1)
            assert torch.equal(x.contiguous(), want)
            with pytest.raises(ValueError, match="strides"):
                ops.adamw([x], [g.contiguous()] if not g.is_contiguous() else [g.flatten()], *a[:2], 1, 0.1, scales=a[2])
    with pytest.raises(ValueError, match="gaps"):
        x = torch.zeros(6, 4, device="cuda")[:, :2]
        ops.adamw([x], [x], [x], [x], 1, 0.1)


def test_a_factor_that_is_not_finite_changes_nothing():
    _say("adamw factor")
    for bits in (32, 8):
        x = [torch.randn(3000, device="cuda"), torch.randn(7, device="cuda")]
        g = [torch.randn_like(t) for t in x]
        c = [torch.zeros_like(t) for t in x]
        a = ops.adamw_states(x, bits)
        ops.adamw(x, g, *a[:2], 1, 0.1, scales=a[2])
        before = [t.clone() for t in (*x, *a[0], *a[1], *(a[2] or []))]
        for value in (NAN, INF, -INF):
            ops.adamw(x, g, *a[:2], 2, 0.1, scales=a[2], copies=c, factor=torch.tensor([value], device="cuda"))
        g[1][3] = INF
        norm, factor = ops.grad_norm(g, 1.0)
        ops.adamw(x, g, *a[:2], 2, 0.1, scales=a[2], copies=c, factor=factor)
        for p, q in zip((*x, *a[0], *a[1], *(a[2] or [])), before):
            assert torch.equal(p, q)
        assert not any(t.any() for t in c)


def test_gradients_that_are_not_finite_without_a_factor():
    """In 32 bits a value by itself, in 8 its block of 256; and so they stay."""
    _say("adamw NaN")
    for value in (NAN, INF):
        for bits in (32, 8):
            x, g = [torch.zeros(1000, device="cuda")], [torch.ones(1000, device="cuda")]
            g[0][300] = value
            a = ops.adamw_states(x, bits)
            ops.adamw(x, g, *a[:2], 1, 0.1, scales=a[2])
            bad = x[0].isnan()
            assert int(bad.sum()) == 1 and bad[300]
            m, v = a[:2] if bits == 32 else ops.adamw_state_values(*a)
            lost = ~m[0].isfinite() | ~v[0].isfinite()
            assert lost[300] and int(lost.sum()) == (1 if bits == 32 else 256)
            if bits == 8:
                assert lost[256:512].all()
                g[0][300] = 1.0
                ops.adamw(x, g, *a[:2], 2, 0.1, scales=a[2])
                assert x[0][256:512].isnan().all() and x[0][:256].isfinite().all() and x[0][512:].isfinite().all()


def test_a_training_step_in_a_graph():
    """Scores, their gradient, the norm and the step together: captured, with the step's number and rate on the
    GPU, replayed between the same eager calls on copies."""
    _say("training graph")
    for bits in (32, 8):
        torch.manual_seed(2)
        rows, width, cols = 200, 48, 777
        feats = torch.randn(rows, width, device="cuda")
        y = torch.randint(0, cols, (rows,), device="cuda", dtype=torch.int32)

        def model():
            return [torch.randn(width, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).mul_(0.1), torch.zeros(cols, device="cuda")]

        def step(x, a, copies, number, rate):
            z = feats @ x[0] + x[1]
            lp, h, _, _, stats = ops.token_scores(z, y)
            dz = ops.token_scores_backward(z, y, stats, h, torch.full_like(lp, -1 / rows), torch.full_like(h, -0.01 / rows))
            g = [feats.t() @ dz, torch.ones(1, rows, device="cuda").matmul(dz)[0]]
            norm, factor = ops.grad_norm(g, max_norm=0.05)
            ops.adamw(x, g, *a[:2], number, rate, weight_decay=[0.1, 0.0], scales=a[2], copies=copies, factor=factor)
            return lp, h, norm, factor
        x, eager = model(), model()
        a, b = ops.adamw_states(x, bits), ops.adamw_states(eager, bits)
        copies = [torch.empty_like(t, dtype=torch.bfloat16) for t in x]
        more = [torch.empty_like(t, dtype=torch.bfloat16) for t in x]
        number, rate = torch.tensor([1], device="cuda"), torch.tensor([0.01], device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(model(), ops.adamw_states(x, bits), copies, number, rate)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(x, a, copies, number, rate)
        first = None
        for t in range(1, 6):
            number.fill_(t)
            rate.fill_(0.01 / t)
            graph.replay()
            torch.cuda.synchronize()
            want = step(eager, b, more, torch.tensor([t], device="cuda"), torch.tensor([0.01 / t], device="cuda"))
            for p, q in zip((*out, *x, *copies, *a[0], *a[1], *(a[2] or [])), (*want, *eager, *more, *b[0], *b[1], *(b[2] or []))):
                assert torch.equal(p, q), t
            assert float(out[2]) > 0.05 and abs(float(out[3]) * float(out[2]) - 0.05) < 1e-6
            first = first or float(out[0].mean())
        assert all(torch.equal(c, t.bfloat16()) for c, t in zip(copies, x))


def test_numbers_on_the_device_mean_the_same():
    _say("adamw device numbers")
    for step in (1, 2, 1000, 10 ** 7):
        x = [torch.randn(5000, device="cuda")]
        g = [torch.randn(5000, device="cuda")]
        y = [x[0].clone()]
        a, b = ops.adamw_states(x), ops.adamw_states(y)
        lr = float(np.float32(0.003))
        ops.adamw(x, g, *a[:2], step, lr, weight_decay=0.25)
        ops.adamw(y, g, *b[:2], torch.tensor(step, device="cuda"), torch.tensor(lr, device="cuda"), weight_decay=0.25)
        # The constants of the two may be one rounding apart.
        assert torch.equal(a[0][0], b[0][0]) and torch.equal(a[1][0], b[1][0])
        assert ((x[0] - y[0]).abs() <= 4 * u * (x[0].abs() + 2 * lr / (1 - 0.9 ** step))).all()


def test_parameters_of_a_graph():
    """Leaves that ask for a gradient are changed in place, and autograd notices what it had saved of them."""
    _say("adamw autograd")
    w = torch.randn(8, 8, device="cuda", requires_grad=True)
    z = torch.randn(4, 8, device="cuda")
    (z @ w).square().sum().backward()
    a = ops.adamw_states([w])
    assert not a[0][0].requires_grad
    before = w.detach().clone()
    ops.adamw([w], [w.grad], *a[:2], 1, 0.1)
    assert w.requires_grad and w.is_leaf and not torch.equal(before, w.detach())
    loss = (w * w).sum()
    ops.adamw([w], [w.grad], *a[:2], 2, 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()
    with pytest.raises(ValueError, match="computed"):
        ops.adamw([w * 1], [w.grad], *a[:2], 3, 0.1)


def test_the_binding_refuses_what_does_not_fit():
    _say("update refusals")
    x, g, m, v = (torch.zeros(300, device="cuda") for _ in range(4))
    s, codes = torch.zeros(2, 2, device="cuda"), [torch.zeros(300, dtype=torch.uint8, device="cuda") for _ in range(2)]
    bad = [
        lambda: ops.adamw(x, [g], [m], [v], 1, 0.1), lambda: ops.adamw([x], [g, g], [m], [v], 1, 0.1), lambda: ops.adamw([x], [g[:5]], [m], [v], 1, 0.1),
        lambda: ops.adamw([x], [g.cpu()], [m], [v], 1, 0.1), lambda: ops.adamw([x], [g], [m.half()], [v], 1, 0.1), lambda: ops.adamw([x], [g.double()], [m], [v], 1, 0.1),
        lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, scales=[s]), lambda: ops.adamw([x], [g], *[[c] for c in codes], 1, 0.1),
        lambda: ops.adamw([x], [g], *[[c] for c in codes], 1, 0.1, scales=[s[:1]]), lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, copies=[g.double()]),
        lambda: ops.adamw([x], [g], [m], [v], torch.tensor(1), 0.1), lambda: ops.adamw([x], [g], [m], [v], torch.tensor([1, 2], device="cuda"), 0.1),
        lambda: ops.adamw([x], [g], [m], [v], torch.tensor(1.0, device="cuda"), 0.1), lambda: ops.adamw([x], [g], [m], [v], 1, torch.tensor(0.1, dtype=torch.float64, device="cuda")),
        lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, factor=torch.ones(2, device="cuda")), lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, weight_decay=[0.1, 0.2]),
        lambda: ops.adamw([x], [None], [m], [v], 1, 0.1), lambda: ops.adamw([x], [g], [m.requires_grad_()], [v], 1, 0.1),
        lambda: ops.adamw_state_values([codes[0]], [codes[1]], [s], torch.float16), lambda: ops.adamw_state_values([x], [x], [s]),
        lambda: ops.grad_norm(g), lambda: ops.grad_norm([]), lambda: ops.grad_norm([g.cpu()]), lambda: ops.grad_norm([g.double()]),
        lambda: ops.grad_norm([torch.zeros(4, 4, device="cuda")[:, :2]]), lambda: ops.adamw_states([x], 16),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)
    m.requires_grad_(False)
    refused = [
        lambda: ops.adamw([x], [g], [m], [v], 0, 0.1), lambda: ops.adamw([x], [g], [m], [v], 1, -0.1), lambda: ops.adamw([x], [g], [m], [v], 1, INF),
        lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, betas=(1.0, 0.9)), lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, betas=(0.9, NAN)),
        lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, eps=0.0), lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, weight_decay=-1.0),
        lambda: ops.adamw([x, x], [g, g], [m, v], [torch.zeros_like(v), torch.zeros_like(v)], 1, 0.1), lambda: ops.adamw([x], [x], [m], [v], 1, 0.1),
        lambda: ops.adamw([x], [g], [m], [m], 1, 0.1), lambda: ops.adamw([x[:200]], [g[:200]], [m[:200]], [m[100:]], 1, 0.1),
        lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, factor=x[:1]), lambda: ops.adamw([x], [g], [m], [v], 1, 0.1, copies=[g]),
        lambda: ops.grad_norm([g], 0.0), lambda: ops.grad_norm([g], NAN), lambda: ops.grad_norm([g], 1.0, INF),
        lambda: ops.adamw_state_values([codes[0]], [codes[1]], [s], out=([x], [x])), lambda: ops.adamw([], [], [], [], 0, 0.1),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(P.PGCError) as e:
            call()
            print("not refused:", i)
        assert e.value.status == P.PGC_EINVAL
    with pytest.raises(TypeError):
        ops.adamw([x], [g], [m], [v], 1.5, 0.1)
    ops.adamw([x, x[:0]], [g, g[:0]], [m, m[:0]], [v, v[:0]], 1, 0.1)     # nothing overlaps an empty tensor
    ops.adamw([], [], [], [], 1, 0.1)
    ops.adamw([x[:0]], [g[:0]], [m[:0]], [v[:0]], 1, 0.1)
    ops.grad_norm([g, g])                                                # the same gradient twice counts twice


def test_a_norm_is_no_part_of_a_graph():
    _say("norm of gradients that ask for gradients")
    w = torch.tensor([3.0, 4.0], device="cuda", requires_grad=True)
    (g,) = torch.autograd.grad((w * w).sum() / 2, w, create_graph=True)
    with pytest.raises(ValueError, match="gradient"):
        ops.grad_norm([g])
    with torch.no_grad():
        assert ops.grad_norm([g])[0].item() == 5.0
    assert ops.grad_norm([g.detach()])[0].item() == 5.0


def test_numbers_whose_reading_changes_the_lists():
    _say("lists that change")
    x, g, m, v = ([torch.zeros(300, device="cuda")] for _ in range(4))

    class Clears:
        def __init__(self, which):
            self.which = which

        def __float__(self):
            self.which.clear()
            return 0.1

    for which in (x, g, m, v):
        kept = list(which)
        with pytest.raises(ValueError, match="as many"):
            ops.adamw(x, g, m, v, 1, 0.1, weight_decay=[Clears(which)])
        which[:] = kept
        with pytest.raises(ValueError, match="as many"):
            ops.adamw(x, g, m, v, 1, 0.1, eps=Clears(which))
        which[:] = kept
    more = [0.1]
    more.insert(0, Clears(more))
    with pytest.raises(ValueError, match="as many"):
        ops.adamw([*x, x[0][:0]], [*g, g[0][:0]], [*m, m[0][:0]], [*v, v[0][:0]], 1, 0.1, weight_decay=more)
