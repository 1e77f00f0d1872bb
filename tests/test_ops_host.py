"""The language-model operators on the host (no GPU): the oracle against differences, known
answers and statistics; the binding against include/pgc_ops.h; the C entry points' refusals,
which come before any device work (addresses below are never touched)."""

import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2607_20739_amd as P
from paper_2607_20739_amd import build as B
from paper_2607_20739_amd import ops
from oracle import ops as O
from oracle import rng as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---- oracle -------------------------------------------------------------------------------

def test_kept_values_are_the_fields_of_the_generator():
    seed, row = 99, 7
    key = R.splitmix64(seed, row)
    fields = [(R.splitmix64(key, w) >> (16 * k)) & 0xFFFF for w in range(3) for k in range(4)]
    for p in (0.0, 0.25, 0.5, 1.0):
        keep = O.keep_mask(p, seed, [row], 11)[0]
        assert keep.tolist() == [f >= int(65536 * p) for f in fields[:11]]
    assert O.keep_mask(0.0, 1, [0], 64).all() and not O.keep_mask(1.0, 1, [0], 64).any()


def test_masks_have_the_stated_rate_and_no_correlation():
    """Of N independent values the kept ones number N q +- 5 sqrt(N q (1 - q)); the same holds for
    those kept in two rows, two columns or under two seeds at once, with q squared."""
    p, rows, cols = 0.3, 64, 256
    q = O.keep_share(p)
    a = O.keep_mask(p, 5, range(rows), cols)
    b = O.keep_mask(p, 6, range(rows), cols)
    for both, rate in [(a, q), (a[1:] & a[:-1], q * q), (a[:, 1:] & a[:, :-1], q * q), (a & b, q * q)]:
        n = both.size
        assert abs(both.sum() - n * rate) < 5 * np.sqrt(n * rate * (1 - rate))


def _differences(loss, z, step=1e-5):
    out = np.zeros_like(z)
    for i in np.ndindex(z.shape):
        up, down = z.copy(), z.copy()
        up[i] += step
        down[i] -= step
        out[i] = (loss(up) - loss(down)) / (2 * step)
    return out


def test_oracle_gradients_are_those_of_differences():
    """Central differences of step 1e-5: truncation of order 1e-10 and rounding of order
    1e-16 / 1e-5; the policy's ratios stay clear of its bounds."""
    rng = np.random.default_rng(2)
    rows, cols = 9, 5
    z = rng.normal(size=(rows, cols)) * 2
    z[:, 3] = np.where(np.arange(rows) % 2, z[:, 3], -np.inf)
    y = rng.integers(0, 3, rows)
    y[4] = -1
    grad = rng.normal(size=rows)
    fin = np.where(np.isfinite(z), z, 0.0)

    def at(v):
        return np.where(np.isfinite(z), v, z)

    d = _differences(lambda v: (grad * O.token_logprobs(at(v), y)).sum(), fin)
    np.testing.assert_allclose(O.token_logprobs_backward(z, y, grad), d, atol=1e-8)

    offsets, ref = [0, 2, 2, 5, 8], rng.normal(size=rows)
    w = np.array([0.7, 1.3])
    kw = dict(ref=ref, beta=0.4, smoothing=0.1, scale=0.5, weights=w)
    g = O.preference(z, y, offsets, **kw)[3]
    d = _differences(lambda v: 0.5 * (w * O.preference(at(v), y, offsets, **kw)[0]).sum(), fin)
    np.testing.assert_allclose(O.token_logprobs_backward(z, y, g), d, atol=1e-8)

    lp = O.token_logprobs(z, y)
    shift = np.array([-.5, -.1, .1, .5, 0, -.5, -.1, .1, .5])
    adv = np.array([1, 1, 1, 1, 1, -1, -1, -1, -1.0])
    kw = dict(ref=lp + rng.normal(size=rows) * .3, kl=0.2, scale=0.25, weights=rng.uniform(size=rows))
    g = O.policy(z, y, lp - shift, adv, **kw)[2]
    d = _differences(lambda v: 0.25 * (kw["weights"] * O.policy(at(v), y, lp - shift, adv, **kw)[0]).sum(), fin)
    np.testing.assert_allclose(O.token_logprobs_backward(z, y, g), d, atol=1e-8)


def test_oracle_edge_rows():
    z = np.array([[0.0, 1.0, -np.inf], [-np.inf] * 3, [np.nan, 0, 0], [np.inf, 0, 0], [-3e38] * 3])
    y = [2, 0, 1, 1, 1]
    lp = O.token_logprobs(z, y)
    assert np.isneginf(lp[:2]).all() and np.isnan(lp[2:4]).all()
    assert lp[4] == pytest.approx(-np.log(3))
    dz = O.token_logprobs_backward(z, y, np.ones(5))
    assert dz[0].tolist()[2] == 1.0 and dz[0, :2].sum() == pytest.approx(-1.0)
    assert not dz[1].any() and np.isnan(dz[2:4]).all()
    assert dz[4].tolist() == pytest.approx([-1 / 3, 2 / 3, -1 / 3])
    assert not O.token_logprobs_backward(z, y, np.zeros(5)).any()


# ---- binding ------------------------------------------------------------------------------

def _header():
    with open(os.path.join(ROOT, "include", "pgc_ops.h")) as f:
        return f.read()


def test_library_exports_every_declared_operator():
    declared = sorted(set(re.findall(r"^(?:int|const char\*)\s+(pgc_\w+)\s*\(", _header(), re.M)))
    assert declared == sorted(ops.exported_symbols())
    for name in declared:
        assert hasattr(P.lib(), name), name


def test_binding_structures_match_the_header(tmp_path):
    """Size and every field's offset, from a C program (which also shows that the header is C99)."""
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc is not available")
    types = [ops.pgc_dropout_args, ops.pgc_logits, ops.pgc_preference_args, ops.pgc_policy_args]
    body, want = [], []
    for t in types:
        name = t.__name__
        body.append('printf("%%zu ", sizeof(%s));' % name)
        want.append(ctypes.sizeof(t))
        for field, _ in t._fields_:
            body.append('printf("%%zu ", offsetof(%s, %s));' % (name, field))
            want.append(getattr(t, field).offset)
    body.append('printf("%d %d %d ", PGC_F32, PGC_BF16, PGC_F16);')
    want += [ops.PGC_F32, ops.PGC_BF16, ops.PGC_F16]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "pgc_ops.h"\nint main(void) {\n%s\nreturn 0; }\n'
                   % "\n".join(body))
    exe = str(tmp_path / "layout")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", exe], check=True, capture_output=True, text=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    assert [int(v) for v in out.split()] == want


# ---- refusals -----------------------------------------------------------------------------

def _refused(status, text):
    assert status == P.PGC_EINVAL, status
    message = ops.lib().pgc_ops_last_error().decode()
    assert text in message, message


BASE = 1 << 40     # addresses that nothing reads: every call below is refused on the host


def _dropout_args(**change):
    a = dict(x=BASE, residual=None, out=BASE * 2, row_ids=None, rows=4, cols=10, x_stride=10, residual_stride=0,
             out_stride=10, first_row=0, seed=1, p=0.1, dtype=ops.PGC_BF16)
    a.update(change)
    return ops.pgc_dropout_args(*[a[f] for f, _ in ops.pgc_dropout_args._fields_])


@pytest.mark.parametrize("change,text", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(cols=1 << 31), "rows"),
    (dict(p=-0.01), "p must"), (dict(p=1.01), "p must"), (dict(p=float("nan")), "p must"),
    (dict(x_stride=9), "x stride"), (dict(out_stride=9), "out stride"), (dict(x_stride=1 << 41), "x stride"),
    (dict(residual=BASE * 3, residual_stride=9), "residual stride"), (dict(x=None), "x is NULL"),
    (dict(out=None), "out is NULL"), (dict(x=BASE + 1), "2-byte aligned"), (dict(out=BASE * 2 + 1), "2-byte aligned"),
    (dict(dtype=ops.PGC_F32, x=BASE + 2), "4-byte aligned"), (dict(row_ids=BASE * 4 + 4), "8-byte aligned"),
    (dict(out=BASE + 20), "overlaps x"), (dict(out=BASE, out_stride=11), "overlaps x"),
    (dict(residual=BASE * 2 + 2, residual_stride=10), "overlaps residual"),
    (dict(row_ids=BASE * 2 + 8), "overlaps row_ids"),
])
def test_dropout_refuses(change, text):
    _refused(ops.lib().pgc_dropout(ctypes.byref(_dropout_args(**change)), None), text)


def test_dropout_backward_takes_no_residual_and_null_arguments_are_refused():
    args = _dropout_args(residual=BASE * 3, residual_stride=10)
    _refused(ops.lib().pgc_dropout_backward(ctypes.byref(args), None), "residual")
    for name in ("pgc_dropout", "pgc_dropout_backward"):
        _refused(getattr(ops.lib(), name)(None, None), "null")
    z = _logits()
    _refused(ops.lib().pgc_token_logprobs(None, 0, 0, 0, None), "null")
    _refused(ops.lib().pgc_token_logprobs_backward(None, 0, 0, 0, 0, 0, None), "null")
    _refused(ops.lib().pgc_preference_loss(ctypes.byref(z), None, None, 0, None), "null")
    _refused(ops.lib().pgc_preference_loss(None, ctypes.byref(_preference()), None, 0, None), "null")
    _refused(ops.lib().pgc_policy_loss(None, ctypes.byref(_policy()), None), "null")
    _refused(ops.lib().pgc_policy_loss(ctypes.byref(z), None, None), "null")


def test_nothing_to_do_is_no_error():
    for change in (dict(rows=0), dict(cols=0, x_stride=0, out_stride=0), dict(rows=0, x=None, out=None)):
        assert ops.lib().pgc_dropout(ctypes.byref(_dropout_args(**change)), None) == P.PGC_OK
    z = _logits(rows=0, data=None)
    assert ops.lib().pgc_token_logprobs(ctypes.byref(z), None, None, None, None) == P.PGC_OK
    assert ops.lib().pgc_token_logprobs_backward(ctypes.byref(z), None, None, None, None, 10, None) == P.PGC_OK
    empty = _policy(targets=None, old_logprobs=None, advantages=None, loss=None, logprobs=None, dlogits=None)
    assert ops.lib().pgc_policy_loss(ctypes.byref(z), ctypes.byref(empty), None) == P.PGC_OK
    empty = _preference(pairs=0, targets=None, loss=None, margins=None, logprobs=None, dlogits=None)
    assert ops.lib().pgc_preference_loss(ctypes.byref(z), ctypes.byref(empty), None, 0, None) == P.PGC_OK


def _logits(**change):
    a = dict(data=BASE, rows=6, cols=10, stride=10, dtype=ops.PGC_F16)
    a.update(change)
    return ops.pgc_logits(*[a[f] for f, _ in ops.pgc_logits._fields_])


LOGITS_REFUSALS = [
    (dict(dtype=9), "dtype"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "one column"), (dict(stride=9), "stride"),
    (dict(data=None), "logits is NULL"), (dict(data=BASE + 1), "2-byte aligned"),
]


@pytest.mark.parametrize("change,text", LOGITS_REFUSALS)
def test_every_operator_refuses_such_logits(change, text):
    z, A = _logits(**change), BASE
    lib = ops.lib()
    _refused(lib.pgc_token_logprobs(ctypes.byref(z), 2 * A, 3 * A, 4 * A, None), text)
    _refused(lib.pgc_token_logprobs_backward(ctypes.byref(z), 2 * A, 3 * A, 4 * A, 5 * A, 10, None), text)
    _refused(lib.pgc_preference_loss(ctypes.byref(z), ctypes.byref(_preference()), 12 * A, 1 << 20, None), text)
    _refused(lib.pgc_policy_loss(ctypes.byref(z), ctypes.byref(_policy()), None), text)


@pytest.mark.parametrize("args,text", [
    ((None, 3 * BASE, None), "targets is NULL"), ((2 * BASE + 2, 3 * BASE, None), "targets must be 4-byte"),
    ((2 * BASE, None, None), "logprobs is NULL"), ((2 * BASE, 3 * BASE, 4 * BASE + 4), "stats must be 8-byte"),
    ((2 * BASE, BASE + 4, None), "logprobs overlaps logits"), ((2 * BASE, 2 * BASE, None), "logprobs overlaps targets"),
    ((2 * BASE, 3 * BASE, 3 * BASE + 16), "stats overlaps logprobs"),
])
def test_token_logprobs_refuse(args, text):
    _refused(ops.lib().pgc_token_logprobs(ctypes.byref(_logits()), *args, None), text)


@pytest.mark.parametrize("args,text", [
    ((None, 4 * BASE, 5 * BASE, 10), "stats is NULL"), ((3 * BASE, None, 5 * BASE, 10), "grad is NULL"),
    ((3 * BASE, 4 * BASE, None, 10), "dlogits is NULL"), ((3 * BASE, 4 * BASE, 5 * BASE, 9), "dlogits stride"),
    ((3 * BASE, 4 * BASE, BASE + 2, 10), "dlogits overlaps logits"), ((3 * BASE, 4 * BASE, BASE, 12), "overlaps logits"),
    ((3 * BASE, 4 * BASE, 4 * BASE, 10), "dlogits overlaps grad"), ((3 * BASE, 4 * BASE, 5 * BASE + 1, 10), "2-byte"),
])
def test_token_logprobs_backward_refuse(args, text):
    _refused(ops.lib().pgc_token_logprobs_backward(ctypes.byref(_logits()), 2 * BASE, *args, None), text)


def _preference(**change):
    A = BASE
    a = dict(targets=2 * A, offsets=3 * A, ref_logprobs=4 * A, pair_weights=None, pairs=2, beta=0.1, label_smoothing=0.0,
             scale=1.0, loss=5 * A, margins=6 * A, logprobs=7 * A, dlogits=8 * A, dlogits_stride=10)
    a.update(change)
    return ops.pgc_preference_args(*[a[f] for f, _ in ops.pgc_preference_args._fields_])


@pytest.mark.parametrize("change,text", [
    (dict(pairs=-1), "pairs"), (dict(pairs=1 << 30), "pairs"), (dict(beta=float("inf")), "beta"),
    (dict(scale=float("nan")), "scale"), (dict(scale=1e39), "scale"), (dict(label_smoothing=-0.1), "smoothing"),
    (dict(label_smoothing=1.5), "smoothing"), (dict(offsets=None), "offsets is NULL"), (dict(loss=None), "loss is NULL"),
    (dict(margins=None), "margins is NULL"), (dict(logprobs=None), "logprobs is NULL"),
    (dict(ref_logprobs=4 * BASE + 1), "ref_logprobs must"), (dict(pair_weights=9 * BASE + 2), "pair_weights must"),
    (dict(dlogits_stride=3), "dlogits stride"), (dict(dlogits=BASE, dlogits_stride=11), "overlaps logits"),
    (dict(margins=5 * BASE + 4), "margins overlaps loss"), (dict(logprobs=4 * BASE), "logprobs overlaps ref"),
    (dict(dlogits=3 * BASE), "dlogits overlaps offsets"),
])
def test_preference_loss_refuses(change, text):
    args = _preference(**change)
    _refused(ops.lib().pgc_preference_loss(ctypes.byref(_logits()), ctypes.byref(args), 12 * BASE, 1 << 20, None), text)


def _workspace(z, pairs):
    out = ctypes.c_size_t(1)
    return ops.lib().pgc_preference_workspace_bytes(ctypes.byref(z), pairs, ctypes.byref(out)), out.value


def test_preference_workspace_sizes_and_refusals():
    lib = ops.lib()
    big = _logits(rows=5000, cols=100, stride=100)
    status, need = _workspace(big, 2)
    assert status == P.PGC_OK and need % 256 == 0 and need >= 5000 * 12
    assert _workspace(_logits(rows=0), 0) == (P.PGC_OK, 0)
    # Few logits need none; as many in one pair, in none, or of long rows, do.
    assert _workspace(_logits(rows=1000, cols=64, stride=64), 8) == (P.PGC_OK, 0)
    for rows, cols, pairs in [(1200, 64, 1), (1000, 64, 0), (40, 8192, 8), (4097, 10, 100), (1000, 64, 5000)]:
        assert _workspace(_logits(rows=rows, cols=cols, stride=cols), pairs)[1] >= rows * 12, (rows, cols, pairs)
    assert ops.preference_workspace_bytes(torch.empty(5000, 100, dtype=torch.float16), 2) == need
    _refused(_workspace(big, -1)[0], "pairs")
    _refused(_workspace(_logits(rows=-1), 1)[0], "rows")
    _refused(_workspace(_logits(dtype=7), 1)[0], "dtype")
    _refused(lib.pgc_preference_workspace_bytes(ctypes.byref(big), 1, None), "null")
    _refused(lib.pgc_preference_workspace_bytes(None, 1, ctypes.byref(ctypes.c_size_t())), "null")
    a = _preference(dlogits_stride=100)
    args = [ctypes.byref(big), ctypes.byref(a)]
    _refused(lib.pgc_preference_loss(*args, 12 * BASE, need - 1, None), "too small")
    _refused(lib.pgc_preference_loss(*args, None, need, None), "workspace is NULL")
    _refused(lib.pgc_preference_loss(*args, 12 * BASE + 128, need, None), "256-byte")
    _refused(lib.pgc_preference_loss(*args, 7 * BASE, need, None), "workspace overlaps logprobs")
    _refused(lib.pgc_preference_loss(*args, BASE, need, None), "workspace overlaps logits")


def _policy(**change):
    A = BASE
    a = dict(targets=2 * A, old_logprobs=3 * A, advantages=4 * A, ref_logprobs=None, token_weights=None, clip_low=0.2,
             clip_high=0.2, kl=0.0, scale=1.0, loss=5 * A, logprobs=6 * A, dlogits=8 * A, dlogits_stride=10)
    a.update(change)
    return ops.pgc_policy_args(*[a[f] for f, _ in ops.pgc_policy_args._fields_])


@pytest.mark.parametrize("change,text", [
    (dict(clip_low=-0.1), "clip_low"), (dict(clip_low=1.1), "clip_low"), (dict(clip_high=-1.0), "clip_high"),
    (dict(clip_high=float("inf")), "clip_high"), (dict(kl=float("nan")), "kl"), (dict(kl=1e300), "kl"),
    (dict(scale=float("inf")), "scale"), (dict(kl=0.1), "ref_logprobs is NULL"), (dict(old_logprobs=None), "old_logprobs"),
    (dict(advantages=None), "advantages"), (dict(loss=None), "loss is NULL"), (dict(logprobs=None), "logprobs is NULL"),
    (dict(token_weights=3), "token_weights must"), (dict(dlogits_stride=9), "dlogits stride"),
    (dict(loss=3 * BASE), "loss overlaps old_logprobs"), (dict(logprobs=BASE), "logprobs overlaps logits"),
    (dict(dlogits=4 * BASE), "dlogits overlaps advantages"), (dict(dlogits=BASE + 4), "dlogits overlaps logits"),
])
def test_policy_loss_refuses(change, text):
    _refused(ops.lib().pgc_policy_loss(ctypes.byref(_logits()), ctypes.byref(_policy(**change)), None), text)


def test_tensors_off_the_gpu_are_refused():
    x, y = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: ops.dropout(x, 0.1, 1), lambda: ops.dropout_backward(x, 0.1, 1),
                 lambda: ops.token_logprobs(x, y), lambda: ops.policy_loss(x, y, x[:, 0], x[:, 0]),
                 lambda: ops.preference_loss(x, y, y)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_the_binding_refuses_tensors_off_the_gpu():
    """The compiled binding is built, takes nothing but tensors on the GPU, and says why."""
    z, y, f = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    for call, what in [(lambda: ops.dropout(z, 0.1, 1), "x must be"), (lambda: ops.dropout_backward(z, 0.1, 1), "x must be"),
                       (lambda: ops.token_logprobs(z, y), "logits must be"),
                       (lambda: ops.token_logprobs_backward(z, y, f, f), "logits must be"),
                       (lambda: ops.preference_loss(z, y, y), "logits must be"),
                       (lambda: ops.policy_loss(z, y, f, f), "logits must be")]:
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(ValueError, match="logits must be a tensor"):
        ops.policy_loss(None, y, f, f)


def test_the_binding_compiles_without_warnings():
    if shutil.which("g++") is None:
        pytest.skip("g++ is not available")
    res = subprocess.run(["g++"] + B.binding_flags() + ["-fsyntax-only", B.BINDING], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "warning" not in res.stderr, res.stderr[-2000:]


@pytest.mark.parametrize("smoothing,losses", [(0.0, [0.0, np.inf]), (0.1, [np.inf, np.inf]), (1.0, [np.inf, 0.0])])
def test_oracle_losses_of_infinite_margins(smoothing, losses):
    """-ln sigma(inf) = 0 and -ln sigma(-inf) = inf, each with its weight; weight 0 leaves a term out."""
    z = np.array([[0.0, -np.inf], [0.0, -np.inf], [0.0, -np.inf], [0.0, -np.inf]])
    loss, margins, _, grad = O.preference(z, [0, 1, 1, 0], [0, 1, 2, 3, 4], beta=0.5, smoothing=smoothing)
    assert margins.tolist() == [np.inf, -np.inf] and loss.tolist() == losses
    want = 0.5 * smoothing, -0.5 * (1 - smoothing)
    assert grad.tolist() == [want[0], -want[0], want[1], -want[1]]


def test_oracle_policy_loss_of_a_target_that_cannot_occur():
    """kl (exp(d) - d - 1) at d = inf is inf; without the KL term the row has the ratio 0."""
    z, y, one = np.array([[0.0, -np.inf, 1.0], [-np.inf] * 3]), [1, 0], np.ones(2)
    loss, lp, grad = O.policy(z, y, -one, one, ref=-one, kl=0.1)
    assert np.isneginf(lp).all() and np.isposinf(loss).all() and np.isneginf(grad).all()
    for advantage, want in [(1.0, 0.0), (-1.0, 0.8)]:
        loss, _, grad = O.policy(z, y, -one, advantage * one)
        assert loss.tolist() == [want, want] and not grad.any()


@pytest.mark.parametrize("offset,apart", [(10, True), (12, True), (-12, True), (-10, True), (9, False), (13, False), (-13, False),
                                          (-9, False), (22 + 12, True), (22 + 13, False), (5, False), (22, False), (-22, False)])
def test_columns_beside_each_other_do_not_overlap(offset, apart):
    """x has columns 0 to 9 of rows of 22 values, the output 10 columns further on (or ahead).  A pointer that is
    refused last tells which refusal it was: that of overlap comes first."""
    out = BASE + 2 * offset
    args = _dropout_args(x_stride=22, out_stride=22, out=out, row_ids=out // 8 * 8)
    _refused(ops.lib().pgc_dropout(ctypes.byref(args), None), "out overlaps row_ids" if apart else "out overlaps x")


@pytest.mark.parametrize("what", [None, 3.0, [[1.0, 2.0]], np.zeros((3, 4), np.float32)])
def test_what_is_no_tensor_is_refused(what):
    y, f = torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    for call, name in [(lambda: ops.dropout(what, 0.1, 1), "x"), (lambda: ops.dropout_backward(what, 0.1, 1), "x"),
                       (lambda: ops.token_logprobs(what, y), "logits"), (lambda: ops.token_logprobs_backward(what, y, f, f), "logits"),
                       (lambda: ops.preference_loss(what, y, y), "logits"), (lambda: ops.policy_loss(what, y, f, f), "logits")]:
        with pytest.raises(ValueError, match=name + " must be a tensor"):
            call()


@pytest.mark.parametrize("logits", [None, torch.zeros(3, 4, dtype=torch.float64), torch.zeros(4), torch.zeros(2, 3, 4), np.zeros((3, 4))])
def test_workspace_bytes_refuse_what_is_no_matrix_of_logits(logits):
    with pytest.raises(ValueError, match="logits must be a 2-D"):
        ops.preference_workspace_bytes(logits, 1)
