"""The scores of tokens, the norm of many gradients and the AdamW step on the host (no GPU): the oracle
against differences and known answers, the binding's structures against include/pgc_ops.h, and the C entry
points' refusals, which come before any device work (addresses below are never touched)."""

import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2607_20739_amd as P
from paper_2607_20739_amd import ops
from oracle import ops as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = 1 << 20
INF, NAN = float("inf"), float("nan")


# ---- oracle -------------------------------------------------------------------------------

def test_oracle_entropy_and_top_tokens_of_known_rows():
    z = np.log(np.array([[0.5, 0.25, 0.25], [1.0, 1.0, 1.0], [1e-300, 1.0, 1e-300]]))
    assert np.allclose(O.entropy(z), [1.5 * np.log(2), np.log(3), 0.0], atol=1e-15)
    lp, tokens = O.top_tokens(np.array([[1.0, 3.0, 3.0, -INF], [-INF] * 4, [0.0, NAN, 0.0, 0.0]]), 5)
    assert tokens.tolist() == [[1, 2, 0, -1, -1], [-1] * 5, [-1] * 5]
    assert np.isneginf(lp[0, 3:]).all() and np.isneginf(lp[1]).all() and np.isnan(lp[2]).all()
    assert abs(np.exp(lp[0, :3]).sum() - 1) < 1e-15
    lp, tokens = O.top_tokens(np.zeros((2, 3)), 2, targets=[-1, 1])
    assert tokens.tolist() == [[-1, -1], [0, 1]] and not lp[0].any()


def test_oracle_scores_gradient_is_that_of_differences():
    """Central differences of step 1e-5: truncation of order 1e-10, rounding of order 1e-16 / 1e-5."""
    rng = np.random.default_rng(1)
    z, y, g, e = rng.normal(size=(4, 6)), np.array([0, 5, -1, 2]), rng.normal(size=4), rng.normal(size=4)
    z[3, 4] = -INF
    got = O.token_scores_backward(z, y, g, e)
    for i in np.ndindex(z.shape):
        if np.isinf(z[i]):
            assert got[i] == 0
            continue
        values = []
        for s in (1e-5, -1e-5):
            x = z.copy()
            x[i] += s
            values.append((O.token_logprobs(x, y) * g).sum() + (O.entropy(x, y) * e).sum())
        assert abs((values[0] - values[1]) / 2e-5 - got[i]) < 1e-8


def test_oracle_step_of_known_numbers():
    """At the first step m'/(1 - beta1) = g and v'/(1 - beta2) = g^2: the step is lr sign(g) but for eps."""
    g = np.array([2.0, -1e-3, 0.0])
    x, m, v = O.adamw(np.ones(3), g, np.zeros(3), np.zeros(3), 1, 0.25, eps=1e-12, weight_decay=0.5)
    assert np.allclose(x, 1 - 0.25 * (0.5 + np.sign(g)), atol=1e-8)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.001 * g * g)
    norm, factor = O.grad_norm([np.array([3.0]), np.array([[4.0]])], max_norm=2.0, scale=0.5)
    assert norm == 2.5 and abs(factor - 0.4) < 1e-16
    assert O.grad_norm([np.zeros(3)], 1.0, 0.5) == (0.0, 0.5) and np.isnan(O.grad_norm([np.array([INF])], 1.0)[1])


@pytest.mark.parametrize("signed,levels", [(True, 127), (False, 255)])
def test_8_bit_states_keep_every_number_that_they_have(signed, levels):
    """Decoding and encoding again gives the same bytes; other values go to the nearest number."""
    codes = np.zeros(256, dtype=np.uint8)
    codes[:levels] = np.arange(1, levels + 1)
    scale = np.array([1.75], np.float32)
    x = O.decode_states(codes, scale, signed)
    assert x[levels - 1] == 1.75 and np.all(np.diff(x[:levels]) > 0) and not x[levels:].any()
    again, s = O.encode_states(x.astype(np.float32), signed)
    assert np.array_equal(again, codes) and np.array_equal(s, scale)
    rng = np.random.default_rng(2)
    y = (np.exp2(-rng.uniform(0, 20 if signed else 40, 256)) * 1.7).astype(np.float32)
    y[0] = 1.75
    got = O.decode_states(*O.encode_states(y, signed), signed)
    numbers = np.concatenate([[0.0], x[:levels]]) if signed else x[:levels]
    nearest = np.abs(numbers[None] - y.astype(np.float64)[:, None]).min(1)
    assert np.all(np.abs(got - y) <= nearest * (1 + 1e-12))
    if signed:
        assert np.array_equal(O.decode_states(*O.encode_states(-y, True), True), -got)
    bad = np.ones(300, np.float32)
    bad[299] = NAN
    codes, s = O.encode_states(bad, signed)
    assert np.isfinite(s[0]) and np.isnan(s[1]) and np.isnan(O.decode_states(codes, s, signed)[256:]).all()


# ---- binding ------------------------------------------------------------------------------

STRUCTURES = [ops.pgc_scores_args, ops.pgc_scores_grad_args, ops.pgc_values, ops.pgc_adamw_tensor, ops.pgc_adamw_args,
              ops.pgc_adamw_state]


def test_structures_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc is not available")
    lines = []
    for s in STRUCTURES:
        name = s.__name__
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "pgc_ops.h"\nint main(void) {\n%s\nreturn 0; }\n' % "\n".join(lines))
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split("\n")
    want = []
    for s in STRUCTURES:
        want.append("%s %d" % (s.__name__, ctypes.sizeof(s)))
        want += ["%s.%s %d" % (s.__name__, f, getattr(s, f).offset) for f, _ in s._fields_]
    assert got[:-1] == want


def _refused(status, text):
    assert status == P.PGC_EINVAL
    message = ops.lib().pgc_ops_last_error().decode()
    assert re.search(text, message), message


def _logits(**change):
    a = dict(data=BASE, rows=6, cols=10, stride=10, dtype=ops.PGC_F16)
    a.update(change)
    return ops.pgc_logits(*[a[f] for f, _ in ops.pgc_logits._fields_])


def _make(kind, base, change):
    base.update(change)
    return kind(*[base[f] for f, _ in kind._fields_])


def _scores(**change):
    A = BASE
    return _make(ops.pgc_scores_args, dict(targets=2 * A, top=3, logprobs=3 * A, entropy=4 * A, stats=5 * A, top_logprobs=6 * A,
                                           top_tokens=7 * A), change)


def _scores_grad(**change):
    A = BASE
    return _make(ops.pgc_scores_grad_args, dict(targets=2 * A, stats=3 * A, entropy=4 * A, grad_logprobs=5 * A, grad_entropy=6 * A,
                                                dlogits=8 * A, dlogits_stride=10), change)


@pytest.mark.parametrize("change,text", [
    (dict(top=-1), "top must"), (dict(top=65), "top must"), (dict(targets=2 * BASE + 1), "targets must"), (dict(targets=None), "need targets"),
    (dict(logprobs=None), "logprobs is NULL"), (dict(entropy=4 * BASE + 2), "entropy must"), (dict(stats=5 * BASE + 4), "stats must be 8"),
    (dict(top_logprobs=None), "top_logprobs is NULL"), (dict(top_tokens=None), "top_tokens is NULL"), (dict(entropy=3 * BASE), "overlaps logprobs"),
    (dict(top_tokens=6 * BASE + 8), "top_tokens overlaps top_logprobs"), (dict(stats=BASE), "stats overlaps logits"),
    (dict(top_logprobs=2 * BASE), "overlaps targets"),
])
def test_token_scores_refuse(change, text):
    _refused(ops.lib().pgc_token_scores(ctypes.byref(_logits()), ctypes.byref(_scores(**change)), None, 0, None), text)


@pytest.mark.parametrize("change,text", [
    (dict(targets=None), "grad_logprobs needs targets"), (dict(stats=None), "stats is NULL"), (dict(entropy=None), "entropy is NULL"),
    (dict(grad_logprobs=None, grad_entropy=None), "neither"), (dict(grad_entropy=6 * BASE + 2), "grad_entropy must"), (dict(dlogits=None), "dlogits is NULL"),
    (dict(dlogits_stride=9), "dlogits stride"), (dict(dlogits=BASE + 2), "overlaps logits"), (dict(dlogits=6 * BASE), "overlaps grad_entropy"),
])
def test_token_scores_backward_refuse(change, text):
    _refused(ops.lib().pgc_token_scores_backward(ctypes.byref(_logits()), ctypes.byref(_scores_grad(**change)), None), text)


@pytest.mark.parametrize("change,text", [
    (dict(dtype=9), "dtype"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "one column"), (dict(stride=9), "stride"),
    (dict(data=None), "logits is NULL"), (dict(data=BASE + 1), "2-byte aligned")])
def test_scores_refuse_such_logits(change, text):
    z = _logits(**change)
    _refused(ops.lib().pgc_token_scores(ctypes.byref(z), ctypes.byref(_scores()), None, 0, None), text)
    _refused(ops.lib().pgc_token_scores_backward(ctypes.byref(z), ctypes.byref(_scores_grad()), None), text)


def test_scores_workspace():
    size = ctypes.c_size_t(1)
    for rows, cols, top in [(0, 10, 0), (1, 10, 5), (1, 131072, 64), (100000, 131072, 20), (6, (1 << 31) - 1, 64)]:
        for dtype in (ops.PGC_F32, ops.PGC_BF16):
            z = _logits(rows=rows, cols=cols, dtype=dtype, stride=cols)
            assert ops.lib().pgc_token_scores_workspace_bytes(ctypes.byref(z), top, ctypes.byref(size)) == P.PGC_OK
            need = size.value
            assert need % 256 == 0 and need < 1 << 30
            if need:
                args = ctypes.byref(z), ctypes.byref(_scores(top=top, targets=(1 << 46) + 0, logprobs=2 << 46, entropy=3 << 46, stats=4 << 46, top_logprobs=5 << 46, top_tokens=6 << 46))
                _refused(ops.lib().pgc_token_scores(*args, None, need, None), "workspace is NULL")
                _refused(ops.lib().pgc_token_scores(*args, 7 << 46, need - 1, None), "too small")
                _refused(ops.lib().pgc_token_scores(*args, (7 << 46) + 128, need, None), "256-byte")
                _refused(ops.lib().pgc_token_scores(*args, 3 << 46, need, None), "workspace overlaps entropy")
    _refused(ops.lib().pgc_token_scores_workspace_bytes(None, 1, ctypes.byref(size)), "null")
    _refused(ops.lib().pgc_token_scores_workspace_bytes(ctypes.byref(_logits()), 1, None), "null")
    _refused(ops.lib().pgc_token_scores_workspace_bytes(ctypes.byref(_logits()), 65, ctypes.byref(size)), "top")
    _refused(ops.lib().pgc_token_scores_workspace_bytes(ctypes.byref(_logits(rows=-1)), 1, ctypes.byref(size)), "rows")


def _tensor(at=1, **change):
    A = at << 24
    return _make(ops.pgc_adamw_tensor, dict(param=A, grad=A + 0x10000, copy=None, m=A + 0x20000, v=A + 0x30000, scales=None, count=1000, weight_decay=0.1,
                                            param_dtype=ops.PGC_F32, grad_dtype=ops.PGC_F32, copy_dtype=0), change)


def _step(**change):
    return _make(ops.pgc_adamw_args, dict(lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, step=1, lr_at=None, step_at=None, factor=None, state_bits=32), change)


def _adamw(tensors, **change):
    return ops.lib().pgc_adamw((ops.pgc_adamw_tensor * len(tensors))(*tensors), len(tensors), ctypes.byref(_step(**change)), None)


@pytest.mark.parametrize("change,text", [
    (dict(lr=-1.0), "lr"), (dict(lr=INF), "lr"), (dict(lr=1e39), "lr"), (dict(beta1=1.0), "beta"), (dict(beta1=-0.1), "beta"), (dict(beta2=NAN), "beta"),
    (dict(beta2=1 - 1e-12), "beta"), (dict(eps=0.0), "eps"), (dict(eps=1e-60), "eps"), (dict(eps=INF), "eps"), (dict(step=0), "step"),
    (dict(lr_at=BASE + 2), "lr_at must"), (dict(step_at=BASE + 4), "step_at must"), (dict(factor=BASE + 1), "factor must"), (dict(state_bits=16), "state_bits"),
    (dict(factor=1 << 24), "param overlaps factor|factor overlaps param"), (dict(state_bits=8), "scales is NULL"),
])
def test_adamw_refuses_arguments(change, text):
    _refused(_adamw([_tensor()], **change), text)


@pytest.mark.parametrize("change,text", [
    (dict(param=None), "param is NULL"), (dict(grad=None), "grad is NULL"), (dict(m=None), "m is NULL"), (dict(v=None), "v is NULL"),
    (dict(param=(2 << 24) + 2), "param must"), (dict(grad_dtype=ops.PGC_F16, grad=(2 << 24) + 0x10001), "grad must"), (dict(count=-1), "counts"),
    (dict(count=(1 << 38) + 1), "counts"), (dict(weight_decay=-0.1), "weight_decay"), (dict(weight_decay=INF), "weight_decay"), (dict(param_dtype=3), "param dtype"),
    (dict(grad_dtype=-1), "grad dtype"), (dict(copy=(2 << 24) + 0x40000, copy_dtype=9), "copy dtype"), (dict(copy=(2 << 24) + 0x40002), "copy must"),
    (dict(copy=2 << 24), "overlaps"), (dict(m=2 << 24), "overlaps"), (dict(v=(2 << 24) + 0x20000 + 3996), "overlaps"), (dict(grad=(2 << 24) + 0x30000), "overlaps"),
    (dict(param=1 << 24), "overlaps"), (dict(m=(1 << 24) + 0x10000), "overlaps"), (dict(grad=(3 << 24) + 3996), "overlaps"), (dict(copy=(1 << 24) - 3996), "overlaps"),
])
def test_adamw_refuses_tensors(change, text):
    """The second of three, against itself and the others, in any order of addresses."""
    for order in ((1, 2, 3), (3, 2, 1)):
        _refused(_adamw([_tensor(at, **(change if at == 2 else {})) for at in order]), text)


def test_adamw_overlaps_of_8_bit_states():
    small = dict(scales=(1 << 24) + 0x50000, state_bits=8)
    step = dict(state_bits=8)
    base = dict(scales=small["scales"])
    _refused(_adamw([_tensor(**{**base, "v": (1 << 24) + 0x20000 + 999})], **step), "overlaps")
    _refused(_adamw([_tensor(**{**base, "scales": (1 << 24) + 0x20000 + 992})], **step), "overlaps")
    _refused(_adamw([_tensor(**{**base, "scales": (1 << 24) + 0x50004})], **step), "8-byte")
    # Apart by a byte: the last refusal of all comes, which shows that no other did.
    apart = _tensor(**{**base, "v": (1 << 24) + 0x20000 + 1000, "scales": (1 << 24) + 0x20000 - 32, "copy": (1 << 24) + 0x20000 - 36 - 4000})
    _refused(_adamw([apart, _tensor(at=2, scales=5 << 24, param=5 << 24)], **step), "overlaps")
    assert "copy" not in ops.lib().pgc_ops_last_error().decode()


def test_lists_refuse():
    lib, size = ops.lib(), ctypes.c_size_t()
    _refused(lib.pgc_adamw(None, 1, ctypes.byref(_step()), None), "NULL")
    _refused(lib.pgc_adamw(None, -1, ctypes.byref(_step()), None), "number of tensors")
    _refused(lib.pgc_adamw(None, (1 << 20) + 1, ctypes.byref(_step()), None), "number of tensors")
    _refused(lib.pgc_adamw(None, 0, None, None), "null")
    assert lib.pgc_adamw(None, 0, ctypes.byref(_step()), None) == P.PGC_OK
    assert _adamw([_tensor(count=0, param=None, grad=None, m=None, v=None)] * 3) == P.PGC_OK
    assert lib.pgc_adamw_state_values(None, 0, None) == P.PGC_OK
    _refused(lib.pgc_adamw_state_values(None, 2, None), "NULL")
    base = dict(m=BASE, v=2 * BASE, scales=3 * BASE, m_values=4 * BASE, v_values=5 * BASE, count=1000, dtype=ops.PGC_BF16)
    for change, text in [(dict(dtype=ops.PGC_F16), "float or bf16"), (dict(m=None), "m is NULL"), (dict(scales=3 * BASE + 4), "scales must"), (dict(count=-5), "counts"),
                         (dict(v_values=4 * BASE + 1998), "overlaps"), (dict(m_values=2 * BASE), "overlaps"), (dict(m_values=4 * BASE + 1), "2-byte")]:
        s = _make(ops.pgc_adamw_state, dict(base), change)
        _refused(lib.pgc_adamw_state_values(ctypes.byref(s), 1, None), text)
    two = (ops.pgc_values * 2)(ops.pgc_values(BASE, 1000, ops.PGC_F32), ops.pgc_values(2 * BASE, 5, ops.PGC_F16))
    assert lib.pgc_grad_norm_workspace_bytes(two, 2, ctypes.byref(size)) == P.PGC_OK and size.value == 256
    need = size.value
    _refused(lib.pgc_grad_norm_workspace_bytes(two, 2, None), "null")
    for args, text in [((0.0, 1.0, 4 * BASE, 5 * BASE, 6 * BASE, need), "max_norm"), ((NAN, 1.0, 4 * BASE, 5 * BASE, 6 * BASE, need), "max_norm"),
                       ((1.0, INF, 4 * BASE, 5 * BASE, 6 * BASE, need), "scale"), ((1.0, 1.0, 4 * BASE + 1, 5 * BASE, 6 * BASE, need), "norm must"),
                       ((1.0, 1.0, 4 * BASE, 4 * BASE, 6 * BASE, need), "overlaps"), ((1.0, 1.0, 4 * BASE, 5 * BASE, None, need), "workspace is NULL"),
                       ((1.0, 1.0, 4 * BASE, 5 * BASE, 6 * BASE, need - 1), "too small"), ((1.0, 1.0, 4 * BASE, 5 * BASE, 6 * BASE + 8, need), "256-byte"),
                       ((1.0, 1.0, BASE + 40, 5 * BASE, 6 * BASE, need), "overlaps"), ((1.0, 1.0, 4 * BASE, 5 * BASE, 2 * BASE, need), "overlaps")]:
        _refused(lib.pgc_grad_norm(two, 2, *args, None), text)
    bad = (ops.pgc_values * 1)(ops.pgc_values(None, 10, ops.PGC_F32))
    _refused(lib.pgc_grad_norm(bad, 1, 1.0, 1.0, 4 * BASE, 5 * BASE, 6 * BASE, 256, None), "gradient is NULL")
    bad = (ops.pgc_values * 1)(ops.pgc_values(BASE, 10, 7))
    _refused(lib.pgc_grad_norm(bad, 1, 1.0, 1.0, 4 * BASE, 5 * BASE, 6 * BASE, 256, None), "dtype")


def test_the_binding_refuses_tensors_off_the_gpu():
    z, y, f = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    for call in [lambda: ops.token_scores(z), lambda: ops.token_scores(z, y, 2), lambda: ops.token_scores_backward(z, y, f, f, f, f),
                 lambda: ops.grad_norm([f]), lambda: ops.adamw([f], [f], [f], [f], 1, 0.1)]:
        with pytest.raises(ValueError, match="GPU"):
            call()
    for what in (None, 3.0, z):
        with pytest.raises(ValueError, match="must be a list of tensors|must be a tensor"):
            ops.grad_norm(what)
        with pytest.raises(ValueError, match="must be a list of tensors"):
            ops.adamw(what, [f], [f], [f], 1, 0.1)
    for what in (None, 3.0):
        with pytest.raises(ValueError, match="must be a tensor"):
            ops.grad_norm([what])
        with pytest.raises(ValueError, match="must be a tensor"):
            ops.token_scores(what)
    with pytest.raises(ValueError, match="bits"):
        ops.adamw_states([f], 4)
    m, v, s = ops.adamw_states([torch.zeros(3, 100, dtype=torch.bfloat16, requires_grad=True)], 8)
    assert m[0].dtype == torch.uint8 and m[0].shape == (3, 100) and s[0].shape == (2, 2) and not s[0].requires_grad
