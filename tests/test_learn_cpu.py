"""Host checks of the learning operators: what they refuse, before anything is launched."""
import ctypes

import pytest

from paper_2510_05421_amd import _abi

A, B, C, D = (1 << 20), (1 << 24), (1 << 28), (1 << 32)   # addresses that no call here reaches


def _logprob(**kw):
    d = dict(rows=4, vocab=100, dtype=_abi.FP32, logits=B, ld=100, tokens=A, temperature=1.0, logp=A + 4096, entropy=None)
    d.update(kw)
    return _abi.LogprobArgs(**d)


def _policy(**kw):
    d = dict(rows=4, vocab=100, dtype=_abi.FP32, logits=B, ld=100, tokens=A, advantages=A + 256, old_logp=None, weights=None,
             ref_logits=None, ref_ld=0, ref_logp=None, temperature=1.0, ref_temperature=1.0, clip_low=0.2, clip_high=0.2,
             c_kl=0.0, c_ent=0.0, grad=C, grad_ld=100, logp=None, terms=A + 8192)
    d.update(kw)
    return _abi.PolicyArgs(**d)


def _adamw(n=2, tensor=None, **kw):
    t = (_abi.AdamwTensor * max(n, 1))()
    for i in range(n):
        d = dict(n=10, param=A + 1024 * i, master=None, grad=B + 1024 * i, m=C + 1024 * i, v=D + 1024 * i, m_scale=None,
                 v_scale=None)
        if i == n - 1:
            d.update(tensor or {})
        t[i] = _abi.AdamwTensor(**d)
    d = dict(dtype=_abi.FP32, grad_dtype=_abi.FP32, state_bits=32, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
             weight_decay=0.0, max_norm=0.0, seed=0, grad_norm=None)
    d.update(kw)
    return t, _abi.AdamwArgs(**d)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(vocab=0), dict(dtype=2), dict(logits=None), dict(tokens=None), dict(logp=None), dict(ld=-1),
    dict(ld=1 << 40), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF),
    dict(logits=B + 2)])
def test_token_logprobs_refuses(kw):
    lib = _abi.load()
    assert lib.dvi_token_logprobs(_logprob(**kw), A, 1 << 20, None) == _abi.ERR_ARG
    assert lib.dvi_op_error()


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(vocab=0), dict(dtype=-1), dict(logits=None), dict(tokens=None), dict(advantages=None),
    dict(terms=None), dict(temperature=0.0), dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_low=NAN),
    dict(clip_high=-0.1), dict(clip_high=NAN), dict(c_kl=0.1), dict(c_kl=NAN), dict(c_ent=INF),
    dict(ref_logits=D, ref_ld=100, ref_logp=A), dict(ref_logits=D, ref_ld=-1), dict(ref_logits=D, ref_ld=100, ref_temperature=0.0),
    dict(ref_logits=D + 1, ref_ld=100), dict(grad_ld=99), dict(grad=C + 2),
    dict(grad=B + 4),                               # overlaps the logits without being them
    dict(grad=B, grad_ld=101),                      # the same start with another stride
    dict(grad=B + 400, ld=150, grad_ld=150),        # rows of one stride that meet
    dict(ref_logits=C, ref_ld=100),                 # the gradient over the reference
    dict(ref_logits=C + 40, ref_ld=0),              # over an expanded reference row
])
def test_policy_loss_refuses(kw):
    lib = _abi.load()
    assert lib.dvi_policy_loss(_policy(**kw), A, 1 << 20, None) == _abi.ERR_ARG
    assert lib.dvi_op_error()


@pytest.mark.parametrize("tensor,kw", [
    ({}, dict(dtype=3)), ({}, dict(grad_dtype=3)), ({}, dict(state_bits=16)), ({}, dict(step=0)), ({}, dict(lr=NAN)),
    ({}, dict(beta1=1.0)), ({}, dict(beta2=-0.1)), ({}, dict(beta2=NAN)), ({}, dict(eps=0.0)), ({}, dict(eps=1e-50)), ({}, dict(lr=1e200)),
    ({}, dict(lr=1e30, weight_decay=1e30)), ({}, dict(max_norm=-1.0)),
    ({}, dict(max_norm=NAN)), ({}, dict(weight_decay=INF)), ({}, dict(grad_norm=A)), ({}, dict(state_bits=8)),
    (dict(n=-1), {}), (dict(param=None), {}), (dict(grad=None), {}), (dict(m=None), {}), (dict(v=None), {}),
    (dict(master=D), {}), (dict(master=D), dict(dtype=_abi.BF16)), (dict(param=A + 2), {}), (dict(m=C + 2), {}),
    (dict(m_scale=D + 2, v_scale=D), dict(state_bits=8)),
])
def test_adamw_refuses(tensor, kw):
    lib = _abi.load()
    t, args = _adamw(tensor=tensor, **kw)
    assert lib.dvi_adamw(t, 2, args, A, 1 << 20, None) == _abi.ERR_ARG
    assert lib.dvi_op_error()


def test_null_arguments_are_refused():
    lib = _abi.load()
    assert lib.dvi_update_policy(None, None, None) == _abi.ERR_ARG
    assert lib.dvi_set_optimizer(None, None) == _abi.ERR_ARG
    t, args = _adamw()
    assert lib.dvi_token_logprobs(None, A, 1 << 20, None) == _abi.ERR_ARG
    assert lib.dvi_policy_loss(None, A, 1 << 20, None) == _abi.ERR_ARG
    assert lib.dvi_adamw(t, 2, None, A, 1 << 20, None) == _abi.ERR_ARG
    assert lib.dvi_adamw(None, 2, args, A, 1 << 20, None) == _abi.ERR_ARG
    assert lib.dvi_adamw(t, -1, args, A, 1 << 20, None) == _abi.ERR_ARG


def test_capacity_and_workspaces():
    lib = _abi.load()
    wide = dict(vocab=200000, ld=200000)     # split over workgroups: sums of the parts
    for name, args in (("dvi_token_logprobs", _logprob(**wide)), ("dvi_policy_loss", _policy(grad_ld=200000, grad=1 << 40, **wide))):
        need = getattr(lib, name + "_workspace_bytes")(4, 200000)
        assert 0 < need < 1 << 20
        assert getattr(lib, name)(args, A, need - 1, None) == _abi.ERR_CAPACITY
        assert getattr(lib, name)(args, A + 128, need, None) == _abi.ERR_ARG      # not aligned
        assert getattr(lib, name)(args, None, need, None) == _abi.ERR_ARG
        assert getattr(lib, name + "_workspace_bytes")(-1, 100) == 0
    assert lib.dvi_token_logprobs(_logprob(rows=1 << 40), A, 1 << 20, None) == _abi.ERR_CAPACITY
    assert lib.dvi_policy_loss(_policy(rows=1 << 40), A, 1 << 20, None) == _abi.ERR_CAPACITY
    assert lib.dvi_policy_loss(_policy(vocab=(1 << 28) + 1, ld=1 << 29, grad_ld=1 << 29), A, 1 << 20, None) == _abi.ERR_CAPACITY
    t, args = _adamw(max_norm=1.0)
    assert lib.dvi_adamw(t, 2, args, A, lib.dvi_adamw_workspace_bytes(2) - 1, None) == _abi.ERR_CAPACITY
    t, args = _adamw(tensor=dict(n=1 << 50))
    assert lib.dvi_adamw(t, 2, args, A, 1 << 20, None) == _abi.ERR_CAPACITY
    t, args = _adamw(tensor=dict(n=(1 << 63) - 1))
    assert lib.dvi_adamw(t, 2, args, A, 1 << 20, None) == _abi.ERR_CAPACITY
    assert lib.dvi_adamw_workspace_bytes(200) > lib.dvi_adamw_workspace_bytes(2)


def test_nothing_to_do_needs_no_gpu():
    lib = _abi.load()
    assert lib.dvi_token_logprobs(_logprob(rows=0, logits=None, tokens=None, logp=None), None, 0, None) == _abi.OK
    t, args = _adamw(n=2, tensor=dict(n=0))
    t[0].n = 0
    assert lib.dvi_adamw(t, 2, args, None, 0, None) == _abi.OK
    assert lib.dvi_adamw(None, 0, args, None, 0, None) == _abi.OK


def test_argument_structures_have_the_headers_layout(tmp_path):
    """Sizes and offsets as a C compiler sees them."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    pairs = [("dvi_policy_update_args", _abi.PolicyUpdateArgs), ("dvi_policy_update_stats", _abi.PolicyUpdateStats),
             ("dvi_optimizer", _abi.Optimizer), ("dvi_logprob_args", _abi.LogprobArgs), ("dvi_policy_args", _abi.PolicyArgs),
             ("dvi_adamw_tensor", _abi.AdamwTensor), ("dvi_adamw_args", _abi.AdamwArgs)]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "dvi.h"', "int main(void) {"]
    for c, py in pairs:
        lines.append('printf("%%zu", sizeof(%s));' % c)
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (c, f[0]) for f in py._fields_]
        lines.append('printf("\\n");')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines()
    for (c, py), line in zip(pairs, out):
        want = [ctypes.sizeof(py)] + [getattr(py, f[0]).offset for f in py._fields_]
        assert [int(x) for x in line.split()] == want, c
