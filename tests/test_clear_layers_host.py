"""Layers in the clear, on the CPU: every call that the header refuses is refused before anything reaches a device, and calls
with nothing to do succeed without one.  No kernel is launched here: the pointers are never followed."""
import math

import pytest
import torch

import paper_1806_03461_amd as T

P = 4096            # a well aligned address that nothing reads
NULL, PARAM, SIZE = -1, -2, -3

DENSE = dict(x=P, ldx=64, w=P, ldw=64, x_scale=P, w_scale=P, bias=P, out=P, ldo=32, kind=T.CLEAR_F32, m=4, n=32, k=64)
NORM = dict(x=P, ldx=64, residual=P, ldr=64, weight=P, eps=1e-5, total=P, ldt=64, q=P, ldq=64, scale=P, type=T.CLEAR_BF16, m=4, k=64)
GATE = dict(gate=P, ldg=64, up=P, ldu=64, act=2, q=P, ldq=64, scale=P, type=T.CLEAR_BF16, m=4, k=64)


def call(name, base, **change):
    a = dict(base, **change)
    assert set(a) == set(base)
    rc = getattr(T.lib(), name)(*a.values(), None)
    return rc, T.lib().tfhe_last_error().decode()


@pytest.mark.parametrize("change, code, word", [
    (dict(kind=-1), PARAM, "kind"), (dict(kind=6), PARAM, "kind"),
    (dict(m=-1), SIZE, "rows"), (dict(k=-1), SIZE, "rows"), (dict(n=-1), SIZE, "channels"),
    (dict(m=2**31), SIZE, "rows"), (dict(n=2**31), SIZE, "channels"), (dict(n=2**63 - 1), SIZE, "channels"),
    (dict(m=2**31 - 1, n=2**31 - 1, ldo=2**31), SIZE, "too many"),
    (dict(k=131072, ldx=131072, ldw=131072), SIZE, "at most 131071"), (dict(k=2**32 + 64, ldx=2**33, ldw=2**33), SIZE, "at most"),
    (dict(ldx=63), SIZE, "stride"), (dict(ldw=63), SIZE, "stride"), (dict(ldo=31), SIZE, "stride"), (dict(ldx=-64), SIZE, "stride"),
    (dict(ldx=2**41), SIZE, "stride"),
    (dict(x=None), NULL, "x"), (dict(w=None), NULL, "w"), (dict(out=None), NULL, "out"),
    (dict(out=P + 2), PARAM, "aligned"), (dict(x_scale=P + 2), PARAM, "aligned"), (dict(w_scale=P + 1), PARAM, "aligned"),
    (dict(bias=P + 3), PARAM, "aligned"), (dict(kind=T.CLEAR_BF16, out=P + 1), PARAM, "aligned"),
    (dict(kind=T.CLEAR_I32), PARAM, "scales"), (dict(kind=T.CLEAR_SIGN, x_scale=None), PARAM, "scales"),
    (dict(kind=T.CLEAR_BITS, w_scale=None), PARAM, "scales")])
def test_product_refusals(change, code, word):
    rc, said = call("bnn_dense_clear", DENSE, **change)
    assert rc == code and word in said, (rc, said)


@pytest.mark.parametrize("change, code, word", [
    (dict(type=3), PARAM, "type"), (dict(type=-1), PARAM, "type"),
    (dict(eps=0.0), PARAM, "eps"), (dict(eps=-1.0), PARAM, "eps"), (dict(eps=math.inf), PARAM, "eps"), (dict(eps=math.nan), PARAM, "eps"),
    (dict(m=-1), SIZE, "rows"), (dict(k=-1), SIZE, "rows"), (dict(m=2**31), SIZE, "rows"),
    (dict(k=32769, ldx=32769, ldr=32769, ldt=32769, ldq=32769), SIZE, "at most 32768"),
    (dict(ldx=63), SIZE, "stride"), (dict(ldr=63), SIZE, "stride"), (dict(ldt=63), SIZE, "stride"), (dict(ldq=63), SIZE, "stride"),
    (dict(x=None), NULL, "x"), (dict(q=None), NULL, "q"), (dict(scale=None), NULL, "scale"),
    (dict(x=P + 1), PARAM, "aligned"), (dict(residual=P + 1), PARAM, "aligned"), (dict(weight=P + 1), PARAM, "aligned"),
    (dict(total=P + 1), PARAM, "aligned"), (dict(scale=P + 2), PARAM, "aligned"), (dict(type=T.CLEAR_F32, x=P + 2), PARAM, "aligned")])
def test_norm_refusals(change, code, word):
    rc, said = call("bnn_rms_norm_clear", NORM, **change)
    assert rc == code and word in said, (rc, said)


@pytest.mark.parametrize("change, code, word", [
    (dict(type=3), PARAM, "type"), (dict(act=-1), PARAM, "activation"), (dict(act=4), PARAM, "activation"),
    (dict(m=-1), SIZE, "rows"), (dict(k=65537, ldg=65537, ldu=65537, ldq=65537), SIZE, "at most 65536"),
    (dict(ldg=63), SIZE, "stride"), (dict(ldu=63), SIZE, "stride"), (dict(ldq=63), SIZE, "stride"),
    (dict(gate=None), NULL, "gate"), (dict(q=None), NULL, "q"), (dict(scale=None), NULL, "scale"),
    (dict(gate=P + 1), PARAM, "aligned"), (dict(up=P + 1), PARAM, "aligned"), (dict(scale=P + 1), PARAM, "aligned")])
def test_gate_refusals(change, code, word):
    rc, said = call("bnn_gate_clear", GATE, **change)
    assert rc == code and word in said, (rc, said)


def test_nothing_to_do_needs_no_device():
    assert call("bnn_dense_clear", DENSE, m=0, x=None, out=None)[0] == 0
    assert call("bnn_dense_clear", DENSE, n=0, w=None, out=None)[0] == 0
    assert call("bnn_rms_norm_clear", NORM, m=0, x=None, q=None, scale=None)[0] == 0
    assert call("bnn_gate_clear", GATE, m=0, gate=None, q=None, scale=None)[0] == 0


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x, w = torch.zeros(2, 8, dtype=torch.int8), torch.zeros(4, 8, dtype=torch.int8)
    with pytest.raises(ValueError, match="on the GPU"):
        T.bnn_dense_clear(x, w, torch.zeros(2, 4))
    with pytest.raises(ValueError, match="on the GPU"):
        T.bnn_rms_norm_clear(torch.zeros(2, 8), None, 1e-5, x, torch.zeros(2))
    with pytest.raises(ValueError, match="on the GPU"):
        T.bnn_gate_clear(torch.zeros(2, 8), None, "relu", x, torch.zeros(2))
