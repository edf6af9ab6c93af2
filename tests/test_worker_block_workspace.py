"""A dense product's workspace without a GPU: a call without it, with less of it or with one that is not
aligned is refused before anything touches a device, whatever the workspace is for."""
import ctypes

import pytest

import paper_2010_05888_amd as gf
from paper_2010_05888_amd import worker

P, WS = 0x1000, 1 << 20  # aligned addresses, never dereferenced
COUNTS = (ctypes.c_int64 * 2)(13, 27)


def _linear(tokens, inputs, outputs, x=P, ldx=None, w=P, ldw=None):
    fn, ldx, ldw = worker._functions(), ldx or inputs, ldw or inputs
    need = fn["garfield_linear_workspace"](x, 1, tokens, inputs, ldx, w, outputs, ldw)
    return need, lambda ws, size: fn["garfield_linear"](
        x, 1, tokens, inputs, ldx, w, outputs, ldw, None, 0, 0, None, 0, P, outputs, None, 0, ws, size, None)


def _linear_backward(tokens, inputs, outputs, x=P, ldx=None, w=P, ldw=None):
    """x: the gradient, of `inputs` columns here, and w inputs x outputs."""
    fn, ldx, ldw = worker._functions(), ldx or inputs, ldw or outputs
    need = fn["garfield_linear_backward_workspace"](x, 1, tokens, inputs, ldx, w, outputs, ldw)
    return need, lambda ws, size: fn["garfield_linear_backward"](
        x, 1, tokens, inputs, ldx, w, outputs, ldw, 0, None, 0, None, 0, P, outputs, ws, size, None)


def _linear_weight_gradient(tokens, inputs, outputs, x=P, ldx=None, w=P, ldw=None):
    """w: the gradient, tokens x outputs."""
    fn, ldx, ldw = worker._functions(), ldx or inputs, ldw or outputs
    counts = COUNTS if tokens == 40 else (ctypes.c_int64 * 2)(0, tokens)
    need = fn["garfield_linear_weight_gradient_workspace"](w, 1, tokens, outputs, ldw, x, inputs, ldx, 2, counts)
    return need, lambda ws, size: fn["garfield_linear_weight_gradient"](
        w, 1, tokens, outputs, ldw, x, inputs, ldx, 2, counts, P, outputs * inputs, None, 0, ws, size, None)


PACKED = [dict(x=P + 2), dict(w=P + 2), dict(ldx=201), dict(ldw=201), dict(inputs=199), dict(x=P + 2, w=P + 2),
          dict(ldx=1 << 22)]  # rows too far apart
# a depth of 4096 of one tile of results is cut into shares
SHARED = {"linear": dict(tokens=40, inputs=4096, outputs=64),
          "linear_backward": dict(tokens=40, inputs=4096, outputs=64),
          "linear_weight_gradient": dict(tokens=4096, inputs=64, outputs=64)}
CALLS = {"linear": _linear, "linear_backward": _linear_backward, "linear_weight_gradient": _linear_weight_gradient}


def _refused(need, call):
    assert need > 0
    for ws, size in ((None, need), (None, 1 << 40), (WS, need - 1), (WS, 0), (WS + 8, need), (WS + 128, 1 << 40)):
        assert call(ws, size) == gf.EINVAL, (ws, size)


@pytest.mark.parametrize("how", PACKED)
@pytest.mark.parametrize("name", CALLS)
def test_packed_rows_need_their_workspace(name, how):
    case = {"tokens": 40, "inputs": 200, "outputs": 200, **how}
    need, call = CALLS[name](**case)
    rows = {"x": 40, "w": 40 if name == "linear_weight_gradient" else 200}
    cols = {"x": case["inputs"], "w": case["inputs"] if name == "linear" else case["outputs"]}
    if name == "linear_backward":
        rows["w"] = case["inputs"]
    odd = [k for k in "xw" if f"ld{k}" in how or k in how or cols[k] % 8]
    assert odd and need >= sum(rows[k] * ((cols[k] + 7) // 8) * 16 for k in odd)  # whole 16-byte pieces
    _refused(need, call)


@pytest.mark.parametrize("name", CALLS)
def test_shares_need_their_workspace(name):
    need, call = CALLS[name](**SHARED[name])
    assert need >= 2 * 64 * 40 * 4  # two shares' sums at least
    _refused(need, call)
    both, call = CALLS[name](**SHARED[name], x=P + 2, w=P + 2)  # and packed rows
    assert both > need
    _refused(both, call)


def test_few_tokens_need_none():
    for how in PACKED:
        case = {"tokens": 16, "inputs": 200, "outputs": 200, **how}
        assert _linear(**case)[0] == 0
