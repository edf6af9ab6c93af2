"""The operators of a worker's residual block without a GPU: what the host refuses before
anything touches a device, and the 64-bit references against autograd."""
import ctypes

import pytest
import torch

import paper_2010_05888_amd as gf
from paper_2010_05888_amd import worker
import block_reference as ref

P = 0x1000  # an aligned address, never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module")
def fn():
    return worker._functions()


def _counts(*c):
    return (ctypes.c_int64 * len(c))(*c)


def test_linear_refuses(fn):
    def call(x=P, t=1, m=4, k=200, ldx=200, w=P, n=7, ldw=200, b=None, bt=0, act=0, r=None, ldr=7,
             out=P, ldo=7, pre=None, ldp=7):
        return fn["garfield_linear"](x, t, m, k, ldx, w, n, ldw, b, bt, act, r, ldr, out, ldo, pre, ldp,
                                     1 << 20, BIG, None)

    for bad in (dict(x=None), dict(x=P + 1), dict(t=3), dict(m=-1), dict(k=-1), dict(ldx=199), dict(w=None),
                dict(w=P + 1), dict(ldw=100), dict(n=-2), dict(b=P + 2), dict(b=P, bt=2), dict(act=5),
                dict(act=-1), dict(r=P + 1), dict(r=P, ldr=6), dict(out=None), dict(ldo=6), dict(pre=P + 1),
                dict(pre=P, ldp=3)):
        assert call(**bad) == gf.EINVAL, bad
    assert call(m=0) == gf.OK and call(n=0) == gf.OK
    assert call(k=(1 << 24) + 1, ldx=1 << 25, ldw=1 << 25) == gf.ETOOBIG
    assert call(m=1 << 26) == gf.ETOOBIG
    need = fn["garfield_linear_workspace"](P + 2, 1, 4, 200, 201, P, 7, 200)
    if need:
        f = fn["garfield_linear"]
        args = (P + 2, 1, 4, 200, 201, P, 7, 200, None, 0, 0, None, 0, P, 7, None, 0)
        assert f(*args, None, need, None) == gf.EINVAL
        assert f(*args, 1 << 20, need - 1, None) == gf.EINVAL
        assert f(*args, (1 << 20) + 8, need, None) == gf.EINVAL
    assert fn["garfield_linear_workspace"](P, 9, 4, 200, 200, P, 7, 200) == 0


def test_linear_backward_refuses(fn):
    def call(dy=P, t=1, m=4, n=7, lddy=7, w=P, k=200, ldw=200, act=2, pre=P, ldp=200, r=None, ldr=200,
             dx=P, lddx=200):
        return fn["garfield_linear_backward"](dy, t, m, n, lddy, w, k, ldw, act, pre, ldp, r, ldr, dx, lddx,
                                              1 << 20, BIG, None)

    for bad in (dict(dy=None), dict(dy=P + 1), dict(t=-1), dict(m=-1), dict(lddy=6), dict(w=None), dict(ldw=199),
                dict(act=9), dict(pre=None), dict(pre=P + 1), dict(ldp=199), dict(r=P + 1), dict(r=P, ldr=1),
                dict(dx=None), dict(lddx=199)):
        assert call(**bad) == gf.EINVAL, bad
    assert call(m=0) == gf.OK
    assert call(n=1 << 25, lddy=1 << 25) == gf.ETOOBIG


def test_activation_backward_refuses(fn):
    def call(dy=P, t=1, m=4, k=200, ld=200, act=2, pre=P, ldp=200, dp=P, lddp=200):
        return fn["garfield_activation_backward"](dy, t, m, k, ld, act, pre, ldp, dp, lddp, None)

    for bad in (dict(dy=None), dict(t=4), dict(ld=1), dict(act=7), dict(pre=None), dict(ldp=3), dict(dp=P + 1),
                dict(lddp=199), dict(k=-1)):
        assert call(**bad) == gf.EINVAL, bad
    assert call(m=0) == gf.OK


def test_linear_weight_gradient_refuses(fn):
    def call(dy=P, t=1, tokens=4, outputs=10, lddy=10, x=P, inputs=200, ldx=200, n=2, counts=(1, 3), dw=P,
             lddw=2000, db=None, lddb=10):
        return fn["garfield_linear_weight_gradient"](
            dy, t, tokens, outputs, lddy, x, inputs, ldx, n, _counts(*counts) if counts else None, dw, lddw,
            db, lddb, 1 << 20, BIG, None)

    for bad in (dict(dy=None), dict(dy=P + 1), dict(t=5), dict(lddy=9), dict(x=None), dict(x=P + 1),
                dict(ldx=100), dict(n=0), dict(counts=None), dict(counts=(1, 1)), dict(counts=(5, -1)),
                dict(dw=None), dict(dw=P + 2), dict(lddw=1999), dict(db=P + 1), dict(db=P, lddb=9)):
        assert call(**bad) == gf.EINVAL, bad
    assert call(n=65, counts=[0] * 65) == gf.ETOOBIG
    assert call(outputs=(1 << 24) + 8, lddy=1 << 25) == gf.ETOOBIG
    assert call(outputs=0, lddy=0) == gf.OK


def _residual(t=1, wt=0, rows=4, cols=200, rms=0, eps=1e-5, w=P, b=None, pw=P, pb=None, gate=P, ldg=0):
    return worker._ResidualBlock(t, wt, rows, cols, rms, eps, 1.0, w, b, pw, pb, gate, ldg)


BAD_BLOCKS = [dict(t=3), dict(wt=2), dict(rows=-1), dict(cols=0), dict(eps=-1.0), dict(eps=float("nan")),
              dict(w=P + 2), dict(b=P + 2), dict(w=None, b=P), dict(pw=None, pb=P), dict(rms=1, b=P),
              dict(rms=1, pb=P), dict(gate=P + 2), dict(gate=P + 1, ldg=200), dict(ldg=199)]


def test_residual_norm_refuses(fn):
    def call(block=None, x=P, ldx=200, h=P, ldh=200, s=P, lds=200, y=P, ldy=200, stats=(P, P, P, P), y8=None):
        return fn["garfield_residual_norm"](block or _residual(), x, ldx, h, ldh, s, lds, y, ldy, *stats, y8,
                                            None)

    for bad in BAD_BLOCKS:
        assert call(_residual(**bad)) == gf.EINVAL, bad
    y8 = worker._Block8(P, P, 4, 199, 256, 4)
    for bad in (dict(x=None), dict(ldx=1), dict(h=P + 1), dict(ldh=199), dict(s=None), dict(lds=2), dict(y=P + 1),
                dict(ldy=100), dict(y8=y8), dict(stats=(None, P, P, P)), dict(stats=(P, None, P, P)),
                dict(stats=(P, P, P + 2, P)), dict(stats=(P, P, P, None)), dict(block=_residual(w=None))):
        assert call(**bad) == gf.EINVAL, bad
    assert call(_residual(rows=0)) == gf.OK
    assert call(_residual(rows=1 << 26)) == gf.ETOOBIG
    assert fn["garfield_residual_norm"](None, P, 200, P, 200, P, 200, P, 200, P, P, P, P, None, None) == gf.EINVAL


def test_residual_norm_backward_refuses(fn):
    def call(block=None, ds=P, ldds=200, dy=P, lddy=200, s=P, lds=200, h=P, ldh=200, stats=(P, P, P, P), dx=P,
             lddx=200, dh=P, lddh=200, dgate=None, lddg=200, n=2, counts=(1, 3), to=None, ws=1 << 20, size=BIG):
        g = worker._ResidualGradients()
        for k, v in (to or {}).items():
            setattr(g, k, v)
        return fn["garfield_residual_norm_backward"](
            block or _residual(), ds, ldds, dy, lddy, s, lds, h, ldh, *stats, dx, lddx, dh, lddh, dgate, lddg, n,
            _counts(*counts), g, ws, size, None)

    for bad in BAD_BLOCKS:
        assert call(_residual(**bad)) == gf.EINVAL, bad
    by_tokens = _residual(ldg=200)
    for bad in (dict(ds=None, dy=None), dict(ds=P + 1), dict(ldds=3), dict(dy=P + 1), dict(lddy=3),
                dict(block=_residual(w=None)), dict(s=None), dict(lds=1), dict(h=None), dict(ldh=199),
                dict(stats=(None, P, P, P)), dict(stats=(P, None, P, P)), dict(stats=(P, P, None, P)),
                dict(stats=(P, P, P, P + 1)), dict(dx=P + 1), dict(lddx=1), dict(dh=P + 1), dict(lddh=1),
                dict(dgate=P), dict(block=by_tokens, dgate=P, lddg=7), dict(block=by_tokens, to=dict(gate=P)),
                dict(n=0), dict(counts=(1, 2)), dict(counts=(-1, 5)), dict(to=dict(weight=P, ld_weight=199)),
                dict(to=dict(bias=P + 2, ld_bias=200)), dict(block=_residual(rms=1), to=dict(bias=P, ld_bias=200)),
                dict(block=_residual(pw=None), to=dict(post_weight=P, ld_post_weight=200)),
                dict(block=_residual(rms=1), to=dict(post_bias=P, ld_post_bias=200)),
                dict(block=_residual(gate=None), to=dict(gate=P, ld_gate=200)), dict(ws=None), dict(ws=P + 8),
                dict(size=16)):
        assert call(**bad) == gf.EINVAL, bad
    assert call(n=65, counts=[0] * 65) == gf.ETOOBIG


def _tensors(*t):
    return (worker._Gradient * len(t))(*[worker._Gradient(*v) for v in t])


def test_clip_refuses(fn):
    def call(tensors=((P, 10, 10, 0), (0x9000, 5, 5, 1)), n=2, most=1.0, norms=P, out=P, ld=15, ws=1 << 20,
             size=BIG):
        return fn["garfield_clip_gradients"](_tensors(*tensors), len(tensors), n, most, norms, out, ld, ws, size,
                                             None)

    for bad in (dict(n=0), dict(most=-1.0), dict(most=float("nan")), dict(norms=None), dict(norms=P + 2),
                dict(out=P + 2), dict(ld=14),
                dict(tensors=((P, 1 << 20, 1 << 20, 0),), ld=1 << 20, ws=None),
                dict(tensors=((P, 1 << 20, 1 << 20, 0),), ld=1 << 20, ws=P + 8),
                dict(tensors=((P, 1 << 20, 1 << 20, 0),), ld=1 << 20, size=8),
                dict(tensors=((None, 10, 10, 0),)), dict(tensors=((P + 2, 10, 10, 0),)),
                dict(tensors=((P, 10, 9, 0),)), dict(tensors=((P, -1, 10, 0),)), dict(tensors=((P, 10, 10, 3),)),
                # in place, tensors may not share memory
                dict(out=None, tensors=((P, 10, 10, 0), (P, 10, 10, 0))),
                dict(out=None, tensors=((P, 10, 30, 0), (P + 36, 10, 30, 0))),
                dict(out=None, tensors=((P, 10, 30, 0), (P + 40, 21, 30, 0))),
                dict(out=None, tensors=((P, 10, 30, 0), (P + 40, 10, 31, 0))),
                dict(out=None, tensors=((P, 10, 30, 0), (P + 40, 10, 60, 1), (P + 56, 5, 30, 0))),
                dict(out=None, n=1, tensors=((P, 10, 0, 0), (P + 39, 10, 0, 1))),
                # nor with the rows that are written
                dict(out=P, ld=10, tensors=((P, 10, 10, 0),)), dict(out=P + 36, ld=30, tensors=((P, 10, 30, 0),)),
                dict(out=P + 40, ld=31, tensors=((P, 10, 30, 0),)),
                dict(out=0x9000 + 8, ld=15), dict(out=P - 40, ld=30, tensors=((P, 11, 30, 0),))):
        assert call(**bad) == gf.EINVAL, bad
    assert call(n=65) == gf.ETOOBIG
    assert call(tensors=((P, (1 << 34) + 1, 1 << 35, 0),)) == gf.ETOOBIG
    assert fn["garfield_gradient_norms"](None, 1, 2, P, 1 << 20, BIG, None) == gf.EINVAL
    assert fn["garfield_gradient_norms"](None, -1, 2, P, 1 << 20, BIG, None) == gf.EINVAL


def test_python_refuses_what_is_not_on_a_gpu():
    x, v = torch.zeros(4, 200), torch.zeros(200)
    r = gf.ResidualNorm(x, x, None, v, v, v, v)
    for call in (lambda: gf.linear(x, x), lambda: gf.linear_backward(x, x),
                 lambda: gf.activation_backward(x, x, "relu"), lambda: gf.linear_weight_gradient(x, x),
                 lambda: gf.residual_norm(x, x, v), lambda: gf.residual_norm_backward(r, x, x),
                 lambda: gf.gradient_norms(x), lambda: gf.clip_gradients([x], 1.0)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("name", [None] + ref.ACTIVATIONS)
def test_reference_slopes_are_the_activations(name):
    p = torch.linspace(-9, 9, 181, dtype=torch.float64, requires_grad=True)
    want, = torch.autograd.grad(ref.activation(name, p).sum(), p)
    assert float((ref.slope(name, p.detach()) - want).abs().max()) < 1e-12


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("by", [None, "columns", "tokens"])
def test_reference_gradients_are_the_forward_passes(by, rms):
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64, requires_grad=True)  # noqa: E731
    x, h, w, pw, ds, dy = n(6, 9), n(6, 9), n(9), n(9), n(6, 9), n(6, 9)
    b, pb = (None, None) if rms else (n(9), n(9))
    gate = {None: None, "columns": n(9), "tokens": n(6, 9)}[by]
    out = ref.residual_norm(x, h, w, b, pw, pb, gate, 0.7, 1e-5, rms)
    wanted = {"x": x, "h": h, "weight": w, "bias": b, "post_weight": pw, "post_bias": pb, "gate": gate}
    wanted = {k: v for k, v in wanted.items() if v is not None}
    grads = dict(zip(wanted, torch.autograd.grad((ds * out["s"][0] + dy * out["y"][0]).sum(),
                                                 list(wanted.values()))))
    stat = lambda k: out[k][0].detach()  # noqa: E731
    got = ref.residual_norm_backward(ds.detach(), dy.detach(), stat("s"), h.detach(), stat("mean"), stat("rstd"),
                                     stat("post_mean"), stat("post_rstd"), w.detach(), pw.detach(),
                                     None if rms else pb.detach(), None if gate is None else gate.detach(), 0.7,
                                     rms, [6])
    for k, v in grads.items():
        have = got["dgate_by_token"] if k == "gate" and by == "tokens" else got["d" + k]
        assert float((have[0].reshape(v.shape) - v).abs().max()) < 1e-12, k
