"""The norms around the residual in the forms that many rows take: several rows of a team at a time,
ragged at the end, and workgroups that go through many rows of a worker; outputs that are not asked
for; and clipping of very many tensors. Against 64 bits on the GPU, with block_reference.py's
bounds."""
import ctypes

import pytest
import torch

import paper_2010_05888_amd as gf
import block_reference as ref
import worker_reference
from paper_2010_05888_amd import worker
from test_gpu_worker import _split
from test_gpu_worker_block import FORMS, _clip_close
from test_gpu_worker_block_tiles import _check, _gpu
from worker_reference import BF16, F16, F32, U, close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [F32, BF16, F16]
LAYOUTS = ["plain", "strided", "offset", "apart"]


@pytest.fixture(scope="module", autouse=True)
def _library():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    gf.load()
    yield
    torch.cuda.empty_cache()


def _cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _block(rows, cols, dtype, i, rms=False, post=True, gate="columns", norm=True):
    """The parameters of FORMS[i]; weights in fp32 and in dtype in turn."""
    def vector(at, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        return (at + 0.3 * torch.randn(cols, generator=g, device=DEV)).to(F32 if i % 2 else dtype)

    return {"weight": vector(1, 1) if norm else None,
            "bias": vector(0, 2) if norm and not rms and i != 3 else None,
            "post_weight": vector(1, 3) if post else None,
            "post_bias": vector(0, 4) if post and not rms and i != 3 else None,
            "gate": {None: None, "columns": vector(0.5, 5),
                     "tokens": _gpu(rows, cols, 6, dtype, 1.0, LAYOUTS[(i + 1) % 4])}[gate]}


def _check_blocks(y8, want, cols):
    """As in test_gpu_worker_block.py: an exponent within the bound, codes half a step off."""
    y, bound = want
    rows, nb = y.shape[0], -(-cols // 128)

    def blocks(v):
        return torch.nn.functional.pad(v, (0, nb * 128 - cols)).view(rows, nb, 128)

    values, off = blocks(y.abs()), blocks(bound)
    top, most = values.amax(2), off.amax(2)
    s = y8.exponents[:, :nb].double() - 127
    assert bool(((worker_reference.shift((top - most).clamp(min=0)) <= s)
                 & (s <= worker_reference.shift(top + most))).all())
    p = torch.exp2(s)[:, :, None]
    step = worker_reference.half_step((values + off) / p) * p
    error = blocks((y8.restore(F32).double() - y).abs())
    assert float((error - step - off).max()) <= 0, "y8"
    assert bool((y8.exponents[:, nb:] == 127).all())
    assert not bool(y8.values[:, cols:].view(torch.uint8).any())


# (rows beyond eight a compute unit, columns): a wave to four rows, and to two; a workgroup to two rows of one
# vector a lane, and of two; eight waves, twelve and sixteen to a row
MANY = [(1, 40), (3, 300), (2, 512), (1, 513), (3, 1000), (1, 1025), (0, 2048), (1, 2055), (3, 4096), (1, 6144),
        (2, 6145), (1, 8192)]
FEW = [(1, 6145), (5, 7001), (3, 8192), (2, 6144), (2, 16384)]


def _forward(rows, cols, dtype):
    for i, form in enumerate(FORMS):
        block, rms, layout = _block(rows, cols, dtype, i, **form), form.get("rms", False), LAYOUTS[i % 4]
        x, h = _gpu(rows, cols, 10, dtype, 1.0, layout), _gpu(rows, cols, 11 + i, dtype, 1.0, layout)
        scale, normed = (1.0, 0.7, -1.5)[i % 3], block["weight"] is not None
        r = gf.residual_norm(x, h, **block, scale=scale, rms=rms, y8=normed)
        want = ref.residual_norm(x, h, **block, scale=torch.tensor(scale).double().item(), eps=1e-5, rms=rms)
        _check(r.s, want["s"], dtype, f"s {form}")
        for name in ("mean", "rstd", "post_mean", "post_rstd"):
            got = getattr(r, name)
            if name not in want or (rms and "mean" in name):
                assert got is None
            else:
                _check(got, want[name], F32, f"{name} {form}")
        if normed:
            _check(r.y, want["y"], dtype, f"y {form}")
            _check_blocks(r.y8, want["y"], cols)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("more,cols", MANY)
def test_residual_norm_of_many_rows(more, cols, dtype):
    _forward(8 * _cus() + more, cols, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", FEW)
def test_residual_norm_of_few_wide_rows(rows, cols, dtype):
    _forward(rows, cols, dtype)


def test_many_rows_keep_what_is_not_finite_in_its_row():
    """Rows that share a wave, and the last one, which fills up for those that are not there."""
    for cols in (300, 700, 1500, 4000):
        rows = 8 * _cus() + 1
        x, h = _gpu(rows, cols, 1, BF16), _gpu(rows, cols, 2, BF16)
        block = _block(rows, cols, BF16, 0)
        clean = gf.residual_norm(x, h, **block, y8=True)
        bad = [0, 5, 1002, rows - 1]
        x[0, 3], h[5, cols - 1], x[1002, 17], h[rows - 1, 0] = (float(v) for v in ("nan", "inf", "-inf", "nan"))
        r = gf.residual_norm(x, h, **block, y8=True)
        keep = torch.ones(rows, dtype=torch.bool, device=DEV)
        keep[bad] = False
        for a, b in ((r.s, clean.s), (r.y, clean.y), (r.rstd, clean.rstd), (r.post_mean, clean.post_mean),
                     (r.y8.restore(), clean.y8.restore())):
            assert torch.equal(a[keep], b[keep])
        assert bool(r.y[bad].isnan().all())


# (workers, rows of a workgroup, rows beyond, columns): the backward pass's forms, and rows beyond 8192 columns
BACKWARD = [(5, 3, 77, 40), (7, 3, 5, 512), (3, 2, 77, 600), (3, 3, 1, 1024), (2, 3, 13, 1500), (19, 4, 9, 2048),
            (3, 3, 77, 3001), (5, 6, 1, 4096), (2, 3, 9, 4097), (4, 5, 11, 8192), (3, 3, 5, 8193)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,each,more,cols", BACKWARD)
def test_residual_norm_backward_of_many_rows(n, each, more, cols, dtype):
    rows = _cus() * (8 if cols <= 512 else 4 if cols <= 1024 else 2 if cols <= 2048 else 1) * each + more
    counts = _split(rows, n, rows)
    plain = worker._ResidualBlock(worker.TYPES[dtype], 0, rows, cols, 0, 0.0, 1.0)
    need = worker._functions()["garfield_residual_norm_backward_workspace"](
        plain, n, (ctypes.c_int64 * n)(*counts))
    chunks = (need - (rows * 8 if cols > 8192 else 0)) // (5 * cols * 4)  # five sums of cols values each
    assert rows > 2 * chunks, "workgroups of two rows alone"
    for i, form in enumerate(FORMS):
        block, rms, layout = _block(rows, cols, dtype, i, **form), form.get("rms", False), LAYOUTS[i % 4]
        block.pop("bias")
        normed, scale = block["weight"] is not None, (1.0, 0.7, -1.5)[i % 3]
        h, s = _gpu(rows, cols, 20, dtype, 1.0, layout), _gpu(rows, cols, 21 + i, dtype, 1.0, layout)
        dy = _gpu(rows, cols, 31, dtype, 0.1, layout) if normed else None
        ds = _gpu(rows, cols, 32, dtype, 0.1, layout) if i != 2 else None
        ones, zeros = torch.ones(cols, device=DEV), torch.zeros(rows, cols, device=DEV).double()
        _, (mean, _), (rstd, _) = ref.norm(s.double(), zeros, ones, None, 1e-5, rms)
        _, (pm, _), (pr, _) = ref.norm(h.double(), zeros, ones, None, 1e-5, rms)
        post = block["post_weight"] is not None
        stats = [None if rms or not normed else mean.float(), rstd.float() if normed else None,
                 None if rms or not post else pm.float(), pr.float() if post else None]
        r = gf.ResidualNorm(s, None, None, *stats)

        def call():
            return gf.residual_norm_backward(r, h, ds, dy, **block, scale=scale, rms=rms, counts=counts)

        got = call()
        want = ref.residual_norm_backward(ds, dy, s, h, *stats, **block, scale=float(torch.tensor(scale)),
                                          rms=rms, counts=counts)
        _check(got.dx, want["dx"], dtype, f"dx {form}")
        _check(got.dh, want["dh"], dtype, f"dh {form}")
        for k in ("weight", "bias", "post_weight", "post_bias"):
            v = getattr(got, "d" + k)
            assert (v is not None) == ((post if "post" in k else normed) and not (rms and "bias" in k))
            if v is not None:
                _check(v, want["d" + k], F32, f"d{k} {form}")
        if block["gate"] is not None and block["gate"].dim() == 1:
            _check(got.dgate, want["dgate"], F32, f"dgate {form}")
        elif block["gate"] is not None:
            _check(got.dgate, want["dgate_by_token"], dtype, f"dgate {form}")
        for a, b in zip(call(), got):
            assert (a is None and b is None) or torch.equal(a, b), "other bits from another call"


def test_wide_rows_sums_go_round():
    """2,000,001 columns: more groups of 64 sums than a launch of the workers' sums has workgroups."""
    cols, rows, counts = 2_000_001, 3, [2, 1]
    x, h = _gpu(rows, cols, 1, BF16), _gpu(rows, cols, 2, BF16)
    block = _block(rows, cols, BF16, 0)
    r = gf.residual_norm(x, h, **block)
    want = ref.residual_norm(x, h, **block, scale=1.0, eps=1e-5, rms=False)
    _check(r.s, want["s"], BF16, "s")
    _check(r.y, want["y"], BF16, "y")
    block.pop("bias")
    ds, dy = _gpu(rows, cols, 3, BF16, 0.1), _gpu(rows, cols, 4, BF16, 0.1)
    got = gf.residual_norm_backward(r, h, ds, dy, **block, counts=counts)
    want = ref.residual_norm_backward(ds, dy, r.s, h, r.mean, r.rstd, r.post_mean, r.post_rstd, **block,
                                      scale=1.0, rms=False, counts=counts)
    _check(got.dx, want["dx"], BF16, "dx")
    _check(got.dh, want["dh"], BF16, "dh")
    for k in ("weight", "bias", "post_weight", "post_bias", "gate"):
        _check(getattr(got, "d" + k), want["d" + k], F32, k)


@pytest.mark.parametrize("gated", ["columns", "tokens"])
@pytest.mark.parametrize("rows,cols", [(37, 129), (50, 2048), (33, 5000), (9, 9000)])
def test_residual_norm_backward_of_some_outputs(rows, cols, gated):
    """dx, dh, a gate's gradient and each parameter's may be left out, at the C boundary."""
    fn, counts = worker._functions(), [rows // 2, 0, rows - rows // 2]
    x, h = _gpu(rows, cols, 1, BF16), _gpu(rows, cols, 2, BF16)
    ds, dy = _gpu(rows, cols, 3, BF16, 0.1), _gpu(rows, cols, 4, BF16, 0.1)
    block = _block(rows, cols, BF16, 1, gate=gated)
    r = gf.residual_norm(x, h, **block)
    block.pop("bias")
    full = gf.residual_norm_backward(r, h, ds, dy, **block, counts=counts)
    b = worker._residual_block(h, rows, cols, 1, block["weight"], None, block["post_weight"],
                               block["post_bias"], block["gate"], 1.0, 0.0, False)
    n, c_counts = len(counts), (ctypes.c_int64 * len(counts))(*counts)
    need = fn["garfield_residual_norm_backward_workspace"](b, n, c_counts)
    space = torch.empty(need, dtype=torch.uint8, device=DEV)
    by_tokens = gated == "tokens"
    for asked in range(1, 1 << len(full)):
        out = [torch.full_like(t, 7.0) for t in full]  # dx, dh, dweight, dbias, dpost_weight, dpost_bias, dgate
        p = [t.data_ptr() if asked >> i & 1 else None for i, t in enumerate(out)]
        to = worker._ResidualGradients(*p[2:6], None if by_tokens else p[6], cols, cols, cols, cols, cols)
        code = fn["garfield_residual_norm_backward"](
            b, ds.data_ptr(), cols, dy.data_ptr(), cols, r.s.data_ptr(), cols, h.data_ptr(), cols,
            r.mean.data_ptr(), r.rstd.data_ptr(), r.post_mean.data_ptr(), r.post_rstd.data_ptr(), p[0], cols,
            p[1], cols, p[6] if by_tokens else None, cols, n, c_counts, to, space.data_ptr(), need,
            torch.cuda.current_stream().cuda_stream)
        assert code == gf.OK
        for i, (got, want) in enumerate(zip(out, full)):
            assert torch.equal(got, want if asked >> i & 1 else torch.full_like(want, 7.0)), (asked, i)


# --------------------------------------------------------------------------- products
@pytest.mark.parametrize("dtype", DTYPES)
def test_products_of_no_depth(dtype):
    """More tokens than the form for few takes: sums of nothing are 0."""
    x, w = torch.empty(40, 0, dtype=dtype, device=DEV), torch.empty(30, 0, dtype=dtype, device=DEV)
    bias, residual = torch.full((30,), 2.0, device=DEV), _gpu(40, 30, 1, dtype)
    r = gf.linear(x, w, bias, "relu", residual, pre=True)
    assert bool(r.pre.eq(2).all())
    want = residual.double() + 2
    _check(r.out, (want, U * want.abs()), dtype, "out")  # added in fp32, then rounded
    got = gf.linear_backward(x, torch.empty(0, 30, dtype=dtype, device=DEV), residual, "gelu", residual)
    assert torch.equal(got, residual)


def test_packed_rows_go_round():
    """2^21 rows of 4099 values, packed: more 16-byte pieces than a launch has threads."""
    m, k, n = 1 << 21, 4099, 3
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.empty(m, k, dtype=BF16, device=DEV).normal_(generator=g)
    w = _gpu(n, k, 2, BF16, k ** -0.5)
    out = gf.linear(x, w).out
    for at in list(range(0, m, 1 << 18)) + [m - 4096]:
        part = x[at:at + 4096]
        _check(out[at:at + 4096], ref.linear(part, w, None, None, None)[0], BF16, f"rows from {at}")
    del x, out


# --------------------------------------------------------------------------- clipping
@pytest.mark.parametrize("types", [[F32], [F16, F32, BF16]])
@pytest.mark.parametrize("n,count", [(3, 256), (3, 257), (2, 1000)])
def test_clip_of_many_tensors(n, count, types):
    """Tables of hundreds of tensors, empty ones among them, some of several chunks."""
    lengths = []
    for i in range(count):
        lengths += [20_000 if i % 50 == 0 else 1 + i * 37 % 50] + [0] * (i % 7 == 3)
    grads = [_gpu(n, k, i, types[i % len(types)]) for i, k in enumerate(lengths)]
    d = sum(lengths)
    limit = 0.9 * float(ref.clip(grads, 1.0)[0].median())
    limit = float(torch.tensor(limit).float())
    norms, rows = ref.clip(grads, limit)
    out = torch.full((n, d + 2), float("nan"), device=DEV)
    close(gf.gradient_norms(grads), norms, 1.01 * U * norms, "norms")
    close(gf.clip_gradients(grads, limit, out=out[:, 1:-1]), norms, 1.01 * U * norms, "norms")
    _clip_close(out[:, 1:-1], rows, F32)
    assert bool(out[:, 0].isnan().all()) and bool(out[:, -1].isnan().all())
    gf.clip_gradients(grads, limit)
    at = 0
    for g in grads:
        _clip_close(g, rows[:, at:at + g.shape[1]], g.dtype)
        at += g.shape[1]


def test_clip_of_more_chunks_than_a_launch_has_workgroups():
    """131,073 tensors of one value of 64 workers: columns of one matrix, each a chunk."""
    n, count = 64, (1 << 17) + 1
    m = _gpu(n, count, 1, F32) * torch.linspace(0.3, 1.5, n, device=DEV)[:, None]
    was, grads = m.clone(), list(m.split(1, dim=1))
    norms, rows = ref.clip([m], 300.0)
    assert 0 < int((norms > 300.0).sum()) < n
    out = torch.empty(n, count, device=DEV)
    close(gf.clip_gradients(grads, 300.0, out=out), norms, 1.01 * U * norms, "norms")
    _clip_close(out, rows, F32)
    assert torch.equal(m, was)
    close(gf.gradient_norms(grads), norms, 1.01 * U * norms, "norms")
    gf.clip_gradients(grads, 300.0)
    _clip_close(m, rows, F32)
