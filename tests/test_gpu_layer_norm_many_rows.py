"""The layer norm where a CTA has many rows, so that the rings reuse their stages, fetch past the first mask word and keep
the columns' sums over all of it: against the formula in float64 (on the GPU: the matrices are large).

Tolerances are those of tests/test_gpu_layer_norm.py: sums of n terms have at most n / 32 + 32 additions on a term's way, g =
(n / 32 + 32) 2^-24; x - mean is off by its rounding, the mean's and the sum's (dh, in units of h); rstd is relative g + 4 u;
a result in bf16 adds half a step. Fixed before the first run.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
TYPES = [(BF, BF), (BF, F32), (F32, BF), (F32, F32)]
EPS = 1e-5


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


# CTAs of a backward launch: 152 at 4,104 and 4,101 columns (34 rows each: more than the 32 whose mask is read at once), 608 to
# 2,432 at the others; stages: 2 to 8. Up to 256 columns rows go several to a warp.
SHAPES = [(5200, 4104, 0, 0), (5200, 4101, 2, 1), (9000, 2048, 8, 0), (9000, 2050, 0, 1), (15000, 1024, 0, 0), (12000, 1001, 3, 1),
          (40000, 512, 0, 0), (24000, 300, 1, 0), (20000, 200, 0, 0), (20000, 130, 3, 1), (20000, 96, 0, 0), (20000, 100, 1, 1),
          (1300, 96, 0, 0)]


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF else U


def matrix(rows, D, dtype, pad, off):
    buf = torch.full((rows * (D + pad) + off + 8,), 777.0, dtype=dtype, device="cuda")
    return buf[off:off + rows * (D + pad)].view(rows, D + pad)[:, :D], buf


def outside_is_untouched(view, buf):
    inside = torch.zeros(buf.shape, dtype=torch.bool, device="cuda")
    off = (view.data_ptr() - buf.data_ptr()) // view.element_size()
    rows, D = view.shape
    inside[off:off + rows * view.stride(0)].view(rows, -1)[:, :D] = True
    return bool((buf[~inside] == 777).all())


def make(rows, D, types, pad, off, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def noise(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    x, _ = matrix(rows, D, types[0], pad, off)
    x.copy_(noise(rows, D) * torch.rand(rows, 1, generator=g, device="cuda").mul(3).exp() + 1.5 * noise(rows, 1))
    dy, _ = matrix(rows, D, types[1], pad, off)
    dy.copy_(noise(rows, D) * 1e-3)
    return x, dy, 1 + 0.3 * noise(D), 0.2 * noise(D), g


def within(err, tol, what):
    assert bool((err <= tol * (1 + 1e-3) + 1e-37).all()), (what, float((err / (tol + 1e-37)).max()))


def check_fwd(got, x, w, b, what):
    y, mean, rstd = (t.double() for t in got)
    x64, w64, b64 = x.double(), w.double(), b.double()
    D = x.shape[1]
    g = (D / 32 + 32) * U
    rm = x64.mean(1)
    rr = ((x64 - rm[:, None]).square().mean(1) + EPS).rsqrt()
    size = x64.abs().mean(1)
    within((mean - rm).abs(), g * size + 2 * U * rm.abs(), (what, "mean"))
    h = (x64 - rm[:, None]) * rr[:, None]
    dh = rr[:, None] * (U * (2 * x64.abs() + 2 * rm.abs()[:, None]) + g * size[:, None])
    rel = g + 4 * U + (h.abs() * dh).mean(1) + dh.square().mean(1)
    within((rstd - rr).abs(), rel * rr, (what, "rstd"))
    ry = h * w64 + b64
    tol = w64.abs() * (dh + (rel[:, None] + 2 * U) * h.abs()) + 2 * U * ry.abs() + half_step(got[0].dtype) * ry.abs()
    tol += U * b64.abs() + half_step(got[0].dtype) * w64.abs() * dh
    within((y - ry).abs(), tol, (what, "y"))


def check_bwd(dx, dw, db, dw0, db0, dy, x, mean, rstd, w, mask, what):
    on = torch.ones(len(x), dtype=torch.bool, device="cuda") if mask is None else mask != 0
    assert bool((dx[~on] == 0).all()), what
    x64, d64, m, r, w64 = x[on].double(), dy[on].double(), mean[on].double()[:, None], rstd[on].double()[:, None], w.double()
    rows, D = x64.shape
    g = (D / 32 + 32) * U
    h = (x64 - m) * r
    dh = r * U * (2 * x64.abs() + m.abs()) + 2 * U * h.abs()
    gr = d64 * w64
    ref = r * (gr - gr.mean(1, keepdim=True) - h * (gr * h).mean(1, keepdim=True))
    s, q = gr.abs().mean(1, keepdim=True), (gr * h).abs().mean(1, keepdim=True)
    qe = g * q + 2 * U * q + (gr.abs() * dh).mean(1, keepdim=True)
    tol = r * (4 * U * gr.abs() + (g + 4 * U) * s + h.abs() * (qe + 4 * U * q) + dh * q)
    tol = tol * (1 + 1e-3) + (half_step(dx.dtype) + 2 * U) * ref.abs() + half_step(dx.dtype) * tol
    within((dx[on].double() - ref).abs(), tol, (what, "dx"))
    gw = (rows / 32 + 32) * U
    for name, got, got0, val, size, extra in (("dw", dw, dw0, (d64 * h).sum(0), (d64 * h).abs().sum(0), (d64.abs() * dh).sum(0)),
                                              ("db", db, db0, d64.sum(0), d64.abs().sum(0), 0.0)):
        err = (got.double() - got0.double() - val).abs()
        within(err, (gw + 2 * U) * size + extra + 2 * U * (got0.double().abs() + size), (what, name))


def masks(rows, g):
    """None; 60% of the rows at random; runs of some thousand rows with and without a gradient, and few in the last of them."""
    rand = torch.rand(2, rows, generator=g, device="cuda")
    at = torch.arange(rows, device="cuda")
    runs = torch.where(at < rows - rows // 7, (at // (rows // 7)) % 2 == 0, rand[1] < 0.02)
    return [None, (rand[0] < 0.6).to(torch.uint8), runs.to(torch.uint8)]


@pytest.mark.parametrize("rows,D,pad,off", SHAPES)
@pytest.mark.parametrize("types", TYPES)
def test_many_rows(R, rows, D, pad, off, types):
    x, dy, w, b, g = make(rows, D, types, pad, off, seed=D)
    what = (rows, D, pad, off, types)
    y, ybuf = matrix(rows, D, types[1], pad, off)
    got = R.rl_layer_norm_fwd(x, weight=w, bias=b, eps=EPS, y=y)
    check_fwd(got, x, w, b, what)
    assert outside_is_untouched(y, ybuf), what
    _, mean, rstd = got
    ws = R.new_layer_norm_workspace(rows, D)
    for kind, mask in enumerate(masks(rows, g)):
        if mask is not None:
            # what is not trained on is not read
            x_, dy_ = x.clone(), dy.clone()
            x_[mask == 0], dy_[mask == 0] = float("nan"), float("inf")
        else:
            x_, dy_ = x, dy
        dw, db = 1e-3 * torch.randn(D, generator=g, device="cuda"), 1e-3 * torch.randn(D, generator=g, device="cuda")
        dw0, db0 = dw.clone(), db.clone()
        dx, dxbuf = matrix(rows, D, types[0], pad, off)
        xs, _ = matrix(rows, D, types[0], pad, off)
        ds, _ = matrix(rows, D, types[1], pad, off)
        xs.copy_(x_)
        ds.copy_(dy_)
        R.rl_layer_norm_bwd(ds, xs, mean, rstd, ws, weight=w, mask=mask, d_x=dx, d_weight=dw, d_bias=db)
        check_bwd(dx, dw, db, dw0, db0, dy, x, mean, rstd, w, mask, (what, kind))
        assert outside_is_untouched(dx, dxbuf), (what, kind)
        again_w = dw0.clone()
        R.rl_layer_norm_bwd(ds, xs, mean, rstd, ws, weight=w, mask=mask, d_x=dx, d_weight=again_w)
        assert torch.equal(again_w, dw), (what, kind)
    assert R.rl_query_status(ws)[1] == 0


@pytest.mark.parametrize("rows,D,pad,off", [s for s in SHAPES if s[0] > 1300])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_rows_in_place(R, rows, D, pad, off, dtype):
    x, dy, w, b, g = make(rows, D, (dtype, dtype), pad, off, seed=rows)
    mask = masks(rows, g)[1]
    y, _ = matrix(rows, D, dtype, pad, off)
    _, mean, rstd = R.rl_layer_norm_fwd(x, weight=w, bias=b, y=y)

    def copy(t):
        c, buf = matrix(rows, D, dtype, pad, off)
        c.copy_(t)
        return c, buf

    over, buf = copy(x)
    R.rl_layer_norm_fwd(over, weight=w, bias=b, y=over)
    assert torch.equal(over, y) and outside_is_untouched(over, buf)
    ws = R.new_layer_norm_workspace(rows, D)
    dws = [torch.zeros(D, device="cuda") for _ in range(3)]
    dx, _ = matrix(rows, D, dtype, pad, off)
    R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w, mask=mask, d_x=dx, d_weight=dws[0])
    for i, first in ((1, True), (2, False)):
        over, buf = copy(dy if first else x)
        R.rl_layer_norm_bwd(over if first else dy, x if first else over, mean, rstd, ws, weight=w, mask=mask, d_x=over,
                            d_weight=dws[i])
        assert torch.equal(over, dx) and torch.equal(dws[i], dws[0]) and outside_is_untouched(over, buf), first
