"""rl_layer_norm_fwd and rl_layer_norm_bwd against their float64 reference.

Tolerances, fixed before the first run. u = 2^-24 is fp32's rounding. A sum of n terms that threads take in turns and
then add up in a tree has at most n / 32 + 32 additions on any term's way: its error is at most g = (n / 32 + 32) u times the
sum of the terms' sizes. x - mean has the error of its rounding, of the mean's rounding and of the sum: dh below, in units
of h. rstd is relative g + 4 u (half the error of the squares' sum, the root, the quotient). A result in bf16 adds half a
step, 2^-8 of it.
"""

import numpy as np
import pytest
import torch

import oracle.model_ends as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF else U


def np64(t):
    return t.detach().double().cpu().numpy()


def strided(rows, D, dtype, pad=0, shift=0, fill=777.0):
    """A [rows, D] view of a buffer filled with `fill`, rows D + pad apart, `shift` elements from its start; and the buffer."""
    buf = torch.full((rows * (D + pad) + shift + 8,), fill, dtype=dtype, device="cuda")
    return buf[shift:shift + rows * (D + pad)].view(rows, D + pad)[:, :D], buf


def outside_is_untouched(view, buf, fill=777.0):
    inside = torch.zeros(buf.shape, dtype=torch.bool, device="cuda")
    rows, D = view.shape
    off = (view.data_ptr() - buf.data_ptr()) // view.element_size()
    ld = view.stride(0) if rows > 1 else D
    inside[(off + torch.arange(rows, device="cuda")[:, None] * ld + torch.arange(D, device="cuda")).reshape(-1)] = True
    return bool((buf[~inside] == fill).all())


def make(rows, D, x_dtype, y_dtype, seed=0, shift=1.5, pad=0, off=0):
    g = torch.Generator().manual_seed(seed)
    x, xbuf = strided(rows, D, x_dtype, pad, off)
    x.copy_(torch.randn(rows, D, generator=g) * torch.rand(rows, 1, generator=g).mul(3).exp() + shift * torch.randn(rows, 1, generator=g))
    dy, _ = strided(rows, D, y_dtype, pad, off)
    dy.copy_(torch.randn(rows, D, generator=g) * 1e-3)
    w = 1 + 0.3 * torch.randn(D, generator=g)
    b = 0.2 * torch.randn(D, generator=g)
    return x, dy, w.cuda(), b.cuda()


def bounds(x, mean, rstd):
    """g of a row's sums; the error of x - mean in units of h, [rows, D]."""
    D = x.shape[1]
    g = (D / 32 + 32) * U
    dh = rstd[:, None] * (U * (2 * np.abs(x) + 2 * np.abs(mean)[:, None]) + g * np.abs(x).mean(1, keepdims=True))
    return g, dh


def check_fwd(got, x, w, b, eps, what):
    y, mean, rstd = got
    x64 = np64(x)
    ry, rm, rr = O.layer_norm(x64, None if w is None else np64(w), None if b is None else np64(b), eps)
    g, dh = bounds(x64, rm, rr)
    assert (np.abs(np64(mean) - rm) <= g * np.abs(x64).mean(1) + 2 * U * np.abs(rm)).all(), what
    # the squares of x - mean: their error 2 |h| dh on average, and dh^2
    h = (x64 - rm[:, None]) * rr[:, None]
    rel = g + 4 * U + (np.abs(h) * dh).mean(1) + (dh * dh).mean(1)
    assert (np.abs(np64(rstd) - rr) <= rel * rr).all(), what
    w64 = np.ones(x64.shape[1]) if w is None else np64(w)
    tol = np.abs(w64) * (dh + (rel[:, None] + 2 * U) * np.abs(h)) + 2 * U * np.abs(ry) + half_step(y.dtype) * np.abs(ry)
    if b is not None:
        tol += U * np.abs(np64(b)) + half_step(y.dtype) * np.abs(w64) * dh
    tol = tol * (1 + 1e-3) + 1e-37
    assert (np.abs(np64(y) - ry) <= tol).all(), (what, np.max(np.abs(np64(y) - ry) / tol))


def check_bwd(dx, dw, db, dw0, db0, dy, x, mean, rstd, w, mask, what):
    x64, dy64, m64, r64 = np64(x), np64(dy), np64(mean), np64(rstd)
    mk = None if mask is None else mask.cpu().numpy()
    rdx, rdw, rdb = O.layer_norm_grad(dy64, x64, m64, r64, None if w is None else np64(w), mk)
    on = np.ones(len(x64), bool) if mk is None else mk != 0
    assert (np64(dx)[~on] == 0).all(), what
    x64, dy64, m64, r64 = x64[on], dy64[on], m64[on], r64[on]
    rows, D = x64.shape
    if rows:
        g = (D / 32 + 32) * U
        h = (x64 - m64[:, None]) * r64[:, None]
        dh = r64[:, None] * U * (2 * np.abs(x64) + np.abs(m64)[:, None]) + 2 * U * np.abs(h)
        gr = dy64 * (1 if w is None else np64(w))
        s, q = np.abs(gr).mean(1, keepdims=True), np.abs(gr * h).mean(1, keepdims=True)
        qe = g * q + 2 * U * q + (np.abs(gr) * dh).mean(1, keepdims=True)
        tol = r64[:, None] * (4 * U * np.abs(gr) + (g + 4 * U) * s + np.abs(h) * (qe + 4 * U * q) + dh * q)
        tol = tol * (1 + 1e-3) + (half_step(dx.dtype) + 2 * U) * np.abs(rdx[on]) + half_step(dx.dtype) * tol + 1e-37
        err = np.abs(np64(dx)[on] - rdx[on])
        assert (err <= tol).all(), (what, np.max(err / tol))
        gw = (rows / 32 + 32) * U
        for got, got0, ref, size, extra in ((dw, dw0, rdw, np.abs(dy64 * h).sum(0), (np.abs(dy64) * dh).sum(0)),
                                            (db, db0, rdb, np.abs(dy64).sum(0), 0.0)):
            if got is not None:
                e = np.abs(np64(got) - np64(got0) - ref)
                lim = (gw + 2 * U) * size + extra + 2 * U * (np.abs(np64(got0)) + size) + 1e-37
                assert (e <= lim * (1 + 1e-3)).all(), (what, np.max(e / lim))
    else:
        for got, got0 in ((dw, dw0), (db, db0)):
            assert got is None or torch.equal(got, got0), what


SHAPES = [(1, 1), (3, 2), (5, 7), (4, 8), (130, 31), (7, 64), (33, 100), (9, 255), (66, 256), (5, 257), (40, 512), (3, 1000),
          (611, 1001), (20, 1024), (17, 2048), (6, 2777), (300, 4096), (2, 4100), (35, 8192), (3, 8200), (5, 16384),
          (4, 20001), (1, 70000), (1, 4096), (2000, 96)]


@pytest.mark.parametrize("rows,D", SHAPES)
@pytest.mark.parametrize("types", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
def test_forward_and_backward(R, rows, D, types):
    for pad, off, seed in ((0, 0, 1), (3, 0, 2), (8, 0, 3), (1, 1, 4)):
        x, dy, w, b = make(rows, D, *types, seed=seed, pad=pad, off=off)
        if seed == 2:
            w = None
        if seed == 3:
            w, b = w.to(BF), b.to(BF)
        if seed == 4:
            b = None
        what = (rows, D, types, pad, off)
        y, ybuf = strided(rows, D, types[1], pad, off)
        got = R.rl_layer_norm_fwd(x, weight=w, bias=b, eps=1e-5, y=y)
        check_fwd(got, x, w, b, 1e-5, what)
        assert outside_is_untouched(y, ybuf), what
        _, mean, rstd = got
        g = torch.Generator().manual_seed(seed)
        mask = None if seed in (1, 4) else (torch.rand(rows, generator=g) < 0.6).to(torch.uint8).cuda()
        dw, db = torch.randn(D, generator=g).cuda() * 1e-3, torch.randn(D, generator=g).cuda() * 1e-3
        if seed == 4:
            db = None
        dw0, db0 = dw.clone(), None if db is None else db.clone()
        dx, dxbuf = strided(rows, D, types[0], pad, off)
        ws = R.new_layer_norm_workspace(rows, D)
        out = R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w, mask=mask, d_x=dx, d_weight=dw, d_bias=db)
        assert out is dx and R.rl_query_status(ws)[1] == 0
        check_bwd(dx, dw, db, dw0, db0, dy, x, mean, rstd, w, mask, what)
        assert outside_is_untouched(dx, dxbuf), what


def test_values_that_are_hard(R):
    """A mean far from zero, equal entries, one large entry, tiny entries."""
    D = 1000
    x = torch.zeros(6, D, device="cuda")
    g = torch.Generator().manual_seed(5)
    x[0] = 1000 + torch.randn(D, generator=g).cuda()
    x[1] = 7.25
    x[2, 17] = 3e4
    x[3] = torch.randn(D, generator=g).cuda() * 1e-12
    x[5] = -1e4 + 1e-2 * torch.randn(D, generator=g).cuda()
    w = torch.ones(D, device="cuda")
    got = R.rl_layer_norm_fwd(x, weight=w, eps=1e-5)
    check_fwd(got, x, w, None, 1e-5, "hard values")
    assert (got[0][1] == 0).all() and (got[0][4] == 0).all()
    with_none = R.rl_layer_norm_fwd(x[1:2], eps=0.0)[0]
    assert torch.isnan(with_none).all()


def test_rows_with_nan_stay_alone(R):
    for D in (100, 4096, 20000):
        x, dy, w, b = make(12, D, BF, BF, seed=9)
        clean = [t.clone() for t in R.rl_layer_norm_fwd(x, weight=w, bias=b)]
        mask = torch.ones(12, dtype=torch.uint8, device="cuda")
        mask[3] = 0
        ws = R.new_layer_norm_workspace(12, D)

        def back():
            dw = torch.zeros(D, device="cuda")
            return R.rl_layer_norm_bwd(dy, x, clean[1], clean[2], ws, weight=w, mask=mask, d_weight=dw), dw

        x[3, D // 2] = float("nan")
        dy[3] = float("inf")
        y, mean, rstd = R.rl_layer_norm_fwd(x, weight=w, bias=b)
        keep = [i for i in range(12) if i != 3]
        assert torch.isnan(y[3]).all()
        assert all(torch.equal(a[keep], c[keep]) for a, c in zip((y, mean, rstd), clean))
        # a masked row's d_y and x are not looked at
        dx, dw = back()
        assert torch.isfinite(dx).all() and torch.isfinite(dw).all() and (dx[3] == 0).all()
        # a row that is not masked makes the columns' sums NaN, and no other row
        x[5, 0] = float("nan")
        bad, bad_w = back()
        assert torch.isnan(bad_w).any() and torch.isnan(bad[5]).any()
        others = [i for i in range(12) if i != 5]
        assert torch.equal(bad[others], dx[others])


@pytest.mark.parametrize("rows,D", [(50, 256), (33, 1001), (70, 4096), (9, 12000)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_place(R, rows, D, dtype):
    x, dy, w, b = make(rows, D, dtype, dtype, seed=11)
    y, mean, rstd = R.rl_layer_norm_fwd(x, weight=w, bias=b)
    z = x.clone()
    R.rl_layer_norm_fwd(z, weight=w, bias=b, y=z)
    assert torch.equal(z, y)
    ws = R.new_layer_norm_workspace(rows, D)
    dws = [torch.zeros(D, device="cuda") for _ in range(3)]
    dx = R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w, d_weight=dws[0])
    over_dy, over_x = dy.clone(), x.clone()
    R.rl_layer_norm_bwd(over_dy, x, mean, rstd, ws, weight=w, d_x=over_dy, d_weight=dws[1])
    R.rl_layer_norm_bwd(dy, over_x, mean, rstd, ws, weight=w, d_x=over_x, d_weight=dws[2])
    assert torch.equal(over_dy, dx) and torch.equal(over_x, dx)
    assert torch.equal(dws[1], dws[0]) and torch.equal(dws[2], dws[0])


def test_masks_that_leave_nothing_and_no_outputs(R):
    for rows, D in ((100, 512), (40, 4096), (7, 9001)):
        x, dy, w, _ = make(rows, D, BF, BF, seed=3)
        _, mean, rstd = R.rl_layer_norm_fwd(x, weight=w)
        ws = R.new_layer_norm_workspace(rows, D)
        dw = torch.full((D,), 2.5, device="cuda")
        none = torch.zeros(rows, dtype=torch.uint8, device="cuda")
        dx = R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w, mask=none, d_weight=dw)
        assert (dx == 0).all() and (dw == 2.5).all()
        # without the columns' sums the rows' gradient is the same
        a = R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w, d_weight=dw)
        assert torch.equal(a, R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w))
    empty = torch.empty(0, 64, device="cuda")
    y, mean, rstd = R.rl_layer_norm_fwd(empty)
    assert y.shape == (0, 64) and R.rl_layer_norm_bwd(empty, empty, mean, rstd, R.new_layer_norm_workspace(0, 64)).numel() == 0


def test_the_gradient_agrees_with_differences(R):
    """sum(y dy) at x + t d and x - t d, in float64, against dx . d: the differences' error is of order t^2."""
    x, dy, w, b = make(5, 300, F32, F32, seed=21)
    _, mean, rstd = R.rl_layer_norm_fwd(x, weight=w, bias=b)
    ws = R.new_layer_norm_workspace(5, 300)
    dw, db = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    dx = np64(R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w, d_weight=dw, d_bias=db))
    x64, dy64, w64, b64 = (np64(t) for t in (x, dy, w, b))
    rng = np.random.default_rng(1)

    def value(dx_, dw_, db_):
        return float((O.layer_norm(x64 + dx_, w64 + dw_, b64 + db_)[0] * dy64).sum())

    for _ in range(5):
        d, e, f = rng.normal(size=x64.shape), rng.normal(size=300), rng.normal(size=300)
        t = 1e-5
        diff = (value(t * d, t * e, t * f) - value(-t * d, -t * e, -t * f)) / (2 * t)
        parts = [dx * d, np64(dw) * e, np64(db) * f]
        ours = sum(float(p.sum()) for p in parts)
        # fp32's roundings over at most 1,500 terms, and the differences' own (their values are about 1)
        assert abs(diff - ours) <= 1e-5 * sum(float(np.abs(p).sum()) for p in parts) + 1e-9


def test_repeats_streams_and_graphs(R):
    rows, D = 777, 1024
    x, dy, w, b = make(rows, D, BF, BF, seed=8)
    ws = R.new_layer_norm_workspace(rows, D)

    def both(ws, dw):
        y, mean, rstd = R.rl_layer_norm_fwd(x, weight=w, bias=b)
        return y, R.rl_layer_norm_bwd(dy, x, mean, rstd, ws, weight=w, d_weight=dw), dw

    first = both(ws, torch.zeros(D, device="cuda"))
    side = torch.cuda.Stream()
    ws2 = R.new_layer_norm_workspace(rows, D)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        second = both(ws2, torch.zeros(D, device="cuda"))
    third = both(ws, torch.zeros(D, device="cuda"))
    torch.cuda.synchronize()
    for got in (second, third):
        assert all(torch.equal(a, c) for a, c in zip(first, got))
    graph = torch.cuda.CUDAGraph()
    dw = torch.zeros(D, device="cuda")
    with torch.cuda.graph(graph):
        y, dx, _ = both(ws, dw)
    for _ in range(2):
        dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(first, (y, dx, dw)))


@pytest.mark.parametrize("rows,D", [(6, 100), (6, 1000), (900, 4096), (2000, 4097), (5, 9001)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_beyond_the_range(R, rows, D, dtype):
    """Squares beyond fp32's range: rstd is 0 and the row comes out as the bias; a sum beyond it: NaN. The rows beside stay."""
    x, _, w, b = make(rows, D, dtype, F32, seed=31)
    clean = [t.clone() for t in R.rl_layer_norm_fwd(x, weight=w, bias=b, y_dtype=F32)]
    x[1] = torch.where(torch.arange(D, device="cuda") % 2 == 0, 1e25, -2e25).to(dtype)
    x[3] = 3e38
    y, mean, rstd = R.rl_layer_norm_fwd(x, weight=w, bias=b, y_dtype=F32)
    assert torch.equal(y[1], b) and float(rstd[1]) == 0.0 and torch.isfinite(mean[1])
    assert torch.isnan(y[3]).all()
    keep = [i for i in range(rows) if i not in (1, 3)]
    assert all(torch.equal(a[keep], c[keep]) for a, c in zip((y, mean, rstd), clean))
