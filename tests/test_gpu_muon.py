"""rl_muon_update against its float64 reference.

Tolerances, fixed before the first run: the products read fp16 operands, and an emulation of the scheme
(fp16 roundings of the operands, fp32 X and diagonals) over random, low-rank and decaying matrices stays
below 1.1e-3 of X in 2-norm and 1e-2 of its root mean square in any element; twice that is allowed,
2^-9 in 2-norm and 2^-8 of an element more for the rounding to bf16. Momentum is one fp32 fused
multiply-add (2^-24 of its two terms); weights are three fp32 roundings and lr s times the error of X.
"""

import numpy as np
import pytest
import torch

import oracle.orthogonal_update as O

pytestmark = pytest.mark.gpu

NS_REL, NS_MAX = 2.2e-3, 2e-2


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


def matrices(law, batch, m, n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(batch, m, n, generator=g)
    r = min(8, m, n)
    u, v = torch.randn(batch, m, r, generator=g), torch.randn(batch, r, n, generator=g)
    if law == "low_rank":
        x = (u / torch.arange(1, r + 1)) @ v + 0.02 * x
    elif law == "one_direction":
        x = u[:, :, :1] @ v[:, :1] + 1e-3 * x
    elif law == "zero_rows":
        x[:, ::3] = 0
    return x


def check_x(got, ref, what, bf16):
    got, ref = got.double().cpu().numpy(), np.asarray(ref)
    assert np.isfinite(got).all(), what
    for b in range(len(ref)):
        norm = np.linalg.norm(ref[b])
        d = got[b] - ref[b]
        rms = norm / np.sqrt(ref[b].size)
        assert np.linalg.norm(d) <= (NS_REL + (2.0 ** -9 if bf16 else 0.0)) * norm, (what, b, np.linalg.norm(d) / norm)
        assert (np.abs(d) <= NS_MAX * rms + (2.0 ** -8 * np.abs(ref[b]) if bf16 else 0.0)).all(), (what, b)


SHAPES = [(1, 1, 1), (1, 1, 7), (1, 7, 1), (2, 5, 3), (1, 64, 64), (1, 128, 128), (1, 127, 129), (3, 129, 127),
          (2, 130, 300), (2, 300, 130), (5, 33, 1000), (1, 1000, 33), (1, 257, 1025), (1, 640, 384), (1, 128, 9000),
          (1, 9001, 100), (12, 256, 256), (1, 1000, 1777), (1, 2305, 2049), (1, 1024, 5000)]


@pytest.mark.parametrize("batch,m,n", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_update(R, batch, m, n, dtype):
    law = ["low_rank", "normal"][(m + n) % 2]
    grad = matrices(law, batch, m, n, 1).to(dtype)
    mom = matrices(law, batch, m, n, 2) * 3
    buf, _, upd, _ = O.muon_update(grad.double().numpy(), mom.numpy(), update_scale=0.5)
    ws = R.new_muon_workspace(batch, m, n)
    d_mom = mom.cuda()
    got = R.rl_muon_update(grad.cuda(), R.make_muon_params(update_scale=0.5), ws, momentum=d_mom)
    assert R.rl_query_status(ws)[1] == 0
    check_x(got, upd, "update", True)
    tol = 2.0 ** -23 * (np.abs(mom.double().numpy()) + np.abs(grad.double().numpy()))
    assert (np.abs(d_mom.cpu().double().numpy() - buf) <= tol + 1e-30).all()


@pytest.mark.parametrize("law", ["normal", "low_rank", "one_direction", "zero_rows"])
@pytest.mark.parametrize("m,n", [(192, 320), (320, 192), (512, 512), (96, 4096)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_weights(R, law, m, n, nesterov):
    batch, lr, scale, wd = 2, 0.05, 0.7, 0.1
    grad, mom, w = (matrices(law, batch, m, n, 3), matrices(law, batch, m, n, 4), matrices("normal", batch, m, n, 5))
    _, X, _, w_ref = O.muon_update(grad.numpy(), mom.numpy(), w.numpy(), lr=lr, nesterov=nesterov, weight_decay=wd,
                                   update_scale=scale)
    ws = R.new_muon_workspace(batch, m, n)
    P = R.make_muon_params(lr=lr, nesterov=nesterov, weight_decay=wd, update_scale=scale)
    # weights in a wider buffer; what lies between the rows stays
    wide = torch.full((batch, m, n + 3), 7.0, device="cuda")
    wide16 = torch.full((batch, m, n + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :, :n] = w.cuda()
    out = R.rl_muon_update(grad.cuda(), P, ws, momentum=mom.cuda(), weights=wide[:, :, :n], weights_bf16=wide16[:, :, :n])
    assert out is None and R.rl_query_status(ws)[1] == 0
    got = wide[:, :, :n].cpu()
    for b in range(batch):
        err = np.linalg.norm(got[b].double().numpy() - w_ref[b])
        assert err <= lr * scale * NS_REL * np.linalg.norm(X[b]) + 4 * 2.0 ** -24 * np.linalg.norm(w_ref[b])
    assert torch.equal(wide16[:, :, :n].cpu(), got.bfloat16())
    assert (wide[:, :, n:] == 7).all() and (wide16[:, :, n:] == 7).all()


def test_interleaved_batch(R):
    """A batch whose rows alternate in memory ([m, batch, n]), for the gradient and for the weights."""
    batch, m, n = 3, 70, 90
    grad, w = matrices("normal", batch, m, n, 6), matrices("normal", batch, m, n, 7)
    P = R.make_muon_params(lr=0.1, momentum=0.0)
    ws = R.new_muon_workspace(batch, m, n)
    plain = w.cuda()
    R.rl_muon_update(grad.cuda(), P, ws, weights=plain)
    g2, w2 = grad.cuda().transpose(0, 1).contiguous(), w.cuda().transpose(0, 1).contiguous()
    R.rl_muon_update(g2.transpose(0, 1), P, ws, weights=w2.transpose(0, 1))
    assert torch.equal(w2.transpose(0, 1), plain)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-20, 1e20, 1e30, 1e37])
@pytest.mark.parametrize("m,n", [(100, 180), (180, 100)])
def test_scale_of_the_gradient(R, scale, m, n):
    """The norm neither overflows nor underflows fp32 (eps is 0 here)."""
    g = (matrices("normal", 1, m, n, 8).double() * scale).float()
    ref = O.newton_schulz(g[0].double().numpy(), eps=0.0)
    ws = R.new_muon_workspace(1, m, n)
    got = R.rl_muon_update(g.cuda(), R.make_muon_params(momentum=0.0, eps=0.0), ws)
    assert R.rl_query_status(ws)[1] == 0
    check_x(got, ref[None], "update", True)


def test_zero_and_non_finite(R):
    batch, m, n = 4, 150, 90
    g = matrices("normal", batch, m, n, 9)
    g[1] = 0
    g[2, 17, 3] = float("nan")
    g[3, 0, 89] = float("inf")
    ws = R.new_muon_workspace(batch, m, n)
    got = R.rl_muon_update(g.cuda(), R.make_muon_params(momentum=0.0), ws)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_VALUE
    check_x(got[:1], O.newton_schulz(g[0].numpy())[None], "update", True)
    assert not got[1].any()
    assert got[2].isnan().all() and got[3].isnan().all()
    # the workspace serves the next call after its status is cleared
    R.rl_workspace_init(ws)
    again = R.rl_muon_update(g[:1].expand(batch, m, n).cuda(), R.make_muon_params(momentum=0.0), ws)
    assert R.rl_query_status(ws)[1] == 0
    assert all(torch.equal(again[k], got[0]) for k in range(batch))


@pytest.mark.parametrize("steps,coef", [(1, O.NS_COEF), (2, (1.5, -0.5, 0.0)), (10, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))])
def test_steps_and_coefficients(R, steps, coef):
    g = matrices("normal", 1, 200, 260, 10)
    ref = O.newton_schulz(g[0].numpy(), steps, coef)
    ws = R.new_muon_workspace(1, 200, 260)
    got = R.rl_muon_update(g.cuda(), R.make_muon_params(momentum=0.0, ns_steps=steps, ns_coef=coef), ws)
    check_x(got, ref[None], "update", True)


@pytest.mark.parametrize("batch,m,n", [(1, 300, 500), (1, 128, 9000), (1, 1500, 1500)])
def test_repeats_streams_and_graphs(R, batch, m, n):
    """The same bits again, on another stream, and from a graph; no workspace contents are relied on."""
    g = matrices("low_rank", batch, m, n, 11).cuda()
    P = R.make_muon_params(momentum=0.5)
    ws = R.new_muon_workspace(batch, m, n)
    first = R.rl_muon_update(g, P, ws, momentum=torch.zeros_like(g))
    ws2 = torch.full_like(ws, 255)
    R.rl_workspace_init(ws2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = R.rl_muon_update(g, P, ws2, momentum=torch.zeros_like(g))
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, second)
    mom, upd = torch.zeros_like(g), torch.empty_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.rl_muon_update(g, P, ws, momentum=mom, update=upd)
    for _ in range(2):
        mom.zero_()
        upd.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, upd)
    assert R.rl_query_status(ws)[1] == 0 and R.rl_query_status(ws2)[1] == 0


def test_binding_refusals(R):
    g = torch.zeros(8, 16, device="cuda")
    ws = R.new_muon_workspace(1, 8, 16)
    P = R.make_muon_params(momentum=0.0)
    for bad in (dict(weights=torch.zeros(8, 15, device="cuda")), dict(weights=torch.zeros(16, 8, device="cuda").T),
                dict(weights=torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda")),
                dict(update=torch.zeros(8, 16, device="cuda")), dict(momentum=torch.zeros(8, 8, device="cuda")),
                dict(weights=torch.zeros(8, 16, device="cuda"),
                     weights_bf16=torch.zeros(8, 32, dtype=torch.bfloat16, device="cuda")[:, ::2])):
        with pytest.raises(ValueError):
            R.rl_muon_update(g, P, ws, **bad)
    for bad in (g.half(), g.T, g[None, None], g.cpu()):
        with pytest.raises((ValueError, R.RLError)):
            R.rl_muon_update(bad, P, ws)
    with pytest.raises(R.RLError):
        R.rl_muon_update(g, P, ws[:512])
    with pytest.raises(R.RLError):
        R.new_muon_workspace(1, 40000, 40000)


@pytest.mark.parametrize("batch,m,n,pad", [(3, 96, 132, 0), (2, 132, 96, 4), (2, 260, 100, 8), (1, 301, 404, 12),
                                           (2, 404, 301, 3), (1, 66, 130, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_and_off_multiples_of_four(R, batch, m, n, pad, dtype):
    """Vectors of four elements and single ones: gradient, momentum, weights and update by both ways."""
    grad = matrices("low_rank", batch, m, n, 12).to(dtype)
    mom, w = matrices("low_rank", batch, m, n, 13), matrices("normal", batch, m, n, 14)
    P = R.make_muon_params(lr=0.1, momentum=0.9, update_scale=0.3, weight_decay=0.5)
    ws = R.new_muon_workspace(batch, m, n)
    buf, X, upd, w_ref = O.muon_update(grad.double().numpy(), mom.numpy(), w.numpy(), lr=0.1, mu=0.9, update_scale=0.3,
                                       weight_decay=0.5)
    results = []
    for shift in (0, 1):  # elements by which everything starts off its alignment
        def place(x, width, dt):
            t = torch.full((batch * m * width + shift,), 5.0, dtype=dt, device="cuda")[shift:].view(batch, m, width)
            t[:, :, :n] = x.cuda()
            return t
        g, d_w = place(grad, n + pad, dtype)[:, :, :n], place(w, n + pad, torch.float32)
        d_m, d_u = place(mom, n, torch.float32), place(torch.zeros(batch, m, n), n, torch.bfloat16)
        d_b = place(torch.zeros(batch, m, n), n + pad, torch.bfloat16)
        R.rl_muon_update(g, P, ws, momentum=d_m, weights=d_w[:, :, :n], weights_bf16=d_b[:, :, :n], update=d_u)
        assert R.rl_query_status(ws)[1] == 0
        check_x(d_u, upd, "update", True)
        tol = 2.0 ** -23 * (np.abs(mom.double().numpy()) + np.abs(grad.double().numpy()))
        assert (np.abs(d_m.cpu().double().numpy() - buf) <= tol + 1e-30).all()
        for b in range(batch):
            err = np.linalg.norm(d_w[b, :, :n].cpu().double().numpy() - w_ref[b])
            assert err <= 0.1 * 0.3 * NS_REL * np.linalg.norm(X[b]) + 4 * 2.0 ** -24 * np.linalg.norm(w_ref[b])
        assert torch.equal(d_b[:, :, :n], d_w[:, :, :n].bfloat16())
        assert (d_w[:, :, n:] == 5).all() and (d_b[:, :, n:] == 5).all()
        results.append([x.clone() for x in (d_m, d_w, d_b, d_u)])
    # both ways round alike, but for the order in which the norm's squares are added
    for a, b in zip(*results):
        assert (a.float() - b.float()).norm() <= 1e-3 * a.float().norm()


def test_strides_of_a_single_row(R):
    """A weight of one row cut out of a wider buffer, its copy contiguous: the row's own stride says nothing."""
    for batch in (1, 3):
        g, w = matrices("normal", batch, 1, 40, 15).cuda(), matrices("normal", batch, 1, 40, 16).cuda()
        P = R.make_muon_params(lr=0.1, momentum=0.0)
        ws = R.new_muon_workspace(batch, 1, 40)
        plain = w.clone()
        R.rl_muon_update(g, P, ws, weights=plain)
        wide = torch.full((batch, 5, 8), 7.0, device="cuda")
        cut = wide.as_strided((batch, 1, 40), (40, 64, 1))
        cut.copy_(w)
        copy = torch.empty(batch, 1, 40, dtype=torch.bfloat16, device="cuda")
        R.rl_muon_update(g, P, ws, weights=cut, weights_bf16=copy)
        assert torch.equal(cut, plain) and torch.equal(copy, plain.bfloat16())


# One or two directions and noise: directions in which the matrix is small, or 0, grow by a per step, and whatever the
# operands' roundings put there with them. Emulated as the file's bounds (these shapes, noises, three seeds): at most
# 2.0e-3 in 2-norm after 3 and 5 steps, 3.8e-3 after 8, and 3.1e-2 of the root mean square in an element; twice that is
# allowed.
FEW_DIRECTIONS = {3: 4e-3, 5: 4e-3, 8: 7.6e-3}


@pytest.mark.parametrize("m,n", [(8, 64), (16, 16), (16, 8000), (8000, 16), (64, 8000), (192, 3000), (256, 256), (300, 700)])
@pytest.mark.parametrize("directions", [1, 2])
@pytest.mark.parametrize("steps", [3, 5, 8])
def test_few_directions(R, m, n, directions, steps):
    ws = R.new_muon_workspace(1, m, n)
    for noise in (1e-1, 1e-3, 1e-5, 0.0):
        g = torch.Generator().manual_seed(17)
        x = torch.randn(m, directions, generator=g) @ torch.randn(directions, n, generator=g)
        x = x + noise * torch.randn(m, n, generator=g)
        ref = O.newton_schulz(x.numpy(), steps)
        norm = np.linalg.norm(ref)
        w = torch.zeros(m, n, device="cuda")
        update = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
        R.rl_muon_update(x.cuda(), R.make_muon_params(lr=-1.0, momentum=0.0, ns_steps=steps), ws, weights=w, update=update)
        assert R.rl_query_status(ws)[1] == 0
        for got, bf16 in ((w, 0.0), (update, 1.0)):
            d = got.double().cpu().numpy() - ref
            assert np.linalg.norm(d) <= (FEW_DIRECTIONS[steps] + bf16 * 2.0 ** -9) * norm, (noise, np.linalg.norm(d) / norm)
            assert (np.abs(d) <= 6.2e-2 * norm / np.sqrt(m * n) + bf16 * 2.0 ** -8 * np.abs(ref)).all(), noise


# Sides above 256: not the kernel that takes a whole matrix. Singles and pairs of CTAs, a padded short side that is an odd
# multiple of 128 (a pair's tile then holds rows of the next matrix), a contraction in parts.
TILED = [(4, 300, 700), (3, 700, 300), (20, 640, 900), (5, 1400, 1150), (3, 640, 6000), (4, 128, 9000)]


@pytest.mark.parametrize("batch,m,n", TILED)
def test_zero_and_non_finite_in_tiles(R, batch, m, n):
    """A NaN or an infinity fills its own matrix and no other; a zero matrix stays zero, also without eps."""
    g = matrices("normal", batch, m, n, 18)
    P, ws = R.make_muon_params(momentum=0.0, eps=0.0), R.new_muon_workspace(batch, m, n)
    clean = R.rl_muon_update(g.cuda(), P, ws)
    assert R.rl_query_status(ws)[1] == 0
    check_x(clean[:1], O.newton_schulz(g[0].numpy(), eps=0.0)[None], "update", True)
    for value in (float("nan"), float("inf"), -float("inf")):
        hurt = g.clone()
        hurt[1, m - 1, 3] = value
        hurt[2] = 0
        got = R.rl_muon_update(hurt.cuda(), P, ws)
        assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_VALUE
        assert got[1].isnan().all() and not got[2].any()
        for b in range(batch):
            assert b in (1, 2) or torch.equal(got[b], clean[b]), b
        R.rl_workspace_init(ws)
    again = R.rl_muon_update(g.cuda(), P, ws)
    assert R.rl_query_status(ws)[1] == 0 and torch.equal(again, clean)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-20, 1e20, 1e30, 1e37])
@pytest.mark.parametrize("m,n", [(300, 520), (520, 300), (100, 5000)])
def test_scale_of_the_gradient_in_tiles(R, scale, m, n):
    """As test_scale_of_the_gradient, with sides above 256."""
    g = (matrices("normal", 1, m, n, 19).double() * scale).float()
    ws = R.new_muon_workspace(1, m, n)
    got = R.rl_muon_update(g.cuda(), R.make_muon_params(momentum=0.0, eps=0.0), ws)
    assert R.rl_query_status(ws)[1] == 0
    check_x(got, O.newton_schulz(g[0].double().numpy(), eps=0.0)[None], "update", True)


@pytest.mark.parametrize("batch,m,n", [(3, 300, 520), (2, 520, 300), (4, 128, 900)])
def test_interleaved_batch_in_tiles(R, batch, m, n):
    """As test_interleaved_batch, with sides above 256, a momentum and a bf16 copy."""
    grad, w, mom = (matrices("normal", batch, m, n, k).cuda() for k in (20, 21, 22))
    P = R.make_muon_params(lr=0.1, weight_decay=0.1)
    ws = R.new_muon_workspace(batch, m, n)
    plain, copy, plain_mom = w.clone(), torch.zeros_like(w, dtype=torch.bfloat16), mom.clone()
    R.rl_muon_update(grad, P, ws, momentum=plain_mom, weights=plain, weights_bf16=copy)
    g2, w2 = grad.transpose(0, 1).contiguous(), w.transpose(0, 1).contiguous()
    copy2, mom2 = torch.zeros_like(w2, dtype=torch.bfloat16), mom.clone()
    R.rl_muon_update(g2.transpose(0, 1), P, ws, momentum=mom2, weights=w2.transpose(0, 1), weights_bf16=copy2.transpose(0, 1))
    assert torch.equal(w2.transpose(0, 1), plain) and torch.equal(copy2.transpose(0, 1), copy)
    assert torch.equal(mom2, plain_mom) and torch.equal(copy, plain.bfloat16())


def known(m, n, seed):
    """(G, X) in float64 on the GPU: G = U S R with U of orthonormal columns (cosines, rows with random signs), R of three
    reflections and decaying singular values, and X after five steps, from those alone."""
    l, s = max(m, n), min(m, n)
    g = torch.Generator(device="cuda").manual_seed(seed)
    f64 = dict(dtype=torch.float64, device="cuda")
    k = torch.arange(s, **f64)
    u = torch.cos((torch.arange(l, **f64) + 0.5)[:, None] * (k * (np.pi / l)))
    u.mul_(torch.where(k == 0, 1.0, 2.0 ** 0.5) / l ** 0.5)
    u.mul_(torch.randint(0, 2, (l, 1), generator=g, device="cuda").double() * 2 - 1)
    sigma = 1 / (1 + k / 8)
    x = sigma / (sigma.norm() + float(np.float32(1e-7)))
    a, b, c = (float(np.float32(t)) for t in O.NS_COEF)
    for _ in range(5):
        x = a * x + b * x ** 3 + c * x ** 5
    grad, ref = u * sigma, u.mul_(x)
    for _ in range(3):
        v = torch.randn(s, generator=g, **f64)
        v /= v.norm()
        for t in (grad, ref):
            t.addr_(t @ v, v, alpha=-2.0)
    return (grad, ref) if m > n else (grad.T.contiguous(), ref.T.contiguous())


@pytest.mark.parametrize("m,n", [(300, 520), (4500, 4600), (151936, 4096), (4096, 20000)])
def test_large_matrices(R, m, n):
    """Sides above 4,096, more tiles per CTA pair than accumulators, and the fused head's d_weight at V = 151,936, D = 4,096.
    To the bound of the roundings comes one unit of fp32 per 16 elements of the longest contraction."""
    grad, ref = known(m, n, 23)
    grad = grad.float()
    ws = R.new_muon_workspace(1, m, n)
    w = torch.zeros(m, n, device="cuda")
    copy = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    update = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    R.rl_muon_update(grad, R.make_muon_params(lr=-1.0, momentum=0.0), ws, weights=w, weights_bf16=copy, update=update)
    assert R.rl_query_status(ws)[1] == 0
    assert torch.equal(copy, w.bfloat16()) and torch.equal(update, copy)
    norm, tol = ref.norm(), NS_REL + max(m, n) / 16 * 2.0 ** -23
    d = ref.sub_(w)
    assert d.norm() <= tol * norm, (d.norm() / norm).item()
    assert d.abs_().max() <= (NS_MAX + tol) * norm / (m * n) ** 0.5
    del grad, ref, d, w, copy, update, ws
    torch.cuda.empty_cache()
