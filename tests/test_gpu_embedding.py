"""rl_embedding_fwd and rl_embedding_bwd against their float64 reference.

Tolerances, fixed before the first run: a product is rounded once to fp32 and once to the output's type (half a step each).
A gradient's sum of n terms has at most n additions on any term's way, its product with the scale and its addition to what
was there one rounding each: (n + 2) 2^-24 of the sum of the terms' sizes, and 2^-24 of the result and of what was there.
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


def np64(t):
    return t.detach().double().cpu().numpy()


def token_ids(law, T, V, seed):
    rng = np.random.default_rng(seed)
    if law == "same":
        return np.full(T, V // 2)
    if law == "two":
        return np.where(rng.random(T) < 0.5, 0, V - 1)
    if law == "all_once":
        return rng.permutation(max(T, V))[:T] % V
    if law == "often":  # frequencies fall with the rank
        return np.minimum((V ** rng.random(T)).astype(np.int64) - 1, V - 1)
    return rng.integers(0, V, T)


def ids_on_device(ids):
    return torch.from_numpy(ids.astype(np.int32)).cuda()


@pytest.mark.parametrize("T,D,V", [(1, 1, 1), (3, 8, 5), (9, 64, 10), (100, 100, 77), (33, 1000, 513), (500, 1024, 1000),
                                   (7, 4096, 151936), (2, 8200, 30), (1000, 24, 3)])
@pytest.mark.parametrize("types", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
def test_forward(R, T, D, V, types):
    rng = np.random.default_rng(T + D)
    ids = rng.integers(0, V, T)
    ws = R.new_workspace(0, 0)
    for pad, off in ((0, 0), (8, 0), (3, 1)):
        w = torch.empty(V * (D + pad) + off, dtype=types[0], device="cuda")[off:].view(V, D + pad)[:, :D]
        w.copy_(torch.from_numpy(rng.normal(size=(V, D))))
        buf = torch.full((T * (D + pad) + off,), 7.0, dtype=types[1], device="cuda")
        out = buf[off:].view(T, D + pad)[:, :D]
        R.rl_embedding_fwd(ids_on_device(ids), w, ws, scale=1.7, out=out)
        ref = O.embedding(ids, np64(w), 1.7)
        step = 2.0 ** -8 if types[1] == BF else 0.0
        assert (np.abs(np64(out) - ref) <= (step + U) * (1 + 1e-3) * np.abs(ref)).all(), (pad, off)
        assert (buf[off:].view(T, D + pad)[:, D:] == 7).all() and (buf[:off] == 7).all()
    assert R.rl_query_status(ws)[1] == 0


def check_grad(R, ids, V, D, dtype, what, scale=0.9, pad=0, off=0, seed=0, ws=None):
    T = len(ids)
    g = torch.Generator().manual_seed(seed)
    d = torch.full((T * (D + pad) + off,), float("nan"), dtype=dtype, device="cuda")[off:].view(T, D + pad)[:, :D]
    d.copy_(torch.randn(T, D, generator=g) * 1e-2)
    dw = torch.randn(V, D, generator=g).cuda()
    before = np64(dw)
    keep = dw.clone()
    ws = R.new_embedding_workspace(T, V, D) if ws is None else ws
    R.rl_embedding_bwd(ids_on_device(ids), d, dw, ws, scale=scale)
    ref, size = O.embedding_grad(ids, np64(d), V, scale)
    counts = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
    tol = (counts + 2) * U * size + U * (np.abs(before) + np.abs(ref)) * (1 + 1e-3)
    err = np.abs(np64(dw) - before - ref)
    assert (err <= tol * (1 + 1e-3)).all(), (what, float(np.max(err / np.maximum(tol, 1e-300))))
    untouched = torch.from_numpy(counts[:, 0] == 0).cuda()
    assert torch.equal(dw[untouched], keep[untouched]), what
    return d, dw


@pytest.mark.parametrize("law", ["same", "two", "all_once", "often", "any"])
@pytest.mark.parametrize("T,D,V", [(1, 8, 4), (2, 1, 1), (15, 33, 7), (16, 64, 40), (17, 128, 600), (64, 100, 5),
                                   (1000, 96, 1000), (1024, 256, 32000), (1025, 40, 511), (4096, 64, 512),
                                   (5000, 72, 151936), (5001, 17, 513), (33000, 16, 9000), (70001, 24, 300000), (180224, 8, 40000),
                                   (180225, 8, 40000)])
def test_backward(R, law, T, D, V):
    ids = token_ids(law, T, V, seed=T)
    for dtype in (BF, F32):
        check_grad(R, ids, V, D, dtype, (law, T, D, V, dtype))


@pytest.mark.parametrize("D", [1, 3, 8, 60, 129, 512, 513, 1024, 1500, 4096, 5000])
def test_backward_widths_and_strides(R, D):
    ids = token_ids("often", 700, 60, seed=D)
    for dtype in (BF, F32):
        for pad, off in ((0, 0), (8, 0), (1, 0), (5, 1)):
            check_grad(R, ids, 60, D, dtype, (D, dtype, pad, off), pad=pad, off=off)


@pytest.mark.parametrize("T,D", [(1025, 1024), (3000, 129), (3000, 513), (3000, 1024), (3000, 4096), (3000, 5000), (9001, 1001),
                                 (9001, 2048), (70001, 129), (70001, 520), (180300, 136)])
@pytest.mark.parametrize("law", ["same", "two", "often", "any"])
def test_backward_of_sorted_tokens_over_many_columns(R, law, T, D):
    """Rows that several CTAs share, whose runs of equal ids are cut at the chunks' borders: the parts and the list of the long
    runs are of all columns. The reference is summed in float64 on the GPU; every tenth id is out of range."""
    V = 60
    ids = ids_on_device(token_ids(law, T, V, seed=T + D))
    ids[5::10] = torch.where(torch.arange(len(ids[5::10]), device="cuda") % 2 == 0, -1, V).int()
    ok = (ids >= 0) & (ids < V)
    g = torch.Generator(device="cuda").manual_seed(D)
    ws = R.new_embedding_workspace(T, V, D)
    for dtype in (BF, F32):
        values = (torch.randn(T, D, generator=g, device="cuda") * 1e-2).to(dtype)
        before = torch.randn(V, D, generator=g, device="cuda")
        # the formula, and the sum of the terms' sizes
        ref, size = torch.zeros(2, V, D, dtype=torch.float64, device="cuda")
        terms = values[ok].double() * float(np.float32(0.9))
        ref.index_add_(0, ids[ok].long(), terms)
        size.index_add_(0, ids[ok].long(), terms.abs())
        del terms
        n = torch.bincount(ids[ok].long(), minlength=V)[:, None]
        tol = (n + 2) * U * size + U * (before.double().abs() + ref.abs())
        for pad, off in ((0, 0), (8, 0), (3, 0), (5, 1)):
            buf = torch.full((T * (D + pad) + off,), float("nan"), dtype=dtype, device="cuda")
            d = buf[off:].view(T, D + pad)[:, :D]
            d.copy_(values)
            d[~ok] = float("nan")  # not read
            dw = before.clone()
            R.rl_embedding_bwd(ids, d, dw, ws, scale=0.9)
            err = (dw.double() - before.double() - ref).abs()
            assert bool((err <= tol * (1 + 1e-3)).all()), (law, T, D, dtype, pad, off, float((err / tol.clamp(min=1e-300)).max()))
            assert torch.equal(dw[n[:, 0] == 0], before[n[:, 0] == 0])
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN


def test_ids_out_of_range(R):
    V, D = 50, 64
    for T in (20, 3000):
        ids = token_ids("any", T, V, seed=2)
        ids[3], ids[7], ids[-1] = -1, V, 2 ** 31 - 1
        ws = R.new_embedding_workspace(T, V, D)
        d = torch.randn(T, D, device="cuda")
        bad = torch.from_numpy((ids < 0) | (ids >= V)).cuda()
        d[bad] = float("nan")  # not read
        dw = torch.zeros(V, D, device="cuda")
        R.rl_embedding_bwd(ids_on_device(ids), d, dw, ws)
        assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN
        good = ids[(ids >= 0) & (ids < V)]
        ref, size = O.embedding_grad(good, np64(d[~bad]), V)
        assert (np.abs(np64(dw) - ref) <= (T + 2) * U * size).all()
        R.rl_workspace_init(ws)
        w = torch.randn(V, D, device="cuda")
        out = R.rl_embedding_fwd(ids_on_device(ids), w, ws)
        assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN
        assert (out[bad] == 0).all() and torch.equal(out[~bad], w[torch.from_numpy(good).cuda()])
        R.rl_workspace_init(ws)
    # many bad ids: their run is longer than any that one CTA adds up
    ids = token_ids("any", 5000, V, seed=3)
    ids[::2] = 2 ** 30
    ws = R.new_embedding_workspace(5000, V, D)
    d = torch.randn(5000, D, device="cuda")
    d[::2] = float("nan")
    dw = R.rl_embedding_bwd(ids_on_device(ids), d, torch.zeros(V, D, device="cuda"), ws)
    ref, size = O.embedding_grad(ids[1::2], np64(d[1::2]), V)
    assert (np.abs(np64(dw) - ref) <= 5000 * U * size).all()
    R.rl_workspace_init(ws)
    # nothing but bad ids
    ids = np.full(100, -5)
    dw = torch.ones(V, D, device="cuda")
    R.rl_embedding_bwd(ids_on_device(ids), torch.randn(100, D, device="cuda"), dw, ws)
    assert (dw == 1).all() and R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN


def test_no_tokens(R):
    w = torch.randn(5, 16, device="cuda")
    ws = R.new_embedding_workspace(0, 5, 16)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert R.rl_embedding_fwd(none, w, ws).shape == (0, 16)
    dw = w.clone()
    R.rl_embedding_bwd(none, torch.empty(0, 16, device="cuda"), dw, ws)
    assert torch.equal(dw, w)


def test_one_workspace_for_fewer_tokens(R):
    """A workspace of the most tokens serves every shorter call."""
    V, D = 300, 40
    ws = R.new_embedding_workspace(5000, V, D)
    for T in (5000, 4097, 4096, 1500, 1024, 1, 16, 3000):
        check_grad(R, token_ids("often", T, V, seed=T), V, D, BF, T, ws=ws)


def test_the_gradient_is_the_transpose(R):
    """sum(out e) = sum(W dW) for d_out = e: the lookup is linear in W."""
    T, V, D = 400, 90, 48
    ids = token_ids("often", T, V, seed=4)
    e = torch.randn(T, D, device="cuda")
    w = torch.randn(V, D, device="cuda")
    ws = R.new_embedding_workspace(T, V, D)
    out = R.rl_embedding_fwd(ids_on_device(ids), w, ws, scale=2.0)
    dw = R.rl_embedding_bwd(ids_on_device(ids), e, torch.zeros(V, D, device="cuda"), ws, scale=2.0)
    a, b = (np64(out) * np64(e)), (np64(w) * np64(dw))
    assert abs(a.sum() - b.sum()) <= (T + 4) * U * np.abs(a).sum()


def test_repeats_streams_and_graphs(R):
    for T, V, D in ((300, 64, 512), (9000, 700, 256)):
        ids = token_ids("often", T, V, seed=6)
        d, first = check_grad(R, ids, V, D, BF, "first")
        i = ids_on_device(ids)
        start = torch.randn(V, D, generator=torch.Generator().manual_seed(0))  # not what check_grad began with
        start = start.cuda()
        ws = R.new_embedding_workspace(T, V, D)
        once = R.rl_embedding_bwd(i, d, start.clone(), ws)
        side = torch.cuda.Stream()
        ws2 = R.new_embedding_workspace(T, V, D)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            other = R.rl_embedding_bwd(i, d, start.clone(), ws2)
        again = R.rl_embedding_bwd(i, d, start.clone(), ws)
        torch.cuda.synchronize()
        assert torch.equal(once, again) and torch.equal(once, other)
        graph = torch.cuda.CUDAGraph()
        dw = start.clone()
        with torch.cuda.graph(graph):
            R.rl_embedding_bwd(i, d, dw, ws)
        for _ in range(2):
            dw.copy_(start)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dw, once)
