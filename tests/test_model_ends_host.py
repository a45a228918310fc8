"""What rl_sample_tokens, the layer norm's and the embedding's calls refuse before any launch (no GPU needed), and the sizes of
their workspaces."""

import ctypes

import pytest

from paper_2608_16798_gb300 import build as B

FAKE = 0x10000  # never dereferenced: every call below fails validation first, or has nothing to do


@pytest.fixture(scope="module")
def R():
    B.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


def sample(R, **over):
    a = dict(z=FAKE, dt=R.RL_BF16, rows=2, V=8, ld=8, u=FAKE, params=R.make_sample_params(), rt=None, rk=None, rp=None, rm=None,
             ids=FAKE, logp=FAKE, among=None, kept=None, ws=FAKE, ws_bytes=256)
    a.update(over)
    P = a["params"]
    return R.lib().rl_sample_tokens(a["z"], a["dt"], a["rows"], a["V"], a["ld"], a["u"], None if P is None else ctypes.byref(P),
                                    a["rt"], a["rk"], a["rp"], a["rm"], a["ids"], a["logp"], a["among"], a["kept"], a["ws"],
                                    a["ws_bytes"], None)


@pytest.mark.parametrize("over,status", [
    (dict(dt=5), 1), (dict(rows=-1), 1), (dict(V=0), 1), (dict(ld=7), 1), (dict(params=None), 1), (dict(z=None), 1),
    (dict(u=None), 1), (dict(ids=None), 1), (dict(logp=None), 1), (dict(ws=None), 1), (dict(z=FAKE + 2), 3),
    (dict(ws=FAKE + 4), 3), (dict(V=(1 << 24) + 1, ld=1 << 25), 2), (dict(dt=1, V=(1 << 23) + 1, ld=1 << 24), 2),
    (dict(rows=(1 << 26) + 1), 2), (dict(ws_bytes=255), 4),
])
def test_sample_refusals(R, over, status):
    assert sample(R, **over) == status
    assert "rl_sample_tokens" in R.rl_last_error_message()


@pytest.mark.parametrize("kw", [dict(temperature=-1.0), dict(temperature=1e-5), dict(temperature=float("nan")),
                                dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.5),
                                dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.1), dict(min_p=float("nan"))])
def test_sample_refused_parameters(R, kw):
    assert sample(R, params=R.make_sample_params(**kw)) == 1


def norm_fwd(R, **over):
    a = dict(x=FAKE, xt=R.RL_BF16, rows=2, D=8, ld_x=8, w=FAKE, b=FAKE, wt=R.RL_F32, eps=1e-5, y=FAKE + 4096, yt=R.RL_BF16, ld_y=8,
             mean=FAKE, rstd=FAKE)
    a.update(over)
    return R.lib().rl_layer_norm_fwd(a["x"], a["xt"], a["rows"], a["D"], a["ld_x"], a["w"], a["b"], a["wt"], a["eps"], a["y"],
                                     a["yt"], a["ld_y"], a["mean"], a["rstd"], None)


@pytest.mark.parametrize("over,status", [
    (dict(xt=3), 1), (dict(yt=-1), 1), (dict(wt=2), 1), (dict(rows=-1), 1), (dict(D=0), 1), (dict(ld_x=7), 1), (dict(ld_y=7), 1),
    (dict(x=None), 1), (dict(y=None), 1), (dict(mean=None), 1), (dict(rstd=None), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(D=(1 << 20) + 1, ld_x=1 << 21, ld_y=1 << 21), 2),
    (dict(rows=1 << 38), 2), (dict(x=FAKE + 1), 3), (dict(y=FAKE + 1), 3), (dict(w=FAKE + 2), 3), (dict(b=FAKE + 1), 3),
    (dict(xt=1, x=FAKE + 2), 3), (dict(y=FAKE, yt=1), 1), (dict(y=FAKE, ld_y=16), 1),
])
def test_norm_forward_refusals(R, over, status):
    assert norm_fwd(R, **over) == status
    assert "rl_layer_norm_fwd" in R.rl_last_error_message()


def norm_bwd(R, **over):
    a = dict(dy=FAKE, dt=R.RL_BF16, ld_dy=8, x=FAKE + 4096, xt=R.RL_BF16, ld_x=8, rows=2, D=8, w=FAKE, wt=R.RL_F32, mean=FAKE,
             rstd=FAKE, mask=None, dx=FAKE + 8192, ld_dx=8, dw=FAKE, db=FAKE, ws=FAKE, ws_bytes=1 << 20)
    a.update(over)
    return R.lib().rl_layer_norm_bwd(a["dy"], a["dt"], a["ld_dy"], a["x"], a["xt"], a["ld_x"], a["rows"], a["D"], a["w"], a["wt"],
                                     a["mean"], a["rstd"], a["mask"], a["dx"], a["ld_dx"], a["dw"], a["db"], a["ws"],
                                     a["ws_bytes"], None)


@pytest.mark.parametrize("over,status", [
    (dict(dt=3), 1), (dict(xt=3), 1), (dict(wt=3), 1), (dict(rows=-1), 1), (dict(D=-4), 1), (dict(ld_dy=7), 1), (dict(ld_x=7), 1),
    (dict(ld_dx=7), 1), (dict(dy=None), 1), (dict(x=None), 1), (dict(dx=None), 1), (dict(mean=None), 1), (dict(rstd=None), 1),
    (dict(ws=None), 1), (dict(ws=FAKE + 8), 3), (dict(dy=FAKE + 1), 3), (dict(x=FAKE + 1), 3), (dict(dx=FAKE + 1), 3),
    (dict(dw=FAKE + 2), 3), (dict(db=FAKE + 1), 3), (dict(mean=FAKE + 1), 3), (dict(rstd=FAKE + 2), 3),
    (dict(dx=FAKE, ld_dx=16), 1), (dict(dx=FAKE, dt=1), 1), (dict(dx=FAKE + 4096, ld_dx=16), 1), (dict(ws_bytes=300), 4),
])
def test_norm_backward_refusals(R, over, status):
    assert norm_bwd(R, **over) == status
    assert "rl_layer_norm_bwd" in R.rl_last_error_message()


def embed_fwd(R, **over):
    a = dict(ids=FAKE, T=2, w=FAKE, wt=R.RL_BF16, V=9, D=8, ld_w=8, scale=1.0, out=FAKE, ot=R.RL_F32, ld_out=8, ws=FAKE,
             ws_bytes=256)
    a.update(over)
    return R.lib().rl_embedding_fwd(a["ids"], a["T"], a["w"], a["wt"], a["V"], a["D"], a["ld_w"], a["scale"], a["out"], a["ot"],
                                    a["ld_out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("over,status", [
    (dict(T=-1), 1), (dict(V=0), 1), (dict(D=0), 1), (dict(wt=4), 1), (dict(ot=4), 1), (dict(ld_w=7), 1), (dict(ld_out=7), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(ids=None), 1), (dict(w=None), 1), (dict(out=None), 1),
    (dict(ws=None), 1), (dict(ids=FAKE + 2), 3), (dict(w=FAKE + 1), 3), (dict(out=FAKE + 2), 3), (dict(ws=FAKE + 4), 3),
    (dict(T=(1 << 30) + 1), 2), (dict(V=1 << 31), 2), (dict(ws_bytes=16), 4),
])
def test_embedding_forward_refusals(R, over, status):
    assert embed_fwd(R, **over) == status
    assert "rl_embedding_fwd" in R.rl_last_error_message()


def embed_bwd(R, **over):
    a = dict(ids=FAKE, T=2, d=FAKE, dt=R.RL_BF16, ld_d=8, V=9, D=8, scale=1.0, dw=FAKE, ws=FAKE, ws_bytes=1 << 20)
    a.update(over)
    return R.lib().rl_embedding_bwd(a["ids"], a["T"], a["d"], a["dt"], a["ld_d"], a["V"], a["D"], a["scale"], a["dw"], a["ws"],
                                    a["ws_bytes"], None)


@pytest.mark.parametrize("over,status", [
    (dict(T=-1), 1), (dict(V=0), 1), (dict(D=0), 1), (dict(dt=4), 1), (dict(ld_d=7), 1), (dict(scale=float("nan")), 1),
    (dict(ids=None), 1), (dict(d=None), 1), (dict(dw=None), 1), (dict(ws=None), 1), (dict(ids=FAKE + 1), 3), (dict(d=FAKE + 1), 3),
    (dict(dw=FAKE + 2), 3), (dict(ws=FAKE + 4), 3), (dict(D=(1 << 20) + 1, ld_d=1 << 21), 2), (dict(T=1 << 31), 2),
    (dict(ws_bytes=256), 4),
])
def test_embedding_backward_refusals(R, over, status):
    assert embed_bwd(R, **over) == status
    assert "rl_embedding_bwd" in R.rl_last_error_message()


def test_nothing_to_do(R):
    assert sample(R, rows=0) == 0 and norm_fwd(R, rows=0) == 0 and norm_bwd(R, rows=0) == 0
    assert embed_fwd(R, T=0) == 0 and embed_bwd(R, T=0) == 0
    assert norm_fwd(R, rows=0, x=None, y=None, mean=None, rstd=None) == 0


def test_workspace_sizes(R):
    assert R.rl_layer_norm_workspace_size(-1, 4) == 0 and R.rl_layer_norm_workspace_size(4, 0) == 0
    assert R.rl_embedding_workspace_size(-1, 4, 4) == 0 and R.rl_embedding_workspace_size(4, 0, 4) == 0
    # parts of the columns' sums: no more than rows, and no more than the device takes at a time
    assert R.rl_layer_norm_workspace_size(1, 1000) <= 256 + 2 * 1000 * 4
    assert R.rl_layer_norm_workspace_size(1 << 20, 4096) == R.rl_layer_norm_workspace_size(1 << 16, 4096) < 16 << 20
    # a workspace serves every call with fewer tokens
    for V, D in ((1000, 64), (151936, 4097)):
        sizes = [R.rl_embedding_workspace_size(T, V, D) for T in
                 (0, 1, 100, 1024, 1025, 8192, 8193, 65536, 65537, 180224, 180225, 1 << 22, 1 << 24)]
        assert sizes == sorted(sizes)
    # 32-bit counts of bytes are passed by a long batch
    assert R.rl_embedding_workspace_size(1 << 24, 151936, 8192) > 1 << 32
