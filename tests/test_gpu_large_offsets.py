"""Matrices of more than 2^31 elements: the rows behind that place come out as the same rows do by themselves."""

import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


def noise(rows, D, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(rows, D, dtype=dtype, device="cuda")
    for a in range(0, rows, 65536):
        x[a:a + 65536] = torch.randn(min(65536, rows - a), D, generator=g, device="cuda")
    return x


def test_sampling(R):
    rows, V = 14500, 151936
    z = noise(rows, V, BF, 1)
    assert z.numel() > 1 << 31
    u = torch.rand(rows, device="cuda")
    P, ws = R.make_sample_params(1.0, 30, 0.9, 0.0), R.new_workspace(0, 0)
    ids, logp = R.rl_sample_tokens(z, u, P, ws)
    for a in (0, rows - 40):
        # (by itself a row may be on more CTAs, whose sums are added up in another order)
        some, lp = R.rl_sample_tokens(z[a:a + 40], u[a:a + 40].contiguous(), P, ws)
        assert (ids[a:a + 40] == some).sum() >= 39 and (logp[a:a + 40] - lp).abs()[ids[a:a + 40] == some].max() < 1e-5
    assert R.rl_query_status(ws)[1] == 0


@pytest.mark.parametrize("D", [4096, 4099, 128])
def test_layer_norm(R, D):
    rows = (1 << 31) // D + 3000
    x = noise(rows, D, BF, 2)
    y, mean, rstd = R.rl_layer_norm_fwd(x)
    few = slice(rows - 700, rows)
    ws = R.new_layer_norm_workspace(rows, D)
    mask = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    mask[few] = 1
    dw = torch.zeros(D, device="cuda")
    dx = R.rl_layer_norm_bwd(y, x, mean, rstd, ws, mask=mask, d_weight=dw)
    y2, mean2, rstd2 = R.rl_layer_norm_fwd(x[few])
    # (fewer rows take another kernel: the last bits of the sums)
    assert (mean[few] - mean2).abs().max() < 1e-6 and (rstd[few] / rstd2 - 1).abs().max() < 1e-6
    assert (y[few].float() - y2.float()).abs().max() <= 2.0 ** -7 * 8
    dw2 = torch.zeros(D, device="cuda")
    dx2 = R.rl_layer_norm_bwd(y[few], x[few], mean[few].clone(), rstd[few].clone(), ws, d_weight=dw2)
    assert (dx[few].float() - dx2.float()).abs().max() <= 2.0 ** -7 and (dw - dw2).abs().max() <= 1e-5 * dw.abs().max()
    assert (dx[:1000] == 0).all() and (dx[rows - 1700:rows - 700] == 0).all()


def test_embedding(R):
    V, D, T = 524300, 4104, 523400
    w = noise(V, D, BF, 3)
    ids = torch.arange(T, device="cuda", dtype=torch.int32) + 900
    ws = R.new_embedding_workspace(T, V, D)
    out = R.rl_embedding_fwd(ids, w, ws)
    assert w.numel() > 1 << 31 and out.numel() > 1 << 31
    assert torch.equal(out[-500:], w[-500:]) and torch.equal(out[:500], w[900:1400])
    del w
    dw = torch.zeros(V, D, device="cuda")
    R.rl_embedding_bwd(ids, out, dw, ws)
    assert torch.equal(dw[-500:], out[-500:].float()) and torch.equal(dw[900:1400], out[:500].float()) and (dw[:900] == 0).all()
    assert R.rl_query_status(ws)[1] == 0
