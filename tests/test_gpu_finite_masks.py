"""Logits masked by finite values (-1e9 to -1e30): rows of which some threads, or whole CTAs, see nothing but masks have
the loss, gradient, statistics and log-probabilities of the softmax over the other entries."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    return R


ROWS = 6


def masked(dtype, V, ld, where, value):
    g = torch.Generator(device="cuda").manual_seed(V + ld)
    z = torch.empty(ROWS, ld, dtype=dtype, device="cuda")[:, :V]
    z.copy_(torch.randn(ROWS, V, device="cuda", generator=g) * 2)
    off = {"front": torch.arange(V, device="cuda") < V - V // 4, "end": torch.arange(V, device="cuda") >= V // 3,
           "most": torch.rand(V, device="cuda", generator=g) < 0.97}[where]
    off[V // 3 - 1 if where == "end" else V - 1] = False
    z[:, off] = value
    ids = torch.nonzero(~off)[:, 0][torch.randint(0, int((~off).sum()), (ROWS,), device="cuda", generator=g)]
    return z, ids.int()


# bf16: warps with 4, 8 and 16 vectors a lane, one CTA and clusters; fp32: warps, the aligned kernel and
# the shifted one, wide rows on both of their shapes
@pytest.mark.parametrize("dtype,V,ld", [
    (torch.bfloat16, 1000, 1000), (torch.bfloat16, 2000, 2003), (torch.bfloat16, 4096, 4096),
    (torch.bfloat16, 12000, 12000), (torch.bfloat16, 32003, 32003), (torch.bfloat16, 151936, 151936),
    (torch.float32, 500, 500), (torch.float32, 2048, 2051), (torch.float32, 32000, 32000),
    (torch.float32, 32000, 32003), (torch.float32, 151936, 151936), (torch.float32, 200001, 200001)])
@pytest.mark.parametrize("where", ["front", "end", "most"])
@pytest.mark.parametrize("ent", [0.0, 0.01])
def test_finite_masks(R, dtype, V, ld, where, ent):
    mask, tt = torch.ones(ROWS, dtype=torch.uint8, device="cuda"), torch.zeros(ROWS, dtype=torch.int32, device="cuda")
    one = torch.ones(1, device="cuda")
    for value in (-1e4, -1e9, -2e9, -3e9, -1e10, -1e15, -1e20, -1e30):
        z, ids = masked(dtype, V, ld, where, value)
        logp = torch.log_softmax(z.double(), -1)
        p, lp = logp.exp(), logp.gather(1, ids.long()[:, None])[:, 0]
        H = -(p * logp.clamp_min(-1e6)).sum(-1)
        # a loss of -ratio - ent H per row, with the ratio 1: the old log-probabilities are the row's own
        ref = p.clone()
        ref[torch.arange(ROWS), ids.long()] -= 1
        ref += ent * p * (logp.clamp_min(-1e6) + H[:, None])
        ws, total = R.new_workspace(ROWS, V), torch.zeros(1, dtype=torch.float64, device="cuda")
        stats = torch.empty(ROWS, 5, device="cuda") if ent else None
        got = R.rl_policy_loss_fwd_bwd(z, ids, mask, tt, one, one, lp.float(), R.make_params(entropy_coef=ent), ws, total,
                                       token_stats=stats)
        assert abs(total.item() + ROWS + ent * H.sum().item()) <= 2e-5 * ROWS, value
        # fp32 sums and exponentials, and the rounding of the gradient to bf16
        tol = 1e-5 + (2.0 ** -8 if dtype is torch.bfloat16 else 0.0) * ref.abs()
        assert ((got.double() - ref).abs() <= tol).all(), (value, (got.double() - ref).abs().max().item())
        for want in (False, True):
            out, entropy, lse = R.rl_token_logprobs(z, ids, ws, want_entropy=want, want_lse=True)
            assert ((out - lp).abs() <= 1e-5 * (1 + lp.abs())).all(), value
            assert ((lse - z.double().logsumexp(-1)).abs() <= 1e-5 * (1 + lp.abs())).all(), value
            assert not want or ((entropy - H).abs() <= 2e-5 * (1 + H)).all(), value
        assert R.rl_query_status(ws)[1] == 0
