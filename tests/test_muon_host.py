"""What rl_muon_update refuses before any launch (no GPU needed), and its workspace."""

import ctypes

import pytest

from paper_2608_16798_gb300 import build as B

FAKE = 0x10000  # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def R():
    B.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


def _call(R, **over):
    a = dict(batch=2, m=4, n=8, grad=FAKE, dt=R.RL_F32, ld_g=8, st_g=32, mom=FAKE, w=FAKE, wb=FAKE, ld_w=8, st_w=32,
             upd=FAKE, params=R.make_muon_params(), ws=FAKE, ws_bytes=1 << 30)
    a.update(over)
    P = a["params"]
    return R.lib().rl_muon_update(a["batch"], a["m"], a["n"], a["grad"], a["dt"], a["ld_g"], a["st_g"], a["mom"],
                                  a["w"], a["wb"], a["ld_w"], a["st_w"], a["upd"],
                                  None if P is None else ctypes.byref(P), a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("over,status", [
    (dict(batch=-1), 1), (dict(m=-1), 1), (dict(n=-3), 1),
    (dict(m=32769, n=32769), 2), (dict(m=1, n=(1 << 24) + 1), 2), (dict(batch=1 << 18), 2),
    (dict(dt=5), 1), (dict(grad=None), 1), (dict(ws=None), 1), (dict(params=None), 1),
    (dict(w=None, wb=None, upd=None), 1), (dict(w=None), 1), (dict(mom=None), 1),
    (dict(ld_g=7), 1), (dict(st_g=-1), 1), (dict(ld_w=7), 1), (dict(st_w=31), 1), (dict(st_w=8, ld_w=15), 1),
    (dict(ws=FAKE + 4), 3), (dict(grad=FAKE + 2), 3), (dict(mom=FAKE + 1), 3), (dict(w=FAKE + 2), 3),
    (dict(wb=FAKE + 1), 3), (dict(upd=FAKE + 1), 3), (dict(grad=FAKE + 1, dt=0), 3),
    (dict(ws_bytes=1024), 4),
])
def test_refusals(R, over, status):
    assert _call(R, **over) == status
    assert "rl_muon_update" in R.rl_last_error_message()


@pytest.mark.parametrize("kw", [dict(ns_steps=0), dict(ns_steps=17), dict(momentum=1.0), dict(momentum=-0.1),
                                dict(momentum=float("nan")), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(lr=float("inf")), dict(weight_decay=float("nan")), dict(update_scale=float("inf")),
                                dict(ns_coef=(9.0, 0.0, 0.0)), dict(ns_coef=(float("nan"), 0.0, 0.0))])
def test_refused_parameters(R, kw):
    assert _call(R, params=R.make_muon_params(**kw)) == 1


def test_nothing_to_do(R):
    for over in (dict(batch=0), dict(m=0), dict(n=0)):
        assert _call(R, **over) == 0


def test_workspace_size(R):
    assert R.rl_muon_workspace_size(0, 5, 5) == 256
    assert R.rl_muon_workspace_size(-1, 5, 5) == 0 and R.rl_muon_workspace_size(1, 40000, 40000) == 0
    one, two = R.rl_muon_workspace_size(1, 1024, 4096), R.rl_muon_workspace_size(2, 1024, 4096)
    assert 8 * 1024 * 4096 <= one < two
    # the transpose needs the same buffers
    assert abs(R.rl_muon_workspace_size(1, 4096, 1024) - one) < 1 << 16
    # 32-bit counts of bytes are passed by a large matrix
    assert R.rl_muon_workspace_size(1, 32768, 32768) > 8 << 30
