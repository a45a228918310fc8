"""What rl_verify_drafts refuses before any launch (no GPU needed)."""

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
    a = dict(t=FAKE, d=FAKE, dt=0, n_seq=2, n_draft=4, K=2, V=64, ld_t=64, ld_d=64, ids=FAKE, off=FAKE, ua=FAKE, us=FAKE,
             params=R.make_verify_params(), out=FAKE, acc=FAKE, lp=FAKE, ws=FAKE, ws_bytes=1 << 20)
    a.update(over)
    P = a["params"]
    return R.lib().rl_verify_drafts(a["t"], a["d"], a["dt"], a["n_seq"], a["n_draft"], a["K"], a["V"], a["ld_t"],
                                    a["ld_d"], a["ids"], a["off"], a["ua"], a["us"],
                                    None if P is None else ctypes.byref(P), a["out"], a["acc"], a["lp"], a["ws"],
                                    a["ws_bytes"], None)


@pytest.mark.parametrize("over,status", [
    (dict(dt=3), 1), (dict(n_seq=-1), 1), (dict(n_draft=-1), 1), (dict(K=-1), 1), (dict(V=0), 1), (dict(ld_t=63), 1),
    (dict(ld_d=63), 1), (dict(params=None), 1), (dict(t=None), 1), (dict(ids=None), 1), (dict(off=None), 1),
    (dict(ua=None), 1), (dict(us=None), 1), (dict(out=None), 1), (dict(acc=None), 1), (dict(lp=None), 1), (dict(ws=None), 1),
    (dict(t=FAKE + 8), 3), (dict(d=FAKE + 2), 3), (dict(ws=FAKE + 4), 3),
    (dict(V=1 << 25, ld_t=1 << 25, ld_d=1 << 25), 2), (dict(K=1 << 26), 2), (dict(n_draft=1 << 30), 2),
    (dict(ws_bytes=256), 4),
])
def test_refusals(R, over, status):
    assert _call(R, **over) == status
    assert "rl_verify_drafts" in R.rl_last_error_message()


@pytest.mark.parametrize("T", [-1.0, float("nan"), float("inf"), 1e-5])
def test_refused_temperatures(R, T):
    assert _call(R, params=R.make_verify_params(T)) == 1


def test_rows_beyond_the_shared_memory(R):
    # two bf16 rows of 16 CTAs x 220 KB, and one without drafts
    big = 1 << 20
    assert _call(R, V=big, ld_t=big, ld_d=big) == 2
    assert _call(R, V=1 << 21, ld_t=1 << 21, d=None) == 2


def test_nothing_to_do(R):
    assert _call(R, n_seq=0, n_draft=0) == 0
