"""rl_sample_tokens against its float64 reference.

Tokens and counts have to be equal (the cases keep the borders away from rounding; rows for which that cannot be done, of
very many equal small masses, are left out by a rule on the reference alone). A log-probability is x - log2(S) times ln 2:
x = (z - max) log2(e) / T is one fused operation whose two rounded factors (c, and max c) make it relative 2^-23 of its
terms, S a sum of exponentials relative 2^-22 + (rounding of z c: 2^-24 |z c|) each, and the sum's additions, at most
V / 2048 + 64 on a term's way. Fixed before the first run.
"""

import numpy as np
import pytest
import torch

import oracle.model_ends as O
import sample_cases as SC

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.0, 40, 1.0, 0.0), (1.3, 7, 0.8, 0.0), (1.0, 0, 1.0, 0.1),
            (0.6, 20, 0.95, 0.05), (0.0, 0, 1.0, 0.0), (1.0, 1, 0.5, 0.0), (1.0, 0, 0.1, 0.0), (2.0, 1000000, 0.999, 1e-6),
            (1e-4, 3, 0.9, 0.0), (1.0, 0, 1.0, 1.0)]


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


def on_device(z, dtype, pad=0):
    buf = torch.full((z.shape[0], z.shape[1] + pad), float("nan"), dtype=DT[dtype], device="cuda")
    buf[:, :z.shape[1]] = torch.from_numpy(z.astype(np.float32)).cuda()
    return buf[:, :z.shape[1]]


def column(x, dtype):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def run(R, z, dtype, settings, u, pad=0, ws=None):
    """settings: (T, top_k, top_p, min_p) of each row."""
    n = len(z)
    T, k, p, m = (np.array(c) for c in zip(*settings))
    out = [torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), 9.0, device="cuda"),
           torch.full((n,), 9.0, device="cuda"), torch.full((n,), -7, dtype=torch.int32, device="cuda")]
    ws = R.new_workspace(0, 0) if ws is None else ws
    R.rl_sample_tokens(on_device(z, dtype, pad), column(u, torch.float32), R.make_sample_params(), ws,
                       row_temperature=column(T, torch.float32), row_top_k=column(k, torch.int32),
                       row_top_p=column(p, torch.float32), row_min_p=column(m, torch.float32), out_ids=out[0],
                       out_logp=out[1], out_filtered_logp=out[2], n_kept=out[3])
    return [t.cpu().numpy() for t in out], R.rl_query_status(ws)[1]


def logp_tolerance(z, T, V):
    c = 1.4427 / (T or 1.0)
    live = z[z > -1e9]
    size = np.abs(live).max(initial=0.0) * c  # the fused operation's terms, where it is taken
    x = min(size, 2.0 ** 24) * 4 * U
    return (x + (4 + V / 2048 + 64) * U) * 0.7 + 4 * U


def check(R, law, n, V, dtype, seed, pad=0, choices=SETTINGS):
    rng = np.random.default_rng(seed)
    z = SC.rows(law, n, V, dtype, rng)
    settings, us = [], []
    for r in range(n):
        T, k, p, m = choices[(r + seed) % len(choices)]
        T = float(np.float32(T))
        p, m, u = SC.away_from_edges(z[r], T, k, p, m, rng.random())
        settings.append((T, k, p, m))
        us.append(u)
    (ids, logp, among, kept), status = run(R, z, dtype, settings, us, pad)
    assert status == 0
    seen = 0
    for r in range(n):
        T = settings[r][0]
        if not SC.solid(z[r], *settings[r], us[r]):
            continue
        seen += 1
        tok, lp, lf, nk = O.sample(z[r], us[r], *settings[r])
        what = (law, V, dtype, r, settings[r], us[r])
        assert kept[r] == nk, (what, kept[r], nk)
        assert ids[r] == tok, (what, ids[r], tok)
        tol = logp_tolerance(z[r], T, V)
        assert abs(logp[r] - lp) <= tol + 2 * U * abs(lp), (what, logp[r], lp)
        assert abs(among[r] - lf) <= tol + 2 * U * abs(lf), (what, among[r], lf)
    return seen


LAWS = ["normal", "likely", "ties", "equal", "signed_zero", "negative", "masked", "one_left", "finite_masks", "far", "close",
        "large"]


@pytest.mark.parametrize("law", LAWS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_laws(R, law, dtype):
    seen = 0
    for V, n in ((1, 12), (2, 12), (9, 24), (100, 36), (1003, 36), (4096, 24), (9001, 24), (33000, 12)):
        seen += check(R, law, n, V, dtype, seed=V)
    assert seen >= 60


@pytest.mark.parametrize("V", [7, 8, 2047, 8192, 8193, 32003, 50257, 131072, 151936, 409600])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_and_strides(R, V, dtype):
    for pad in (0, 5, 64):
        for law in ("likely", "normal"):
            assert check(R, law, 13, V, dtype, seed=pad + 1, pad=pad) >= 6


@pytest.mark.parametrize("law", ["likely", "normal", "ties", "close", "far", "negative"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_kept_around_what_a_list_holds(R, law, dtype):
    choices = [(1.0, k, p, m) for k in (1, 2, 33, 1000, 1023, 1024, 1025, 3000) for p, m in ((1.0, 0.0), (0.9, 0.0), (0.97, 0.01))]
    seen = sum(check(R, law, len(choices), V, dtype, seed=0, choices=choices) for V in (1500, 30000))
    assert seen >= 20


@pytest.mark.parametrize("V,dtype", [(800000, "f32"), (1600001, "bf16")])
def test_the_longest_rows(R, V, dtype):
    assert check(R, "likely", 6, V, dtype, seed=3) >= 3


@pytest.mark.parametrize("rows", [1, 2, 19, 40, 77, 153, 400, 2000])
def test_numbers_of_rows(R, rows):
    """A row's results do not hang on its company: every row of a batch as alone, bit for bit in ids and counts."""
    for V, dtype in ((1000, "f32"), (20000, "bf16")):
        n = min(rows, 60)
        rng = np.random.default_rng(rows)
        z = SC.rows("likely", n, V, dtype, rng)
        settings, us = [], []
        for r in range(n):
            T, k, p, m = SETTINGS[r % len(SETTINGS)]
            p, m, u = SC.away_from_edges(z[r], float(np.float32(T)), k, p, m, rng.random())
            settings.append((T, k, p, m))
            us.append(u)
        rep = -(-rows // n)
        zz, ss, uu = np.tile(z, (rep, 1))[:rows], (settings * rep)[:rows], (us * rep)[:rows]
        (ids, logp, among, kept), status = run(R, zz, dtype, ss, uu)
        assert status == 0
        for r in range(n):
            if SC.solid(z[r], float(np.float32(settings[r][0])), *settings[r][1:], us[r]):
                tok, _, _, nk = O.sample(z[r], us[r], float(np.float32(settings[r][0])), *settings[r][1:])
                assert ids[r] == tok and kept[r] == nk
        for r in range(n, rows):
            assert ids[r] == ids[r % n] and logp[r] == logp[r % n] and among[r] == among[r % n] and kept[r] == kept[r % n]


def test_scalar_settings_and_optional_outputs(R):
    rng = np.random.default_rng(4)
    V, n = 5000, 9
    z = SC.rows("likely", n, V, "f32", rng)
    ws = R.new_workspace(0, 0)
    for T, k, p, m in SETTINGS:
        u = rng.random(n).astype(np.float32)
        a, st = run(R, z, "f32", [(T, k, p, m)] * n, u)
        ids, logp = R.rl_sample_tokens(on_device(z, "f32"), column(u, torch.float32), R.make_sample_params(T, k, p, m), ws)
        assert np.array_equal(ids.cpu().numpy(), a[0]) and np.array_equal(logp.cpu().numpy(), a[1])
        assert st == 0 and R.rl_query_status(ws)[1] == 0


def test_draws_without_filters_are_those_of_the_verification(R):
    """rl_verify_drafts without drafts draws from the same numbers by the same rule."""
    rng = np.random.default_rng(8)
    V, n = 30000, 64
    z = SC.rows("likely", n, V, "bf16", rng)
    u = np.array([SC.away_from_edges(z[r], 1.0, 0, 1.0, 0.0, rng.random())[2] for r in range(n)])
    dev, ws = on_device(z, "bf16"), R.new_workspace(n, V)
    ids, logp = R.rl_sample_tokens(dev, column(u, torch.float32), R.make_sample_params(), ws)
    none_i, none_f = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    ids2, _, logp2 = R.rl_verify_drafts(dev, none_i, torch.zeros(n + 1, dtype=torch.int32, device="cuda"), none_f,
                                        column(u, torch.float32), 0, R.make_verify_params(1.0), ws)
    assert torch.equal(ids, ids2) and (logp - logp2).abs().max() <= 2 * logp_tolerance(z, 1.0, V)


def test_rows_that_cannot_be_drawn_from(R):
    """NaN, +infinity, nothing but -infinity, and settings out of range: token -1, and the other rows as without them."""
    V = 3000
    rng = np.random.default_rng(6)
    for dtype in ("bf16", "f32"):
        z = SC.rows("likely", 16, V, dtype, rng)
        settings = [(1.0, 20, 0.9, 0.01)] * 16
        u = np.full(16, 0.4)
        clean, st = run(R, z, dtype, settings, u)
        assert st == 0
        z[1, 7] = np.nan
        z[2, 8] = np.inf
        z[3] = -np.inf
        z[4] = np.nan
        settings[5], settings[6], settings[7], settings[8] = (-1.0, 0, 1, 0), (1, -2, 1, 0), (1, 0, 0.0, 0), (1, 0, 1, 1.5)
        settings[9], settings[10], settings[11] = (np.nan, 0, 1, 0), (1, 0, np.nan, 0), (1, 0, 1, np.nan)
        u[12], u[13], u[14] = 1.0, -0.1, np.nan
        got, st = run(R, z, dtype, settings, u)
        assert st == R.RL_DEV_BAD_VALUE
        for r in range(16):
            if r in (0, 15):
                assert all(a[r] == b[r] for a, b in zip(got, clean))
            else:
                assert got[0][r] == -1 and np.isnan(got[1][r]) and np.isnan(got[2][r]) and got[3][r] == 0, r


def test_the_frequencies_of_many_draws(R):
    """65,536 evenly spread numbers on one row: each kept token comes as often as its share says, within its two edges."""
    V, n = 600, 65536
    rng = np.random.default_rng(2)
    row = SC.rows("normal", 1, V, "f32", rng)
    dev = on_device(row, "f32").expand(n, V).contiguous()
    u = (np.arange(n) + 0.5) / n
    ws = R.new_workspace(0, 0)
    ids, _ = R.rl_sample_tokens(dev, column(u, torch.float32), R.make_sample_params(0.9, 100, 0.9, 0.0), ws)
    p, left = O.kept_tokens(row[0], float(np.float32(0.9)), 100, float(np.float32(0.9)))
    share = np.zeros(V)
    share[left] = p[left] / p[left].sum()
    count = np.bincount(ids.cpu().numpy(), minlength=V)
    assert (np.abs(count - share * n) <= 2 + 1e-5 * n).all() and (count[share == 0] == 0).all()
    assert (np.diff(ids.cpu().numpy()) >= 0).all()


def test_repeats_streams_and_graphs(R):
    rng = np.random.default_rng(12)
    V, n = 40000, 33
    z = on_device(SC.rows("likely", n, V, "bf16", rng), "bf16")
    u = column(rng.random(n), torch.float32)
    P = R.make_sample_params(0.8, 50, 0.9, 0.01)
    ws, ws2 = R.new_workspace(0, 0), R.new_workspace(0, 0)
    first = R.rl_sample_tokens(z, u, P, ws)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        second = R.rl_sample_tokens(z, u, P, ws2)
    third = R.rl_sample_tokens(z, u, P, ws)
    torch.cuda.synchronize()
    for got in (second, third):
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = R.rl_sample_tokens(z, u, P, ws)
    for _ in range(2):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, out))


ALONE = [("greedy", (0.0, 0, 1.0, 0.0)), ("top_k", (1.0, 1, 1.0, 0.0)), ("top_k, cold", (0.7, 1, 0.9, 0.1)),
         ("top_p", (0.7, 0, 1e-6, 0.0)), ("min_p", (0.6, 0, 1.0, 1.0))]


@pytest.mark.parametrize("rows,V", [(1, 5), (3, 151936), (61, 32003), (300, 4001), (1833, 1472)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,settings", ALONE, ids=[n for n, _ in ALONE])
def test_a_token_kept_alone_has_the_whole_mass(R, name, settings, dtype, rows, V):
    """Its share is 1, whatever its value: the logarithm is 0, not the rounding of the weight's own exponential."""
    rng = np.random.default_rng(rows + V)
    z = rng.normal(0, 2.0, (rows, V))
    z[np.arange(rows), rng.integers(0, V, rows)] = rng.uniform(14.0, 25.0, rows)  # the only largest one, in bf16 too
    z = SC.values(z, dtype)
    (ids, _, among, kept), status = run(R, z, dtype, [settings] * rows, rng.random(rows))
    assert status == 0
    assert (kept == 1).all() and (ids == z.argmax(1)).all()
    assert (among == 0.0).all(), among[among != 0.0][:8]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_share_is_above_the_whole(R, dtype):
    """Two tokens, the smaller down to a 2^-30 of the larger: the logarithm of the larger one's share is never positive."""
    rows = 512
    rng = np.random.default_rng(5)
    z = np.full((rows, 700), -40.0)
    z[:, 3] = rng.uniform(1.0, 20.0, rows)
    z = SC.values(z, dtype)
    z[:, 600] = SC.values(z[:, 3] - rng.uniform(5.0, 21.0, rows), dtype)
    (ids, _, among, kept), status = run(R, z, dtype, [(1.0, 2, 1.0, 0.0)] * rows, np.zeros(rows))
    assert status == 0 and (kept == 2).all() and (ids == 3).all()
    assert (among <= 0.0).all(), among[among > 0.0][:8]


def where_top_p_may_end(V):
    """How far from top_p, as a share of the mass, the border may come out: a thread adds up at most min(V / 4096, 256) tiles of
    a row, 8 entries on a way within one, and 20 sums of others, each of them rounded; an exponential is relative 2^-22 here and in
    the row's normaliser, and its mass is rounded to 2^-38."""
    return (48 + min(V / 4096, 256)) * U + V * 2.0 ** -39


@pytest.mark.parametrize("V,dtype,low,top_k", [
    (1 << 24, "bf16", -9.6875, 0), (1 << 24, "bf16", -9.0, 0), (1 << 24, "bf16", -9.6875, 1 << 23), (1 << 24, "bf16", 16.0, 0),
    (1 << 23, "f32", -9.7, 0), (1 << 23, "f32", -9.7, 6000000), (1 << 23, "f32", 16.0, 0), (1 << 20, "f32", -2.0, 0)])
@pytest.mark.parametrize("rows", [1, 3])
def test_where_top_p_ends_in_a_long_flat_tail(R, V, dtype, low, top_k, rows):
    """One entry and millions of equal ones, each of them down to 2^-37 of its mass: half of what they have together is kept
    (and not all of it, as where their masses come out as nothing)."""
    z = torch.full((rows, V), low, dtype=DT[dtype], device="cuda")
    z[:, V // 3] = 16.0
    w = float(np.exp(low - 16.0))
    of_k = top_k - 1 if top_k else V - 1
    total = 1.0 + of_k * w
    top_p = float(np.float32((1.0 + 0.5 * of_k * w) / total))
    kept = torch.empty(rows, dtype=torch.int32, device="cuda")
    ws = R.new_workspace(0, 0)
    R.rl_sample_tokens(z, column(np.full(rows, 0.5), torch.float32), R.make_sample_params(1.0, top_k, top_p, 0.0), ws, n_kept=kept)
    assert R.rl_query_status(ws)[1] == 0
    for n in kept.cpu().numpy().astype(np.float64):
        before, upto = (1.0 + (n - 2) * w) / total, (1.0 + (n - 1) * w) / total
        tol = where_top_p_may_end(V)
        assert before < top_p + tol and upto >= top_p - tol, (n, (upto - top_p) / U)

@pytest.mark.parametrize("rows,V", [(1, 700), (1, 151936), (61, 32003), (300, 4001), (600, 20000), (1833, 1472)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("settings", [(1.0, 6, 1.0, 0.0), (0.7, 6, 0.9999999, 0.0), (1.0, 0, 1.0, 1e-16), (1.0, 0, 1.0, 0.0)])
def test_a_share_close_to_the_whole(R, settings, dtype, rows, V):
    """The largest entry and five others 4 to 30 below it: the logarithm of its share is as exact, relative, as the others'
    weights. An exponent (z - max) c has c's two roundings and its own, 2.5 2^-24 of its size in all; the two exponentials are
    relative 2^-22, five weights are added up, and the quotient (two units, and its divisor's rounding), the series and the
    result are 10 roundings."""
    rng = np.random.default_rng(rows + V)
    z = np.full((rows, V), -np.inf)
    at = np.argsort(rng.random((rows, V)), axis=1)[:, :6] if V < 2000 else rng.integers(0, V // 6, (rows, 6)) + np.arange(6) * (V // 6)
    r = np.arange(rows)
    z[r, at[:, 0]] = rng.uniform(14.0, 25.0, rows)
    for i in range(1, 6):
        z[r, at[:, i]] = z[r, at[:, 0]] - rng.uniform(4.0, 30.0, rows) * settings[0]
    z = SC.values(z, dtype)
    (ids, _, among, kept), status = run(R, z, dtype, [settings] * rows, np.full(rows, 0.5))
    assert status == 0 and (ids == at[:, 0]).all()
    T = float(np.float32(settings[0]))
    for k in range(rows):
        p, left = O.kept_tokens(z[k], T, 6)
        if settings[2] == 1.0 and settings[3] == 0.0:
            assert kept[k] == 6
        order = left[np.argsort(-z[k][left], kind="stable")][: kept[k]]
        x = (z[k][order[1:]] - z[k][order[0]]) / T
        ref = -np.log1p(np.exp(x).sum())
        tol = (2.5 * np.abs(x).max(initial=0.0) + 8 + 5 + 10) * U
        assert abs(among[k] - ref) <= tol * abs(ref), (k, among[k], ref, (among[k] / ref - 1) / U)

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_temperatures(R, dtype):
    """Every finite temperature is one that the header allows; these make all entries equally likely."""
    V = 1000
    rng = np.random.default_rng(1)
    u = (np.arange(V) + 0.5) / V
    z = np.tile(SC.rows("normal", 1, V, dtype, rng), (V, 1))
    largest = float(np.finfo(np.float32).max)
    for T in (2.9e38, 3e38, 3.3e38, largest):
        (ids, logp, among, kept), status = run(R, z, dtype, [(T, 0, 1.0, 0.0)] * V, u)
        assert status == 0 and (ids == np.arange(V)).all() and (kept == V).all()
        assert (np.abs(logp + np.log(V)) <= 100 * U).all() and (np.abs(among + np.log(V)) <= 100 * U).all()
        ws = R.new_workspace(0, 0)
        once, _ = R.rl_sample_tokens(on_device(z, dtype), column(u, torch.float32), R.make_sample_params(T), ws)
        assert (once.cpu().numpy() == np.arange(V)).all() and R.rl_query_status(ws)[1] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_number_takes_the_last_of_the_mass(R, dtype):
    """sample_u = 1 - 2^-24: where the rounded goal is not passed, the last kept token of any weight is taken; the mass behind
    it stays within the bound of the header (the sums' error)."""
    last = 1 - 2.0 ** -24
    for V, n in ((100, 300), (5000, 300), (40000, 60)):
        rng = np.random.default_rng(V)
        z = rng.normal(0, 2.0, (n, V))
        z[:, V // 2:] -= 3.0
        z = SC.values(z, dtype)
        order = np.argsort(-z, axis=1, kind="stable")
        for T, k, p, m in SETTINGS:
            T = float(np.float32(T))
            (ids, _, among, kept), status = run(R, z, dtype, [(T, k, p, m)] * n, np.full(n, last))
            assert status == 0
            for r in range(n):
                if T == 0:
                    assert ids[r] == z[r].argmax() and among[r] == 0
                    continue
                left = np.sort(order[r][: kept[r]])
                w = np.exp((z[r][left] - z[r].max()) / T)
                at = np.nonzero(left == ids[r])[0]
                assert len(at) == 1, (V, T, k, p, m, r)
                share = w / w.sum()
                behind = share[at[0] + 1:].sum()
                assert behind <= (48 + V / 4096) * U + 2.0 ** -24, (V, T, k, p, m, r, behind)
                tol = logp_tolerance(z[r], T, V)
                assert abs(among[r] - np.log(share[at[0]])) <= tol + 2 * U * abs(among[r]), (V, T, k, p, m, r)
