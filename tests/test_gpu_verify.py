"""rl_verify_drafts against its float64 reference: tokens and counts are equal, log-probabilities within
2e-5 (1 + |logp|): float32 differences and products of the logits (2^-24 of up to 60 each), exponentials
(2^-22) and sums of at most 1,000 terms per lane, of errors that mostly cancel."""

import numpy as np
import pytest
import torch

import verify_cases as VC

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


def rows(x, dtype, pad=0):
    t = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    out = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")[:, :x.shape[1]]
    out.copy_(t)
    return out


def call(R, c, ws=None, pad=0, draft_pad=0, max_draft=None, **kw):
    t = rows(c["target"], c["dtype"], pad)
    d = None if c["draft"] is None else rows(c["draft"], c["dtype"], draft_pad)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    ws = R.new_workspace(t.shape[0], t.shape[1]) if ws is None else ws
    out = R.rl_verify_drafts(t, dev(c["ids"]), dev(c["offsets"]), dev(c["u"]), dev(c["s"]),
                             c["max_draft"] if max_draft is None else max_draft, R.make_verify_params(c["T"]), ws,
                             draft_logits=d, **kw)
    return out, ws


def check(R, c, out, ws, word=0):
    ids, n, lp = (x.cpu().numpy() for x in out)
    r_ids, r_n, r_lp = VC.expected(c)
    assert R.rl_query_status(ws)[1] == word
    assert np.array_equal(n, r_n), (n, r_n)
    assert np.array_equal(ids, r_ids), (np.nonzero(ids != r_ids), ids[ids != r_ids], r_ids[ids != r_ids])
    assert (np.abs(lp - r_lp) <= 2e-5 * (1 + np.abs(r_lp))).all(), np.abs(lp - r_lp).max()


@pytest.mark.parametrize("V", [1, 2, 7, 8, 64, 257, 1000, 4096, 4099, 32003])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
def test_vocabularies(R, V, dtype, draft):
    c = VC.make([3, 0, 1, 5, 2], V, dtype, draft, seed=V)
    check(R, c, *call(R, c))


@pytest.mark.parametrize("counts", [[0], [1], [4], [0, 0, 0], [0, 0, 0, 0], [7, 0, 3], [1] * 40, [0, 9, 0, 2] * 8])
@pytest.mark.parametrize("T", [1.0, 0.6, 0.0])
def test_sequences(R, counts, T):
    for seed, draft in ((1, True), (2, False)):
        c = VC.make(counts, 2000, "bf16", draft, T=T, seed=seed)
        check(R, c, *call(R, c))


@pytest.mark.parametrize("dtype,pads", [("bf16", (1, 1)), ("bf16", (3, 0)), ("bf16", (8, 5)), ("f32", (1, 2)), ("f32", (0, 3))])
@pytest.mark.parametrize("V", [1000, 1003, 30001])
def test_leading_dimensions(R, dtype, pads, V):
    """Rows that begin at any element, a target row and its draft row at different places of a 16-byte block."""
    c = VC.make([2, 4, 0, 3, 1, 6], V, dtype, True, noise=1.5, seed=7)
    check(R, c, *call(R, c, pad=pads[0], draft_pad=pads[1]))


@pytest.mark.parametrize("V,dtype", [(151936, "bf16"), (151936, "f32"), (200003, "bf16"), (200003, "f32")])
@pytest.mark.parametrize("counts", [[4], [2, 1, 0, 3, 2, 1]])
def test_wide_rows(R, V, dtype, counts):
    c = VC.make(counts, V, dtype, True, noise=1.0, seed=11)
    check(R, c, *call(R, c))
    c = VC.make(counts, V, dtype, False, seed=12)
    check(R, c, *call(R, c))


@pytest.mark.parametrize("value", [-np.inf, float(np.finfo(np.float32).min), -1e30, -1e4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
def test_masked_entries(R, value, dtype, draft):
    if dtype == "bf16" and value < -3.3e38:
        value = -3.3895313892515355e38  # the type's lowest
    c = VC.make([3, 2, 0, 5], 3000, dtype, draft, masked=0.95, mask_value=value, T=0.5, seed=13)
    check(R, c, *call(R, c))


@pytest.mark.parametrize("T", [1.0, 0.0])
def test_one_entry_left_and_all_entries_at_the_lowest(R, T):
    """A row with one entry is drawn from it; a row whose entries are all the type's lowest value is uniform."""
    V = 1024
    c = VC.make([1, 0], V, "f32", False, T=T, seed=14)
    c["target"][:] = -np.inf
    c["target"][0, 700] = 3.0
    c["target"][1] = float(np.finfo(np.float32).min)
    c["target"][2, 5] = float(np.finfo(np.float32).min)
    c["ids"][:] = 700
    c["s"][:] = [(300 + 0.5) / V, 0.9]
    check(R, c, *call(R, c))


def test_many_sequences_skip_rows_behind_a_refusal(R):
    """More clusters than run at once: rows behind a refusal may be skipped, and nothing else changes."""
    rng = np.random.default_rng(15)
    for noise in (0.3, 3.0):
        c = VC.make(rng.integers(0, 8, 900), 1500, "bf16", True, noise=noise, seed=16)
        out, ws = call(R, c)
        check(R, c, out, ws)
        again, _ = call(R, c, ws=ws, max_draft=12)
        for a, b in zip(out, again):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n", [1, 3, 4])
def test_calls_leave_their_words_at_zero(R, n):
    """Sequences of one call after another in one workspace, accepted and refused in turn."""
    ws = R.new_workspace(64, 600)
    for seed in range(6):
        c = VC.make([seed % 4] * n, 600, "f32", True, noise=[0.0, 5.0][seed % 2], seed=seed)
        check(R, c, call(R, c, ws=ws)[0], ws)


def test_refused_rows_of_numbers(R):
    """A NaN, an infinity, or nothing but minus infinity ends the sequence with -1 and NaN and is reported."""
    for where, value in (("target", np.nan), ("target", np.inf), ("draft", np.nan), ("target", None), ("draft", None)):
        c = VC.make([2, 2, 2, 2], 500, "f32", True, noise=0.0, likely=0.0, seed=17)
        t_row = [0, 1, 3, 4, 6, 7, 9, 10]
        c["draft"] = c["target"][t_row].copy()  # equal rows: every token is accepted
        ref = VC.expected(c)
        hit = 4 if where == "target" else 3  # sequence 1, its second token
        if value is None:
            c[where][hit] = -np.inf
        else:
            c[where][hit, 123] = value
        (ids, n, lp), ws = call(R, c)
        assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_VALUE
        ids, n, lp = ids.cpu().numpy(), n.cpu().numpy(), lp.cpu().numpy()
        assert n.tolist() == [2, 1, 2, 2]
        assert ids[4] == -1 and np.isnan(lp[4]) and ids[5] == -1 and lp[5] == 0
        keep = [0, 1, 2, 3, 6, 7, 8, 9, 10, 11]
        assert np.array_equal(ids[keep], ref[0][keep])


def test_bad_tokens_and_offsets(R):
    c = VC.make([2, 2, 1, 1], 500, "f32", True, noise=0.0, likely=0.0, seed=18)
    c["draft"] = c["target"][[0, 1, 3, 4, 6, 8]].copy()
    bad = dict(c, ids=c["ids"].copy())
    bad["ids"][2] = 500
    (ids, n, _), ws = call(R, bad)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN
    assert n.cpu().tolist() == [2, 0, 1, 1] and 0 <= ids[3] < 500
    bad = dict(c, ids=c["ids"].copy())
    bad["ids"][0] = -7
    (ids, n, _), ws = call(R, bad)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN and n.cpu().tolist() == [0, 2, 1, 1]
    for offsets in ([0, 2, 1, 5, 6], [-1, 2, 4, 5, 6], [0, 2, 4, 5, 7], [0, 2, 4, 2000000000, 6]):
        out = dict(n_accepted=torch.full((4,), 99, dtype=torch.int32, device="cuda"))
        (ids, n, _), ws = call(R, dict(c, offsets=np.array(offsets, np.int32)), **out)
        assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_OFFSETS
        assert (n.cpu().numpy() == -1).any() and (n.cpu().numpy()[np.diff(offsets) < 0] == -1).all()
    # a sequence with more tokens than was said
    (ids, n, _), ws = call(R, c, max_draft=1)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_OFFSETS and n.cpu().tolist() == [-1, -1, 1, 1]


@pytest.mark.parametrize("n", [2, 50])
def test_streams_graphs_and_repeats(R, n):
    c = VC.make([4] * n, 3000, "bf16", True, noise=1.0, seed=19)
    first, ws = call(R, c)
    t, d = rows(c["target"], "bf16"), rows(c["draft"], "bf16")
    dev = [torch.from_numpy(np.ascontiguousarray(c[k])).cuda() for k in ("ids", "offsets", "u", "s")]
    P = R.make_verify_params(c["T"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws2 = torch.full_like(ws, 255)
    R.rl_workspace_init(ws2)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = R.rl_verify_drafts(t, *dev, 4, P, ws2, draft_logits=d)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    out = [torch.empty_like(x) for x in first]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.rl_verify_drafts(t, *dev, 4, P, ws, draft_logits=d, out_ids=out[0], n_accepted=out[1], out_logp=out[2])
    for _ in range(3):
        for x in out:
            x.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, out))
    assert R.rl_query_status(ws)[1] == 0


def test_the_first_token_follows_the_target(R):
    """Stratified numbers over a small vocabulary: the shares of the emitted first tokens are p."""
    V, g = 6, 64
    rng = np.random.default_rng(20)
    z, zd = VC.values(rng.normal(0, 1.5, (2, V)), "f32"), VC.values(rng.normal(0, 1.5, (1, V)), "f32")
    import oracle.draft_verification as O

    p, q = O.softmax(z[0], 1.0), O.softmax(zd[0], 1.0)
    grid = (np.arange(g) + 0.5) / g
    x, u, s = (a.ravel() for a in np.meshgrid(np.arange(V), grid, grid, indexing="ij"))
    n = len(x)
    c = dict(target=np.tile(z, (n, 1)), draft=np.tile(zd, (n, 1)), ids=x.astype(np.int32),
             offsets=np.arange(n + 1).astype(np.int32), u=u.astype(np.float32), s=s.astype(np.float32), T=1.0, dtype="f32",
             max_draft=1)
    (ids, _, _), ws = call(R, c)
    first = ids.cpu().numpy()[0::2]
    share = np.bincount(first, weights=q[x] / (g * g), minlength=V)
    # each of the V x 64 strata of u, and of s within it, is off by at most one of 64
    assert np.abs(share - p).max() <= 2.0 / g


def test_binding_refusals(R):
    t = torch.zeros(3, 16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    ids, off = torch.zeros(2, **i32), torch.tensor([0, 2], **i32)
    u, s = torch.zeros(2, device="cuda"), torch.zeros(1, device="cuda")
    ws, P = R.new_workspace(3, 16), R.make_verify_params()
    R.rl_verify_drafts(t, ids, off, u, s, 2, P, ws, draft_logits=torch.zeros(2, 16, device="cuda"))
    for a, kw in (((t[:2], ids, off, u, s), {}), ((t.double(), ids, off, u, s), {}), ((t.T, ids, off, u, s), {}),
                  ((t, ids.long(), off, u, s), {}), ((t, ids, off.long(), u, s), {}), ((t, ids, off, u[:1], s), {}),
                  ((t, ids, off, u, s[:0]), {}), ((t, ids, off, u, s.cpu()), {}),
                  ((t, ids, off, u, s), dict(draft_logits=torch.zeros(1, 16, device="cuda"))),
                  ((t, ids, off, u, s), dict(draft_logits=torch.zeros(2, 15, device="cuda"))),
                  ((t, ids, off, u, s), dict(draft_logits=torch.zeros(2, 16, dtype=torch.bfloat16, device="cuda"))),
                  ((t, ids, off, u, s), dict(out_ids=torch.zeros(2, **i32)))):
        with pytest.raises(ValueError):
            R.rl_verify_drafts(*a, 2, P, ws, **kw)
    with pytest.raises(R.RLError):
        R.rl_verify_drafts(t, ids, off, u, s, 2, R.make_verify_params(-1.0), ws)
    with pytest.raises(R.RLError):
        R.rl_verify_drafts(t, ids, off, u, s, 2, P, ws[:256])


@pytest.mark.parametrize("V,dtype,pad", [(40000, "bf16", 0), (33003, "bf16", 0), (33003, "bf16", 5), (20001, "f32", 0),
                                         (20000, "f32", 3)])
@pytest.mark.parametrize("draft,T", [(True, 1.0), (True, 0.6), (False, 1.0), (True, 0.0)])
def test_many_long_rows(R, V, dtype, pad, draft, T):
    """More rows than run at once, each of several CTAs."""
    rng = np.random.default_rng(21)
    c = VC.make(rng.integers(0, 5, 140), V, dtype, draft, T=T, noise=1.2, masked=0.2, seed=V + pad)
    assert len(c["ids"]) + 140 >= 304
    out, ws = call(R, c, pad=pad, draft_pad=(pad * 2) % 7)
    check(R, c, out, ws)
    again, _ = call(R, c, ws=ws, pad=pad, draft_pad=(pad * 2) % 7, max_draft=6)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


def test_many_long_rows_and_only_draws(R):
    c = VC.make([0] * 400, 70001, "bf16", False, T=0.7, seed=22)
    ws = R.new_workspace(400, 70001)
    for _ in range(3):
        check(R, c, call(R, c, ws=ws)[0], ws)


def test_many_long_rows_without_numbers(R):
    """As test_refused_rows_of_numbers and test_bad_tokens_and_offsets, with more rows than run at once."""
    n, V = 160, 40000
    c = VC.make([1] * n, V, "bf16", True, noise=0.0, likely=0.0, seed=23)
    t_row = 2 * np.arange(n)
    c["draft"] = c["target"][t_row].copy()
    c["ids"][9] = -1
    for r, value in ((2 * 3, np.nan), (2 * 5 + 1, np.inf)):
        c["target"][r, 77] = value
    c["target"][2 * 7] = -np.inf
    c["draft"][11, 5] = np.nan
    c["offsets"][150] = 2000
    (ids, acc, lp), ws = call(R, c)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_VALUE | R.RL_DEV_BAD_TOKEN | R.RL_DEV_BAD_OFFSETS
    ids, acc, lp = ids.cpu().numpy(), acc.cpu().numpy(), lp.cpu().numpy()
    want = np.ones(n, np.int64)
    want[[3, 7, 9, 11]] = 0
    want[[149, 150]] = -1
    assert np.array_equal(acc, want)
    assert (ids[[6, 14, 22]] == -1).all() and np.isnan(lp[[6, 14, 22]]).all() and ids[11] == -1 and np.isnan(lp[11])
    assert 0 <= ids[18] < V and ids[19] == -1
    R.rl_workspace_init(ws)
    good = VC.make([1] * n, 33000, "bf16", True, seed=24)
    check(R, good, call(R, good, ws=ws)[0], ws)


@pytest.mark.parametrize("V,dtype", [(900, "f32"), (30000, "bf16")])
@pytest.mark.parametrize("longest", [31, 32, 70])
def test_long_drafts(R, V, dtype, longest):
    """Rows behind a refusal finish before and after it is known."""
    rng = np.random.default_rng(25)
    counts = list(rng.integers(0, longest, 6)) + [longest, 0, longest]
    c = VC.make(counts, V, dtype, True, noise=0.05, likely=0.9, seed=longest)
    assert c["max_draft"] == longest
    for _ in range(2):
        check(R, c, *call(R, c))
    c = VC.make(counts, V, dtype, False, T=0.0, seed=longest)
    check(R, c, *call(R, c))


@pytest.mark.parametrize("V,dtype,pad", [(12289, "f32", 0), (20000, "f32", 3), (33003, "bf16", 5), (25000, "bf16", 0)])
@pytest.mark.parametrize("T", [1.0, 0.0])
def test_more_draws_than_run_at_once(R, V, dtype, pad, T):
    n = 330
    c = VC.make([0] * n, V, dtype, False, T=T, masked=0.3, seed=V)
    out, ws = call(R, c, pad=pad)
    check(R, c, out, ws)
    again, _ = call(R, c, ws=ws, pad=pad)
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    c["target"][7] = -np.inf
    c["target"][311, V - 1] = np.nan
    (ids, acc, lp), ws = call(R, c, pad=pad)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_VALUE
    lp, bad = lp.cpu().numpy(), np.isin(np.arange(n), [7, 311])
    assert (acc == 0).all() and np.array_equal(np.isnan(lp), bad)
    assert np.array_equal(ids.cpu().numpy()[~bad], out[0].cpu().numpy()[~bad])
    assert (ids.cpu().numpy()[bad] == -1).all()


@pytest.mark.parametrize("V,dtype,n", [(20000, "bf16", 400), (11000, "f32", 400), (150000, "f32", 40)])
def test_clusters_of_several_ctas_that_skip(R, V, dtype, n):
    """Clusters of two CTAs and of more, in more turns than one: all CTAs of a row behind a refusal leave, or
    none does. Most sequences are refused early, and the same call repeats bit for bit."""
    rng = np.random.default_rng(26)
    counts = rng.integers(1, 4 if n == 40 else 6, n)
    assert n != 40 or counts.sum() + n < 152  # not a CTA per row
    c = VC.make(counts, V, dtype, True, noise=3.0, likely=0.0, seed=V)
    out, ws = call(R, c)
    check(R, c, out, ws)
    for max_draft in (None, 9):
        again, _ = call(R, c, ws=ws, max_draft=max_draft)
        assert R.rl_query_status(ws)[1] == 0
        assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("V,dtype", [(33003, "bf16"), (151936, "bf16"), (33003, "f32")])
def test_tables_of_tile_weights(R, V, dtype):
    """A CTA per row, all three readers of its table: draws, draws without the looked-up token, and draws from p
    where nothing is left without it. The tokens are those of the sums in 64 bits, each time."""
    n = 170
    for counts, draft in (([0] * n, False), ([1] * n, False)):
        c = VC.make(counts, V, dtype, draft, noise=0.0, likely=0.0, seed=V)
        if counts[0]:
            c["u"][:] = np.float32(1 - 2.0 ** -24)  # every looked-up token is refused
            for b in range(n):
                p = VC.O.softmax(c["target"][2 * b], 1.0)
                q = np.zeros(V)
                q[c["ids"][b]] = 1.0
                c["s"][b] = VC.inside(VC.O.residual(p, q), float(c["s"][b]))
        ws = R.new_workspace(2 * n, V)
        for _ in range(4):
            check(R, c, call(R, c, ws=ws)[0], ws)
    # one token, drafted and refused by its number: nothing is left of p without it, so the draw is from p
    c["target"][0::2] = -np.inf
    c["target"][np.arange(0, 2 * n, 2), c["ids"]] = 1.0
    c["u"][:] = 1.0
    for _ in range(4):
        out, ws = call(R, c)
        check(R, c, out, ws)
        assert torch.equal(out[0][0::2].cpu(), torch.from_numpy(c["ids"])) and not out[1].any()


# few rows: clusters; many long ones: a CTA per row
FEW, MANY = ([3, 2, 0, 5], 3000), ([2] * 54, 33003)


@pytest.mark.parametrize("value", [-1e9, -1e10, -1e15, -1e20])
@pytest.mark.parametrize("T", [1.0, 0.3, 0.1, 0.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,V", [FEW, MANY])
def test_finite_masks(R, value, T, dtype, counts, V):
    """Masks whose exponent has a rounding error of more than fp32's range: single entries, and whole stretches, so
    that some threads see nothing else."""
    for draft in (True, False):
        c = VC.make(counts, V, dtype, draft, masked=0.3, mask_value=value, mask_from=V // 3, T=T, seed=27)
        check(R, c, *call(R, c))
        c = VC.make(counts, V, dtype, draft, masked=0.95, mask_value=value, T=T, seed=28)
        check(R, c, *call(R, c))


@pytest.mark.parametrize("T", [1.0, 0.3])
@pytest.mark.parametrize("V", [151936])
def test_padded_vocabulary(R, T, V):
    """Draws from rows whose last 293 entries are padding at -1e10."""
    for n in (3, 160):
        c = VC.make([0] * n, V, "bf16", False, masked=1e-9, mask_value=-1e10, mask_from=V - 293, T=T, seed=29)
        check(R, c, *call(R, c))


# log2(e) 11629080 is 2^24
@pytest.mark.parametrize("shift", [11629080, -11629080, 1e10, -1e10, 1e20, -1e20, 3e38, -3e38])
@pytest.mark.parametrize("T", [1.0, 0.3, 0.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,V", [FEW, MANY])
def test_rows_of_large_entries(R, shift, T, dtype, counts, V):
    """Rows whose entries, the largest among them, all have a large exponent. In fp32 the first two shifts leave whole
    numbers next to each other, on both sides of 2^24 as exponents; beyond them the rows are uniform."""
    for draft in (True, False):
        c = VC.make(counts, V, dtype, draft, shift=shift, T=T, seed=30)
        if V == 33003 and dtype == "f32" and abs(shift) < 1e9:
            assert (np.abs(c["target"]) < 2.0 ** 24 / np.log2(np.e)).any() and (np.abs(c["target"]) > 2.0 ** 24 / np.log2(np.e)).any()
        check(R, c, *call(R, c))


@pytest.mark.parametrize("n,V,dtype", [(4, 500, "f32"), (4, 3000, "bf16"), (400, 1500, "bf16"), (60, 33003, "bf16"), (60, 20000, "f32")])
@pytest.mark.parametrize("T", [1.0, 0.0])
def test_status_of_rows_behind_a_refusal(R, n, V, dtype, T):
    """What is wrong with rows and tokens behind a sequence's end is not reported, whether or not they were looked
    at; what is wrong with the row that ends it is, by itself."""
    c = VC.make([3] * n, V, dtype, True, T=T, noise=0.0, likely=0.0, seed=31)
    row, drow = 4 * np.arange(n), 3 * np.arange(n)
    c["target"][row, 5] = 30.0  # the first token, another one, is refused
    c["ids"][drow] = 7
    c["u"][drow] = 0.5
    c["s"][:] = 0.5
    ref = VC.expected(c)
    assert (ref[1] == 0).all()
    hurt = dict(c, target=c["target"].copy(), draft=c["draft"].copy(), ids=c["ids"].copy())
    hurt["target"][row + 1, 11] = np.nan
    hurt["target"][row + 2] = -np.inf
    hurt["target"][row + 3, V - 1] = np.inf
    hurt["draft"][drow + 1, 3] = np.nan
    hurt["ids"][drow + 1], hurt["ids"][drow + 2] = -5, V
    for max_draft in (3, 5):
        out, ws = call(R, hurt, max_draft=max_draft)
        ids, acc, lp = (x.cpu().numpy() for x in out)
        assert R.rl_query_status(ws)[1] == 0
        assert np.array_equal(ids, ref[0]) and np.array_equal(acc, ref[1])
        assert (np.abs(lp - ref[2]) <= 2e-5 * (1 + np.abs(ref[2]))).all()
    hurt["ids"][drow[-1]] = V + 3
    out, ws = call(R, hurt)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN and not out[1].any()
    hurt["ids"][drow[-1]] = 7
    hurt["target"][row[1], 9] = np.nan
    out, ws = call(R, hurt, ws=ws)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_TOKEN | R.RL_DEV_BAD_VALUE and not out[1].any()
    R.rl_workspace_init(ws)
    out, ws = call(R, hurt, ws=ws)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_VALUE and out[0][4].item() == -1


def test_status_texts(R):
    """Each bit of the status word that the call can set has its words in the error's text."""
    c = VC.make([1, 1, 1], 500, "f32", True, noise=0.0, likely=0.0, seed=32)
    c["target"][0, 3], c["ids"][1], c["offsets"][3] = np.nan, -1, 9
    _, ws = call(R, c)
    assert R.rl_query_status(ws) == (6, R.RL_DEV_BAD_VALUE | R.RL_DEV_BAD_TOKEN | R.RL_DEV_BAD_OFFSETS)
    text = R.rl_last_error_message()
    assert "token id out of range" in text and "inconsistent offsets" in text and "non-finite" in text
    R.rl_workspace_init(ws)
    c["ids"][1], c["offsets"][3] = 0, 3
    call(R, c, ws=ws)
    assert R.rl_query_status(ws)[1] == R.RL_DEV_BAD_VALUE and "non-finite" in R.rl_last_error_message()


# the most entries of which 16 CTAs hold a row, or a row and its draft row, and the first of that segment size
@pytest.mark.parametrize("draft,V", [(True, 899073), (True, 900096), (False, 1800193), (False, 1801216)])
def test_rows_that_fill_the_shared_memory(R, draft, V):
    c = VC.make([1, 0] if draft else [0, 0], V, "bf16", draft, seed=33)
    check(R, c, *call(R, c))


@pytest.mark.parametrize("V,dtype", [(500000, "f32"), (523264, "f32"), (900097, "bf16"), (1046528, "bf16")])
def test_rows_beyond_the_shared_memory(R, V, dtype):
    """A row and its draft row that 16 CTAs do not hold: whether they are taken depends on V alone, not on the rows."""
    c = VC.make([1, 0], V, dtype, True, noise=1.0, seed=34)
    check(R, c, *call(R, c))
    c = VC.make([1, 2], V, dtype, True, T=0.0, seed=35)
    check(R, c, *call(R, c))
    c = VC.make([3], 523265 if dtype == "f32" else 1046529, dtype, True, seed=36)
    with pytest.raises(R.RLError):
        call(R, c)
