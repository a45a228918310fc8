"""Three operators at the two ends of the policy model, as cases that can be timed and compared.

  sample   the next token of every request from its logits row (``rl_sample_tokens``): temperature,
           top-k, top-p and min-p, each request with its own, from given random numbers. Out come the
           token, its log-probability under softmax(z / T) (the rollout log-probability of the loss),
           its log-probability among the tokens that were kept, and how many were.
  norm     layer norm before the LM head (``rl_layer_norm_fwd``, ``rl_layer_norm_bwd``): the hidden
           states that the fused head reads; backward, from the head's d hidden, the gradient of the
           input and the reductions for the weight and the bias. Rows that are not trained on have no
           gradient.
  embed    the embedding of the tokens, scaled (``rl_embedding_fwd``), and its gradient
           (``rl_embedding_bwd``), added to the fp32 gradient that a tied LM head adds to as well.

With ``own`` false a pass computes the operators in their plain form, elementary torch operations in
32 bits (64 for the sums of the probabilities); with ``own`` true it makes the calls of
the library's binding. ``exact`` states the results in 64 bits.

The token that a given number selects and the number of tokens that are kept are whole numbers, so
the given numbers, top_p and min_p are kept a little away from the edges at which these change:
every correct implementation takes the same ones.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EDGE = 2e-5          # distance of a given number, and of top_p, from the edges of its token's interval
LEAST_MASS = 6e-5    # tokens that a number selects, or at which top_p ends, have at least this probability
NORM_EPS = 1e-5


def _sample(name, rows, V, dtype, temp=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, std=2.0, masked=0.0, pad=0):
    c = dict(kind="sample", rows=rows, V=V, dtype=dtype, temp=temp, top_k=top_k, top_p=top_p, min_p=min_p, mixed=mixed,
             std=std, masked=masked, pad=pad)
    return dict(c, name=name) if name else c


def _norm(name, back, rows, D, x_dtype, y_dtype, bias=True, trained=1.0, pad=0):
    c = dict(kind="norm", back=back, rows=rows, D=D, x_dtype=x_dtype, y_dtype=y_dtype, bias=bias, trained=trained,
             pad=pad)
    return dict(c, name=name) if name else c


def _embed(name, back, T, D, V, w_dtype, a_dtype, zipf=1.0, pad=0):
    c = dict(kind="embed", back=back, T=T, D=D, V=V, w_dtype=w_dtype, a_dtype=a_dtype, zipf=zipf, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request that decodes by itself: one row, latency counts
        _sample("sample_one", 1, 151936, "bf16", temp=0.7, top_k=50, top_p=0.8),
        # a decoding step of the multi-turn batch: all 128 rollouts, top-p alone
        _sample("sample_group", 128, 151936, "bf16", top_p=0.95),
        # a large batch of requests, each with its own settings (greedy ones and unfiltered ones among them)
        _sample("sample_mixed", 509, 151936, "bf16", mixed=True),
        # fp32 logits of a vocabulary with three added tokens, entries cut off before, in a wider buffer
        _sample("sample_f32", 61, 32003, "f32", temp=0.8, top_k=200, min_p=0.02, masked=0.3, std=3.0, pad=5),
        # the norm of a decoding step: one row for each of 128 rollouts
        _norm("norm_fwd_step", False, 128, 4096, "bf16", "bf16"),
        # a microbatch whose residual stream is kept in fp32
        _norm("norm_fwd_batch", False, 32768, 4096, "f32", "bf16"),
        # its backward pass from the head's bf16 d hidden, 60% of the tokens trained on
        _norm("norm_bwd_batch", True, 32768, 4096, "bf16", "bf16", trained=0.6),
        # an odd width in wider buffers, fp32 gradients, no bias
        _norm("norm_bwd_odd", True, 4999, 1001, "bf16", "f32", bias=False, pad=6),
        # the embedding of a microbatch at the full hidden size
        _embed("embed_fwd_batch", False, 32768, 4096, 151936, "bf16", "bf16"),
        # the gradient of a short microbatch of a small model
        _embed("embed_bwd_small", True, 512, 1024, 32000, "bf16", "bf16"),
        # the gradient of the microbatch at the full hidden size
        _embed("embed_bwd_batch", True, 32768, 4096, 151936, "bf16", "bf16"),
        # the whole multi-turn batch of a small model: an odd width, fp32 gradients, frequent tokens that come often
        _embed("embed_bwd_multiturn", True, 155959, 1001, 32003, "f32", "f32", zipf=1.2, pad=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "norm", "embed"])
    if kind == "sample":
        V = _log_int(rng, 1000, 151936)
        if rng.random() < 0.5:
            V = V // 64 * 64
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = int(154e6 / (V * (2 if dtype == "bf16" else 4)))
        return _sample(None, min(_log_int(rng, 1, 2048), most), V, dtype, temp=rng.choice([1.0, 1.0, 0.7, 0.6, 0.0]),
                       top_k=rng.choice([0, 0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 0.95, 0.9, 0.8]),
                       min_p=rng.choice([0.0, 0.0, 0.05, 0.1]), mixed=rng.random() < 0.3, std=rng.choice([2.0, 3.0]),
                       masked=rng.choice([0.0, 0.0, 0.3]), pad=rng.choice([0, 0, 5, 64]))
    if kind == "norm":
        D = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            D = D // 64 * 64
        rows = min(_log_int(rng, 1, 65536), int(1.3e8 / D))
        return _norm(None, rng.random() < 0.5, rows, D, rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"]),
                     bias=rng.random() < 0.7, trained=rng.choice([1.0, 0.6]), pad=rng.choice([0, 0, 6, 64]))
    D = _log_int(rng, 64, 4096)
    if rng.random() < 0.6:
        D = D // 64 * 64
    T = min(_log_int(rng, 1, 160000), int(1.3e8 / D))
    return _embed(None, rng.random() < 0.6, T, D, _log_int(rng, 1000, 151936), rng.choice(["bf16", "f32"]),
                  rng.choice(["bf16", "bf16", "f32"]), zipf=rng.choice([0.0, 1.0, 1.2]), pad=rng.choice([0, 0, 3, 64]))


# ----------------------------------------------------------------------------- inputs

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + stream * 7919) & 0x7FFFFFFFFFFF)
    return g


def _chunks(rows, V, elements=1 << 26):
    step = max(1, elements // V)
    return [(r, min(rows, r + step)) for r in range(0, rows, step)]


def _settings(case, g):
    """(temperature, top_k, top_p, min_p) of every row: the case's, or one of what requests ask for."""
    rows = case["rows"]
    t = torch.full((rows,), case["temp"], device=DEV)
    k = torch.full((rows,), case["top_k"], dtype=torch.int32, device=DEV)
    p = torch.full((rows,), case["top_p"], device=DEV)
    m = torch.full((rows,), case["min_p"], device=DEV)
    if case["mixed"]:
        pick = torch.tensor([[1.0, 0, 1.0, 0.0], [1.0, 0, 0.95, 0.0], [0.7, 20, 0.8, 0.0], [0.6, 20, 0.95, 0.0],
                             [1.0, 50, 1.0, 0.0], [1.0, 0, 1.0, 0.05], [0.8, 1000, 0.9, 0.02], [0.0, 0, 1.0, 0.0]],
                            device=DEV)[torch.randint(0, 8, (rows,), generator=g, device=DEV)]
        t, k, p, m = pick[:, 0].clone(), pick[:, 1].int(), pick[:, 2].clone(), pick[:, 3].clone()
    return t, k, p, m


def _prepare_sample(case, seed):
    """Rows N(0, std^2) in which half the rows have one likely token (of 10 to 60%), as a language model's have."""
    rows, V, std = case["rows"], case["V"], case["std"]
    g = _gen(seed, 1)
    z = torch.empty(rows, V + case["pad"], dtype=DT[case["dtype"]], device=DEV)[:, :V]
    temp, top_k, top_p, min_p = _settings(case, g)
    u = torch.empty(rows, dtype=torch.float32, device=DEV)
    for a, b in _chunks(rows, V, 1 << 25):
        n = b - a
        t = torch.where(temp[a:b] > 0, temp[a:b], 1.0).double()[:, None]
        spike = t[:, 0].float() * (math.log(V) + 0.5 * std * std / t[:, 0].float() ** 2)
        x = torch.randn(n, V, generator=g, device=DEV).mul_(std)
        if case["masked"]:
            x[torch.rand(n, V, generator=g, device=DEV) < case["masked"]] = -math.inf
        hot = torch.rand(n, generator=g, device=DEV) < 0.5
        v = spike + t[:, 0].float() * (torch.rand(n, generator=g, device=DEV) * 2.5 - 2.0)
        i = torch.arange(n, device=DEV)
        x[i, torch.randint(0, V, (n,), generator=g, device=DEV)] = torch.where(hot, v, torch.full_like(v, 2.0 * std))
        z[a:b] = x
        # where the borders lie: the sorted probabilities, the most likely first and the lower index first
        zz = z[a:b].double()
        prob = torch.exp((zz - zz.amax(1, keepdim=True)) / t)
        order = zz.sort(dim=1, descending=True, stable=True).indices
        srt = prob.gather(1, order)
        live = (srt > 0).sum(1, keepdim=True)
        k = top_k[a:b].long()[:, None]
        n_k = torch.where(k > 0, torch.minimum(k, live), live)
        at = torch.arange(V, device=DEV)
        srt_k = torch.where(at < n_k, srt, 0.0)
        run = srt_k.cumsum(1) / srt_k.sum(1, keepdim=True)
        mass = srt_k / srt_k.sum(1, keepdim=True)
        # top_p: inside the interval of a token that is likely enough
        wanted = torch.minimum((run < top_p[a:b, None].double()).sum(1, keepdim=True),
                               ((mass >= LEAST_MASS).sum(1, keepdim=True) - 1).clamp(min=0))
        inside = 0.25 + 0.5 * torch.rand(n, 1, generator=g, device=DEV, dtype=torch.float64)
        moved = (run.gather(1, wanted) - mass.gather(1, wanted) * inside)[:, 0].float()
        off = top_p[a:b] >= 1.0
        n_p = torch.where(off[:, None], n_k, wanted + 1)
        top_p[a:b] = torch.where(off, top_p[a:b], moved)
        # min_p: in the widest gap between two neighbours of the order near its border
        rel = srt / srt[:, :1]
        n0 = (rel >= min_p[a:b, None].double()).sum(1, keepdim=True).clamp(1, V - 1)
        near = (n0 + torch.arange(-8, 9, device=DEV)).clamp(1, V - 1)
        hi, lo = rel.gather(1, near - 1), rel.gather(1, near).clamp(min=1e-300)
        best = (hi / lo).nan_to_num(posinf=0.0).argmax(1, keepdim=True)
        cut = (hi.gather(1, best) * torch.maximum(lo.gather(1, best), 0.25 * hi.gather(1, best))).sqrt()
        use = (min_p[a:b] > 0)[:, None]
        n_m = torch.where(use, (rel >= cut).sum(1, keepdim=True), live)
        min_p[a:b] = torch.where(use, cut, 0.0)[:, 0].float()
        # the numbers: inside the interval, in the order of the vocabulary, of a token that was kept
        kept = torch.zeros_like(prob).scatter_(1, order, (at < torch.minimum(torch.minimum(n_k, n_p), n_m)).double())
        c = prob * kept
        c /= c.sum(1, keepdim=True)
        us = torch.rand(n, 2, generator=g, device=DEV, dtype=torch.float64)
        pick = torch.where(c >= LEAST_MASS, c, 0.0).cumsum(1)
        tok = torch.searchsorted(pick, us[:, :1] * pick[:, -1:], right=True).clamp_(max=V - 1)
        tok = torch.where(c.gather(1, tok) >= LEAST_MASS, tok, c.argmax(1, keepdim=True))
        m1 = c.gather(1, tok)[:, 0]
        low = c.cumsum(1).gather(1, tok)[:, 0] - m1
        u[a:b] = (low + EDGE + us[:, 1] * (m1 - 2 * EDGE).clamp(min=0)).float()
    s = dict(case=case, z=z, u=u.clamp_(0.0, 1.0 - 2.0 ** -24), temp=temp, top_k=top_k, top_p=top_p, min_p=min_p)
    if own:
        import paper_2608_16798_gb300.rl_loss as R

        s.update(params=R.make_sample_params(), ws=R.new_workspace(rows, V),
                 out=[torch.empty(rows, dtype=d, device=DEV) for d in (torch.int32, torch.float32, torch.float32, torch.int32)])
    return s


def _prepare_norm(case, seed):
    """Rows of a residual stream: a few wide channels, a mean of its own for every row; gradients of
    the size that a mean over the batch's tokens gives."""
    rows, D, pad = case["rows"], case["D"], case["pad"]
    g = _gen(seed, 2)
    wide = 1.0 + 8.0 * (torch.rand(D, generator=g, device=DEV) < 0.02)
    x = torch.empty(rows, D + pad, dtype=DT[case["x_dtype"]], device=DEV)[:, :D]
    for a, b in _chunks(rows, D):
        x[a:b] = torch.randn(b - a, D, generator=g, device=DEV) * wide + torch.randn(b - a, 1, generator=g, device=DEV)
    s = dict(case=case, x=x, w=1.0 + 0.2 * torch.randn(D, generator=g, device=DEV))
    if not case["back"]:
        s["b"] = 0.1 * torch.randn(D, generator=g, device=DEV) if case["bias"] else None
        s["y"] = torch.empty(rows, D + pad, dtype=DT[case["y_dtype"]], device=DEV)[:, :D]
        s["mean"], s["rstd"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        return s
    dy = torch.empty(rows, D + pad, dtype=DT[case["y_dtype"]], device=DEV)[:, :D]
    mask = (torch.rand(rows, generator=g, device=DEV) < case["trained"]).to(torch.uint8) if case["trained"] < 1 else None
    s["mean"], s["rstd"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    for a, b in _chunks(rows, D):
        r = torch.randn(b - a, D, generator=g, device=DEV) * 1e-4
        dy[a:b] = r if mask is None else r * mask[a:b, None]
        v = x[a:b].double()
        s["mean"][a:b] = v.mean(1)
        s["rstd"][a:b] = (v.var(1, unbiased=False) + NORM_EPS).rsqrt()
    s.update(dy=dy, mask=mask, dx=torch.empty(rows, D + pad, dtype=DT[case["x_dtype"]], device=DEV)[:, :D],
             dw=torch.randn(D, generator=g, device=DEV) * 1e-3,
             db=torch.randn(D, generator=g, device=DEV) * 1e-3 if case["bias"] else None)
    if own:
        import paper_2608_16798_gb300.rl_loss as R

        s["ws"] = R.new_layer_norm_workspace(rows, D)
    return s


def _frequencies(case):
    r = np.arange(case["V"], dtype=np.float64)
    p = (r + 2.7) ** -case["zipf"]
    return p / p.sum()


def _prepare_embed(case, seed):
    """Token ids whose frequencies fall with their rank, ranks spread over the vocabulary."""
    T, D, V, pad = case["T"], case["D"], case["V"], case["pad"]
    g = _gen(seed, 3)
    cdf = torch.from_numpy(np.cumsum(_frequencies(case))).to(DEV)
    rank = torch.searchsorted(cdf, torch.rand(T, generator=g, device=DEV, dtype=torch.float64)).clamp_(max=V - 1)
    ids = torch.randperm(V, generator=g, device=DEV)[rank].int()
    s = dict(case=case, ids=ids, scale=math.sqrt(D))
    if not case["back"]:
        s["w"] = (torch.randn(V, D, generator=g, device=DEV) * 0.02).to(DT[case["w_dtype"]])
        s["out"] = torch.empty(T, D + pad, dtype=DT[case["a_dtype"]], device=DEV)[:, :D]
    else:
        s["d"] = torch.empty(T, D + pad, dtype=DT[case["a_dtype"]], device=DEV)[:, :D]
        s["d"].copy_(torch.randn(T, D, generator=g, device=DEV) * 1e-4)
        s["dw"] = torch.randn(V, D, generator=g, device=DEV) * 1e-3  # what a tied head has left there
    if own:
        import paper_2608_16798_gb300.rl_loss as R

        s["ws"] = R.new_embedding_workspace(T, V, D)
    return s


def prepare(case, seed):
    return dict(sample=_prepare_sample, norm=_prepare_norm, embed=_prepare_embed)[case["kind"]](case, seed)


# ----------------------------------------------------------------------------- one pass

def _first(cond):
    """The lowest index along the rows at which `cond` holds (the row's length if none)."""
    n = cond.shape[1]
    return torch.where(cond, torch.arange(n, device=cond.device), n).amin(1)


def _sample_plain(s):
    z, V = s["z"].float(), s["case"]["V"]
    greedy = (s["temp"] <= 0)[:, None]
    t = torch.where(greedy, 1.0, s["temp"][:, None])
    x = (z - z.amax(1, keepdim=True)) / t
    e = x.exp()
    logp = (x - e.double().sum(1, keepdim=True).log()).float()
    # the order: the most likely first, the lower index first among equals
    order = z.sort(dim=1, descending=True, stable=True).indices
    srt = x.gather(1, order)
    at = torch.arange(V, device=DEV)
    live = (srt > -math.inf).sum(1, keepdim=True)
    k = s["top_k"].long()[:, None]
    n = torch.where(k > 0, torch.minimum(k, live), live)
    mass = torch.where(at < n, srt.exp(), 0.0).double()
    run = mass.cumsum(1)
    n_p = 1 + (run < s["top_p"][:, None] * run[:, -1:]).sum(1, keepdim=True)
    n_m = (srt.exp() >= s["min_p"][:, None]).sum(1, keepdim=True)
    n = torch.where(s["top_p"][:, None] < 1, torch.minimum(n, n_p), n)
    n = torch.where(s["min_p"][:, None] > 0, torch.minimum(n, n_m), n)
    n = torch.where(greedy, 1, n)
    kept = torch.empty_like(order, dtype=torch.bool).scatter_(1, order, at < n)
    run = torch.where(kept, e, 0.0).double().cumsum(1)
    tok = _first((run > s["u"][:, None] * run[:, -1:]) & kept).clamp(max=V - 1)[:, None]
    lp = logp.gather(1, tok)[:, 0]
    among = (x.gather(1, tok) - run[:, -1:].log())[:, 0]
    return dict(ids=tok[:, 0].int(), logp=lp, filtered_logp=among.float(), n_kept=n[:, 0].int())


def _norm_plain(s):
    case, x = s["case"], s["x"].float()
    if not case["back"]:
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = 1.0 / (c.square().mean(1) + NORM_EPS).sqrt()
        y = c * rstd[:, None] * s["w"]
        s["y"].copy_(y + s["b"] if s["b"] is not None else y)
        s["mean"].copy_(mean)
        s["rstd"].copy_(rstd)
        return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
    dy = s["dy"].float()
    if s["mask"] is not None:
        dy = dy * s["mask"][:, None]
    h = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["w"]
    dx = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * s["rstd"][:, None]
    s["dx"].copy_(dx)
    s["dw"].add_((dy * h).sum(0))
    if s["db"] is None:
        return dict(dx=s["dx"], dw=s["dw"])
    s["db"].add_(dy.sum(0))
    return dict(dx=s["dx"], dw=s["dw"], db=s["db"])


def _embed_plain(s):
    ids = s["ids"].long()
    if not s["case"]["back"]:
        s["out"].copy_(s["w"][ids].float() * s["scale"])
        return dict(out=s["out"])
    s["dw"].index_add_(0, ids, s["d"].float() * s["scale"])
    return dict(dw=s["dw"])


def run(s):
    case = s["case"]
    if not own:
        return dict(sample=_sample_plain, norm=_norm_plain, embed=_embed_plain)[case["kind"]](s)
    import paper_2608_16798_gb300.rl_loss as R

    if case["kind"] == "sample":
        ids, logp, among, kept = s["out"]
        R.rl_sample_tokens(s["z"], s["u"], s["params"], s["ws"], row_temperature=s["temp"], row_top_k=s["top_k"],
                           row_top_p=s["top_p"], row_min_p=s["min_p"], out_ids=ids, out_logp=logp,
                           out_filtered_logp=among, n_kept=kept)
        return dict(ids=ids, logp=logp, filtered_logp=among, n_kept=kept)
    if case["kind"] == "norm":
        if not case["back"]:
            R.rl_layer_norm_fwd(s["x"], weight=s["w"], bias=s["b"], eps=NORM_EPS, y=s["y"], mean=s["mean"], rstd=s["rstd"])
            return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        R.rl_layer_norm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["ws"], weight=s["w"], mask=s["mask"], d_x=s["dx"],
                            d_weight=s["dw"], d_bias=s["db"])
        out = dict(dx=s["dx"], dw=s["dw"])
        return out if s["db"] is None else dict(out, db=s["db"])
    if not case["back"]:
        R.rl_embedding_fwd(s["ids"], s["w"], s["ws"], scale=s["scale"], out=s["out"])
        return dict(out=s["out"])
    R.rl_embedding_bwd(s["ids"], s["d"], s["dw"], s["ws"], scale=s["scale"])
    return dict(dw=s["dw"])


# ----------------------------------------------------------------------------- what a pass cannot do without

def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["V"]
        return dict(bytes=float(n * _size(case["dtype"]) + 36 * case["rows"]), flops=4.0 * n)
    if case["kind"] == "norm":
        n, D = case["rows"] * case["D"], case["D"]
        sx, sy = _size(case["x_dtype"]), _size(case["y_dtype"])
        if not case["back"]:
            return dict(bytes=float(n * (sx + sy) + 8 * case["rows"] + 8 * D), flops=8.0 * n)
        t = case["trained"]
        return dict(bytes=float(n * (t * (sx + sy) + sx) + 8 * t * case["rows"] + 12 * D + (8 * D if case["bias"] else 0)),
                    flops=14.0 * n * t)
    T, D = case["T"], case["D"]
    used = float((1.0 - (1.0 - _frequencies(case)) ** T).sum())  # rows of the matrix that some token names
    if not case["back"]:
        return dict(bytes=used * D * _size(case["w_dtype"]) + T * D * _size(case["a_dtype"]) + 4.0 * T, flops=1.0 * T * D)
    return dict(bytes=used * D * 8.0 + T * D * _size(case["a_dtype"]) + 4.0 * T, flops=1.0 * T * D)


# ----------------------------------------------------------------------------- the results in 64 bits

def _exact_sample(case, seed):
    s = _prepare_sample(case, seed)
    temp, top_k, top_p, min_p = (s[k].tolist() for k in ("temp", "top_k", "top_p", "min_p"))
    u = s["u"].tolist()
    out = dict(ids=[], logp=[], filtered_logp=[], n_kept=[])
    for r in range(case["rows"]):
        x = s["z"][r].double()
        lp = torch.log_softmax(x / (temp[r] or 1.0), 0)
        p = lp.exp()
        if temp[r] == 0:
            n, tok = 1, int((x == x.max()).nonzero()[0])
            among = 0.0
        else:
            # by value, then by index
            order = torch.sort(-x, stable=True).indices
            p_o = p[order]
            n = int((x > -math.inf).sum())
            if 0 < top_k[r] < n:
                n = top_k[r]
            within = p_o[:n].cumsum(0)
            least = n
            if top_p[r] < 1:
                least = min(least, 1 + int((within < top_p[r] * within[-1]).sum()))
            if min_p[r] > 0:
                least = min(least, int((p_o >= min_p[r] * p_o[0]).sum()))
            n = least
            left = order[:n].sort().values
            cdf = p[left].cumsum(0)
            tok = int(left[int((cdf > u[r] * cdf[-1]).nonzero()[0])])
            among = float((p[tok] / cdf[-1]).log())
        out["ids"].append(tok)
        out["logp"].append(float(lp[tok]))
        out["filtered_logp"].append(among)
        out["n_kept"].append(n)
    return dict(ids=np.array(out["ids"], np.int64), logp=np.array(out["logp"]),
                filtered_logp=np.array(out["filtered_logp"]), n_kept=np.array(out["n_kept"], np.int64))


def _exact_norm(case, seed):
    s = _prepare_norm(case, seed)
    x, w = s["x"].double(), s["w"].double()
    if not case["back"]:
        var, mean = torch.var_mean(x, 1, correction=0)
        r = (var + NORM_EPS) ** -0.5
        y = torch.addcmul(torch.zeros_like(w) if s["b"] is None else s["b"].double(), (x - mean[:, None]) * r[:, None], w)
        return dict(y=y, mean=mean, rstd=r)
    # dx from the row's Jacobian: rstd (I - 1 1^T / D - h h^T / D) applied to w dy
    dy = s["dy"].double()
    if s["mask"] is not None:
        dy[s["mask"] == 0] = 0.0
    r = s["rstd"].double()[:, None]
    h = (x - s["mean"].double()[:, None]) * r
    v = dy * w
    D = case["D"]
    dx = r * (v - v.sum(1, keepdim=True) / D - h * torch.einsum("td,td->t", h, v)[:, None] / D)
    out = dict(dx=dx, dw=s["dw"].double() + torch.einsum("td,td->d", dy, h))
    if s["db"] is not None:
        out["db"] = s["db"].double() + torch.ones(case["rows"], dtype=torch.float64, device=DEV) @ dy
    return out


def _exact_embed(case, seed):
    s = _prepare_embed(case, seed)
    ids = s["ids"].long()
    if not case["back"]:
        return dict(out=torch.nn.functional.one_hot(ids, case["V"]).double() @ s["w"].double() * s["scale"]
                    if case["T"] * case["V"] < 1 << 22 else s["w"].double().index_select(0, ids) * s["scale"])
    # sums of consecutive runs of the tokens in the order of their ids
    out = s["dw"].double()
    srt, order = ids.sort()
    v, n = torch.unique_consecutive(srt, return_counts=True)
    for a, b in _chunks(case["D"], case["T"], 1 << 28):
        run = torch.zeros(case["T"] + 1, b - a, dtype=torch.float64, device=DEV)
        torch.cumsum(s["d"][:, a:b].double()[order], 0, out=run[1:])
        end = n.cumsum(0)
        out[v, a:b] += (run[end] - run[end - n]) * s["scale"]
    return dict(dw=out)


def exact(case, seed):
    return dict(sample=_exact_sample, norm=_exact_norm, embed=_exact_embed)[case["kind"]](case, seed)
