"""Two operators on either side of the policy loss, as cases that can be timed and compared.

  verify   verification of drafted tokens against the target's probabilities (``rl_verify_drafts``):
           the rollout that answers with tokens. Per sequence, drafted tokens are accepted while
           u q(x) < p(x); the first one that is not is replaced by a draw from max(p - q, 0), and a
           sequence whose tokens are all accepted gets one more from p. The emitted tokens carry
           their log-probabilities, which are the rollout log-probabilities of the loss.
  muon     the update that learns from the gradient (``rl_muon_update``): momentum, the update
           orthogonalised by Newton-Schulz products, and the step on the weights.

With ``own`` false a pass computes the operators in their plain form, elementary torch operations in
32 bits; with ``own`` true it makes the calls of the library's binding. ``exact`` states the results
in 64 bits.

The token that a given number selects is a whole number, so the given numbers are kept a little away
from the edges at which it changes (as the log-ratios of the policy loss are kept away from its clip
bounds): every correct implementation takes the same token.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ACCEPT_BAND = 1e-4   # relative distance of an acceptance number from p(x) / q(x)
CDF_BAND = 2e-5      # distance of a sampling number from the edges of its token's interval
LEAST_MASS = 6e-5    # tokens that a sampling number selects have at least this probability
NS_COEF = (3.4445, -4.7750, 2.0315)
NS_STEPS = 5
NS_EPS = 1e-7


def _verify(name, seqs, lo, hi, V, dtype, draft="logits", temp=1.0, std=2.0, noise=0.5, masked=0.0, pad=0):
    c = dict(kind="verify", seqs=seqs, lo=lo, hi=hi, V=V, dtype=dtype, draft=draft, temp=temp, std=std, noise=noise,
             masked=masked, pad=pad)
    return dict(c, name=name) if name else c


def _muon(name, batch, m, n, dtype, apply, nesterov=True, momentum=True, pad=0):
    c = dict(kind="muon", batch=batch, m=m, n=n, dtype=dtype, apply=apply, nesterov=nesterov, momentum=momentum,
             pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one rollout decoding by itself: five rows, latency counts
        _verify("verify_one_rollout", 1, 4, 4, 151936, "bf16"),
        # a small model's group of eight, at the smallest configuration's vocabulary
        _verify("verify_small_vocab", 8, 1, 5, 4096, "bf16", temp=0.7, std=3.0),
        # the multi-turn batch: all 128 rollouts decode together, four drafted tokens each
        _verify("verify_multiturn", 128, 4, 4, 151936, "bf16", noise=0.3),
        # drafts looked up in the prompt (no distribution of their own), none to eight a rollout
        _verify("verify_lookup", 256, 0, 8, 151936, "bf16", draft="ids", temp=0.8),
        # fp32 logits of a vocabulary with three added tokens, entries cut off by a filter, odd counts
        _verify("verify_filtered_f32", 61, 1, 7, 32003, "f32", masked=0.3, std=3.0),
        # nothing drafted: the draw of the next token of every rollout of a large batch
        _verify("sample_only", 509, 0, 0, 151936, "bf16"),
        # one small matrix: launches and latency
        _muon("muon_small", 1, 256, 256, "f32", False),
        # the square projections of the layers of a small model, stepped together
        _muon("muon_layers", 12, 1024, 1024, "bf16", True),
        # one square projection of the full hidden size: weights in fp32 and their bf16 copy
        _muon("muon_square", 1, 4096, 4096, "bf16", True),
        # an odd shape in a wider buffer, no momentum
        _muon("muon_odd", 1, 1000, 2777, "f32", False, momentum=False, pad=7),
        # the fp32 gradient of a small model's LM head as the fused head leaves it: tall
        _muon("muon_head", 1, 32000, 1024, "f32", False),
        # a wide projection of the full hidden size
        _muon("muon_wide", 1, 4096, 16384, "bf16", False, nesterov=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        V = _log_int(rng, 1000, 151936)
        if rng.random() < 0.5:
            V = V // 64 * 64
        dtype = rng.choice(["bf16", "bf16", "f32"])
        lo = rng.choice([0, 1, 2, 4])
        hi = lo + rng.choice([0, 0, 1, 3, 4])
        row = V * (2 if dtype == "bf16" else 4)
        most = max(1, int(320e6 / (row * (lo + hi + 1))))
        return _verify(None, min(_log_int(rng, 1, 512), most), lo, hi, V, dtype,
                       draft=rng.choice(["logits", "logits", "ids"]), temp=rng.choice([1.0, 1.0, 0.7, 0.6, 0.0]),
                       std=rng.choice([2.0, 3.0]), noise=rng.choice([0.2, 0.5, 0.8]), masked=rng.choice([0.0, 0.0, 0.3]),
                       pad=rng.choice([0, 0, 5, 64]))
    s = _log_int(rng, 64, 4096)
    if rng.random() < 0.5:
        s = s // 64 * 64
    apply = rng.random() < 0.5
    most = 3.5e7 if apply else 5.5e7  # elements
    long = int(s * math.exp(rng.uniform(0.0, math.log(12.0)))) if rng.random() < 0.7 else s
    long = min(long, 32000, int(most / s), int((4.0e12 / NS_STEPS - s ** 3) / (3.0 * s * s)))
    m, n = (s, long) if rng.random() < 0.5 else (long, s)
    batch = max(1, min(_log_int(rng, 1, 16), int(4.0e12 / _muon_flops(1, m, n)), int(most / (m * n))))
    return _muon(None, batch, m, n, rng.choice(["bf16", "f32"]), apply, nesterov=rng.random() < 0.7,
                 momentum=rng.random() < 0.8, pad=rng.choice([0, 0, 3, 64]))


# ----------------------------------------------------------------------------- inputs

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + stream * 7919) & 0x7FFFFFFFFFFF)
    return g


def _counts(case):
    """Drafted tokens of each sequence: the case's own, whatever the seed."""
    rng = np.random.default_rng([case["seqs"], case["lo"], case["hi"], case["V"]])
    return rng.integers(case["lo"], case["hi"] + 1, case["seqs"])


def _chunks(rows, V):
    step = max(1, (1 << 26) // V)
    return [(r, min(rows, r + step)) for r in range(0, rows, step)]


def _softmax64(z, temp):
    e = torch.exp((z.double() - z.amax(-1, keepdim=True).double()) / temp)
    return e / e.sum(-1, keepdim=True)


def _prepare_verify(case, seed):
    """Target rows N(0, std^2) in which half the rows have one likely token, as a language model's
    have; draft rows are the target's with noise, the drafted ids are drawn from them. Looked-up ids
    are the row's likely token four times in five, else any."""
    V, temp, std = case["V"], case["temp"], case["std"]
    K = _counts(case)
    nd, nr = int(K.sum()), int(K.sum()) + case["seqs"]
    offs = np.concatenate([[0], np.cumsum(K)])
    first_row = offs[:-1] + np.arange(case["seqs"])
    t_row = np.concatenate([np.arange(k) + r for k, r in zip(K, first_row)] + [np.zeros(0)]).astype(np.int64)
    dt, ld = DT[case["dtype"]], V + case["pad"]
    g = _gen(seed, 1)
    zt = torch.empty(nr, ld, dtype=dt, device=DEV)[:, :V]
    top = torch.randint(0, V, (nr,), generator=g, device=DEV)
    spike = math.log(V) + 0.5 * std * std
    for a, b in _chunks(nr, V):
        x = torch.randn(b - a, V, generator=g, device=DEV).mul_(std)
        if case["masked"]:
            x[torch.rand(b - a, V, generator=g, device=DEV) < case["masked"]] = -math.inf
        hot = torch.rand(b - a, generator=g, device=DEV) < 0.5
        v = spike + torch.rand(b - a, generator=g, device=DEV) * 7.0 - 2.0
        i = torch.arange(b - a, device=DEV)
        x[i, top[a:b]] = torch.where(hot, v, torch.full_like(v, 2.0 * std))
        zt[a:b] = x
    t_row_d = torch.from_numpy(t_row).to(DEV)
    ids = torch.empty(nd, dtype=torch.int64, device=DEV)
    px = torch.empty(nd, dtype=torch.float64, device=DEV)
    qx = torch.ones(nd, dtype=torch.float64, device=DEV)
    scale = temp if temp > 0 else 1.0
    zd = None
    if case["draft"] == "logits" and nd:
        zd = torch.empty(nd, ld, dtype=dt, device=DEV)[:, :V]
    for a, b in _chunks(nd, V):
        zr = zt[t_row_d[a:b]]
        if zd is not None:
            zd[a:b] = zr.float() + torch.randn(b - a, V, generator=g, device=DEV).mul_(case["noise"] * scale)
            e = torch.rand(b - a, V, generator=g, device=DEV).clamp_(min=1e-30).log_().neg_().log_().neg_()
            ids[a:b] = e.add_(zd[a:b].float() / scale).argmax(1)
            qx[a:b] = _softmax64(zd[a:b], scale).gather(1, ids[a:b, None])[:, 0]
        else:
            other = torch.randint(0, V, (b - a,), generator=g, device=DEV)
            ids[a:b] = torch.where(torch.rand(b - a, generator=g, device=DEV) < 0.8, top[t_row_d[a:b]], other)
        px[a:b] = _softmax64(zr, scale).gather(1, ids[a:b, None])[:, 0]
    # acceptance numbers, a little away from p(x) / q(x)
    ua = torch.rand(nd, generator=g, device=DEV, dtype=torch.float64)
    r = px / qx
    near = (ua - r).abs() <= ACCEPT_BAND * r
    ua = torch.where(near, torch.where(r < 0.9, r * (1 + 4 * ACCEPT_BAND) + 1e-6, r * (1 - 4 * ACCEPT_BAND)), ua)
    ua = ua.float().clamp_(max=1.0 - 2.0 ** -24)
    if temp > 0:
        no = (ua.double() * qx >= px).cpu().numpy()
    else:
        no = np.zeros(nd, bool)
    # sampling numbers, in the inside of the interval of a token of the last distribution
    us = torch.rand(case["seqs"], 2, generator=g, device=DEV, dtype=torch.float64)
    n_acc = np.array([next((j for j in range(k) if no[o + j]), k) for k, o in zip(K, offs)], dtype=np.int64)
    last = torch.from_numpy(first_row + n_acc).to(DEV)
    at = torch.from_numpy(np.where(n_acc < K, offs[:-1] + n_acc, -1)).to(DEV)
    u = torch.empty(case["seqs"], dtype=torch.float32, device=DEV)
    for a, b in _chunks(case["seqs"], V * 4):
        c = _softmax64(zt[last[a:b]], scale)
        if nd:
            has = (at[a:b] >= 0)[:, None]
            i = at[a:b].clamp(min=0)
            if zd is not None:
                q = _softmax64(zd[i], scale)
            else:
                q = torch.zeros_like(c).scatter_(1, ids[i][:, None], 1.0)
            c = torch.where(has, (c - q).clamp(min=0), c)
        c /= c.sum(1, keepdim=True)
        ok = torch.where(c >= LEAST_MASS, c, torch.zeros_like(c))
        pick = ok.cumsum(1)
        tok = torch.searchsorted(pick, us[a:b, :1] * pick[:, -1:], right=True).clamp_(max=V - 1)
        tok = torch.where(ok.gather(1, tok) > 0, tok, c.argmax(1, keepdim=True))
        hi = c.cumsum(1).gather(1, tok)[:, 0]
        mass = c.gather(1, tok)[:, 0]
        u[a:b] = (hi - mass + CDF_BAND + us[a:b, 1] * (mass - 2 * CDF_BAND).clamp(min=0)).float()
    s = dict(case=case, zt=zt, zd=zd, ids=ids.int(), offs=torch.from_numpy(offs.astype(np.int32)).to(DEV),
             ua=ua, us=u.clamp_(0.0, 1.0 - 2.0 ** -24), K=int(K.max(initial=0)))
    # the layout of the rows, as a program that packs ragged drafts has it
    s.update(t_row=t_row_d, first_row=torch.from_numpy(first_row).to(DEV), n=torch.from_numpy(K.astype(np.int64)).to(DEV))
    if own:
        import paper_2608_16798_gb300.rl_loss as R

        s.update(params=R.make_verify_params(temperature=temp), ws=R.new_workspace(nr, V),
                 out=(torch.empty(nr, dtype=torch.int32, device=DEV),
                      torch.empty(case["seqs"], dtype=torch.int32, device=DEV), torch.empty(nr, device=DEV)))
    return s


def _spectrum(u, v, g):
    """A sum of outer products whose sizes fall as 1 / k, over noise: what gradients look like."""
    rank = u.shape[2]
    w = (1.0 + torch.rand(rank, generator=g, device=DEV)) / torch.arange(1, rank + 1, device=DEV)
    return (u * w) @ v + torch.randn(u.shape[0], u.shape[1], v.shape[2], generator=g, device=DEV) * 0.05


def _prepare_muon(case, seed):
    B, m, n = case["batch"], case["m"], case["n"]
    g = _gen(seed, 2)
    rank = min(24, m, n)
    left = torch.randn(B, m, rank, generator=g, device=DEV)
    right = torch.randn(B, rank, n, generator=g, device=DEV)
    grad = torch.empty(B, m, n + case["pad"], dtype=DT[case["dtype"]], device=DEV)[:, :, :n]
    grad.copy_(_spectrum(left, right, g) * 1e-3)
    s = dict(case=case, grad=grad, lr=2e-5, wd=0.1, mu=0.95 if case["momentum"] else 0.0, scale=0.2 * math.sqrt(max(m, n)))
    if case["momentum"]:
        s["mom"] = _spectrum(left, right, g) * 8e-3
    if case["apply"]:
        s["w"] = torch.randn(B, m, n, generator=g, device=DEV) * 0.02
        s["wb"] = torch.empty(B, m, n, dtype=torch.bfloat16, device=DEV)
    else:
        s["upd"] = torch.empty(B, m, n, dtype=torch.bfloat16, device=DEV)
    if own:
        import paper_2608_16798_gb300.rl_loss as R

        s.update(ws=R.new_muon_workspace(B, m, n),
                 params=R.make_muon_params(lr=s["lr"], momentum=s["mu"], nesterov=case["nesterov"], weight_decay=s["wd"],
                                           update_scale=s["scale"], ns_coef=NS_COEF, ns_steps=NS_STEPS, eps=NS_EPS))
    return s


def prepare(case, seed):
    return _prepare_verify(case, seed) if case["kind"] == "verify" else _prepare_muon(case, seed)


# ----------------------------------------------------------------------------- one pass

def _softmax_rows(z, temp):
    """(probabilities, log-probabilities) of logits rows / temp, in 32 bits."""
    z = z.float()
    z = (z - z.amax(-1, keepdim=True)) / temp
    e = z.exp()
    s = e.sum(-1, keepdim=True)
    return e / s, z - s.log()


def _first(cond):
    """The lowest index along the rows at which `cond` holds (the row's length if none)."""
    n = cond.shape[1]
    return torch.where(cond, torch.arange(n, device=cond.device), n).amin(1)


def _verify_plain(s):
    case = s["case"]
    V, temp, n = case["V"], case["temp"], s["n"]
    B, nd = n.numel(), s["ids"].numel()
    zt, ids = s["zt"], s["ids"].long()
    p, logp = _softmax_rows(zt, temp if temp > 0 else 1.0)
    best = _first(zt == zt.amax(1, keepdim=True)) if temp == 0 else None
    if nd:
        q = None
        if temp == 0:
            yes = best[s["t_row"]] == ids
        else:
            px = p[s["t_row"], ids]
            if s["zd"] is None:
                yes = s["ua"] < px
            else:
                q, _ = _softmax_rows(s["zd"], temp)
                yes = s["ua"] * q.gather(1, ids[:, None])[:, 0] < px
        # the first refusal of each sequence, or the number of its drafted tokens
        j = torch.arange(s["K"], device=DEV)
        at = s["offs"][:-1, None].long() + j
        stop = (j >= n[:, None]) | ~yes[at.clamp(max=nd - 1)]
        n_acc = _first(stop).clamp(max=s["K"])
    else:
        n_acc = torch.zeros(B, dtype=torch.int64, device=DEV)
    last = s["first_row"] + n_acc
    if temp == 0:
        tok = best[last]
    else:
        r = p[last]
        if nd:
            refused = (n_acc < n)[:, None]
            i = (s["offs"][:-1].long() + n_acc).clamp(max=nd - 1)
            sub = q[i] if q is not None else (torch.arange(V, device=DEV) == ids[i][:, None]).float()
            r = torch.where(refused, (r - sub).clamp(min=0), r)
        # sums of blocks first, so that 32 bits hold the running sum of a long row
        pad = torch.zeros(B, -(-V // 512) * 512, device=DEV)
        pad[:, :V] = r
        pad = pad.view(B, -1, 512)
        block = pad.sum(2)
        run = block.cumsum(1)
        cdf = (pad.cumsum(2) + (run - block)[:, :, None]).view(B, -1)[:, :V]
        tok = _first((cdf > s["us"][:, None] * run[:, -1:]) & (r > 0)).clamp(max=V - 1)
    # what is emitted: the accepted tokens, then the one drawn
    row = torch.arange(zt.shape[0], device=DEV)
    seq = torch.searchsorted(s["first_row"], row, right=True) - 1
    pos = row - s["first_row"][seq]
    drafted = ids[(s["offs"][seq].long() + pos).clamp(max=max(nd - 1, 0))] if nd else torch.zeros_like(row)
    out = torch.where(pos < n_acc[seq], drafted, torch.where(pos == n_acc[seq], tok[seq], -1))
    lp = torch.where(out >= 0, logp.gather(1, out.clamp(min=0)[:, None])[:, 0], 0.0)
    return dict(ids=out.int(), n_accepted=n_acc.int(), logp=lp)


def _muon_plain(s):
    case = s["case"]
    a, b, c = NS_COEF
    u = g = s["grad"].float()
    if case["momentum"]:
        s["mom"].mul_(s["mu"]).add_(g)
        u = g + s["mu"] * s["mom"] if case["nesterov"] else s["mom"]
    x = u / (u.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    tall = case["m"] > case["n"]
    x = x.transpose(1, 2) if tall else x
    for _ in range(NS_STEPS):
        y = x @ x.transpose(1, 2)
        x = a * x + (b * y + c * (y @ y)) @ x
    x = x.transpose(1, 2) if tall else x
    out = dict(momentum=s["mom"]) if case["momentum"] else {}
    if not case["apply"]:
        s["upd"].copy_(x * s["scale"])
        return dict(out, update=s["upd"])
    s["w"].mul_(1.0 - s["lr"] * s["wd"]).sub_(x * (s["lr"] * s["scale"]))
    s["wb"].copy_(s["w"])
    return dict(out, weights=s["w"], weights_bf16=s["wb"])


def run(s):
    case = s["case"]
    if not own:
        return _verify_plain(s) if case["kind"] == "verify" else _muon_plain(s)
    import paper_2608_16798_gb300.rl_loss as R

    if case["kind"] == "verify":
        ids, n_acc, logp = R.rl_verify_drafts(s["zt"], s["ids"], s["offs"], s["ua"], s["us"], s["K"], s["params"],
                                              s["ws"], draft_logits=s["zd"], out_ids=s["out"][0], n_accepted=s["out"][1],
                                              out_logp=s["out"][2])
        return dict(ids=ids, n_accepted=n_acc, logp=logp)
    R.rl_muon_update(s["grad"], s["params"], s["ws"], momentum=s.get("mom"), weights=s.get("w"),
                     weights_bf16=s.get("wb"), update=s.get("upd"))
    out = dict(momentum=s["mom"]) if case["momentum"] else {}
    if not case["apply"]:
        return dict(out, update=s["upd"])
    return dict(out, weights=s["w"], weights_bf16=s["wb"])


# ----------------------------------------------------------------------------- what a pass cannot do without

def _muon_flops(batch, m, n):
    """Each step: the symmetric product X X^T and the symmetric square of it (half their elements
    each), and the product with X."""
    s, l = min(m, n), max(m, n)
    return batch * NS_STEPS * (3.0 * s * s * l + 1.0 * s ** 3)


def work(case):
    if case["kind"] == "verify":
        es = 2 if case["dtype"] == "bf16" else 4
        # rows after a sequence's first refusal need not be read: the expected number of the others,
        # by the rate at which a drafted token is accepted (the noise is felt in the rows without a likely token)
        if case["draft"] == "logits" and case["temp"] > 0:
            alpha = 1.0 - 0.6 * math.erf(case["noise"] / 2.0 / math.sqrt(2.0))
        else:
            alpha = 0.35
        K = _counts(case)
        tested = sum(float((1 - alpha ** k) / (1 - alpha)) for k in K)
        rows = tested + sum(alpha ** int(k) for k in K)
        if case["draft"] == "logits" and case["temp"] > 0:
            rows += tested
        return dict(bytes=rows * case["V"] * es + 20.0 * (int(K.sum()) + case["seqs"]), flops=rows * case["V"] * 4.0)
    B, m, n = case["batch"], case["m"], case["n"]
    es = 2 if case["dtype"] == "bf16" else 4
    per = es + (8 if case["momentum"] else 0) + (10 if case["apply"] else 2)
    return dict(bytes=float(B * m * n * per), flops=_muon_flops(B, m, n))


# ----------------------------------------------------------------------------- the results in 64 bits

def _exact_verify(case, seed):
    s = _prepare_verify(case, seed)
    zt, zd, ids = s["zt"], s["zd"], s["ids"].tolist()
    offs, ua, us = s["offs"].tolist(), s["ua"].double().tolist(), s["us"].double().tolist()
    V, T = case["V"], case["temp"]
    out_ids, out_lp, out_n = [], [], []
    for b in range(case["seqs"]):
        k, got, lps, tok = offs[b + 1] - offs[b], [], [], -1
        for j in range(k + 1):
            z = zt[offs[b] + b + j].double()
            lp = torch.log_softmax(z / (T or 1.0), 0)
            p = lp.exp()
            if T == 0:
                tok = int((z == z.max()).nonzero()[0])
                if j < k and ids[offs[b] + j] == tok:
                    got.append(tok)
                    lps.append(float(lp[tok]))
                    continue
            elif j < k:
                x = ids[offs[b] + j]
                if zd is None:
                    q = torch.zeros_like(p)
                    q[x] = 1.0
                else:
                    q = torch.softmax(zd[offs[b] + j].double() / T, 0)
                if ua[offs[b] + j] * float(q[x]) < float(p[x]):
                    got.append(x)
                    lps.append(float(lp[x]))
                    continue
                p = (p - q).clamp(min=0)
            if T > 0:
                cdf = p.cumsum(0)
                tok = int(((cdf > us[b] * cdf[-1]) & (p > 0)).nonzero()[0])
            out_n.append(len(got))
            got.append(tok)
            lps.append(float(lp[tok]))
            break
        out_ids += got + [-1] * (k + 1 - len(got))
        out_lp += lps + [0.0] * (k + 1 - len(lps))
    return dict(ids=np.array(out_ids, np.int64), n_accepted=np.array(out_n, np.int64), logp=np.array(out_lp))


def _exact_muon(case, seed):
    s = _prepare_muon(case, seed)
    a, b, c = NS_COEF
    g = s["grad"].double()
    out = {}
    u = g
    if case["momentum"]:
        buf = s["mu"] * s["mom"].double() + g
        u = g + s["mu"] * buf if case["nesterov"] else buf
        out["momentum"] = buf
    o = torch.empty_like(u)
    for i in range(case["batch"]):  # one matrix at a time, on its shorter side
        x = u[i] / (torch.linalg.norm(u[i]) + NS_EPS)
        x = x.T if case["m"] > case["n"] else x
        for _ in range(NS_STEPS):
            y = x @ x.T
            x = a * x + b * (y @ x) + c * (y @ (y @ x))
        o[i] = x.T if case["m"] > case["n"] else x
    if not case["apply"]:
        return dict(out, update=s["scale"] * o)
    w = s["w"].double()
    w = w - s["lr"] * (s["wd"] * w + s["scale"] * o)
    return dict(out, weights=w, weights_bf16=w)


def exact(case, seed):
    return _exact_verify(case, seed) if case["kind"] == "verify" else _exact_muon(case, seed)
