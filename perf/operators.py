"""The operators of a model's head over a table of rows, as cases that can be timed.

Two operators, each in both directions:

  norm, norm_grad    layer norm of hidden states, the last step of the encoder that
                     the queries come from, and its gradients (input, weight, bias).
  score, score_grad  log probabilities of given rows under the softmax of all rows'
                     scores scale <q, x> + bias, the softmax' entropy, its largest
                     alternatives; and the gradients of the queries, of the rows and
                     of the bias: the full-softmax loss that encoders are trained with.

`own` selects between the plain form (elementary torch operations in 32 bits,
in 64 where rows have to be put in order) and the framework's kernels.  Rows are
unit-norm mixtures like the repository's inner-product workloads, queries lie
near the row that is asked for, and the scale is an inverse temperature.
"""
import math

import torch

own = False

DEV = "cuda"
PAD = -1            # ANN_PAD_ID as int32: no row is given
EPS = 1e-5
NEAR = 8            # rows beyond k that the plain form puts in order in 64 bits
CHUNK = 1 << 28     # scores that the plain form holds at a time
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def _norm(name, n, d, dtype, grad=False, **more):
    case = dict(name=name, kind="norm_grad" if grad else "norm", n=n, d=d, dtype=dtype, weight="same", affine=True, pad=0)
    case.update(more)
    return case


def _score(name, nq, n, d, dtype, k=0, grad=False, **more):
    case = dict(name=name, kind="score_grad" if grad else "score", nq=nq, n=n, d=d, dtype=dtype, k=k, entropy=True, bias="none", scale=20.0,
                pad=0)
    if grad:
        case["rows_grad"] = True
    case.update(more)
    return case


def listed():
    return [
        # one query's hidden state on its way to a search: a launch
        _norm("norm_one_768", 1, 768, "bf16"),
        # a corpus of long rows that is normalised before it is encoded, 32 bits
        _norm("norm_200k_960", 200_000, 960, "f32"),
        # a training batch of token states: both gradients' reductions, 16 bits with 32-bit weights
        _norm("norm_grad_80k_768", 80_000, 768, "bf16", grad=True, weight="f32"),
        # odd sizes and a row stride of its own, half precision
        _norm("norm_grad_5003_100", 5_003, 100, "f16", grad=True, pad=4),
        # one query answered with its ten likeliest rows of the headline workload's table: bound by reading the rows
        _score("score_one_1m_128", 1, 1_000_000, 128, "bf16", k=10),
        # a few requests over long rows with a bias per row and rows left out, 32 bits
        _score("score_8_200k_960", 8, 200_000, 960, "f32", k=5, bias="holes"),
        # the headline workload's batch and table: the largest; as many exponentials as scores
        _score("score_10k_1m_128", 10_000, 1_000_000, 128, "bf16", k=10),
        # a batch over long rows, half precision: the matrix cores count
        _score("score_4k_100k_768", 4_000, 100_003, 768, "f16", k=20),
        # a fine-tuning step of the encoder: queries' gradient only, entropy as a regulariser
        _score("score_grad_256_50k_96", 256, 50_000, 96, "bf16", grad=True, rows_grad=False),
        # a training step of both towers on short rows: gradients of queries and rows
        _score("score_grad_4k_100k_128", 4_096, 100_000, 128, "bf16", grad=True, entropy=False),
        # the same on long rows, half precision with a loss scale
        _score("score_grad_2k_50k_768", 2_048, 50_000, 768, "f16", grad=True),
        # odd sizes, 32 bits, bias with rows left out and its gradient
        _score("score_grad_513_20k_100", 513, 20_011, 100, "f32", grad=True, bias="holes", pad=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "score", "score", "score_grad", "score_grad"])
    dtype = rng.choice(list(TYPES))
    if kind.startswith("norm"):
        d = rng.choice([96, 100, 128, 768, 960, _log_int(rng, 16, 8192)])
        n = _log_int(rng, 1, min(200_000, 192_000_000 // d))
        return _norm("", n, d, dtype, grad=kind == "norm_grad", weight=rng.choice(["same", "f32"]), affine=rng.random() < 0.8,
                     pad=rng.choice([0, 0, 1, 8]))
    grad = kind == "score_grad"
    # (a few rows of a few dimensions leave nothing but the rounding of probabilities near one)
    d = rng.choice([96, 100, 128, 768, 960, _log_int(rng, 16, 1024)])
    n = _log_int(rng, 64, 200_000 if grad else 1_000_000)
    nq = _log_int(rng, 1, 4_096 if grad else 10_000)
    nq = max(1, min(nq, (100_000_000_000 if grad else 400_000_000_000) // (n * d), (400_000_000 if grad else 4_000_000_000) // n))
    more = dict(bias=rng.choice(["none", "none", "plain", "holes"]), entropy=rng.random() < 0.7, pad=rng.choice([0, 0, 0, 1, 8]),
                scale=rng.choice([1.0, 10.0, 20.0]))
    if grad:
        more["rows_grad"] = rng.random() < 0.7
    else:
        more["k"] = min(n, rng.choice([0, 1, 5, 10, 20, 32]))
    case = _score("", nq, n, d, dtype, grad=grad, **more)
    return case


# ------------------------------------------------------------------ what a program has in hand
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _padded(x, pad):
    """x with a row stride of its own: a view into a wider array."""
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _norm_inputs(case, g):
    n, d, t = case["n"], case["d"], TYPES[case["dtype"]]
    wt = t if case["weight"] == "same" else torch.float32
    # hidden states: every dimension with a spread and an offset of its own
    spread = torch.exp(0.5 * torch.randn(d, generator=g, device=DEV))
    offset = torch.randn(d, generator=g, device=DEV)
    s = dict(x=_padded(torch.randn(n, d, generator=g, device=DEV).mul_(spread).add_(offset).to(t), case["pad"]), weight=None, bias=None)
    if case["affine"]:
        s["weight"] = (1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(wt)
        s["bias"] = (0.2 * torch.randn(d, generator=g, device=DEV)).to(wt)
    if case["kind"] == "norm":
        s["y"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"])
        s["mean"], s["rstd"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        return s
    s["dy"] = _padded(torch.randn(n, d, generator=g, device=DEV).to(t), case["pad"])
    x64 = s["x"].double()
    mean = x64.mean(1)
    s["mean"], s["rstd"] = mean.float(), ((x64 - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
    s["dx"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"])
    if case["affine"]:
        s["dweight"], s["dbias"] = torch.empty(d, dtype=wt, device=DEV), torch.empty(d, dtype=wt, device=DEV)
    return s


def _score_inputs(case, g):
    nq, n, d, t = case["nq"], case["n"], case["d"], TYPES[case["dtype"]]
    clusters = max(8, n // 1000)
    centres = torch.randn(clusters, d, generator=g, device=DEV)

    def unit(v):
        return v / v.norm(dim=1, keepdim=True).clamp_min(1e-6)

    of = torch.randint(clusters, (n,), generator=g, device=DEV)
    rows = unit(centres[of] + 0.3 * torch.randn(n, d, generator=g, device=DEV))
    target = torch.randint(n, (nq,), generator=g, device=DEV)
    q = unit(rows[target] + 0.3 / math.sqrt(d) * torch.randn(nq, d, generator=g, device=DEV))
    s = dict(q=_padded(q.to(t), case["pad"]), rows=_padded(rows.to(t), case["pad"]), bias=None)
    if case["bias"] != "none":
        s["bias"] = 0.5 * torch.randn(n, generator=g, device=DEV)
    if case["bias"] == "holes":
        s["bias"][torch.rand(n, generator=g, device=DEV) < 0.05] = -math.inf
        s["bias"][0] = 0.0
        target[s["bias"][target] == -math.inf] = 0
    if nq > 4:
        target[nq // 2] = PAD
    s["target"] = target.int()
    if case["kind"] == "score":
        s["logprob"], s["lse"] = torch.empty(nq, device=DEV), torch.empty(nq, device=DEV)
        s["entropy"] = torch.empty(nq, device=DEV) if case["entropy"] else None
        s["alt_ids"] = torch.empty(nq, case["k"], dtype=torch.int32, device=DEV) if case["k"] else None
        s["alt_logprob"] = torch.empty(nq, case["k"], device=DEV) if case["k"] else None
        return s
    # the forward pass' statistics, and the loss' gradient: mean over a few, scaled as half precision asks for
    lse, entropy = torch.empty(nq, device=DEV), torch.empty(nq, device=DEV)
    for b, e in _chunks(nq, n, 8):
        z = s["q"][b:e].double() @ s["rows"].double().T
        z *= case["scale"]
        if s["bias"] is not None:
            z += s["bias"].double()
        lse[b:e] = torch.logsumexp(z, 1)
        logp = z - torch.logsumexp(z, 1, keepdim=True)
        entropy[b:e] = -(logp.exp() * logp.masked_fill(logp == -math.inf, 0.0)).sum(1)
        del z, logp
    s["lse"], s["entropy"] = lse, entropy
    s["g_logprob"] = -0.5 - torch.rand(nq, generator=g, device=DEV)
    s["g_entropy"] = 0.1 * torch.randn(nq, generator=g, device=DEV) if case["entropy"] else None
    s["dq"] = _padded(torch.empty(nq, d, dtype=t, device=DEV), case["pad"])
    s["drows"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"]) if case["rows_grad"] else None
    s["dbias"] = torch.empty(n, device=DEV) if case["rows_grad"] and s["bias"] is not None else None
    return s


def _workspace(nbytes):
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    make = _norm_inputs if case["kind"].startswith("norm") else _score_inputs
    s = make(case, _generator(seed))
    s["case"] = case
    if own:
        import paper_2503_17911_amd as ann
        n, d = case["n"], case["d"]
        if case["kind"] == "norm_grad":
            s["workspace"] = _workspace(ann.ann_layer_norm_backward_workspace(n, d))
        elif case["kind"] == "score":
            s["workspace"] = _workspace(ann.ann_row_logprobs_workspace(case["nq"], n, d, _ann_type(ann, case["dtype"]), case["k"]))
        elif case["kind"] == "score_grad":
            s["workspace"] = _workspace(ann.ann_row_logprobs_backward_workspace(case["nq"], n, d, _ann_type(ann, case["dtype"])))
    return s


# ------------------------------------------------------------------ plain forms
def _chunks(nq, n, bytes_each=4):
    step = max(1, CHUNK * 4 // bytes_each // max(n, 1))
    return [(b, min(nq, b + step)) for b in range(0, nq, step)]


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    centred = x - mean[:, None]
    rstd = 1.0 / torch.sqrt(centred.square().mean(1) + EPS)
    y = centred * rstd[:, None]
    if s["weight"] is not None:
        y = y * s["weight"].float() + s["bias"].float()
    return dict(y=y.to(s["x"].dtype), mean=mean, rstd=rstd)


def _plain_norm_grad(s):
    t = s["x"].dtype
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    a = dy if s["weight"] is None else dy * s["weight"].float()
    dx = s["rstd"][:, None] * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    out = dict(dx=dx.to(t))
    if s["weight"] is not None:
        out["dweight"] = (dy * xh).sum(0).to(s["weight"].dtype)
        out["dbias"] = dy.sum(0).to(s["weight"].dtype)
    return out


def _plain_scores(q, rows, scale, bias):
    z = (q @ rows.T) * scale
    return z if bias is None else z + bias


def _plain_score(s):
    case, rows, bias = s["case"], s["rows"].float(), s["bias"]
    nq, n, k, scale = case["nq"], case["n"], case["k"], case["scale"]
    logprob, lse, entropy = (torch.empty(nq, device=DEV) for _ in range(3))
    ids = torch.full((nq, k), PAD, dtype=torch.int32, device=DEV)
    alt = torch.full((nq, k), -math.inf, device=DEV)
    for b, e in _chunks(nq, n):
        q = s["q"][b:e].float()
        z = _plain_scores(q, rows, scale, bias)
        top = z.max(1, keepdim=True).values
        if k:
            near = z.topk(min(n, k + NEAR), 1).indices.sort(1).values
            part = max(1, CHUNK // (near.shape[1] * case["d"]) // 2)
            for c in range(0, e - b, part):
                at = near[c:c + part]
                z64 = (s["q"][b + c:min(e, b + c + part)].double()[:, None, :] * s["rows"][at].double()).sum(2) * scale
                if bias is not None:
                    z64 = z64 + bias[at].double()
                z64, order = z64.sort(dim=1, descending=True, stable=True)
                at = at.gather(1, order)[:, :k].int()
                z64 = z64[:, :k]
                alt[b + c:b + c + len(at)] = z64.float()
                ids[b + c:b + c + len(at)] = at.masked_fill(z64 == -math.inf, PAD)
        given = s["target"][b:e].long()
        z -= top
        picked = z.gather(1, given.clamp_min(0)[:, None])[:, 0]
        p = z.exp()
        total = p.sum(1)
        lse[b:e] = top[:, 0] + total.log()
        logprob[b:e] = torch.where(given < 0, torch.zeros_like(picked), picked - total.log())
        if case["entropy"]:
            entropy[b:e] = total.log() - (p * (z if bias is None else z.clamp_min(-1e30))).sum(1) / total
        if k:
            alt[b:e] -= lse[b:e, None]
    out = dict(logprob=logprob, lse=lse)
    if case["entropy"]:
        out["entropy"] = entropy
    if k:
        out.update(alt_ids=ids, alt_logprob=alt)
    return out


def _plain_score_grad(s):
    case, rows, bias, scale = s["case"], s["rows"].float(), s["bias"], s["case"]["scale"]
    nq, n, t = case["nq"], case["n"], s["q"].dtype
    dq = torch.empty(nq, case["d"], device=DEV)
    drows = torch.zeros(n, case["d"], device=DEV) if s["drows"] is not None else None
    dbias = torch.zeros(n, device=DEV) if s["dbias"] is not None else None
    for b, e in _chunks(nq, n):
        q = s["q"][b:e].float()
        logp = _plain_scores(q, rows, scale, bias) - s["lse"][b:e, None]
        p = logp.exp()
        given = s["target"][b:e].long()
        g = torch.where(given < 0, torch.zeros_like(s["lse"][b:e]), s["g_logprob"][b:e])
        dz = p * -g[:, None]
        if s["g_entropy"] is not None:
            if bias is not None:
                logp = logp.clamp_min(-1e30)
            dz -= s["g_entropy"][b:e, None] * p * (logp + s["entropy"][b:e, None])
        dz.scatter_add_(1, given.clamp_min(0)[:, None], g[:, None])
        dq[b:e] = (dz @ rows) * scale
        if drows is not None:
            drows += (dz.T @ q) * scale
        if dbias is not None:
            dbias += dz.sum(0)
    out = dict(dq=dq.to(t))
    if drows is not None:
        out["drows"] = drows.to(t)
    if dbias is not None:
        out["dbias"] = dbias
    return out


# ------------------------------------------------------------------ the framework's calls
def _ann_type(ann, dtype):
    return {"f32": ann.F32, "f16": ann.F16, "bf16": ann.BF16}[dtype]


def _own(s):
    import paper_2503_17911_amd as ann
    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    n, d, kind, t = case["n"], case["d"], case["kind"], _ann_type(ann, case["dtype"])
    if kind.startswith("norm"):
        wt = t if case["weight"] == "same" else ann.F32
        if kind == "norm":
            ann.ann_layer_norm(s["x"], n, d, s["x"].stride(0), t, s["weight"], s["bias"], wt, EPS, s["y"], s["y"].stride(0), s["mean"],
                               s["rstd"], stream)
            return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        dw, db = s.get("dweight"), s.get("dbias")
        ann.ann_layer_norm_backward(s["dy"], s["dy"].stride(0), s["x"], s["x"].stride(0), n, d, t, s["weight"], wt, s["mean"], s["rstd"],
                                    s["dx"], s["dx"].stride(0), dw, db, s["workspace"], s["workspace"].numel(), stream)
        return dict(dx=s["dx"]) if dw is None else dict(dx=s["dx"], dweight=dw, dbias=db)
    table = dict(q=s["q"], nq=case["nq"], q_stride=s["q"].stride(0), rows=s["rows"], n=n, row_stride=s["rows"].stride(0), d=d, type=t,
                 scale=case["scale"], row_bias=s["bias"], targets=s["target"])
    if kind == "score":
        ann.ann_row_logprobs(**table, k=case["k"], logprob=s["logprob"], entropy=s["entropy"], lse=s["lse"], alt_ids=s["alt_ids"],
                             alt_logprobs=s["alt_logprob"], workspace=s["workspace"], workspace_bytes=s["workspace"].numel(), stream=stream)
        out = dict(logprob=s["logprob"], lse=s["lse"])
        if case["entropy"]:
            out["entropy"] = s["entropy"]
        if case["k"]:
            out.update(alt_ids=s["alt_ids"], alt_logprob=s["alt_logprob"])
        return out
    ann.ann_row_logprobs_backward(**table, lse=s["lse"], entropy=s["entropy"], g_logprob=s["g_logprob"], g_entropy=s["g_entropy"],
                                  dq=s["dq"], dq_stride=s["dq"].stride(0), drows=s["drows"],
                                  drows_stride=s["drows"].stride(0) if s["drows"] is not None else 0, drow_bias=s["dbias"],
                                  workspace=s["workspace"], workspace_bytes=s["workspace"].numel(), stream=stream)
    out = dict(dq=s["dq"])
    if s["drows"] is not None:
        out["drows"] = s["drows"]
    if s["dbias"] is not None:
        out["dbias"] = s["dbias"]
    return out


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "score": _plain_score, "score_grad": _plain_score_grad}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    n, d = case["n"], case["d"]
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("norm"):
        wsize = 4 if case["weight"] == "f32" else size
        affine = 2 * d * wsize if case["affine"] else 0
        if case["kind"] == "norm":
            return dict(bytes=2 * n * d * size + 8 * n + affine, flops=8 * n * d)
        return dict(bytes=3 * n * d * size + 8 * n + (affine * 3 // 2 if case["affine"] else 0), flops=15 * n * d)
    nq = case["nq"]
    read = (nq + n) * d * size + 4 * nq + (4 * n if case["bias"] != "none" else 0)
    if case["kind"] == "score":
        return dict(bytes=read + (12 if case["entropy"] else 8) * nq + 8 * nq * case["k"], flops=2 * nq * n * d)
    written = nq * d * size
    if case["rows_grad"]:
        written += n * d * size + (4 * n if case["bias"] != "none" else 0)
    return dict(bytes=read + written + (16 if case["entropy"] else 8) * nq, flops=(6 if case["rows_grad"] else 4) * nq * n * d)


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_norm(s):
    x = s["x"].to(torch.float64)
    n, d = x.shape
    if s["case"]["kind"] == "norm":
        mean = x.sum(1) / d
        var = ((x - mean.unsqueeze(1)) ** 2).sum(1) / d
        rstd = (var + EPS) ** -0.5
        y = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
        if s["weight"] is not None:
            y = torch.addcmul(s["bias"].to(torch.float64), y, s["weight"].to(torch.float64))
        return dict(y=y, mean=mean, rstd=rstd)
    mean, rstd, dy = (s[f].to(torch.float64) for f in ("mean", "rstd", "dy"))
    out = {}
    up = dy
    xh = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
    if s["weight"] is not None:
        out["dweight"] = torch.einsum("nd,nd->d", dy, xh)
        out["dbias"] = dy.sum(0)
        up = dy * s["weight"].to(torch.float64)
    along = torch.einsum("nd,nd->n", up, xh) / d
    dx = rstd.unsqueeze(1) * (up - (up.sum(1) / d).unsqueeze(1) - along.unsqueeze(1) * xh)
    return dict(dx=dx, **out)


def _exact_score(s):
    case = s["case"]
    nq, n, k = case["nq"], case["n"], case["k"]
    rows_t = s["rows"].to(torch.float64).t().contiguous()
    parts = []
    step = max(1, (1 << 27) // n)
    for i in range(0, nq, step):
        z = torch.mm(s["q"][i:i + step].to(torch.float64), rows_t).mul_(case["scale"])
        if s["bias"] is not None:
            z.add_(s["bias"].to(torch.float64))
        lse = torch.logsumexp(z, dim=1)
        t = s["target"][i:i + step].to(torch.int64)
        one = dict(logprob=torch.where(t >= 0, z[torch.arange(len(t), device=DEV), t.clamp(min=0)] - lse, 0.0), lse=lse)
        if k:
            # the largest k, equal ones by their number: candidates in the order of their numbers, then a stable order by value
            val, at = torch.topk(z, min(n, k + 2 * NEAR), dim=1)
            at, by_id = torch.sort(at, dim=1)
            val, by_val = torch.sort(val.gather(1, by_id), dim=1, descending=True, stable=True)
            at = at.gather(1, by_val)
            one["alt_logprob"] = val[:, :k] - lse.unsqueeze(1)
            one["alt_ids"] = torch.where(torch.isinf(val[:, :k]), PAD, at[:, :k]).to(torch.int32)
        if case["entropy"]:
            z.sub_(lse.unsqueeze(1))
            one["entropy"] = torch.special.entr(z.exp_()).sum(1)
        parts.append(one)
        del z
    out = {f: torch.cat([p[f] for p in parts]) for f in parts[0]}
    order = ["logprob", "lse"] + (["entropy"] if case["entropy"] else []) + (["alt_ids", "alt_logprob"] if k else [])
    return {f: out[f] for f in order}


def _exact_score_grad(s):
    case = s["case"]
    nq, n, d = case["nq"], case["n"], case["d"]
    rows = s["rows"].to(torch.float64)
    dq = torch.zeros(nq, d, dtype=torch.float64, device=DEV)
    drows = torch.zeros(n, d, dtype=torch.float64, device=DEV)
    dbias = torch.zeros(n, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 27) // n)
    for i in range(0, nq, step):
        at = slice(i, min(nq, i + step))
        q = s["q"][at].to(torch.float64)
        z = torch.mm(q, rows.t()) * case["scale"]
        if s["bias"] is not None:
            z = z + s["bias"].to(torch.float64)
        z = z - s["lse"][at].to(torch.float64).unsqueeze(1)
        p = torch.exp(z)
        there = s["target"][at] >= 0
        g = s["g_logprob"][at].to(torch.float64) * there
        grad = -p * g.unsqueeze(1)
        if s["g_entropy"] is not None:
            slope = torch.where(p > 0, p * (z + s["entropy"][at].to(torch.float64).unsqueeze(1)), 0.0)
            grad = grad - s["g_entropy"][at].to(torch.float64).unsqueeze(1) * slope
        lines = torch.nonzero(there).squeeze(1)
        grad[lines, s["target"][at][lines].to(torch.int64)] += g[lines]
        dq[at] = torch.mm(grad, rows) * case["scale"]
        if s["drows"] is not None:
            drows += torch.mm(grad.t(), q) * case["scale"]
        dbias += grad.sum(0)
    out = dict(dq=dq)
    if s["drows"] is not None:
        out["drows"] = drows
    if s["dbias"] is not None:
        out["dbias"] = dbias
    return out


def exact(case, seed):
    make = _norm_inputs if case["kind"].startswith("norm") else _score_inputs
    s = make(case, _generator(seed))
    s["case"] = case
    if case["kind"].startswith("norm"):
        return _exact_norm(s)
    return _exact_score(s) if case["kind"] == "score" else _exact_score_grad(s)
