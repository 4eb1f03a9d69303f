"""More operators of the model that the queries come from, as cases that can be timed.

Three operators, each in both directions:

  embed, embed_grad      the encoder's first step: rows of a table of token embeddings
                         times a scale, and the table's gradient.
  rms, rms_grad          the norm between its layers: root-mean-square norm of the sum of
                         a layer's output and the residual, the sum itself, and their
                         gradients; "rms" with a group also in 8 bits (e4m3) with a scale
                         to every group of columns, as a product in 8 bits takes it.
  distill, distill_grad  its loss where a larger encoder teaches it: how far the softmax of
                         all rows' scores scale <q, x> + bias is from the teacher's k
                         likeliest rows and their probabilities; gradients of the queries,
                         of the rows and of the bias.

`own` selects between the plain form (elementary torch operations in 32 bits) and
the framework's kernels.  Tokens are drawn by Zipf's law with a few that are
padding; rows are unit-norm mixtures like the repository's inner-product
workloads; the teacher's queries are less noisy ones than the student's.
"""
import math

import torch

own = False

DEV = "cuda"
PAD = -1            # ANN_PAD_ID as int32: no token, no row
EPS = 1e-6
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -100   # a group's largest value counts as this at least
CHUNK = 1 << 28     # scores that the plain form holds at a time
PART = 1000         # rows that it sums at a time
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def _embed(name, n, d, rows, dtype, grad=False, **more):
    return dict(dict(name=name, kind="embed_grad" if grad else "embed", n=n, d=d, rows=rows, dtype=dtype, table="same", scale=math.sqrt(d), pad=0), **more)


def _rms(name, n, d, dtype, grad=False, **more):
    case = dict(name=name, kind="rms_grad" if grad else "rms", n=n, d=d, dtype=dtype, weight="same", residual=True, pad=0)
    if not grad:
        case.update(bits=16 if dtype != "f32" else 32, group=0)
    return dict(case, **more)


def _distill(name, nq, n, d, dtype, k, grad=False, **more):
    case = dict(name=name, kind="distill_grad" if grad else "distill", nq=nq, n=n, d=d, dtype=dtype, k=k, bias="none", scale=10.0, pad=0)
    if grad:
        case["rows_grad"] = True
    return dict(case, **more)


def listed():
    return [
        # one new token of a request: a launch
        _embed("embed_one_768", 1, 768, 50_000, "bf16"),
        # a training batch's tokens from the optimizer's 32-bit table, states in 16 bits
        _embed("embed_80k_960", 80_000, 960, 100_003, "bf16", table="f32"),
        # its gradient: frequent tokens occur thousands of times, most rows of the table not at all
        _embed("embed_grad_80k_768", 80_000, 768, 50_000, "bf16", grad=True, table="f32"),
        # a small batch, odd sizes, a row stride of its own, half precision: launches and the tokens' order
        _embed("embed_grad_5003_100", 5_003, 100, 20_011, "f16", grad=True, pad=4),
        # one token's state between two layers
        _rms("rms_one_768", 1, 768, "bf16"),
        # a batch's states on their way to a product in 8 bits
        _rms("rms_e4m3_80k_768", 80_000, 768, "bf16", weight="f32", bits=8, group=128),
        # the gradient of a training batch, with what arrives over the residual
        _rms("rms_grad_80k_768", 80_000, 768, "bf16", grad=True, weight="f32"),
        # a few queries against the headline workload's table: bound by reading the rows
        _distill("distill_8_1m_128", 8, 1_000_000, 128, "bf16", k=10),
        # a fine-tuning step of the encoder: queries' gradient only
        _distill("distill_grad_256_50k_96", 256, 50_000, 96, "bf16", k=10, grad=True, rows_grad=False),
        # a training step of both towers on short rows
        _distill("distill_grad_4k_100k_128", 4_096, 100_000, 128, "bf16", k=32, grad=True),
        # the same on long rows, half precision
        _distill("distill_grad_2k_50k_768", 2_048, 50_000, 768, "f16", k=20, grad=True),
        # odd sizes, 32 bits, bias with rows left out and its gradient
        _distill("distill_grad_513_20k_100", 513, 20_011, 100, "f32", k=5, grad=True, bias="holes", pad=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "rms", "rms", "rms_grad", "distill", "distill_grad", "distill_grad"])
    dtype = rng.choice(list(TYPES))
    if not kind.startswith("distill"):
        d = rng.choice([96, 100, 128, 768, 960, _log_int(rng, 16, 8192)])
        n = _log_int(rng, 1, min(200_000, 128_000_000 // d))
        pad = rng.choice([0, 0, 1, 8])
        if kind.startswith("embed"):
            rows = _log_int(rng, 64, min(200_000, 128_000_000 // d))
            return _embed("", n, d, rows, dtype, grad=kind == "embed_grad", table=rng.choice(["same", "f32"]), scale=rng.choice([1.0, math.sqrt(d)]), pad=pad)
        case = _rms("", n, d, dtype, grad=kind == "rms_grad", weight=rng.choice(["same", "f32", "none"]), residual=rng.random() < 0.7, pad=pad)
        if kind == "rms" and rng.random() < 0.5:
            case.update(bits=8, group=rng.choice([0, 32, 64, 128]))
        return case
    grad = kind == "distill_grad"
    d = rng.choice([96, 100, 128, 768, 960, _log_int(rng, 16, 1024)])
    n = _log_int(rng, 64, 200_000 if grad else 1_000_000)
    nq = _log_int(rng, 8, 4_096)
    nq = max(1, min(nq, 100_000_000_000 // (n * d), 400_000_000 // n))
    more = dict(bias=rng.choice(["none", "none", "plain", "holes"]), pad=rng.choice([0, 0, 0, 1, 8]), scale=rng.choice([8.0, 10.0]))
    if grad:
        more["rows_grad"] = rng.random() < 0.7
    return _distill("", nq, n, d, dtype, k=min(n, rng.choice([1, 5, 10, 20, 32, 64])), grad=grad, **more)


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


def _table_type(case):
    return torch.float32 if case["table"] == "f32" else TYPES[case["dtype"]]


def _embed_inputs(case, g):
    n, d, rows, t = case["n"], case["d"], case["rows"], TYPES[case["dtype"]]
    ids = (torch.exp(torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * math.log(rows + 1.0)) - 1.0).long().clamp_(0, rows - 1)
    if n > 16:
        ids[torch.rand(n, generator=g, device=DEV) < 0.02] = PAD
    s = dict(ids=ids.int())
    if case["kind"] == "embed":
        s["table"] = _padded((torch.randn(rows, d, generator=g, device=DEV) / math.sqrt(d)).to(_table_type(case)), case["pad"])
        s["y"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"])
    else:
        s["dy"] = _padded(torch.randn(n, d, generator=g, device=DEV).to(t), case["pad"])
        s["dtable"] = _padded(torch.empty(rows, d, dtype=_table_type(case), device=DEV), case["pad"])
    return s


def _rms_inputs(case, g):
    n, d, t = case["n"], case["d"], TYPES[case["dtype"]]
    wt = t if case["weight"] == "same" else torch.float32
    # a residual stream with a spread per dimension, and a layer's smaller output
    spread = torch.exp(0.5 * torch.randn(d, generator=g, device=DEV))
    stream = torch.randn(n, d, generator=g, device=DEV).mul_(spread)
    s = dict(weight=None if case["weight"] == "none" else (1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(wt))
    if case["kind"] == "rms":
        s["rstd"] = torch.empty(n, device=DEV)
        if case["residual"]:
            s["residual"] = _padded(stream.to(t), case["pad"])
            s["x"] = _padded(torch.randn(n, d, generator=g, device=DEV).mul_(0.3).to(t), case["pad"])
            s["sum"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"])
        else:
            s["x"], s["residual"], s["sum"] = _padded(stream.to(t), case["pad"]), None, None
        if case["bits"] == 8:
            groups = 1 if case["group"] == 0 else -(-d // case["group"])
            s["y"] = torch.empty(n, d, dtype=torch.float8_e4m3fn, device=DEV)
            s["scales"] = torch.empty(n, groups, device=DEV)
        else:
            s["y"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"])
        return s
    s["h"] = _padded(stream.to(t), case["pad"])
    s["rstd"] = (s["h"].double().square().mean(1) + EPS).rsqrt().float()
    s["dy"] = _padded(torch.randn(n, d, generator=g, device=DEV).to(t), case["pad"])
    s["dsum"] = _padded(torch.randn(n, d, generator=g, device=DEV).to(t), case["pad"]) if case["residual"] else None
    s["dx"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"])
    s["dweight"] = None if s["weight"] is None else torch.empty(d, dtype=wt, device=DEV)
    return s


def _distill_inputs(case, g):
    nq, n, d, k, t = case["nq"], case["n"], case["d"], case["k"], TYPES[case["dtype"]]
    centres = torch.randn(max(8, n // 1000), d, generator=g, device=DEV)

    def unit(v):
        return v / v.norm(dim=1, keepdim=True).clamp_min(1e-6)

    of = torch.randint(len(centres), (n,), generator=g, device=DEV)
    rows = unit(centres[of] + torch.randn(n, d, generator=g, device=DEV))
    near = rows[torch.randint(n, (nq,), generator=g, device=DEV)]
    teacher = unit(near + 0.3 / math.sqrt(d) * torch.randn(nq, d, generator=g, device=DEV))
    s = dict(q=_padded(unit(near + 1.0 / math.sqrt(d) * torch.randn(nq, d, generator=g, device=DEV)).to(t), case["pad"]),
             rows=_padded(rows.to(t), case["pad"]), bias=None)
    if case["bias"] != "none":
        s["bias"] = 0.5 * torch.randn(n, generator=g, device=DEV)
    if case["bias"] == "holes":
        s["bias"][torch.rand(n, generator=g, device=DEV) < 0.05] = -math.inf
        s["bias"][0] = 0.0
    ids, logp = torch.empty(nq, k, dtype=torch.int64, device=DEV), torch.empty(nq, k, device=DEV)
    for b, e in _chunks(nq, n):
        z = _plain_scores(teacher[b:e], rows, case["scale"], s["bias"])
        val, ids[b:e] = z.topk(k, 1)
        logp[b:e] = val - torch.logsumexp(z, 1, keepdim=True)
        del z
    # lists that end early as the teacher's do, and a query that it says nothing of
    ids[logp == -math.inf] = PAD
    if k > 2:
        ids[::7, k - 1], logp[::7, k - 1] = PAD, -math.inf
    if nq > 4:
        ids[nq // 2], logp[nq // 2] = PAD, -math.inf
    s["ids"], s["given"] = ids.int(), logp
    if case["kind"] == "distill":
        s["loss"], s["lse"], s["logprobs"] = torch.empty(nq, device=DEV), torch.empty(nq, device=DEV), torch.empty(nq, k, device=DEV)
        return s
    # the forward pass' statistics, and the loss' gradient: a mean over a few
    s["lse"], s["logprobs"] = torch.empty(nq, device=DEV), torch.empty(nq, k, device=DEV)
    for b, e in _chunks(nq, n, 8):
        z = s["q"][b:e].double() @ s["rows"].double().T
        z *= case["scale"]
        if s["bias"] is not None:
            z += s["bias"].double()
        lse = torch.logsumexp(z, 1, keepdim=True)
        s["lse"][b:e] = lse[:, 0]
        s["logprobs"][b:e] = torch.where(ids[b:e] < 0, 0.0, z.gather(1, ids[b:e].clamp_min(0)) - lse)
        del z
    s["g"] = 0.5 + torch.rand(nq, generator=g, device=DEV)
    s["dq"] = _padded(torch.empty(nq, d, dtype=t, device=DEV), case["pad"])
    s["drows"] = _padded(torch.empty(n, d, dtype=t, device=DEV), case["pad"]) if case["rows_grad"] else None
    s["dbias"] = torch.empty(n, device=DEV) if case["rows_grad"] and s["bias"] is not None else None
    return s


def _inputs(case, seed):
    make = {"embed": _embed_inputs, "rms": _rms_inputs, "distill": _distill_inputs}[case["kind"].split("_")[0]]
    return dict(make(case, _generator(seed)), case=case)


def _workspace(nbytes):
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2503_17911_amd as ann
        kind, t = case["kind"], _ann_type(ann, case["dtype"])
        if kind == "embed_grad":
            s["workspace"] = _workspace(ann.ann_embedding_backward_workspace(case["n"], case["rows"], case["d"]))
        elif kind == "rms_grad":
            s["workspace"] = _workspace(ann.ann_rms_norm_backward_workspace(case["n"], case["d"]))
        elif kind == "distill":
            s["workspace"] = _workspace(ann.ann_row_distillation_workspace(case["nq"], case["n"], case["d"], t, case["k"]))
        elif kind == "distill_grad":
            s["workspace"] = _workspace(ann.ann_row_distillation_backward_workspace(case["nq"], case["n"], case["d"], t, case["k"]))
    return s


# ------------------------------------------------------------------ plain forms
def _chunks(nq, n, bytes_each=4):
    step = max(1, CHUNK * 4 // bytes_each // max(n, 1))
    return [(b, min(nq, b + step)) for b in range(0, nq, step)]


def _plain_embed(s):
    ids = s["ids"].long()
    y = s["table"][ids.clamp_min(0)].float() * s["case"]["scale"]
    return dict(y=y.masked_fill((ids < 0)[:, None], 0.0).to(s["y"].dtype))


def _plain_embed_grad(s):
    ids, case = s["ids"].long(), s["case"]
    # (a row more takes what belongs to no token)
    total = torch.zeros(case["rows"] + 1, case["d"], device=DEV)
    total.index_add_(0, torch.where(ids < 0, case["rows"], ids), s["dy"].float())
    return dict(dtable=(total[:-1] * case["scale"]).to(s["dtable"].dtype))


def _plain_rms(s):
    case, t = s["case"], s["x"].dtype
    h = s["x"].float()
    out = {}
    if s["residual"] is not None:
        out["sum"] = (h + s["residual"].float()).to(t)
        h = out["sum"].float()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None]
    if s["weight"] is not None:
        y = y * s["weight"].float()
    if case["bits"] != 8:
        return dict(out, y=y.to(t), rstd=rstd)
    n, d = y.shape
    group = case["group"] or d
    whole = torch.nn.functional.pad(y, (0, -d % group)).view(n, -1, group)
    scales = whole.abs().amax(2).clamp_min(SMALLEST) / E4M3_MAX
    codes = (whole / scales[:, :, None]).to(torch.float8_e4m3fn).view(n, -1)[:, :d]
    return dict(out, y=codes, scales=scales, rstd=rstd)


def _plain_rms_grad(s):
    t = s["h"].dtype
    xh = s["h"].float() * s["rstd"][:, None]
    dy = s["dy"].float()
    a = dy if s["weight"] is None else dy * s["weight"].float()
    dx = s["rstd"][:, None] * (a - xh * (a * xh).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    out = dict(dx=dx.to(t))
    if s["weight"] is not None:
        out["dweight"] = (dy * xh).sum(0).to(s["weight"].dtype)
    return out


def _plain_scores(q, rows, scale, bias):
    z = (q @ rows.T) * scale
    return z if bias is None else z + bias


def _plain_distill(s):
    case, rows = s["case"], s["rows"].float()
    nq, n = case["nq"], case["n"]
    loss, lse, logprobs = torch.empty(nq, device=DEV), torch.empty(nq, device=DEV), torch.empty(nq, case["k"], device=DEV)
    for b, e in _chunks(nq, n):
        z = _plain_scores(s["q"][b:e].float(), rows, case["scale"], s["bias"])
        ids, given = s["ids"][b:e].long(), s["given"][b:e]
        top = z.max(1, keepdim=True).values
        z -= top
        picked = z.gather(1, ids.clamp_min(0))
        total = z.exp().sum(1).log()
        lse[b:e] = top[:, 0] + total
        there = ids >= 0
        logprobs[b:e] = torch.where(there, picked - total[:, None], 0.0)
        there = there & (given > -math.inf)
        loss[b:e] = torch.where(there, given.exp() * (given.masked_fill(~there, 0.0) - logprobs[b:e]), 0.0).sum(1)
    return dict(loss=loss, lse=lse, logprobs=logprobs)


def _over_rows(dz, rows):
    """dz @ rows as sums over a thousand rows each: like terms of very many rows lose 2e-5 of one sum in 32 bits."""
    whole, d = len(rows) // PART * PART, rows.shape[1]
    total = dz[:, whole:] @ rows[whole:]
    if whole:
        total += torch.bmm(dz[:, :whole].reshape(len(dz), -1, PART).transpose(0, 1).contiguous(), rows[:whole].reshape(-1, PART, d)).sum(0)
    return total


def _plain_distill_grad(s):
    case, rows, scale = s["case"], s["rows"].float(), s["case"]["scale"]
    nq, n, t = case["nq"], case["n"], s["q"].dtype
    dq = torch.empty(nq, case["d"], device=DEV)
    drows = torch.zeros(n, case["d"], device=DEV) if s["drows"] is not None else None
    dbias = torch.zeros(n, device=DEV) if s["dbias"] is not None else None
    for b, e in _chunks(nq, n):
        q, ids = s["q"][b:e].float(), s["ids"][b:e].long()
        weight = s["g"][b:e, None] * torch.where(ids < 0, 0.0, s["given"][b:e].exp())
        dz = (_plain_scores(q, rows, scale, s["bias"]) - s["lse"][b:e, None]).exp() * weight.sum(1, keepdim=True)
        dz.scatter_add_(1, ids.clamp_min(0), -weight)
        dq[b:e] = (_over_rows(dz, rows) if t == torch.float32 else dz @ rows) * scale
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
    if kind.startswith("embed"):
        tt = ann.F32 if case["table"] == "f32" else t
        if kind == "embed":
            ann.ann_embedding(s["table"], case["rows"], d, s["table"].stride(0), tt, s["ids"], n, case["scale"], s["y"], s["y"].stride(0), t, stream)
            return dict(y=s["y"])
        ann.ann_embedding_backward(s["dy"], s["dy"].stride(0), t, s["ids"], n, case["scale"], case["rows"], d, s["dtable"], s["dtable"].stride(0), tt,
                                   workspace=s["workspace"], workspace_bytes=s["workspace"].numel(), stream=stream)
        return dict(dtable=s["dtable"])
    if kind.startswith("rms"):
        wt = ann.F32 if case["weight"] == "f32" else t
        if kind == "rms":
            more = {}
            if case["residual"]:
                more = dict(residual=s["residual"], residual_stride=s["residual"].stride(0), sum=s["sum"], sum_stride=s["sum"].stride(0))
            if case["bits"] == 8:
                ann.ann_rms_norm_e4m3(s["x"], n, d, s["x"].stride(0), t, s["weight"], wt, EPS, s["y"], s["y"].stride(0), case["group"], s["scales"],
                                      s["scales"].stride(0), rstd=s["rstd"], stream=stream, **more)
                out = dict(y=s["y"], scales=s["scales"], rstd=s["rstd"])
            else:
                ann.ann_rms_norm(s["x"], n, d, s["x"].stride(0), t, s["weight"], wt, EPS, s["y"], s["y"].stride(0), rstd=s["rstd"], stream=stream, **more)
                out = dict(y=s["y"], rstd=s["rstd"])
            return dict(out, sum=s["sum"]) if case["residual"] else out
        more = dict(dsum=s["dsum"], dsum_stride=s["dsum"].stride(0)) if case["residual"] else {}
        ann.ann_rms_norm_backward(s["dy"], s["dy"].stride(0), s["h"], s["h"].stride(0), n, d, t, s["weight"], wt, s["rstd"], s["dx"], s["dx"].stride(0),
                                  dweight=s["dweight"], workspace=s["workspace"], workspace_bytes=s["workspace"].numel(), stream=stream, **more)
        return dict(dx=s["dx"]) if s["dweight"] is None else dict(dx=s["dx"], dweight=s["dweight"])
    table = dict(q=s["q"], nq=case["nq"], q_stride=s["q"].stride(0), rows=s["rows"], n=n, row_stride=s["rows"].stride(0), d=d, type=t,
                 scale=case["scale"], row_bias=s["bias"], k=case["k"], given_ids=s["ids"], given_logprobs=s["given"], lse=s["lse"],
                 logprobs=s["logprobs"], workspace=s["workspace"], workspace_bytes=s["workspace"].numel(), stream=stream)
    if kind == "distill":
        ann.ann_row_distillation(**table, loss=s["loss"])
        return dict(loss=s["loss"], lse=s["lse"], logprobs=s["logprobs"])
    ann.ann_row_distillation_backward(**table, g_loss=s["g"], dq=s["dq"], dq_stride=s["dq"].stride(0), drows=s["drows"],
                                      drows_stride=s["drows"].stride(0) if s["drows"] is not None else 0, drow_bias=s["dbias"])
    out = dict(dq=s["dq"])
    if s["drows"] is not None:
        out["drows"] = s["drows"]
    if s["dbias"] is not None:
        out["dbias"] = s["dbias"]
    return out


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "rms": _plain_rms, "rms_grad": _plain_rms_grad, "distill": _plain_distill,
            "distill_grad": _plain_distill_grad}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def _distinct(n, rows):
    """How many different tokens n draws have, by the law that they are drawn by."""
    p = torch.log1p(1.0 / torch.arange(1, rows + 1, dtype=torch.float64)) / math.log(rows + 1.0)
    return float((1.0 - torch.exp(n * torch.log1p(-p.clamp(max=1.0 - 1e-12)))).sum())


def work(case):
    n, d, kind = case["n"], case["d"], case["kind"]
    size = 4 if case["dtype"] == "f32" else 2
    if kind.startswith("embed"):
        tsize = 4 if case["table"] == "f32" else size
        if kind == "embed":
            return dict(bytes=4 * n + _distinct(n, case["rows"]) * d * tsize + n * d * size, flops=n * d)
        return dict(bytes=4 * n + n * d * size + case["rows"] * d * tsize, flops=n * d)
    if kind.startswith("rms"):
        weight = {"none": 0, "f32": 4 * d, "same": size * d}[case["weight"]]
        if kind == "rms_grad":
            return dict(bytes=(4 if case["residual"] else 3) * n * d * size + 4 * n + 2 * weight, flops=10 * n * d)
        out = n * d + 4 * n * (1 if case["group"] == 0 else -(-d // case["group"])) if case["bits"] == 8 else n * d * size
        return dict(bytes=(3 if case["residual"] else 1) * n * d * size + out + 4 * n + weight, flops=5 * n * d)
    nq, k = case["nq"], case["k"]
    read = (nq + n) * d * size + 8 * nq * k + (4 * n if case["bias"] != "none" else 0)
    if kind == "distill":
        return dict(bytes=read + 8 * nq + 4 * nq * k, flops=2 * nq * n * d)
    written = nq * d * size
    if case["rows_grad"]:
        written += n * d * size + (4 * n if case["bias"] != "none" else 0)
    return dict(bytes=read + written + 8 * nq + 4 * nq * k, flops=(6 if case["rows_grad"] else 4) * nq * n * d)


# ------------------------------------------------------------------ the definitions in 64 bits
F64 = torch.float64


def _exact_embed(s):
    case = s["case"]
    there = s["ids"] != PAD
    if case["kind"] == "embed":
        y = torch.zeros(case["n"], case["d"], dtype=F64, device=DEV)
        y[there] = s["table"].to(F64)[s["ids"][there].long()] * case["scale"]
        return dict(y=y)
    # runs of equal tokens, as differences of a running sum over the tokens in order
    order = torch.argsort(s["ids"], stable=True)
    ids = s["ids"][order].long()
    running = torch.cumsum(s["dy"].to(F64)[order], 0)
    end = torch.ones(case["n"], dtype=torch.bool, device=DEV)
    end[:-1] = ids[1:] != ids[:-1]
    of, sums = ids[end], running[end]
    sums = torch.cat([sums[:1], sums[1:] - sums[:-1]])
    table = torch.zeros(case["rows"], case["d"], dtype=F64, device=DEV)
    table[of[of >= 0]] = sums[of >= 0] * case["scale"]
    return dict(dtable=table)


def _exact_rms(s):
    case = s["case"]
    d = case["d"]
    w = None if s["weight"] is None else s["weight"].to(F64)
    if case["kind"] == "rms_grad":
        h, rstd, dy = s["h"].to(F64), s["rstd"].to(F64).unsqueeze(1), s["dy"].to(F64)
        up = dy if w is None else dy * w
        dx = rstd * up - h * rstd ** 3 * torch.einsum("nd,nd->n", up, h).unsqueeze(1) / d
        out = dict(dx=dx if s["dsum"] is None else dx + s["dsum"].to(F64))
        if w is not None:
            out["dweight"] = torch.einsum("nd,nd->d", dy, h * rstd)
        return out
    out = {}
    h = s["x"].to(F64)
    if case["residual"]:
        out["sum"] = h + s["residual"].to(F64)
        h = out["sum"].to(s["x"].dtype).to(F64)  # (the norm is that of the sum as it is kept)
    rstd = (torch.einsum("nd,nd->n", h, h) / d + EPS) ** -0.5
    y = h * rstd.unsqueeze(1)
    if w is not None:
        y = y * w
    if case["bits"] != 8:
        return dict(out, y=y, rstd=rstd)
    group = case["group"] or d
    parts = torch.split(y, group, dim=1)
    scales = torch.stack([torch.clamp(p.abs().max(1).values, min=SMALLEST) / E4M3_MAX for p in parts], 1)
    # (what the codes stand for before they are rounded to 8 bits)
    codes = torch.cat([p / scales[:, i:i + 1] for i, p in enumerate(parts)], 1)
    return dict(out, y=codes, scales=scales, rstd=rstd)


def _exact_distill(s):
    case = s["case"]
    nq, n, d = case["nq"], case["n"], case["d"]
    rows_t = s["rows"].to(F64).t().contiguous()
    grad = case["kind"] == "distill_grad"
    drows, dbias = torch.zeros(n, d, dtype=F64, device=DEV), torch.zeros(n, dtype=F64, device=DEV)
    parts = []
    step = max(1, (1 << 27) // n)
    for i in range(0, nq, step):
        at = slice(i, min(nq, i + step))
        q = s["q"][at].to(F64)
        z = torch.mm(q, rows_t).mul_(case["scale"])
        if s["bias"] is not None:
            z.add_(s["bias"].to(F64))
        line, entry = torch.nonzero(s["ids"][at] != PAD, as_tuple=True)
        row = s["ids"][at][line, entry].long()
        given = s["given"][at][line, entry].to(F64)
        if grad:
            mass = torch.exp(given) * s["g"][at].to(F64)[line]
            whole = torch.zeros(len(q), dtype=F64, device=DEV).index_add_(0, line, mass)
            z.sub_(s["lse"][at].to(F64).unsqueeze(1)).exp_().mul_(whole.unsqueeze(1))
            z.index_put_((line, row), -mass, accumulate=True)
            parts.append(dict(dq=torch.mm(z, rows_t.t().contiguous()) * case["scale"]))
            if s["drows"] is not None:
                drows += torch.mm(z.t().contiguous(), q) * case["scale"]
            dbias += z.sum(0)
            continue
        lse = torch.logsumexp(z, dim=1)
        own_logp = z[line, row] - lse[line]
        logprobs = torch.zeros(len(q), case["k"], dtype=F64, device=DEV)
        logprobs[line, entry] = own_logp
        loss = torch.zeros(len(q), dtype=F64, device=DEV).index_add_(0, line, torch.exp(given) * (given - own_logp))
        parts.append(dict(loss=loss, lse=lse, logprobs=logprobs))
        del z
    out = {f: torch.cat([p[f] for p in parts]) for f in parts[0]}
    if grad and s["drows"] is not None:
        out["drows"] = drows
    if grad and s["dbias"] is not None:
        out["dbias"] = dbias
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return {"embed": _exact_embed, "rms": _exact_rms, "distill": _exact_distill}[case["kind"].split("_")[0]](s)
