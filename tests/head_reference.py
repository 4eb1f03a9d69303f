"""Layer norm and the rows' log probabilities, with their gradients, from their
definitions in 64 bits on the CPU, and how far a result may lie from them."""
import math

import torch

F64 = torch.float64
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24        # half a step of fp32, relative


def half_step(dtype):
    """What rounding to a type may take, relative to the value."""
    return torch.finfo(dtype).eps / 2


def smallest_step(dtype):
    """What rounding to a type may take of values below its normal ones (bf16 and fp32 have fp32's range: not seen here)."""
    return 2.0 ** -25 if dtype == torch.float16 else 0.0


def layer_norm(x, w, b, eps):
    x = x.to(F64)
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    y = (x - mean) * rstd
    return (y if w is None else y * w.to(F64)) + (0.0 if b is None else b.to(F64)), mean[:, 0], rstd[:, 0]


def layer_norm_grad(dy, x, w, mean, rstd):
    dy, x = dy.to(F64), x.to(F64)
    xh = (x - mean.to(F64)[:, None]) * rstd.to(F64)[:, None]
    a = dy if w is None else dy * w.to(F64)
    dx = rstd.to(F64)[:, None] * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def scores(q, rows, scale, bias):
    """Rows that are left out come as -infinity whatever they hold."""
    rows = rows.to(F64)
    if bias is not None:
        out = bias == -math.inf
        rows = torch.where(out[:, None], torch.zeros_like(rows), rows)
    z = scale * (q.to(F64) @ rows.T)
    return z if bias is None else z + bias.to(F64)


def log_probabilities(z, targets):
    """lse, log probabilities of the targets (0 where none is given), entropy."""
    nq, n = z.shape
    lse = torch.logsumexp(z, 1) if n else torch.full((nq,), -math.inf, dtype=F64)
    logp = z - lse[:, None]
    p = torch.where(z == -math.inf, torch.zeros_like(z), logp.exp())
    entropy = -(p * torch.where(p > 0, logp, torch.zeros_like(z))).sum(1)
    entropy = torch.where(lse == -math.inf, torch.zeros_like(lse), entropy)
    given = (targets >= 0) & (targets < n)
    at = targets.clamp(0, max(n - 1, 0))
    lp = torch.zeros(nq, dtype=F64)
    if n:
        picked = z.gather(1, at[:, None])[:, 0]
        lp = torch.where(given, torch.where(picked == -math.inf, picked, picked - lse), lp)
    return lse, lp, entropy


def alternatives(z, k):
    """The k largest of every line, equal ones by their number; -1 behind the last."""
    nq, n = z.shape
    val, ids = z.sort(dim=1, descending=True, stable=True)
    val = torch.cat([val, torch.full((nq, k), -math.inf, dtype=F64)], 1)[:, :k]
    ids = torch.cat([ids, torch.full((nq, k), -1)], 1)[:, :k]
    return torch.where(val == -math.inf, torch.full_like(ids, -1), ids), val


def score_gradient(z, lse, entropy, targets, g, h):
    """G of the definition; lse and entropy as the forward pass returned them."""
    nq, n = z.shape
    lse = lse.to(F64)
    logp = z - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None]
    p = torch.where(z == -math.inf, torch.zeros_like(z), logp.exp())
    given = (targets >= 0) & (targets < n)
    G = torch.zeros_like(z)
    if g is not None:
        gg = torch.where(given, g.to(F64), torch.zeros_like(lse))
        G -= gg[:, None] * p
        line = torch.nonzero(given)[:, 0]
        G[line, targets[line]] += gg[line]
    if h is not None:
        G -= h.to(F64)[:, None] * torch.where(p > 0, p * (logp + entropy.to(F64)[:, None]), torch.zeros_like(z))
    G[z == -math.inf] = 0.0
    return G, p


def score_error(q, rows, scale, bias):
    """The most a score in fp32 may err, per query: d additions (fp32 elements: six products of bf16 parts to an
    element), each rounding a partial sum of at most |q| |x|, twice for the order inside the matrix instruction; the
    products of parts left out; a product and an addition at the end."""
    d = q.shape[1]
    rows = rows.to(F64)
    if bias is not None:
        rows = rows[bias != -math.inf]
        bias = bias[bias != -math.inf]
    if rows.shape[0] == 0:
        return torch.zeros(q.shape[0], dtype=F64)
    size = abs(scale) * q.to(F64).norm(dim=1) * rows.norm(dim=1).max()
    most = size + (0.0 if bias is None else bias.abs().max().to(F64))
    return ((6 if q.dtype == torch.float32 else 1) * d + 64) * 2 * U32 * size + 4 * U32 * most


def sum_error(n):
    """Relative error of a sum of n exponentials (one unit in the last place each, and their arguments' rounding) in fp32."""
    return (n + 64) * U32 + 8 * U32
