"""Token embeddings and root-mean-square norm, with their gradients, from their
definitions in 64 bits on the CPU, and codes of 8 bits by their definition."""
import torch

F64 = torch.float64


def embedding(table, ids, scale):
    """ids that are not below the table's rows give zeros."""
    there = (ids >= 0) & (ids < table.shape[0])
    y = torch.zeros(len(ids), table.shape[1], dtype=F64)
    y[there] = table.to(F64)[ids[there]] * scale
    return y


def embedding_grad(dy, ids, scale, rows):
    """The gradient, the sums of the terms' sizes, and how many terms a row has."""
    there = (ids >= 0) & (ids < rows)
    total, size, count = torch.zeros(rows, dy.shape[1], dtype=F64), torch.zeros(rows, dy.shape[1], dtype=F64), torch.zeros(rows, dtype=F64)
    total.index_add_(0, ids[there], dy[there].to(F64))
    size.index_add_(0, ids[there], dy[there].to(F64).abs())
    count.index_add_(0, ids[there], torch.ones(int(there.sum()), dtype=F64))
    return total * scale, size * abs(scale), count


def rms_norm(h, w, eps):
    h = h.to(F64)
    rstd = (h.square().mean(1) + eps).rsqrt()
    y = h * rstd[:, None]
    return (y if w is None else y * w.to(F64)), rstd


def rms_norm_grad(dy, h, dsum, w, rstd):
    """dx, dw, and the sums of the sizes of their terms."""
    dy, h, rstd = dy.to(F64), h.to(F64), rstd.to(F64)[:, None]
    xh = h * rstd
    a = dy if w is None else dy * w.to(F64)
    dx = rstd * (a - xh * (a * xh).mean(1, keepdim=True))
    size = rstd * (a.abs() + xh.abs() * (a * xh).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx, size = dx + dsum.to(F64), size + dsum.to(F64).abs()
    return dx, (dy * xh).sum(0), size, (dy * xh).abs().sum(0)


def e4m3_values():
    """What each of the 256 codes stands for: 1 bit of sign, 4 of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are no numbers."""
    code = torch.arange(256)
    e, m = (code >> 3) & 15, (code & 7).to(F64)
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e.to(F64) - 7))
    v = torch.where(code >= 128, -v, v)
    v[127] = v[255] = float("nan")
    return v


def scales(v, group):
    """The scale of every group of columns (0: of the row)."""
    parts = torch.split(v, group or v.shape[1], dim=1)
    return torch.stack([p.abs().amax(1).clamp_min(2.0 ** -100) / 448 for p in parts], 1)
