"""Fits the last layers of a query encoder to a table of rows, then asks the table.

    python examples/train_query_encoder.py [--rows N] [--dim D] [--hidden H] [--queries B] [--steps K]

An encoder's hidden states go through a layer norm and a projection; the
projected states are the queries.  The loss is the negative log probability of
the row that belongs to each query, under the softmax of the scores of ALL rows
(no sampled negatives), less a little of the softmax' entropy.  Layer norm, log
probabilities and their gradients are the library's calls, wrapped for
torch.autograd; the projection is a torch product.  At the end the likeliest rows
with their probabilities answer new queries, next to an exhaustive search by inner
product for the same rows in the same order.  Data are synthetic.
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
import paper_2503_17911_amd as ann  # noqa: E402

DEV = "cuda"
TYPES = {torch.float32: ann.F32, torch.float16: ann.F16, torch.bfloat16: ann.BF16}


def stream():
    return torch.cuda.current_stream().cuda_stream


def scratch(nbytes):
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=DEV)


class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        n, d = x.shape
        y = torch.empty_like(x)
        mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        ann.ann_layer_norm(x, n, d, x.stride(0), TYPES[x.dtype], weight, bias, TYPES[weight.dtype], eps, y, y.stride(0), mean, rstd, stream())
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        n, d = x.shape
        dy = dy.contiguous()
        dx, dweight, dbias = torch.empty_like(x), torch.empty_like(weight), torch.empty_like(weight)
        room = scratch(ann.ann_layer_norm_backward_workspace(n, d))
        ann.ann_layer_norm_backward(dy, dy.stride(0), x, x.stride(0), n, d, TYPES[x.dtype], weight, TYPES[weight.dtype], mean, rstd,
                                    dx, dx.stride(0), dweight, dbias, room, room.numel(), stream())
        return dx, dweight, dbias, None


class RowLogProbs(torch.autograd.Function):
    """Log probability of targets[i] and the entropy of the softmax of scale <q_i, rows_j>."""

    @staticmethod
    def forward(ctx, q, rows, targets, scale):
        (nq, d), n, t = q.shape, rows.shape[0], TYPES[q.dtype]
        logprob, lse, entropy = (torch.empty(nq, device=DEV) for _ in range(3))
        room = scratch(ann.ann_row_logprobs_workspace(nq, n, d, t))
        ann.ann_row_logprobs(q, nq, q.stride(0), rows, n, rows.stride(0), d, t, scale=scale, targets=targets, logprob=logprob, lse=lse,
                             entropy=entropy, workspace=room, workspace_bytes=room.numel(), stream=stream())
        ctx.save_for_backward(q, rows, targets, lse, entropy)
        ctx.scale = scale
        return logprob, entropy

    @staticmethod
    def backward(ctx, g_logprob, g_entropy):
        q, rows, targets, lse, entropy = ctx.saved_tensors
        (nq, d), n, t = q.shape, rows.shape[0], TYPES[q.dtype]
        g_logprob, g_entropy = g_logprob.contiguous(), g_entropy.contiguous()
        dq = torch.empty_like(q)
        drows = torch.empty_like(rows) if ctx.needs_input_grad[1] else None
        room = scratch(ann.ann_row_logprobs_backward_workspace(nq, n, d, t))
        ann.ann_row_logprobs_backward(q, nq, q.stride(0), rows, n, rows.stride(0), d, t, scale=ctx.scale, targets=targets, lse=lse,
                                      entropy=entropy, g_logprob=g_logprob, g_entropy=g_entropy, dq=dq, dq_stride=dq.stride(0),
                                      drows=drows, drows_stride=drows.stride(0) if drows is not None else 0,
                                      workspace=room, workspace_bytes=room.numel(), stream=stream())
        return dq, drows, None, None


def answers(q, rows, scale, k):
    """The k likeliest rows of every query with their log probabilities."""
    (nq, d), n, t = q.shape, rows.shape[0], TYPES[q.dtype]
    logprob, lse, values = torch.empty(nq, device=DEV), torch.empty(nq, device=DEV), torch.empty(nq, k, device=DEV)
    ids = torch.empty(nq, k, dtype=torch.int32, device=DEV)
    room = scratch(ann.ann_row_logprobs_workspace(nq, n, d, t, k))
    ann.ann_row_logprobs(q, nq, q.stride(0), rows, n, rows.stride(0), d, t, scale=scale, k=k, logprob=logprob, lse=lse, alt_ids=ids,
                         alt_logprobs=values, workspace=room, workspace_bytes=room.numel(), stream=stream())
    return ids, values


def train(n=50_000, d=96, hidden=768, batch=256, steps=60, scale=20.0, k=10, report=print):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    rows = torch.randn(n, d, generator=g, device=DEV)
    rows = (rows / rows.norm(dim=1, keepdim=True)).bfloat16()
    lift = torch.randn(d, hidden, generator=g, device=DEV)

    def hidden_states(count):  # what the encoder's body would give for queries that belong to these rows
        target = torch.randint(n, (count,), generator=g, device=DEV)
        h = rows[target].float() @ lift + 0.3 * torch.randn(count, hidden, generator=g, device=DEV) + 0.5
        return h.bfloat16(), target.int()

    weight, bias = torch.ones(hidden, device=DEV, requires_grad=True), torch.zeros(hidden, device=DEV, requires_grad=True)
    project = (torch.randn(hidden, d, generator=g, device=DEV) / hidden**0.5).requires_grad_()
    adam = torch.optim.Adam([weight, bias, project], lr=0.01)

    def queries(h):
        return LayerNorm.apply(h, weight, bias, 1e-5) @ project.bfloat16()

    losses = []
    for step in range(steps):
        h, target = hidden_states(batch)
        logprob, entropy = RowLogProbs.apply(queries(h), rows, target, scale)
        loss = -(logprob + 0.01 * entropy).mean()
        adam.zero_grad()
        loss.backward()
        adam.step()
        losses.append(loss.detach())
        if step % 20 == 0 or step == steps - 1:
            report(f"step {step}: loss {loss.item():.3f}, entropy {entropy.mean().item():.3f}")
    with torch.no_grad():
        h, target = hidden_states(batch)
        q = queries(h)
    ids, values = answers(q, rows, scale, k)
    near, dist = torch.empty(batch, k, dtype=torch.int32, device=DEV), torch.empty(batch, k, device=DEV)
    ann.ann_bruteforce_topk(rows.float(), n, d, q.float(), batch, k, ann.IP, near, dist, stream())
    hit = (ids[:, 0] == target).float().mean().item()
    report(f"new queries: their row is the likeliest for {hit:.3f} of them, probability {values[:, 0].exp().mean().item():.3f}; "
           f"the search by inner product agrees in {(ids == near).float().mean().item():.4f} of the answers")
    return dict(losses=torch.stack(losses).tolist(), hit=hit, ids=ids, near=near, values=values)


def main(argv=None):
    p = argparse.ArgumentParser()
    p.add_argument("--rows", type=int, default=50_000)
    p.add_argument("--dim", type=int, default=96)
    p.add_argument("--hidden", type=int, default=768)
    p.add_argument("--queries", type=int, default=256)
    p.add_argument("--steps", type=int, default=60)
    a = p.parse_args(argv)
    train(a.rows, a.dim, a.hidden, a.queries, a.steps)


if __name__ == "__main__":
    main()
