"""The workspace of distillation's gradients stays within what the header says of it (no GPU)."""
import random

import pytest

import paper_2503_17911_amd as ann

MIB = 1 << 20


def bound(nq, n, d, t, k):
    """What ann_row_logprobs_backward asks for and what is said to come on top, each array up to 256 bytes more."""
    entries, row = nq * k, 4 * (d + 4)
    chunks = min(-(-entries // (8 if entries <= 16384 else 32)), 32768)
    more = 4 * n + 4 * nq * d + 4 * nq + 30 * entries + 2 * chunks * row + min(n, entries) * row + 20 * 256 + 64 * 1024
    if t != ann.F32:
        # (a tile of 128 rows at least, of all queries)
        more += 256 * MIB if d <= 128 else max(512 * MIB, 2 * 2 * 128 * nq) if 2 * nq * n > 512 * MIB else 2 * nq * (n + 128) + nq * n // 1024
    return ann.ann_row_logprobs_backward_workspace(nq, n, d, t) + more


SIZES = [(4096, 70_000, 128, 20), (4096, 65_537, 128, 1), (4096, 131_073, 128, 32), (65_536, 1_000_000, 128, 20), (65_536, 66_000, 96, 3), (434, 4173, 96, 20),
         (4096, 100_000, 128, 32), (100_000, 30_000, 64, 5), (2048, 50_000, 768, 20), (200, 50_000, 768, 10), (5000, 60_000, 144, 12), (300, 200_000_000, 16, 1),
         (1_000_000, 2000, 256, 4), (3000, 2_000_000, 768, 10), (1_000_000, 5000, 64, 2), (1, 5000, 128, 1)]


@pytest.mark.parametrize("nq, n, d, k", SIZES)
def test_bound(nq, n, d, k):
    for t in (ann.F32, ann.F16, ann.BF16):
        need = ann.ann_row_distillation_backward_workspace(nq, n, d, t, k)
        assert 0 < need <= bound(nq, n, d, t, k), t


def test_bound_of_many_sizes():
    rng = random.Random(3)
    for _ in range(3000):
        nq, n, d = round(2 ** rng.uniform(0, 17)), round(2 ** rng.uniform(10.1, 22)), rng.choice([8, 64, 96, 100, 128, 136, 200, 768, 1000])
        k, t = rng.choice([1, 5, 20, 64]), rng.choice([ann.F32, ann.F16, ann.BF16])
        assert ann.ann_row_distillation_backward_workspace(nq, n, d, t, k) <= bound(nq, n, d, t, k), (nq, n, d, k, t)


def test_parts_of_short_rows_sums():
    """A million short rows: their parts would be 512 MB each."""
    more = ann.ann_row_distillation_backward_workspace(65_536, 1_000_000, 128, ann.BF16, 1) - ann.ann_row_logprobs_backward_workspace(65_536, 1_000_000, 128, ann.BF16)
    assert more < 256 * MIB
