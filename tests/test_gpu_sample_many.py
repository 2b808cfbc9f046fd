"""Many rows of few tokens, each against the float64 oracle: two tokens that finish within a thousandth of one another (told
apart in 64 bits), rows whose first look finds nobody, and long rows of few distinct logits come up in such numbers that each of
those ways is taken.  Bounds as in test_gpu_sample.py."""
import numpy as np
import pytest
import torch

from oracle import answer_oracle as ao
from tests.test_gpu_sample import check, draw, logits, numbers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(temperature=2.0), dict(min_p=0.2), dict(top_k=9), dict(top_p=0.8), dict(top_k=30, top_p=0.95, min_p=0.01)])
def test_four_thousand_rows(kw):
    rows = 4000
    for V, dtype in ((33, torch.float32), (61, torch.bfloat16)):
        check(logits(rows, V, dtype, V, scale=0.5), numbers(rows, V), **kw)


def test_near_finishers_were_among_them():
    """The rows above hold about eight pairs within a thousandth: without them the test would say nothing about those."""
    z, seeds = logits(4000, 33, torch.float32, 33, scale=0.5).cpu().numpy(), numbers(4000, 33)
    lead = np.array([ao.sample(z[b], int(seeds[b]) % 2 ** 64)[2] for b in range(4000)])
    assert (lead < 1e-3).sum() >= 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_flat_rows_over_several_blocks(dtype):
    """All logits equal, or of two values: every block has the same to say, and the winner is anywhere."""
    V = 70001
    z = torch.zeros(24, V, dtype=dtype)
    z[12:, ::3] = -2.0
    ids = check(z.cuda(), numbers(24, 5))
    assert len(set(ids // 8751)) > 3                       # (eight pieces of the row)
    check(z.cuda(), numbers(24, 6), top_k=60000)
    check(z.cuda(), numbers(24, 7), top_p=0.9)
    check(z.cuda(), numbers(24, 8), top_k=300)


def test_top_k_around_the_sizes_that_are_sorted_at_once():
    z = logits(6, 30000, torch.float32, 4)
    for k in (255, 256, 257, 400, 511, 512, 513, 700):
        check(z, numbers(6, k), top_k=k)
        check(z, numbers(6, k + 1), top_k=k, top_p=0.7, temperature=1.5)


def test_one_row_drawn_many_times():
    """ld 0: the logits of one prompt, the first tokens of its answers."""
    z = logits(1, 5000, torch.bfloat16, 3).expand(300, 5000)
    check(z, numbers(300, 1), top_p=0.9)
    ids, _ = draw(z, numbers(300, 2))
    assert len(set(ids)) > 5
