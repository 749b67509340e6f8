"""Attention over the 8-bit cache where queries and keys are at opposite ends of bf16's range and scores are ordinary."""
import pytest
import torch

import serving_oracle as so
from test_gpu_attention_kv8 import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group,counts", [(1, [1, 1]), (4, [1, 1]), (4, [7, 9]), (4, [70, 50])])
@pytest.mark.parametrize("power", [-126, -112, -100])
def test_small_queries_and_large_keys(dim, group, counts, power):
    """Queries below 2^power, subnormal ones among them, by keys of 2^-power: scores of a few units."""
    g = so.generator(dim, group, -power)

    def change(kv):
        for k, _ in kv:
            k.copy_((torch.randn(k.shape, generator=g) * 0.4).clamp(-1.9, 1.9) * 2.0 ** (1 - power))
    t = Case([90, 130], 1, dim, 64, torch.bfloat16, change=change)
    q = torch.randint(-127, 128, (sum(counts), group, dim), generator=g).double() * 2.0 ** (power - 7)
    q = q.to(torch.bfloat16)
    k, _ = t.held[1].values()
    s = torch.einsum("qhd,td->qht", q[counts[0]:].double(), k[:, 0]) / dim ** 0.5
    assert 0.2 < s.std() < 50 and torch.isfinite(s).all()
    t.check(q, counts, t.run(q, counts))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("counts", [[1, 1], [3, 2], [40, 50]])
@pytest.mark.parametrize("power", [-126, -123, -120, -117])
def test_scores_that_decide(dim, counts, power):
    """Few tokens whose scores differ by some units: a scale of few bits would move the weights between them."""
    g = so.generator(dim, len(counts), -power)

    def change(kv):
        for k, _ in kv:
            k.copy_((torch.randn(k.shape[0], 1, 1, generator=g) * 0.4).clamp(-1.9, 1.9).expand_as(k) * 2.0 ** (1 - power))
    lens = [max(5, counts[0]), max(4, counts[1])]
    t = Case(lens, 1, dim, 64, torch.bfloat16, change=change)
    q = (torch.randint(64, 128, (sum(counts), 4, 1), generator=g).double() * 2.0 ** (power - 7)).expand(-1, -1, dim)
    q = q.to(torch.bfloat16).contiguous()
    t.check(q, counts, t.run(q, counts))
