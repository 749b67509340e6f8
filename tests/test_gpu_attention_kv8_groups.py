"""Attention over the 8-bit cache where one key head serves many query heads: up to the 1024 that a call takes."""
import pytest
import torch

import fp8_oracle as fo
from test_gpu_attention_kv8 import HALF, Case, mq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim,heads,group,lens,counts", [
    (128, 1, 64, [500, 33, 1, 700], [1, 1, 1, 1]), (64, 2, 65, [500, 33, 90], [1, 1, 1]), (128, 1, 128, [1200, 40, 7], [1, 1, 1]),
    (64, 1, 1024, [300, 5], [1, 1]), (128, 1, 1024, [700], [1]), (64, 1, 128, [300, 2, 900], [9, 1, 2]), (128, 2, 16, [900, 65], [4, 5])])
def test_many_query_heads(dtype, dim, heads, group, lens, counts):
    t = Case(lens, heads, dim, 32, dtype)
    q = t.queries(counts, group)
    o = t.run(q, counts)
    t.check(q, counts, o)
    # the same under a bound of the contexts that makes one chunk of each, or many
    for max_kv in {max(lens), t.table.shape[1] * 32}:
        t.check(q, counts, t.run(q, counts, max_kv=max_kv))


def test_more_is_refused():
    m = mq()
    t = Case([40], 1, 64, 32, torch.float16)
    with pytest.raises(m.MQError):
        t.run(t.queries([1], 1025), [1])
