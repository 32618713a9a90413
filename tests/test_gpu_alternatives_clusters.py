"""The top alternatives by clusters of two, four and eight blocks, with one row and with
several to a cluster, some of which take no part."""
import pytest
import torch

from . import distillation_reference as R
from .test_gpu_alternatives import BF16, F32, call, check, gpu, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [5, 128])
@pytest.mark.parametrize("rows,vocab,dtype", [(9, 32003, BF16), (18, 32003, BF16), (37, 50257, BF16), (18, 50257, BF16), (74, 50257, BF16), (75, 50257, BF16),
                                              (37, 128259, BF16), (148, 128259, BF16), (296, 128259, BF16), (297, 128259, BF16), (74, 32001, F32),
                                              (148, 50257, F32)])
def test_rows_that_clusters_share(rows, vocab, dtype, k):
    x = make(rows, vocab, dtype, seed=rows)
    labels = torch.randint(0, vocab, (rows,), generator=gpu(rows), device="cuda")
    off = torch.rand(rows, generator=gpu(rows + 1), device="cuda") < 0.4
    labels[off] = -100
    got = call(x, k, labels=labels, temperature=1.3)
    pick = torch.cat([torch.arange(0, rows, max(1, rows // 12), device="cuda"), torch.nonzero(off)[:3, 0]])
    want = R.alternatives(x[pick], k, labels[pick], 1.3)
    check({n: v[pick] for n, v in got.items()}, want, k)
    assert bool((got["ids"][off] == -1).all()) and bool(torch.isinf(got["lse"][off]).all())
    # Every row against a call of its own.
    for t in range(0, rows, max(1, rows // 40)):
        one = call(x[t:t + 1], k, labels=labels[t:t + 1], temperature=1.3)
        assert torch.equal(one["ids"], got["ids"][t:t + 1])
