"""What an id that a teacher lists twice is to the distillation loss: two entries of the
divergence, and one token of the gradient."""
import math

import pytest
import torch

from . import distillation_reference as R
from .test_gpu_distillation import call, gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rest", [False, True])
def test_entries_of_one_id(rest):
    x = torch.randn((1, 301), generator=gpu(50), device="cuda")
    log_p = torch.log_softmax(x[0].double(), 0).tolist()
    q = [0.3, 0.1, 0.2, 0.4] if not rest else [0.3, 0.1, 0.2, 0.15]
    ids = [7, 300, 7, 0]
    values = torch.tensor([[math.log(v) for v in q]], device="cuda")
    loss, _, dx = call(x, torch.tensor([ids], dtype=torch.int32, device="cuda"), values, rest=rest)
    q0 = 1.0 - math.fsum(q) if rest else 0.0
    p0 = 1.0 - math.fsum(math.exp(log_p[i]) for i in set(ids))
    left = q0 * math.log(q0 / p0) if rest else 0.0
    entries = math.fsum(v * (math.log(v) - log_p[i]) for v, i in zip(q, ids)) + left
    merged = {i: math.fsum(v for v, j in zip(q, ids) if j == i) for i in ids}
    summed = math.fsum(v * (math.log(v) - log_p[i]) for i, v in merged.items()) + left
    # Logarithms of up to 8, each and the values given in binary32, good to a few half steps.
    bound = 64 * R.ULP * 8
    assert abs(float(loss) - entries) <= bound < summed - entries
    for i, v in merged.items():
        assert abs(float(dx[0, i]) - (math.exp(log_p[i]) - v)) <= bound

    # The same gradient as that of the sums.
    once = torch.tensor([list(merged)], dtype=torch.int32, device="cuda")
    _, _, same = call(x, once, torch.tensor([[math.log(v) for v in merged.values()]], device="cuda"), rest=rest)
    assert float((dx - same).abs().max()) <= bound
