"""The top alternatives, and their backward pass, of a row of the most logits: its indexes
are the last that 32 bits hold."""
import pytest
import torch

from . import distillation_reference as R

pytestmark = pytest.mark.gpu


def test_the_most_logits():
    from paper_2512_09685_b200 import binding as B
    vocab, k = (1 << 31) - 1, 5
    up = torch.nextafter(torch.tensor(1.0), torch.tensor(2.0)).item()
    x = torch.zeros((1, vocab), device="cuda")
    x[0, 100:2100] = 1.0                                 # more equals than candidates are kept
    x[0, vocab - 2:] = up                                # and a few above them: they are counted, and found at the end
    ids, top = torch.empty((1, k), dtype=torch.int32, device="cuda"), torch.empty((1, k), device="cuda")
    lse, entropy = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    B.star_token_alternatives(x, ids, top, lse=lse, entropy=entropy)
    assert ids[0].tolist() == [vocab - 2, vocab - 1, 100, 101, 102]
    sizes = torch.tensor([vocab - 2002, 2000, 2], dtype=torch.float64)
    values = torch.tensor([0.0, 1.0, up], dtype=torch.float64)
    want = float(torch.log((sizes * values.exp()).sum()))
    # A thread of eight blocks of 256 adds up 2^20 logits, 16 of them at a time; log p and lse are then rounded.
    bound = R.ULP * (1 << 16) + 4 * R.ULP * want
    assert abs(float(lse) - want) <= bound
    assert float((top[0].cpu().double() - (values[[2, 2, 1, 1, 1]] - want)).abs().max()) <= bound

    # The gradient goes to elements of another phase, one by one.
    dx = torch.full((vocab + 1,), 5.0, device="cuda")[1:].view(1, vocab)
    labels, one = torch.tensor([vocab - 1], device="cuda"), torch.ones(1, device="cuda")
    d_top = torch.arange(1.0, k + 1, device="cuda")[None]
    B.star_token_alternatives_backward(dx, x, lse, labels=labels, d_logp=one, top_ids=ids, d_top_logp=d_top)
    p = torch.exp(values - float(lse))
    total = 16.0                                         # 1 + (1 + ... + 5)
    dense = (-p * total)
    # An exponent of about 21: a half step for each of its units; the product's, and that of the sum with what names an element.
    close = lambda got, want: bool(((got.double() - want).abs() <= 32 * R.ULP * abs(want)).all())  # noqa: E731
    assert close(dx[0, :100], float(dense[0])) and close(dx[0, 103:2100], float(dense[1]))
    rest = dx[0, 2100:vocab - 2]
    assert close(torch.stack([rest.min(), rest.max()]), float(dense[0]))
    for at, g in ((vocab - 2, 1.0), (vocab - 1, 2.0 + 1.0), (100, 3.0), (101, 4.0), (102, 5.0)):
        which = 2 if at >= vocab - 2 else 1
        assert close(dx[0, at], g + float(dense[which]))
