"""Arguments that the operators of a distillation step refuse, before anything is
launched: addresses that are never read stand in for device memory, no GPU is needed."""
import ctypes
import math

import pytest
import torch

from paper_2512_09685_b200 import binding as B

OK, NULL, INVALID, SMALL, UNSUPPORTED = B.STAR_OK, B.STAR_ERR_NULL_POINTER, B.STAR_ERR_INVALID_ARG, B.STAR_ERR_WORKSPACE_TOO_SMALL, B.STAR_ERR_UNSUPPORTED
MB = 1 << 20


def address(k):
    """The k-th of many address ranges of 1 GiB that do not meet."""
    return (k + 16) << 30


TOP = dict(logits=address(0), dtype=0, rows=8, vocab=100, ld=100, labels=address(1), temperature=1.0, k=5, ids=address(2), top=address(3), ld_top=5,
           logp=address(4), lse=address(5), entropy=address(6), stream=None)
TOP_BACK = dict(dlogits=address(9), ld_dlogits=100, logits=address(0), dtype=1, rows=8, vocab=100, ld=100, labels=address(1), temperature=1.0,
                lse=address(2), entropy=address(3), d_logp=address(4), d_entropy=address(5), k=5, ids=address(6), ld_top=5, d_top=address(7), ld_d_top=6,
                stream=None)
DISTILL = dict(logits=address(0), dtype=0, rows=8, vocab=100, ld=100, ids=address(1), ld_ids=5, values=address(2), ld_values=6, k=5, rest=1,
               teacher_temperature=1.0, labels=address(3), weights=address(4), temperature=1.0, soft=1.0, hard=0.5, token_loss=address(5), sums=address(6),
               dlogits=address(7), ld_dlogits=100, workspace=address(8), ws_bytes=MB, stream=None)
NORM = dict(y=address(0), ld_y=100, x=address(1), ld_x=100, residual=address(2), ld_residual=100, total=address(3), ld_total=100, dtype=1, rows=8, cols=100,
            gain=address(4), gain_dtype=0, eps=1e-5, rstd=address(5), codes=address(6), scales=address(7), stream=None)
NORM_BACK = dict(dx=address(0), ld_dx=100, dgain=address(1), dgain_dtype=0, accumulate=0, dy=address(2), ld_dy=100, total=address(3), ld_total=100,
                 codes=None, scales=None, d_total=address(4), ld_d_total=100, dtype=1, rows=8, cols=100, gain=address(5), gain_dtype=1, rstd=address(6),
                 workspace=address(7), ws_bytes=MB, stream=None)
CALLS = {"star_token_alternatives": TOP, "star_token_alternatives_backward": TOP_BACK, "star_distillation_loss": DISTILL, "star_rms_norm": NORM,
         "star_rms_norm_backward": NORM_BACK}

ROWS = [(dict(dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(vocab=-1), INVALID), (dict(ld=99), INVALID), (dict(logits=None), NULL),
        (dict(logits=address(0) + 1), INVALID), (dict(labels=address(1) + 4), INVALID), (dict(temperature=0.0), INVALID), (dict(temperature=math.nan), INVALID),
        (dict(temperature=1e-40), INVALID), (dict(rows=1 << 50, ld=1 << 30), INVALID), (dict(vocab=1 << 31, ld=1 << 31), UNSUPPORTED), (dict(k=-1), INVALID),
        (dict(k=129, ld_top=129, ld_d_top=129, ld_ids=129, ld_values=129), UNSUPPORTED), (dict(ids=None), NULL)]
KNOWN = lambda name, cases: [(c, s) for c, s in ((({k: v for k, v in c.items() if k in CALLS[name]}), s) for c, s in cases) if c]  # noqa: E731

REFUSED = {
    "star_token_alternatives": KNOWN("star_token_alternatives", ROWS) + [
        (dict(ld_top=4), INVALID), (dict(top=None), NULL), (dict(ids=address(2) + 2), INVALID), (dict(labels=None), NULL), (dict(logp=address(0) + 4), INVALID),
        (dict(lse=address(4)), INVALID), (dict(entropy=address(2) + 8), INVALID), (dict(top=address(2)), INVALID), (dict(ids=address(1)), INVALID)],
    "star_token_alternatives_backward": KNOWN("star_token_alternatives_backward", ROWS) + [
        (dict(lse=None), NULL), (dict(entropy=None), NULL), (dict(labels=None), NULL), (dict(d_top=None), NULL), (dict(ld_top=4), INVALID),
        (dict(ld_d_top=4), INVALID), (dict(dlogits=None), NULL), (dict(ld_dlogits=99), INVALID), (dict(dlogits=address(0) + 2), INVALID),
        (dict(dlogits=address(0), ld_dlogits=101), INVALID), (dict(dlogits=address(2)), INVALID), (dict(dlogits=address(7)), INVALID),
        (dict(d_entropy=address(5) + 1), INVALID)],
    "star_distillation_loss": [c for c in KNOWN("star_distillation_loss", ROWS) if "labels" not in c[0]] + [
        (dict(labels=address(3) + 4), INVALID), (dict(labels=None), NULL), (dict(values=None), NULL), (dict(ld_ids=4), INVALID), (dict(ld_values=4), INVALID),
        (dict(teacher_temperature=0.0), INVALID), (dict(teacher_temperature=math.inf), INVALID), (dict(teacher_temperature=1e-40), INVALID),
        (dict(soft=math.nan), INVALID), (dict(hard=math.inf), INVALID), (dict(token_loss=None), NULL), (dict(sums=None), NULL), (dict(workspace=None), NULL),
        (dict(workspace=address(8) + 8), INVALID), (dict(ws_bytes=16), SMALL), (dict(ld_dlogits=99), INVALID), (dict(dlogits=address(0) + 4), INVALID),
        (dict(dlogits=address(1)), INVALID), (dict(dlogits=address(8)), INVALID), (dict(sums=address(2)), INVALID), (dict(token_loss=address(6)), INVALID),
        (dict(vocab=425985, ld=425985, ld_dlogits=425985), UNSUPPORTED), (dict(dtype=1, vocab=851969, ld=851969, ld_dlogits=851969), UNSUPPORTED)],
    "star_rms_norm": [
        (dict(dtype=2), INVALID), (dict(gain_dtype=3), INVALID), (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID),
        (dict(eps=math.inf), INVALID), (dict(rows=-1), INVALID), (dict(cols=-1), INVALID), (dict(ld_x=99), INVALID), (dict(ld_y=99), INVALID),
        (dict(ld_residual=99), INVALID), (dict(ld_total=99), INVALID), (dict(x=None), NULL), (dict(y=None), NULL), (dict(codes=None), NULL),
        (dict(scales=None), NULL), (dict(codes=address(6) + 8), INVALID), (dict(scales=address(7) + 4), INVALID), (dict(x=address(1) + 1), INVALID),
        (dict(gain=address(4) + 2), INVALID), (dict(y=address(1)), INVALID), (dict(y=address(2)), INVALID), (dict(y=address(4) + 8), INVALID),
        (dict(total=address(1), ld_total=101), INVALID), (dict(total=address(2) + 2), INVALID), (dict(total=address(0)), INVALID), (dict(total=address(4)), INVALID),
        (dict(rstd=address(0)), INVALID), (dict(rstd=address(5) + 2), INVALID), (dict(codes=address(7)), INVALID), (dict(total=address(6)), INVALID),
        (dict(rows=1 << 31, codes=None, scales=None), UNSUPPORTED)],
    "star_rms_norm_backward": [
        (dict(dtype=2), INVALID), (dict(gain_dtype=3), INVALID), (dict(dgain_dtype=2), INVALID), (dict(ld_dx=99), INVALID), (dict(ld_dy=99), INVALID),
        (dict(ld_total=99), INVALID), (dict(ld_d_total=99), INVALID), (dict(dx=None), NULL), (dict(dy=None), NULL), (dict(total=None), NULL),
        (dict(rstd=None), NULL), (dict(codes=address(9), scales=address(10)), INVALID), (dict(total=None, codes=address(9)), NULL),
        (dict(total=None, codes=address(9) + 8, scales=address(10)), INVALID), (dict(workspace=None), NULL), (dict(workspace=address(7) + 4), INVALID),
        (dict(ws_bytes=3200), SMALL), (dict(dx=address(2) + 2), INVALID), (dict(dx=address(2), ld_dx=101), INVALID), (dict(dx=address(3)), INVALID),
        (dict(dx=address(4), ld_dx=104), INVALID), (dict(dx=address(6)), INVALID), (dict(dgain=address(0)), INVALID), (dict(dgain=address(5)), INVALID),
        (dict(dgain=address(1) + 2), INVALID), (dict(workspace=address(0)), INVALID), (dict(rows=-1), INVALID), (dict(dy=address(2) + 1), INVALID),
        (dict(rows=1 << 31, dgain=None), UNSUPPORTED)],
}


def call(name, **changes):
    return getattr(B._lib, name)(*{**CALLS[name], **changes}.values())


@pytest.mark.parametrize("name,changes,status", [(n, c, s) for n, cases in REFUSED.items() for c, s in cases])
def test_refused(name, changes, status):
    before = B.star_launch_count()
    assert call(name, **changes) == status
    assert B.star_launch_count() == before


def test_calls_without_work_succeed_without_a_device():
    assert call("star_token_alternatives", rows=0, logits=None, labels=None, ids=None, top=None, logp=None, lse=None, entropy=None) == OK
    assert call("star_token_alternatives_backward", rows=0, dlogits=None, logits=None, labels=None, lse=None, entropy=None, d_logp=None, d_entropy=None,
                ids=None, d_top=None) == OK
    assert call("star_token_alternatives_backward", vocab=0, dlogits=None, logits=None) == OK
    assert call("star_rms_norm", rows=0, x=None, y=None, residual=None, total=None, rstd=None, codes=None, scales=None) == OK
    assert call("star_rms_norm", cols=0, x=None, y=None, residual=None, total=None, gain=None, codes=None, scales=None) == OK
    assert call("star_rms_norm_backward", cols=0, dx=None, dy=None, total=None, d_total=None, gain=None, dgain=None) == OK
    assert call("star_rms_norm_backward", rows=0, dgain=None, dx=None, dy=None, total=None, d_total=None, rstd=None) == OK


def test_workspace_bytes():
    assert B.star_rms_norm_workspace_bytes(1, 100) >= 400
    assert B.star_rms_norm_workspace_bytes(0, 100) >= 0
    assert B.star_rms_norm_workspace_bytes(1 << 40, 100) == B.star_rms_norm_workspace_bytes(1 << 20, 100)
    out = ctypes.c_size_t(0)
    assert B._lib.star_rms_norm_workspace_bytes(1, 1, None) == NULL
    assert B._lib.star_rms_norm_workspace_bytes(-1, 1, ctypes.byref(out)) == INVALID
    assert B._lib.star_rms_norm_workspace_bytes(1, -1, ctypes.byref(out)) == INVALID
    assert B._lib.star_rms_norm_workspace_bytes(1, 1 << 55, ctypes.byref(out)) == INVALID


def test_the_binding_refuses_wrong_tensors():
    x, v, ids = torch.zeros(4, 10), torch.zeros(4), torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(TypeError):                        # not on a GPU
        B.star_token_alternatives(x)
    with pytest.raises(TypeError):
        B.star_token_alternatives_backward(x, x, v)
    with pytest.raises(TypeError):
        B.star_distillation_loss(x, ids, ids.float(), v, v, v)
    with pytest.raises(TypeError):
        B.star_rms_norm(x, x)
    with pytest.raises(TypeError):
        B.star_rms_norm_backward(x, None, x, None, v, total=x)
    with pytest.raises(TypeError):
        B._listed(ids.long(), 4, 2, "ids", torch.int32)
    with pytest.raises(ValueError):
        B._optional_kept(ids, None, 4, 10)
