"""Arguments that the operators of a worker's step refuse.  Every refusal comes
before anything is launched, so addresses that are never read stand in for
device memory and no GPU is needed."""
import ctypes
import math

import pytest
import torch

from paper_2512_09685_b200 import binding as B

OK, NULL, INVALID, SMALL = B.STAR_OK, B.STAR_ERR_NULL_POINTER, B.STAR_ERR_INVALID_ARG, B.STAR_ERR_WORKSPACE_TOO_SMALL
MB = 1 << 20


def address(k):
    """The k-th of many address ranges of 1 GiB that do not meet."""
    return (k + 16) << 30


LOGPROBS = dict(logits=address(0), dtype=0, rows=8, vocab=100, ld=100, labels=address(1), temperature=1.0, logp=address(2),
                lse=address(3), stream=None)
POLICY = dict(logits=address(0), dtype=0, rows=8, vocab=100, ld=100, labels=address(1), weights=address(2), advantages=address(3),
              old=address(4), ref=address(5), temperature=1.0, clip_low=0.2, clip_high=0.2, kl=0.1, logp=address(6),
              token_loss=address(7), sums=address(8), dlogits=address(9), ld_dlogits=100, workspace=address(10), ws_bytes=MB,
              stream=None)
PREFERENCE = dict(logits=address(0), dtype=1, rows=8, vocab=100, ld=100, labels=address(1), offsets=address(2), pairs=2,
                  ref=address(3), temperature=1.0, beta=0.1, smoothing=0.0, average=0, scale=1.0, seq_logp=address(4),
                  pair_loss=address(5), margin=address(6), loss=address(7), dlogits=address(8), ld_dlogits=100,
                  workspace=address(9), ws_bytes=MB, stream=None)
PACK = dict(codes=address(0), scales=address(1), x=address(2), dtype=0, rows=8, cols=100, ld=100, act=1, act_out=address(3),
            ld_act=100, stream=None)
UNPACK = dict(out=address(2), dtype=0, ld=100, codes=address(0), scales=address(1), rows=8, cols=100, act=0, stream=None)
BACKWARD = dict(dx=address(2), ld_dx=100, dy=address(3), ld_dy=100, dtype=1, codes=address(0), scales=address(1), rows=8, cols=100,
                act=3, stream=None)
WEIGHT = dict(dw=address(2), dw_dtype=0, ld_dw=100, transposed=0, dy=address(3), dy_dtype=1, ld_dy=48, codes=address(0),
              scales=address(1), rows=8, cols=100, outs=48, accumulate=0, stream=None)
CALLS = {"star_token_logprobs": LOGPROBS, "star_policy_loss": POLICY, "star_preference_loss": PREFERENCE,
         "star_checkpoint_pack": PACK, "star_checkpoint_unpack": UNPACK, "star_checkpoint_act_backward": BACKWARD,
         "star_checkpoint_weight_grad": WEIGHT}

COMMON_ROWS = [(dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(rows=-1), INVALID), (dict(vocab=-1), INVALID),
               (dict(ld=99), INVALID), (dict(logits=None), NULL), (dict(labels=None), NULL), (dict(logits=address(0) + 1), INVALID),
               (dict(labels=address(1) + 4), INVALID), (dict(temperature=0.0), INVALID), (dict(temperature=-1.0), INVALID),
               (dict(temperature=math.nan), INVALID), (dict(temperature=math.inf), INVALID), (dict(temperature=1e-40), INVALID),
               (dict(rows=1 << 50, ld=1 << 30), INVALID), (dict(vocab=1 << 31, ld=1 << 31), B.STAR_ERR_UNSUPPORTED), (dict(logp=address(0) + 4), INVALID), (dict(logp=address(1)), INVALID)]

REFUSED = {
    "star_token_logprobs": COMMON_ROWS + [(dict(logp=None), NULL), (dict(lse=address(2)), INVALID), (dict(logp=address(2) + 2), INVALID)],
    "star_policy_loss": COMMON_ROWS + [
        (dict(advantages=None), NULL), (dict(logp=None), NULL), (dict(token_loss=None), NULL), (dict(sums=None), NULL),
        (dict(clip_low=-0.1), INVALID), (dict(clip_low=1.1), INVALID), (dict(clip_high=-0.1), INVALID), (dict(clip_low=math.nan), INVALID),
        (dict(kl=math.inf), INVALID), (dict(ld_dlogits=99), INVALID), (dict(dlogits=address(0) + 4), INVALID),
        (dict(dlogits=address(0), ld_dlogits=101), INVALID), (dict(dlogits=address(6)), INVALID), (dict(dlogits=address(10)), INVALID),
        (dict(workspace=None), NULL), (dict(workspace=address(10) + 8), INVALID), (dict(ws_bytes=8), SMALL),
        (dict(sums=address(3)), INVALID), (dict(token_loss=address(6) + 4), INVALID), (dict(workspace=address(4)), INVALID)],
    "star_preference_loss": [c for c in COMMON_ROWS if "logp" not in c[0]] + [
        (dict(offsets=None), NULL), (dict(pairs=-1), INVALID), (dict(seq_logp=None), NULL), (dict(pair_loss=None), NULL),
        (dict(margin=None), NULL), (dict(loss=None), NULL), (dict(beta=math.inf), INVALID), (dict(smoothing=-0.1), INVALID),
        (dict(smoothing=1.5), INVALID), (dict(scale=math.nan), INVALID), (dict(ld_dlogits=99), INVALID),
        (dict(dlogits=address(0) + 2), INVALID), (dict(dlogits=address(9)), INVALID), (dict(workspace=None), NULL),
        (dict(ws_bytes=16), SMALL), (dict(margin=address(5) + 4), INVALID), (dict(loss=address(3)), INVALID),
        (dict(offsets=address(2) + 2), INVALID), (dict(pairs=1 << 40), INVALID)],
    "star_checkpoint_pack": [
        (dict(dtype=5), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(rows=-1), INVALID), (dict(cols=-1), INVALID),
        (dict(ld=99), INVALID), (dict(ld_act=99), INVALID), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(x=None), NULL),
        (dict(codes=address(0) + 8), INVALID), (dict(scales=address(1) + 4), INVALID), (dict(x=address(2) + 2), INVALID),
        (dict(act_out=address(2) + 4), INVALID), (dict(act_out=address(2), ld_act=104), INVALID), (dict(act_out=address(0)), INVALID),
        (dict(x=address(1)), INVALID), (dict(scales=address(0) + 16), INVALID), (dict(rows=1 << 53), INVALID),
        (dict(rows=1 << 40, cols=1 << 30, ld=1 << 30), INVALID)],
    "star_checkpoint_unpack": [
        (dict(dtype=5), INVALID), (dict(act=9), INVALID), (dict(ld=99), INVALID), (dict(out=None), NULL), (dict(codes=None), NULL),
        (dict(scales=None), NULL), (dict(out=address(0)), INVALID), (dict(out=address(1)), INVALID), (dict(rows=-2), INVALID)],
    "star_checkpoint_act_backward": [
        (dict(dtype=2), INVALID), (dict(act=4), INVALID), (dict(ld_dx=99), INVALID), (dict(ld_dy=99), INVALID), (dict(dx=None), NULL),
        (dict(dy=None), NULL), (dict(dx=address(3) + 2), INVALID), (dict(dx=address(3), ld_dx=101), INVALID),
        (dict(dx=address(0)), INVALID), (dict(dx=address(1)), INVALID), (dict(dy=address(3) + 1), INVALID)],
    "star_checkpoint_weight_grad": [
        (dict(dw_dtype=2), INVALID), (dict(dy_dtype=3), INVALID), (dict(outs=-1), INVALID), (dict(ld_dw=99), INVALID),
        (dict(ld_dw=100, transposed=1, outs=101, ld_dy=101), INVALID), (dict(ld_dy=47), INVALID), (dict(dw=None), NULL),
        (dict(dy=None), NULL), (dict(dw=address(3)), INVALID), (dict(dw=address(0)), INVALID), (dict(dw=address(1)), INVALID),
        (dict(dw=address(2) + 2), INVALID), (dict(codes=None), NULL)],
}


def call(name, **changes):
    return getattr(B._lib, name)(*{**CALLS[name], **changes}.values())


@pytest.mark.parametrize("name,changes,status", [(n, c, s) for n, cases in REFUSED.items() for c, s in cases])
def test_refused(name, changes, status):
    before = B.star_launch_count()
    assert call(name, **changes) == status
    assert B.star_launch_count() == before


def test_calls_without_work_succeed_without_a_device():
    assert call("star_token_logprobs", rows=0, logits=None, labels=None, logp=None, lse=None) == OK
    assert call("star_checkpoint_pack", rows=0, codes=None, scales=None, x=None, act_out=None) == OK
    assert call("star_checkpoint_unpack", cols=0, codes=None, scales=None, out=None) == OK
    assert call("star_checkpoint_act_backward", rows=0, codes=None, scales=None, dx=None, dy=None) == OK
    assert call("star_checkpoint_weight_grad", outs=0, dw=None, dy=None, ld_dy=0) == OK
    assert call("star_checkpoint_weight_grad", rows=0, accumulate=1, dy=None, codes=None, scales=None) == OK


def test_sizes():
    assert B.star_checkpoint_sizes(0, 0) == (0, 0, 0)
    assert B.star_checkpoint_sizes(1, 1) == (16, 16, 256)
    assert B.star_checkpoint_sizes(65, 129) == (144, 65 * 144, 2 * 128 * 4)
    assert B.star_checkpoint_sizes(64, 128) == (128, 8192, 256)
    out = ctypes.c_int64(0)
    assert B._lib.star_checkpoint_sizes(1, 1, None, ctypes.byref(out), ctypes.byref(out)) == NULL
    assert B._lib.star_loss_workspace_bytes(1, 1, None) == NULL
    assert B._lib.star_loss_workspace_bytes(-1, 0, ctypes.byref(out)) == INVALID
    assert B.star_loss_workspace_bytes(1000, 4) >= 16000


def test_the_binding_refuses_wrong_tensors():
    x, labels, v = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    with pytest.raises(TypeError):                        # not on a GPU
        B.star_token_logprobs(x, labels, v)
    with pytest.raises(TypeError):
        B.star_token_logprobs(x.double(), labels, v)
    codes, scales = B.star_checkpoint_empty(4, 10, device="cpu")
    assert codes.shape == (4, 16) and scales.shape == (1, 64, 4)
    with pytest.raises(TypeError):
        B.star_checkpoint_unpack(x, codes, scales)
    with pytest.raises(ValueError):
        B._act("relu")
