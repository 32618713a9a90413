"""Activations kept in 8 bits on the GPU against the format's definition and the
formulas in binary64.

Tolerances, derived before the first run (u = 2^-24, 2-norm over 2-norm):
  codes, scales, restored values: exact (every step is a power of two).
  activations and their slopes in fp32: sigmoid from ex2 and a division, 2 ulp
      each, on an exponent that is off by u of |2 y| <= 20 (beyond, the sigmoid is 0
      or 1): a few 1e-6 relative where it matters; erf a few ulp.  Bound 3e-6.
  bf16 outputs: one rounding to 8 significant bits, 2^-8 each: bound 4e-3.
  weight gradient: exact products summed in binary32.  The sum of n terms is off
      by at most n u of the sum of magnitudes; for random signs the result is
      sqrt(n) times smaller than that sum and the error grows like sqrt(n) or, if
      additions cut instead of rounding, like n: bound 2 u (16 + n / 16) for
      fp32 results (one addition per 16 products in the matrix instructions), plus
      2^-8 for bf16 results.
"""
import math

import pytest
import torch

from tests import worker_step_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ACT = {torch.float32: 3e-6, torch.bfloat16: 4e-3}


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


def matrix(T, C, dtype, offset=0, pad=0, fill=5.0):
    ld = C + pad
    store = torch.full((offset + T * ld + 64,), fill, device="cuda").to(dtype)
    return store[offset: offset + T * ld].view(T, ld)[:, :C]


def make(T, C, dtype, seed, offset=0, pad=0, spread=4.0):
    """Values whose blocks' magnitudes lie up to 2^spread apart."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = matrix(T, C, dtype, offset, pad)
    size = torch.exp2(spread * (torch.rand((T, C), generator=g, device="cuda") - 0.5))
    x.copy_(torch.randn((T, C), generator=g, device="cuda") * size)
    return x, g


def keep(B, x, **kw):
    codes, scales = B.star_checkpoint_empty(*x.shape)
    codes.fill_(99)
    scales.fill_(99)
    B.star_checkpoint_pack(codes, scales, x, **kw)
    torch.cuda.synchronize()
    return codes, scales


SHAPES = [(1, 1), (1, 16), (2, 31), (3, 32), (5, 33), (64, 128), (65, 129), (7, 1000), (130, 257), (1, 4096), (33, 8200), (200, 1024)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,C", SHAPES)
def test_codes_scales_and_restored_values_are_exact(B, T, C, dtype):
    for offset, pad in ((0, 0), (0, 16), (1, 0), (3, 7)):
        x, _ = make(T, C, dtype, seed=T + C, offset=offset, pad=pad)
        codes, scales = keep(B, x)
        want_codes, want_scale, values = R.kept(x)
        assert torch.equal(codes[:, :C], want_codes)
        assert bool((codes[:, C:] == 0).all())
        assert torch.equal(R.scale_bytes(scales, T, C), want_scale)
        for out_dtype in (torch.float32, torch.bfloat16):
            out = matrix(T, C, out_dtype, offset, pad)
            base = out._base if out._base is not None else out
            B.star_checkpoint_unpack(out, codes, scales)
            assert torch.equal(out.double(), values)
            keep_out = torch.full_like(base.reshape(-1), 5.0)
            keep_out[offset: offset + T * (C + pad)].view(T, C + pad)[:, :C] = out
            assert torch.equal(base.reshape(-1), keep_out)               # nothing outside was written


def test_special_values(B):
    for dtype in (torch.float32, torch.bfloat16):
        x, _ = make(10, 70, dtype, seed=4)
        x[0] = 0.0
        x[1, 3] = math.nan
        x[2, 40] = math.inf
        x[3, 69] = -math.inf
        x[4, :32] = 1e-40 if dtype == torch.float32 else 9.2e-41          # subnormal
        x[5, 5] = 3e38
        x[6, 5] = 2.5e33                                                 # the largest that fits is just above
        x[7] = -0.0
        x[8, :32] = 127.4
        x[9, :32] = 127.5 * 2.0 ** 104 if dtype == torch.float32 else 2.0 ** 111
        codes, scales = keep(B, x)
        want_codes, want_scale, values = R.kept(x)
        assert torch.equal(codes[:, :70], want_codes)
        assert torch.equal(R.scale_bytes(scales, 10, 70), want_scale)
        out = torch.empty((10, 70), device="cuda")
        B.star_checkpoint_unpack(out, codes, scales)
        assert R.rel(out, values) == 0.0
        assert bool(torch.isnan(out[1, :32]).all()) and bool(torch.isfinite(out[1, 32:]).all())
        assert bool(torch.isnan(out[3, 64:]).all()) and bool(torch.isnan(out[9, :32]).all())
        # the error bound of the format, on finite blocks
        ok = torch.isfinite(out)
        blocks = torch.nn.functional.pad(x.double(), (0, 26)).view(10, 3, 32).abs().amax(2).repeat_interleave(32, 1)[:, :70]
        assert bool(((out.double() - x.double()).abs()[ok] <= blocks[ok] / 127 + 2.0 ** -127).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("T,C", [(1, 1), (3, 50), (65, 129), (40, 1024), (9, 4104)])
def test_activation_forward_and_backward(B, T, C, act, dtype):
    for offset, pad in ((0, 0), (1, 0), (2, 14)):
        x, g = make(T, C, dtype, seed=T * C + 1, offset=offset, pad=pad)
        h = matrix(T, C, dtype, offset, pad)
        codes, scales = keep(B, x, act=act, act_out=h)
        assert R.rel(h, R.act(x.double(), act)) <= ACT[dtype]
        plain_codes, plain_scales = keep(B, x)
        assert torch.equal(codes, plain_codes)
        values = R.kept(x)[2]
        out = matrix(T, C, dtype, offset, pad)
        B.star_checkpoint_unpack(out, codes, scales, act=act)
        assert R.rel(out, R.act(values, act)) <= ACT[dtype]
        dy, _ = make(T, C, dtype, seed=T + C + 9, offset=offset, pad=pad)
        dx = matrix(T, C, dtype, offset, pad)
        B.star_checkpoint_act_backward(dx, dy, codes, scales, act)
        assert R.rel(dx, dy.double() * R.act_slope(values, act)) <= ACT[dtype]
        got = dx.clone()
        B.star_checkpoint_act_backward(dy, dy, codes, scales, act)       # in place
        assert torch.equal(dy, got)
        B.star_checkpoint_pack(codes, scales, x, act=act, act_out=x)     # in place
        assert torch.equal(x, h)
        assert torch.equal(codes, plain_codes) and torch.equal(R.scale_bytes(scales, T, C), R.scale_bytes(plain_scales, T, C))


@pytest.mark.parametrize("act", R.ACTS[1:])
def test_slope_against_differences(B, act):
    """Central differences of the forward activation on kept values, h = 2^-7:
    3e-6 * |act| / 2h = 8e-4 |act|, third derivative h^2 / 6 = 1e-5."""
    x = torch.arange(-64, 64, device="cuda").float().view(4, 32) / 16.0
    codes, scales = keep(B, x)
    value = torch.empty_like(x)
    B.star_checkpoint_unpack(value, codes, scales)
    dx = torch.empty_like(x)
    B.star_checkpoint_act_backward(dx, torch.ones_like(x), codes, scales, act)
    h, up, down = 2.0 ** -7, torch.empty_like(x), torch.empty_like(x)
    keep(B, value + h, act=act, act_out=up)
    keep(B, value - h, act=act, act_out=down)
    assert bool(((up - down) / (2 * h) - dx).abs().max() <= 8e-4 * 4 + 1e-5)


def test_large_activations_stay_finite(B):
    x = torch.tensor([[1e30, -1e30, 1e20, -1e20, 100.0, -100.0, 0.0, 5.0]], device="cuda")
    for act in R.ACTS:
        for j in range(8):                                # one value a block
            one = x[:, j: j + 1].contiguous()
            codes, scales = keep(B, one)
            value, dx = torch.empty_like(one), torch.empty_like(one)
            B.star_checkpoint_unpack(value, codes, scales)
            B.star_checkpoint_act_backward(dx, torch.ones_like(one), codes, scales, act)
            want = 1.0 if act == "none" or float(one) > 50 else 0.0 if float(one) < -50 else float(R.act_slope(value.double(), act))
            assert abs(float(dx) - want) <= 1e-5, (act, j)


def grad_bound(n, dtype):
    return 2 * U * (16 + n / 16) + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)


def weight_case(B, T, C, O, dy_dtype, dw_dtype, seed, dy_offset=0, dy_pad=0, dw_offset=0, dw_pad=0, transposed=False, accumulate=False):
    x, g = make(T, C, torch.bfloat16, seed=seed, spread=6.0)
    codes, scales = keep(B, x)
    values = R.kept(x)[2]
    dy = matrix(T, O, dy_dtype, dy_offset, dy_pad, fill=1e30)            # what lies between the rows must not matter
    dy.copy_(torch.randn((T, O), generator=g, device="cuda") * 0.01)
    shape = (C, O) if transposed else (O, C)
    dw = matrix(*shape, dw_dtype, dw_offset, dw_pad, fill=3.0)
    if accumulate:
        dw.copy_(torch.randn(shape, generator=g, device="cuda"))
    before = dw.double().clone()
    base = dw._base.reshape(-1) if dw._base is not None else dw.reshape(-1)
    B.star_checkpoint_weight_grad(dw, dy, codes, scales, transposed=transposed, accumulate=accumulate)
    torch.cuda.synchronize()
    want = dy.double().t() @ values
    if transposed:
        want = want.t()
    if accumulate:
        want = want + before
    assert R.rel(dw, want) <= grad_bound(T, dw_dtype)
    rest = torch.full_like(base, 3.0)
    rest[dw_offset: dw_offset + shape[0] * (shape[1] + dw_pad)].view(shape[0], -1)[:, :shape[1]] = dw
    assert torch.equal(base, rest)                                       # nothing outside was written


# around the tile sizes 32 / 64 / 128 / 256 of rows, columns and outputs
WEIGHT_SHAPES = [(1, 1, 1), (1, 128, 256), (2, 17, 40), (63, 128, 256), (64, 130, 8), (65, 127, 264), (200, 256, 512), (128, 1000, 72),
                 (515, 200, 300), (1000, 384, 520), (4100, 144, 136)]


@pytest.mark.parametrize("dw_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dy_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,C,O", WEIGHT_SHAPES)
def test_weight_grad_over_sizes(B, T, C, O, dy_dtype, dw_dtype):
    weight_case(B, T, C, O, dy_dtype, dw_dtype, seed=T + C + O)
    weight_case(B, T, C, O, dy_dtype, dw_dtype, seed=T + C + O + 1, transposed=True, accumulate=True)


@pytest.mark.parametrize("dw_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dy_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offsets", [(1, 0, 0, 0), (0, 3, 1, 0), (0, 8, 0, 8), (8, 0, 3, 5), (4, 4, 2, 2)])
def test_weight_grad_strides_and_alignments(B, offsets, dy_dtype, dw_dtype):
    for transposed in (False, True):
        weight_case(B, 190, 129, 271, dy_dtype, dw_dtype, 5, *offsets, transposed=transposed, accumulate=not transposed)
        weight_case(B, 70, 256, 256, dy_dtype, dw_dtype, 6, *offsets, transposed=transposed)


@pytest.mark.parametrize("T,C,O", [(2048, 1024, 1024), (8192, 256, 512), (16384, 128, 128), (3000, 1000, 2000)])
def test_weight_grad_larger(B, T, C, O):
    for dy_dtype, dw_dtype in ((torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)):
        weight_case(B, T, C, O, dy_dtype, dw_dtype, seed=T)


def test_weight_grad_is_the_same_every_time(B):
    x, g = make(3000, 512, torch.bfloat16, seed=1)
    codes, scales = keep(B, x)
    dy = torch.randn((3000, 768), generator=g, device="cuda").to(torch.bfloat16)
    first = torch.empty((768, 512), device="cuda")
    B.star_checkpoint_weight_grad(first, dy, codes, scales)
    for _ in range(5):
        again = torch.empty_like(first)
        B.star_checkpoint_weight_grad(again, dy, codes, scales)
        assert torch.equal(again, first)


def test_weight_grad_against_differences(B):
    """The loss sum(dy * (x_kept W^T)) is linear in W: its difference quotient is the gradient itself."""
    T, C, O = 20, 40, 24
    x, g = make(T, C, torch.float32, seed=2)
    codes, scales = keep(B, x)
    values = torch.empty_like(x)
    B.star_checkpoint_unpack(values, codes, scales)
    dy = torch.randn((T, O), generator=g, device="cuda")
    dw = torch.empty((O, C), device="cuda")
    B.star_checkpoint_weight_grad(dw, dy, codes, scales)
    W = torch.randn((O, C), generator=g, device="cuda").double()
    loss = lambda w: (dy.double() * (values.double() @ w.t())).sum()  # noqa: E731
    for o, c in ((0, 0), (23, 39), (5, 17)):
        step = torch.zeros_like(W)
        step[o, c] = 0.5
        size = float((dy[:, o].abs() * values[:, c].abs()).sum())
        assert abs(float(loss(W + step) - loss(W - step)) - float(dw[o, c])) <= 40 * U * size


def test_overflowed_block_reaches_the_weight_gradient(B):
    x, g = make(100, 200, torch.bfloat16, seed=3)
    x[50, 70] = math.inf
    codes, scales = keep(B, x)
    for dy_dtype in (torch.bfloat16, torch.float32):
        dy = torch.randn((100, 96), generator=g, device="cuda").to(dy_dtype)
        dw = torch.empty((96, 200), device="cuda")
        B.star_checkpoint_weight_grad(dw, dy, codes, scales)
        assert bool(torch.isnan(dw[:, 64:96]).all())
        assert bool(torch.isfinite(dw[:, :64]).all()) and bool(torch.isfinite(dw[:, 96:]).all())


def test_extreme_scales_in_the_weight_gradient(B):
    for size in (2.0 ** -120, 2.0 ** 100):
        x = torch.randn((70, 64), device="cuda") * size
        codes, scales = keep(B, x)
        dy = torch.randn((70, 32), device="cuda").to(torch.bfloat16)
        dw = torch.empty((32, 64), device="cuda")
        B.star_checkpoint_weight_grad(dw, dy, codes, scales)
        want = dy.double().t() @ R.kept(x)[2]
        # results below binary32's normal range may be flushed
        assert float((dw.double() - want).abs().max()) <= grad_bound(70, torch.float32) * float(want.abs().max()) + 2.0 ** -126


def test_empty_sizes(B):
    for T, C in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty((T, C), device="cuda")
        codes, scales = B.star_checkpoint_empty(T, C)
        B.star_checkpoint_pack(codes, scales, x)
        B.star_checkpoint_unpack(x, codes, scales)
        B.star_checkpoint_act_backward(x, x, codes, scales, "silu")
        dy = torch.empty((T, 7), device="cuda")
        dw = torch.full((7, C), 2.0, device="cuda")
        B.star_checkpoint_weight_grad(dw, dy, codes, scales, accumulate=True)
        assert bool((dw == 2.0).all())
        B.star_checkpoint_weight_grad(dw, dy, codes, scales)
        assert bool((dw == 0.0).all())


def test_other_streams_and_graph_replay(B):
    x, g = make(300, 520, torch.bfloat16, seed=9)
    dy = torch.randn((300, 264), generator=g, device="cuda").to(torch.bfloat16)
    dh, _ = make(300, 520, torch.bfloat16, seed=10)
    codes, scales = keep(B, x)
    h, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty((264, 520), device="cuda", dtype=torch.bfloat16)

    def step(stream=None):
        B.star_checkpoint_pack(codes, scales, x, act="gelu_tanh", act_out=h, stream=stream)
        B.star_checkpoint_act_backward(dx, dh, codes, scales, "gelu_tanh", stream=stream)
        B.star_checkpoint_weight_grad(dw, dy, codes, scales, stream=stream)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (h, dx, dw)]
    side = torch.cuda.Stream()
    for t in (h, dx, dw):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((h, dx, dw), want))
    for t in (h, dx, dw):
        t.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((h, dx, dw), want))
