"""The residual root-mean-square norm, its checkpoint and its backward pass against
the formulas in binary64."""
import math

import pytest
import torch

from . import distillation_reference as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def gpu(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def matrix(rows, cols, dtype, seed, ld=None, offset=0, scale=1.0):
    ld = ld or cols
    store = torch.full((offset + rows * ld + 64,), 7.0, dtype=dtype, device="cuda")
    x = store[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    x.copy_(torch.randn((rows, cols), generator=gpu(seed), device="cuda") * scale)
    return x


def near(got, want, bound):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = torch.isfinite(want)
    off = (got - want).abs()[fine]
    assert bool((off <= bound.expand_as(want)[fine]).all()), float((off / bound.expand_as(want)[fine]).max())


def forward(x, gain=None, residual=None, total="own", keep=True, eps=1e-5, y=None):
    from paper_2512_09685_b200 import binding as B
    rows, cols = x.shape
    before = x.clone(), None if residual is None else residual.clone()
    y = torch.full((rows, cols), 5.0, dtype=x.dtype, device="cuda") if y is None else y
    if isinstance(total, str):
        total = torch.full((rows, cols), 5.0, dtype=x.dtype, device="cuda")
    rstd = torch.full((rows,), 5.0, device="cuda")
    codes, scales = B.star_checkpoint_empty(rows, cols) if keep else (None, None)
    B.star_rms_norm(y, x, gain, residual=residual, total=total, rstd=rstd, codes=codes, scales=scales, eps=eps)
    torch.cuda.synchronize()
    stream = before[0] if residual is None else (before[0].float() + before[1].float()).to(x.dtype)
    if total is not None:
        assert torch.equal(total.float(), stream.float()) or torch.equal(torch.isnan(total), torch.isnan(stream))
    want, r = R.norm(stream, gain, eps)
    bound = R.norm_bound(cols)
    near(rstd, r, bound * r.abs())
    near(y, want, (bound + 4 * R.ULP + R.half_step(x.dtype)) * want.abs() + 1e-38)
    if keep:
        codes2, scales2 = B.star_checkpoint_empty(rows, cols)
        B.star_checkpoint_pack(codes2, scales2, y.contiguous())
        a, b = torch.empty((rows, cols), device="cuda"), torch.empty((rows, cols), device="cuda")
        assert torch.equal(codes, codes2)
        B.star_checkpoint_unpack(a, codes, scales)
        B.star_checkpoint_unpack(b, codes2, scales2)
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
    return y, total, rstd, codes, scales


SIZES = [(1, 1), (3, 7), (1, 4096), (5, 32), (64, 33), (70, 1000), (17, 1001), (200, 1024), (33, 4096), (9, 4095), (3, 8192), (600, 2048), (2, 16384), (4, 32768), (2, 40000),
         (3000, 64), (5000, 40), (2, 70001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, dtype):
    x, res = matrix(rows, cols, dtype, 1), matrix(rows, cols, dtype, 2)
    gain = 1 + 0.1 * torch.randn(cols, generator=gpu(3), device="cuda")
    forward(x, gain.to(BF16), res)
    forward(x, gain, None, total=None)
    forward(x, None, res, total=None, keep=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(1, 0), (3, 1), (8, 8), (16, 32), (0, 3)])
def test_strides_and_alignment(dtype, offset, extra):
    x, res = matrix(6, 520, dtype, 1, 520 + extra, offset), matrix(6, 520, dtype, 2, 544)
    gain = torch.full((531,), 2.0, device="cuda")[3:523]
    y = torch.full((6, 600), 5.0, dtype=dtype, device="cuda")[:, 1:521]
    forward(x, gain, res, y=y)
    forward(x, gain, res)
    forward(x, gain, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [512, 513, 4096])
def test_total_in_place(dtype, cols):
    for which in range(2):
        x, res = matrix(40, cols, dtype, 1), matrix(40, cols, dtype, 2)
        y0, total0, *_ = forward(x.clone(), None, res.clone())
        y1, *_ = forward(x, None, res, total=(x, res)[which])
        assert torch.equal(y0, y1) and torch.equal((x, res)[which], total0)
    x = matrix(40, cols, dtype, 1)
    forward(x, None, None, total=x)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_extremes(dtype):
    x = matrix(9, 1000, dtype, 1)
    x[0] = 0.0
    x[1] = 1e-20
    x[2] = 1e15
    x[3, 5] = math.nan
    x[4, 5] = math.inf
    x[5] = 0.0
    x[5, 999] = 1.0
    x[6] = 3e19                                          # squares beyond binary32
    x[7, ::2] = 0.0
    from paper_2512_09685_b200 import binding as B
    gain = torch.ones(1000, device="cuda")
    bad = [3, 4, 6]
    good = [t for t in range(9) if t not in bad]
    for cols in (1000, 999):
        part = x[:, :cols]
        y, rstd = torch.empty_like(part), torch.empty(9, device="cuda")
        codes, scales = B.star_checkpoint_empty(9, cols)
        B.star_rms_norm(y, part, gain[:cols], rstd=rstd, codes=codes, scales=scales, eps=1e-5)
        kept = torch.empty((9, cols), device="cuda")
        B.star_checkpoint_unpack(kept, codes, scales)
        assert bool(torch.isnan(rstd[bad]).all()) and bool(torch.isnan(y[bad]).all()) and bool(torch.isnan(kept[bad]).all())
        want, r = R.norm(part[good], gain[:cols], 1e-5)
        near(rstd[good], r, R.norm_bound(cols) * r)
        near(y[good], want, (R.norm_bound(cols) + 4 * R.ULP + R.half_step(dtype)) * want.abs() + 1e-38)


def backward(dy, stream, gain=None, d_total=None, kept=False, dgain_dtype=F32, accumulate=False, dx=None, eps=1e-5):
    from paper_2512_09685_b200 import binding as B
    rows, cols = dy.shape
    rstd = R.norm(stream, None, eps)[1].float()
    more, s = {"total": stream}, stream
    if kept:
        codes, scales = B.star_checkpoint_empty(rows, cols)
        B.star_checkpoint_pack(codes, scales, stream)
        s = torch.empty((rows, cols), device="cuda")
        B.star_checkpoint_unpack(s, codes, scales)
        more = {"codes": codes, "scales": scales}
    want, dgain_want, bound, dgain_bound = R.norm_backward(dy, s, rstd, gain, d_total)
    dgain = None
    if dgain_dtype is not None:
        dgain = torch.randn(cols, generator=gpu(9), device="cuda").to(dgain_dtype)
        if accumulate:
            dgain_want = dgain_want + dgain.double()
    dx = torch.full((rows, cols), 5.0, dtype=dy.dtype, device="cuda") if dx is None else dx
    ws = torch.full((B.star_rms_norm_workspace_bytes(rows, cols),), 0xff, dtype=torch.uint8, device="cuda")       # NaNs
    B.star_rms_norm_backward(dx, dgain, dy, gain, rstd, ws if dgain is not None else None, d_total=d_total, accumulate=accumulate, **more)
    torch.cuda.synchronize()
    near(dx, want, bound + R.half_step(dy.dtype) * want.abs() + 1e-38)
    if dgain is not None:
        near(dgain, dgain_want, dgain_bound + (R.half_step(dgain_dtype) + R.ULP) * dgain_want.abs() + 1e-38)
    return dx, dgain


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward_sizes(rows, cols, dtype, kept):
    dy, s, d = matrix(rows, cols, dtype, 1), matrix(rows, cols, dtype, 2), matrix(rows, cols, dtype, 3)
    gain = 1 + 0.1 * torch.randn(cols, generator=gpu(3), device="cuda")
    backward(dy, s, gain.to(BF16), d, kept, BF16)
    backward(dy, s, gain, None, kept, F32, True)
    backward(dy, s, None, d, kept, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(1, 0), (3, 1), (8, 8), (16, 32), (0, 3)])
def test_backward_strides_and_in_place(dtype, offset, extra):
    make = lambda seed: matrix(6, 520, dtype, seed, 520 + extra, offset)  # noqa: E731
    gain = torch.full((531,), 2.0, device="cuda", dtype=BF16)[3:523]
    a, ga = backward(make(1), make(2), gain, make(3))
    dy = make(1)
    b, gb = backward(dy, make(2), gain, make(3), dx=dy)
    d = make(3)
    c, gc = backward(make(1), make(2), gain, d, dx=d)
    assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(ga, gb) and torch.equal(ga, gc)
    out = torch.full((6, 600), 5.0, dtype=dtype, device="cuda")[:, 1:521]
    backward(make(1), make(2), gain, make(3), dx=out)
    backward(make(1), make(2), gain, make(3), kept=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_backward_of_many_rows(dtype):
    dy, s = matrix(20011, 128, dtype, 1), matrix(20011, 128, dtype, 2)
    backward(dy, s, None, None, False, dtype)
    backward(dy.abs(), s.abs(), None, None, True, dtype, True)      # sums of one sign


def test_backward_without_rows():
    from paper_2512_09685_b200 import binding as B
    e = torch.empty((0, 40), device="cuda")
    dgain = torch.ones(40, device="cuda")
    ws = torch.empty(64, dtype=torch.uint8, device="cuda")
    B.star_rms_norm_backward(e.clone(), dgain, e, None, torch.empty(0, device="cuda"), ws, total=e, accumulate=True)
    assert float(dgain.sum()) == 40.0
    B.star_rms_norm_backward(e.clone(), dgain, e, None, torch.empty(0, device="cuda"), ws, total=e)
    assert float(dgain.abs().max()) == 0.0


def test_backward_of_a_row_that_is_not_finite():
    dy, s = matrix(5, 300, BF16, 1), matrix(5, 300, BF16, 2)
    from paper_2512_09685_b200 import binding as B
    rstd = torch.ones(5, device="cuda")
    rstd[2] = math.nan
    dx, dgain = torch.empty_like(dy), torch.empty(300, device="cuda")
    ws = torch.empty(B.star_rms_norm_workspace_bytes(5, 300), dtype=torch.uint8, device="cuda")
    B.star_rms_norm_backward(dx, dgain, dy, None, rstd, ws, total=s)
    assert bool(torch.isnan(dx[2]).all()) and bool(torch.isfinite(dx[[0, 1, 3, 4]]).all()) and bool(torch.isnan(dgain).all())


def test_the_same_call_gives_the_same_bits():
    dy, s = matrix(5000, 1024, BF16, 1), matrix(5000, 1024, BF16, 2)
    a, b = backward(dy, s), backward(dy, s)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_backward_against_differences():
    """y' g along a direction of the stream and of the gain, in binary32 with a step of 2^-6."""
    from paper_2512_09685_b200 import binding as B
    s, g = matrix(4, 300, F32, 1), matrix(4, 300, F32, 2)
    gain = 1 + 0.1 * torch.randn(300, generator=gpu(3), device="cuda")
    rstd = R.norm(s, None, 1e-5)[1].float()
    dx, dgain = torch.empty_like(s), torch.empty(300, device="cuda")
    ws = torch.empty(B.star_rms_norm_workspace_bytes(4, 300), dtype=torch.uint8, device="cuda")
    B.star_rms_norm_backward(dx, dgain, g, gain, rstd, ws, total=s)

    def value(stream, weight):
        y = torch.empty_like(s)
        B.star_rms_norm(y, stream, weight, eps=1e-5)
        return float((y.double() * g.double()).sum())

    step = 2.0 ** -6
    for seed in range(3):
        v, u = torch.randn(s.shape, generator=gpu(seed), device="cuda"), torch.randn(300, generator=gpu(seed + 9), device="cuda")
        v, u = v / v.norm(), u / u.norm()
        slope = (value(s + step * v, gain + step * u) - value(s - step * v, gain - step * u)) / (2 * step)
        inner = float((dx.double() * v.double()).sum() + (dgain.double() * u.double()).sum())
        # The value is a sum of 1200 terms near 1, each off by a few half steps (their root sum: 35 of them); derivatives of order 1.
        assert abs(slope - inner) <= 4 * step ** 2 + 8 * 35 * R.ULP / step
