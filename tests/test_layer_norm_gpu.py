"""Layer normalisation against its 64-bit form: widths on and off every split of a row over lanes, few and many rows, strides, values that a
single pass over squares would lose, gradients against the formula and against differences."""
import pytest
import torch

import layer_reference as ref
import paper_2401_04658_amd as la2

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
EPS = 1e-5


def make(rows, width, dtype, seed=0, pad=0, affine=True):
    g = torch.Generator().manual_seed(seed)
    full = torch.full((rows, width + pad), float("nan"))
    full[:, :width] = torch.randn(rows, width, generator=g) * (0.5 + torch.rand(rows, 1, generator=g)) + torch.randn(rows, 1, generator=g)
    dy = torch.full((rows, width + pad), float("nan"))
    dy[:, :width] = torch.randn(rows, width, generator=g)
    w = 1 + 0.3 * torch.randn(width, generator=g) if affine else None
    b = 0.3 * torch.randn(width, generator=g) if affine else None
    to = lambda t: None if t is None else t.cuda()
    return full.to(dtype).cuda()[:, :width], dy.to(dtype).cuda()[:, :width], to(w), to(b)


def check(x, dy, w, b):
    dt, width = x.dtype, x.shape[-1]
    y, mean, rstd = la2.la2_layer_norm_fwd(x, w, b, eps=EPS)
    ry, rmean, rrstd = ref.norm_fwd(x, w, b, EPS)
    n = min(width, 96)   # additions that one term goes through: a lane's pieces, then the lanes (a thousandth of the width where rows are read anew)
    n = max(n, width // 1024 + 16)
    xa = ref.d(x).abs().mean(-1)
    em = n * ref.U32 * xa
    er = rrstd * (n + 8) * ref.U32 + rrstd ** 2 * 2 * em   # the spread's share of the mean's error: at most |x - mean| em twice
    ref.within("mean", mean, rmean, em + ref.U32 * rmean.abs())
    ref.within("rstd", rstd, rrstd, er)
    h = ((ref.d(x) - rmean.unsqueeze(-1)) * rrstd.unsqueeze(-1))
    wa = ref.d(w).abs() if w is not None else 1.0
    ey = wa * ((em * rrstd).unsqueeze(-1) + h.abs() * (er / rrstd).unsqueeze(-1) + 4 * ref.U32 * h.abs()) + 4 * ref.U32 * ry.abs()
    ref.within("y", y, ry, ey + ref.U[dt] * (ry.abs() + ey) + ref.TINY[dt])
    # backward, from the statistics that the forward pass kept
    dx, dw, db = la2.la2_layer_norm_bwd(dy, x, mean, rstd, w)
    rdx, rdw, rdb = ref.norm_bwd(dy, x, mean, rstd, w)
    r = ref.d(rstd).unsqueeze(-1)
    h = (ref.d(x) - ref.d(mean).unsqueeze(-1)) * r
    eh = 4 * ref.U32 * (h.abs() + r * ref.d(mean).abs().unsqueeze(-1))
    g = ref.d(dy).abs() * wa
    eg = (n + 8) * ref.U32
    ex = r * (4 * ref.U32 * g + eg * g.mean(-1, keepdim=True) + (h.abs() + eh) * ((eg * g * h.abs()) + g * eh).mean(-1, keepdim=True)
              + eh * (g * h.abs()).mean(-1, keepdim=True) + 4 * ref.U32 * h.abs() * (g * h.abs()).mean(-1, keepdim=True))
    ref.within("dx", dx, rdx, ex + ref.U[dt] * (rdx.abs() + ex) + ref.TINY[dt])
    rows = x.numel() // width
    da = ref.d(dy).abs()
    ref.within("d_weight", dw, rdw, ((rows + 8) * ref.U32 * da * h.abs() + da * eh).reshape(-1, width).sum(0))
    ref.within("d_bias", db, rdb, (rows + 8) * ref.U32 * da.reshape(-1, width).sum(0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 63, 64, 65, 128, 200, 256, 257, 511, 512, 513, 1001, 1024, 2048, 2049, 4097, 5120, 8192,
                                   8200, 16384, 16391])
def test_widths(width, dtype):
    check(*make(5, width, dtype, seed=width))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 31, 33, 1000, 5001])
def test_rows(rows, dtype):
    check(*make(rows, 96, dtype, seed=rows))
    check(*make(rows, 1000, dtype, seed=rows))


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_at_a_distance_and_leading_dimensions(dtype):
    for width, pad in ((64, 8), (1001, 7), (640, 1), (8191, 3)):
        x, dy, w, b = make(37, width, dtype, seed=pad, pad=pad)   # NaN between the rows
        check(x, dy, w, b)
    x, dy, w, b = make(24, 320, dtype)
    check(x.view(2, 3, 4, 320), dy.view(2, 3, 4, 320), w, b)
    check(x[0], dy[0], w, b)


def test_rows_wider_than_any_group_of_lanes_holds():
    for dtype, width in ((torch.float32, 8193), (torch.float32, 40001), (torch.bfloat16, 33000)):
        check(*make(70, width, dtype, seed=3))


def test_without_weight_and_bias():
    x, dy, _, _ = make(100, 777, torch.bfloat16, affine=False)
    check(x, dy, None, None)
    _, mean, rstd = la2.la2_layer_norm_fwd(x)
    dx, dw, db = la2.la2_layer_norm_bwd(dy, x, mean, rstd, want_d_weight=False, want_d_bias=False)
    assert dw is None and db is None
    full = la2.la2_layer_norm_bwd(dy, x, mean, rstd)
    assert torch.equal(dx, full[0])
    for one in (0, 1):
        got = la2.la2_layer_norm_bwd(dy, x, mean, rstd, want_d_weight=one == 0, want_d_bias=one == 1)
        assert got[2 - one] is None and torch.equal(got[1 + one], full[1 + one])


def test_a_large_mean_does_not_swallow_the_spread():
    g = torch.Generator().manual_seed(5)
    x = (1000.0 + torch.randn(64, 1536, generator=g)).cuda()
    y, mean, rstd = la2.la2_layer_norm_fwd(x)
    ry, _, rr = ref.norm_fwd(x, None, None, EPS)
    # the mean of numbers near 1000 is off by 64 roundings at most, 64 * 1000 * 2^-24 = 0.004 of the spread
    ref.within("y", y, ry, 0.0041 + 1e-5 * ry.abs())
    ref.within("rstd", rstd, rr, 2e-4)   # the mean's error enters squared, the subtraction is exact to 1000 * 2^-24


def test_constant_rows_and_no_rows():
    x = torch.full((3, 500), 2.5, device="cuda", dtype=torch.bfloat16)
    b = torch.randn(500, device="cuda")
    y, mean, rstd = la2.la2_layer_norm_fwd(x, None, b, eps=EPS)
    assert torch.equal(y, b.bfloat16().expand(3, 500)) and bool((mean == 2.5).all())
    ref.within("rstd", rstd, torch.full((3,), EPS).double().rsqrt(), 1e-4)
    e = x[:0]
    y, mean, rstd = la2.la2_layer_norm_fwd(e, None, b)
    assert y.shape == (0, 500) and mean.shape == (0,)
    dx, dw, db = la2.la2_layer_norm_bwd(e, e, mean, rstd)
    assert dx.shape == (0, 500) and bool((dw == 0).all()) and bool((db == 0).all())


def test_an_infinite_or_missing_value_stays_in_its_row():
    x, dy, w, b = make(9, 300, torch.float32)
    good = la2.la2_layer_norm_fwd(x, w, b)
    x2 = x.clone()
    x2[4, 7], x2[6, 299] = float("inf"), float("nan")
    y, mean, rstd = la2.la2_layer_norm_fwd(x2, w, b)
    keep = [i for i in range(9) if i not in (4, 6)]
    for got, want in zip((y, mean, rstd), good):
        assert torch.equal(got[keep], want[keep]) and not bool(torch.isfinite(got[[4, 6]]).all())


def test_gradient_against_differences():
    x, dy, w, b = make(3, 40, torch.float32, seed=11)
    y, mean, rstd = la2.la2_layer_norm_fwd(x, w, b, eps=EPS)
    dx, dw, db = la2.la2_layer_norm_bwd(dy, x, mean, rstd, w)
    loss = lambda X, W, B: float((ref.norm_fwd(X, W, B, EPS)[0] * ref.d(dy)).sum())
    step = 1e-5   # central differences in 64 bits: error of order step^2, 1e-9, and 1e-16 / step
    X, W, B = ref.d(x), ref.d(w), ref.d(b)
    for r, c in ((0, 0), (1, 17), (2, 39)):
        e = torch.zeros_like(X)
        e[r, c] = step
        want = (loss(X + e, W, B) - loss(X - e, W, B)) / (2 * step)
        assert abs(float(dx[r, c]) - want) <= 2e-5 * max(1.0, abs(want))
    for c in (0, 23, 39):
        e = torch.zeros_like(W)
        e[c] = step
        assert abs(float(dw[c]) - (loss(X, W + e, B) - loss(X, W - e, B)) / (2 * step)) <= 2e-5
        assert abs(float(db[c]) - (loss(X, W, B + e) - loss(X, W, B - e)) / (2 * step)) <= 2e-5


def test_same_bits_in_every_run_in_place_and_on_another_stream():
    x, dy, w, b = make(3000, 1536, torch.bfloat16, seed=2)
    y, mean, rstd = la2.la2_layer_norm_fwd(x, w, b)
    first = la2.la2_layer_norm_bwd(dy, x, mean, rstd, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = la2.la2_layer_norm_bwd(dy, x, mean, rstd, w)
        z = x.clone()
        la2.la2_layer_norm_fwd(z, w, b, out=z)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(first, again)) and torch.equal(z, y)
    for width in (1536, 20000):   # dx in dy's place; the wide rows' kernels read dy twice
        x, dy, w, b = make(70, width, torch.float32, seed=width)
        _, mean, rstd = la2.la2_layer_norm_fwd(x, w, b)
        want = la2.la2_layer_norm_bwd(dy, x, mean, rstd, w)
        got = la2.la2_layer_norm_bwd(dy, x, mean, rstd, w, out=dy)
        assert got[0] is not None and all(torch.equal(a, c) for a, c in zip(got, want))


def test_offsets_beyond_32_bits():
    rows, width, last = (1 << 32) // (2 * 2048) + 700, 2048, 1000   # 4 GiB and a little more a tensor
    x = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda").normal_()
    w, b = torch.randn(width, device="cuda"), torch.randn(width, device="cuda")
    y, mean, rstd = la2.la2_layer_norm_fwd(x, w, b)
    tail = la2.la2_layer_norm_fwd(x[-last:], w, b)
    assert torch.equal(y[-last:], tail[0]) and torch.equal(mean[-last:], tail[1]) and torch.equal(rstd[-last:], tail[2])
    dx, dw, db = la2.la2_layer_norm_bwd(y, x, mean, rstd, w)
    assert torch.equal(dx[-last:], la2.la2_layer_norm_bwd(y[-last:], x[-last:], mean[-last:], rstd[-last:], w)[0])
    # the sums over a million rows, in 64 bits a part at a time; a million terms in fp32 are off by a million roundings at most, in fact by far
    # fewer: rows are summed by 512 workgroups of 256 lanes first
    want = sum(p.double().sum(0) for p in y.split(1 << 16))
    mag = sum(p.abs().sum(0, dtype=torch.float64) for p in y.split(1 << 16))
    assert bool(((db.double() - want).abs() <= (rows / 512 + 520) * ref.U32 * mag).all())
