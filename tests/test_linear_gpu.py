"""Linear layers and their gradients against their 64-bit form: few and many rows, sizes on and off the tiles, rows that are no whole 16-byte
pieces, reductions that are cut, every activation, bias, residual, strides with NaN between the rows."""
import pytest
import torch

import layer_reference as ref
import paper_2401_04658_amd as la2

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
ACTS = ["none", "relu", "gelu", "silu"]


def matrix(g, rows, cols, dtype, pad=0, scale=1.0):
    full = torch.full((rows, cols + pad), float("nan"))
    full[:, :cols] = torch.randn(rows, cols, generator=g) * scale
    return full.to(dtype).cuda()[:, :cols]


def check(m, n, k, dtype, act="silu", bias=True, residual=True, pads=(0, 0, 0), seed=0, forward=True, backward=True):
    g = torch.Generator().manual_seed(seed + 7 * m + 3 * n + k)
    x, w = matrix(g, m, k, dtype, pads[0]), matrix(g, n, k, dtype, pads[1], max(1, k) ** -0.5)
    b = (torch.randn(n, generator=g) * 0.3).cuda() if bias else None
    r = matrix(g, m, n, dtype, pads[2]) if residual else None
    if forward:
        y, pre = la2.la2_linear_fwd(x, w, b, residual=r, act=act, want_pre=True)
        ry, ey, rz, ez = ref.linear_fwd(x, w, b, r, act)
        ref.within("pre", pre, rz, ez)
        ref.within("y", y, ry, ey)
        alone, none = la2.la2_linear_fwd(x, w, b, residual=r, act=act)
        assert none is None and torch.equal(alone, y)
    if backward:
        dy, z = matrix(g, m, n, dtype, pads[2]), matrix(g, m, n, dtype, pads[2])
        dx, dw, db = la2.la2_linear_bwd(dy, x, w, pre=z if act != "none" else None, act=act)
        rdx, edx, rdw, edw, rdb, edb = ref.linear_bwd(dy, x, w, z, act)
        ref.within("dx", dx, rdx, edx)
        ref.within("dw", dw, rdw, edw)
        ref.within("d_bias", db, rdb, edb)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 2, 4, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 257])
def test_rows(m, dtype):
    check(m, 192, 256, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m", [3, 200])
def test_activations_bias_and_residual(m, act, dtype):
    for bias in (False, True):
        for residual in (False, True):
            check(m, 160, 136, dtype, act, bias, residual)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (1, 64), (64, 1), (7, 9), (8, 8), (63, 65), (100, 100), (129, 255), (256, 31), (300, 520), (513, 96)])
def test_odd_sizes(n, k, dtype):
    for m in (1, 5, 40, 131):
        check(m, n, k, dtype, "gelu")


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_at_a_distance(dtype):
    for m in (6, 90):
        check(m, 72, 136, dtype, pads=(8, 16, 24))
        check(m, 71, 135, dtype, pads=(1, 9, 1))     # whole pieces apart, but not whole pieces long
        check(m, 72, 136, dtype, pads=(3, 1, 5))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(40, 64, 8192), (70, 128, 5001), (3000, 64, 72), (1025, 200, 136), (24, 3000, 200), (520, 520, 520)])
def test_long_reductions_and_long_sides(m, n, k, dtype):
    check(m, n, k, dtype, "relu")


@pytest.mark.parametrize("m,n,k", [(4096, 4096, 512), (2100, 4100, 260), (8200, 2056, 136)])
def test_large_tiles(m, n, k):
    """Enough tiles of 256 x 256 for every unit, whole and ragged."""
    check(m, n, k, torch.bfloat16, "silu")


def test_empty_extents():
    dt = torch.bfloat16
    z = lambda *s: torch.zeros(*s, dtype=dt, device="cuda")
    assert la2.la2_linear_fwd(z(0, 64), z(32, 64))[0].shape == (0, 32)
    assert la2.la2_linear_fwd(z(5, 64), z(0, 64))[0].shape == (5, 0)
    b = torch.randn(32, device="cuda")
    for m in (5, 50):   # no features: the bias alone
        y, _ = la2.la2_linear_fwd(z(m, 0), z(32, 0), b)
        assert torch.equal(y, b.to(dt).expand(m, 32))
    dx, dw, db = la2.la2_linear_bwd(z(0, 32), z(0, 64), z(32, 64))
    assert dx.shape == (0, 64) and bool((dw == 0).all()) and bool((db == 0).all())
    dx, dw, db = la2.la2_linear_bwd(z(50, 0), z(50, 64), z(0, 64))
    assert bool((dx == 0).all()) and dw.shape == (0, 64) and db.shape == (0,)
    dx, dw, db = la2.la2_linear_bwd(torch.ones(50, 32, dtype=dt, device="cuda"), z(50, 0), z(32, 0))
    assert dx.shape == (50, 0) and dw.shape == (32, 0) and bool((db == 50).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_and_missing_values_stay_in_their_rows(dtype):
    for m in (8, 80):
        g = torch.Generator().manual_seed(m)
        x, w, dy = matrix(g, m, 100, dtype), matrix(g, 70, 100, dtype), matrix(g, m, 70, dtype)
        good, gx = la2.la2_linear_fwd(x, w, act="silu")[0], la2.la2_linear_bwd(dy, x, w)[0]
        x[1, 99], x[5, 0], dy[2, 69] = float("inf"), float("nan"), float("nan")
        y, dx = la2.la2_linear_fwd(x, w, act="silu")[0], la2.la2_linear_bwd(dy, x, w)[0]
        keep = [i for i in range(m) if i not in (1, 5)]
        assert torch.equal(y[keep], good[keep]) and bool(torch.isnan(y[5]).all()) and bool(((y[1] == float("inf")) | (y[1] == 0)).all())
        keep = [i for i in range(m) if i != 2]
        assert torch.equal(dx[keep], gx[keep]) and bool(torch.isnan(dx[2]).all())


@pytest.mark.parametrize("act", ACTS)
def test_activations_at_their_ends(act):
    """Sums of any size, the infinite ones among them: what the 64-bit form gives, no NaN from 0 * inf."""
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 0.5, -0.5, 3.0, -3.0, 6.0, -6.0, 12.0, -12.0, 40.0, -40.0, 1e4, -1e4, 3e38, -3e38,
                      float("inf"), float("-inf"), float("nan")])
    x, w = z.view(-1, 1).cuda(), torch.ones(1, 1, device="cuda")
    want = {"none": z.double(), "relu": torch.relu(z.double()), "gelu": ref.act(z.double(), "gelu"), "silu": ref.act(z.double(), "silu")}[act]
    want[-2] = float("-inf") if act == "none" else 0.0   # the limit
    for x in (x, torch.cat([x, x])):                     # few rows, and more
        y = la2.la2_linear_fwd(x, w, act=act)[0].cpu().double().view(-1)[:21]
        assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y[18:20], want[18:20])
        assert bool(((y - want).abs()[:18] <= 4e-6 * want.abs()[:18].clamp(max=1e38) + 4e-7 * z.abs().double()[:18].clamp(max=10.0)).all()), (y, want)
        one = torch.ones(x.shape[0], 1, device="cuda")
        if act != "none":
            dz = la2.la2_linear_bwd(one, one, w, pre=x, act=act)[0].cpu().double().view(-1)[:21]
            s = ref.slope(z.double(), act)
            s[18], s[19] = 1.0, 0.0
            s[16], s[17] = 1.0, 0.0
            assert bool(((dz - s).abs()[:20] <= 4e-6 * (1 + z.abs().double()[:20].clamp(max=8.0))).all()), (dz, s)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    for m in (4, 40):
        g = torch.Generator().manual_seed(3)
        x, w, b = matrix(g, m, 24, torch.float32), matrix(g, 20, 24, torch.float32, scale=0.2), torch.randn(20, generator=g).cuda()
        dy = matrix(g, m, 20, torch.float32)
        _, pre = la2.la2_linear_fwd(x, w, b, act=act, want_pre=True)
        dx, dw, db = la2.la2_linear_bwd(dy, x, w, pre=pre, act=act)
        X, W, B, DY = ref.d(x), ref.d(w), ref.d(b), ref.d(dy)
        loss = lambda X, W, B: float((ref.act(X @ W.T + B, act) * DY).sum())
        step = 1e-6
        for t, got, at in ((0, dx, (1, 5)), (0, dx, (m - 1, 23)), (1, dw, (0, 0)), (1, dw, (19, 11)), (2, db, (7,))):
            args = [X, W, B]
            e = torch.zeros_like(args[t])
            e[at] = step
            lo, hi = list(args), list(args)
            lo[t], hi[t] = args[t] - e, args[t] + e
            want = (loss(*hi) - loss(*lo)) / (2 * step)
            assert abs(float(got[at]) - want) <= 1e-4 * max(1.0, abs(want)), (t, at)   # slope bound 4e-6 over up to 40 terms of size 3


def test_leading_dimensions_outputs_and_what_is_not_wanted():
    g = torch.Generator().manual_seed(1)
    x, w = matrix(g, 60, 96, torch.bfloat16), matrix(g, 80, 96, torch.bfloat16)
    y, _ = la2.la2_linear_fwd(x, w)
    assert torch.equal(la2.la2_linear_fwd(x.view(3, 4, 5, 96), w)[0], y.view(3, 4, 5, 80))
    assert torch.equal(la2.la2_linear_fwd(x[7], w)[0], la2.la2_linear_fwd(x[7:8], w)[0][0])
    out, pre = torch.empty_like(y), torch.empty_like(y)
    got = la2.la2_linear_fwd(x, w, out=out, pre=pre)
    assert got[0].data_ptr() == out.data_ptr() and got[1].data_ptr() == pre.data_ptr() and torch.equal(out, y) and torch.equal(pre, y)
    r = matrix(g, 60, 80, torch.bfloat16)
    want = la2.la2_linear_fwd(x, w, residual=r)[0]
    la2.la2_linear_fwd(x, w, residual=r, out=r)   # in place of the residual
    assert torch.equal(r, want)
    dy = matrix(g, 60, 80, torch.bfloat16)
    full = la2.la2_linear_bwd(dy, x, w)
    for i in range(3):
        want = [i == j for j in range(3)]
        one = la2.la2_linear_bwd(dy, x, w, want_dx=want[0], want_dw=want[1], want_d_bias=want[2])
        assert [o is not None for o in one] == want and torch.equal(one[i], full[i])


def test_same_bits_in_every_run_on_another_stream_and_in_a_graph():
    g = torch.Generator().manual_seed(4)
    x, w, b = matrix(g, 300, 999, torch.bfloat16), matrix(g, 131, 999, torch.bfloat16, scale=0.03), torch.randn(131, generator=g).cuda()
    dy = matrix(g, 300, 131, torch.bfloat16)

    def step():
        n, mean, rstd = la2.la2_layer_norm_fwd(x)
        y, pre = la2.la2_linear_fwd(n, w, b, act="gelu", want_pre=True)
        dn, dw, db = la2.la2_linear_bwd(dy, n, w, pre=pre, act="gelu")
        return (y, dw, db) + la2.la2_layer_norm_bwd(dn, x, mean, rstd)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        for o in out:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, out))
        step()


def test_offsets_beyond_32_bits():
    rows, k, n, last = (1 << 32) // (2 * 2048) + 300, 2048, 72, 500   # x, and dx, of 4 GiB and a little more
    x = torch.empty(rows, k, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn(n, k, device="cuda").mul_(0.02).bfloat16()
    y, _ = la2.la2_linear_fwd(x, w)
    ry, ey, _, _ = ref.linear_fwd(x[-last:], w, None, None, "none")
    ref.within("y", y[-last:], ry, ey)
    dx, _, _ = la2.la2_linear_bwd(y, x, w, want_dw=False)
    rdx, edx = ref.linear_bwd(y[-last:], x[-last:], w, None, "none")[:2]
    ref.within("dx", dx[-last:], rdx, edx)
