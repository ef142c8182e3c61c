"""fpde_rms_norm and fpde_rms_norm_bwd against float64, at the widths where the
kernels change layout, odd widths, strided rows, in place, and 8-bit output."""
from __future__ import annotations

import pytest
import torch

from tests import network_ref as R

pytestmark = pytest.mark.gpu

# (float32: 4 columns a lane, 16 bits: 8) the edges of every layout, odd widths, one column, wide rows
WIDTHS = [1, 3, 16, 63, 64, 65, 127, 128, 130, 256, 257, 511, 512, 1000, 1024, 1160, 2049, 4096, 8193, 16385, 20001]
# roundings along a row's sums: at most 64 columns a lane, 10 levels of lanes and waves, rho and the products
CHAIN = 96


@pytest.fixture(scope="module")
def N():
    from paper_2607_18020_amd import network
    network.lib()
    return network


def inputs(rows, width, dt, seed=0):
    g = torch.Generator().manual_seed(seed + rows * 131 + width)
    x, r = R.randn(g, rows, width, dtype=dt), (2 * R.randn(g, rows, width)).to(dt)
    w = 1 + 0.3 * R.randn(g, width)
    return x, r, w, R.randn(g, rows, width, dtype=dt), R.randn(g, rows, width, dtype=dt)


def check_bwd(what, ds, dw, dy, s, w, dsum, eps):
    """ds, dw against the formula; magnitudes are those of the terms added."""
    rds, rdw = R.rms_norm_bwd(R.d(dy), R.d(s), R.d(w), R.d(dsum), eps)
    s64, dy64 = R.d(s), R.d(dy)
    rho = (s64.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    g = dy64 if w is None else dy64 * R.d(w)
    mag = (rho * g).abs() + rho ** 3 * (g * s64).abs().mean(-1, keepdim=True) * s64.abs()
    if dsum is not None:
        mag = mag + R.d(dsum).abs()
    R.close(what + " ds", ds, rds, CHAIN, mag)
    if w is not None:
        # (rows of a workgroup, then its row groups, then the partial rows)
        R.close(what + " dw", dw, rdw, CHAIN + 64 + dy.shape[0] // 256, (dy64 * s64 * rho).abs().sum(0))


@pytest.mark.parametrize("dt", R.DTYPES, ids=str)
@pytest.mark.parametrize("width", WIDTHS)
def test_forward_and_backward(N, width, dt):
    for rows in (1, 5, 67):
        print(f"case norm {rows} x {width} {dt}", flush=True)
        x, r, w, dy, dsum = inputs(rows, width, dt)
        c = [t.cuda() for t in (x, r, w, dy, dsum)]
        y, s = N.fpde_rms_norm(c[0], c[2], residual=c[1], eps=1e-6)
        ry, rs = R.rms_norm(R.d(x), R.d(w), R.d(r), 1e-6)
        R.close("s", s, rs, 1)
        R.close("y", y, ry, CHAIN)
        ds, dw = N.fpde_rms_norm_bwd(c[3], s, c[2], dsum=c[4], eps=1e-6)
        check_bwd("full", ds, dw, dy, s, w, dsum, 1e-6)
        # neither residual, weight nor dsum
        y, s = N.fpde_rms_norm(c[0], eps=1e-5)
        assert s is c[0]
        R.close("plain y", y, R.rms_norm(R.d(x), None, None, 1e-5)[0], CHAIN)
        ds, dw = N.fpde_rms_norm_bwd(c[3], c[0], eps=1e-5)
        assert dw is None
        check_bwd("plain", ds, None, dy, x, None, None, 1e-5)


@pytest.mark.parametrize("rows,width,dt", [(5000, 64, torch.float32), (3001, 130, torch.bfloat16),
                                           (2500, 1024, torch.float16), (300, 17000, torch.bfloat16)], ids=str)
def test_many_rows(N, rows, width, dt):
    """More rows than workgroups times rows: partial sums of dw over the walk."""
    print(f"case norm {rows} x {width} {dt}", flush=True)
    x, r, w, dy, dsum = inputs(rows, width, dt)
    c = [t.cuda() for t in (x, r, w, dy, dsum)]
    y, s = N.fpde_rms_norm(c[0], c[2], residual=c[1])
    R.close("y", y, R.rms_norm(R.d(x), R.d(w), R.d(r), 1e-6)[0], CHAIN)
    ds, dw = N.fpde_rms_norm_bwd(c[3], s, c[2], dsum=c[4])
    check_bwd("many", ds, dw, dy, s, w, dsum, 1e-6)
    again = N.fpde_rms_norm_bwd(c[3], s, c[2], dsum=c[4])
    assert torch.equal(again[0], ds) and torch.equal(again[1], dw)


@pytest.mark.parametrize("dt", R.DTYPES, ids=str)
def test_weight_in_the_data_type_strides_and_in_place(N, dt):
    rows, width = 37, 200
    x, r, w, dy, dsum = inputs(rows, width, dt)
    wt = w.to(dt)
    wide = torch.full((rows, 3 * width + 5), float("nan"), dtype=dt).cuda()
    xs, rs_ = wide[:, 1:1 + width], wide[:, width + 3:2 * width + 3]  # (2-byte aligned rows)
    xs.copy_(x), rs_.copy_(r)
    y, s = N.fpde_rms_norm(xs, wt.cuda(), residual=rs_)
    ry, rs = R.rms_norm(R.d(x), R.d(wt), R.d(r), 1e-6)
    R.close("y", y, ry, CHAIN)
    R.close("s", s, rs, 1)
    # the residual stream updated in place
    stream = r.cuda()
    y2, s2 = N.fpde_rms_norm(x.cuda(), wt.cuda(), residual=stream, sum_out=stream)
    assert s2 is stream and torch.equal(s2, s) and torch.equal(y2, y)
    dyc, dsc = dy.cuda(), dsum.cuda()
    ds, dw = N.fpde_rms_norm_bwd(dyc, s, wt.cuda(), dsum=dsc)
    assert dw.dtype is dt
    for inplace in ("dy", "dsum"):
        a, b = dyc.clone(), dsc.clone()
        ds2, dw2 = N.fpde_rms_norm_bwd(a, s, wt.cuda(), dsum=b, ds=a if inplace == "dy" else b)
        assert torch.equal(ds2, ds) and torch.equal(dw2, dw)
    # leading axes fold
    y3, s3 = N.fpde_rms_norm(x.cuda().view(1, rows, 1, width), wt.cuda())
    assert y3.shape == (1, rows, 1, width)


def test_wide_rows_in_place(N):
    """ds over dy where dw is summed by a launch of its own."""
    x, r, w, dy, dsum = inputs(9, 20000, torch.bfloat16)
    c = [t.cuda() for t in (x, r, w, dy, dsum)]
    ds, dw = N.fpde_rms_norm_bwd(c[3], c[0], c[2], dsum=c[4])
    a = c[3].clone()
    ds2, dw2 = N.fpde_rms_norm_bwd(a, c[0], c[2], dsum=c[4], ds=a)
    assert ds2 is a and torch.equal(ds, ds2) and torch.equal(dw, dw2)
    s = c[1].clone()
    y, _ = N.fpde_rms_norm(c[0], c[2], residual=c[1])
    y2, s2 = N.fpde_rms_norm(c[0], c[2], residual=s, sum_out=s)
    assert torch.equal(y, y2)
    R.close("s", s2, R.d(x) + R.d(r), 1)


@pytest.mark.parametrize("dt", R.DTYPES, ids=str)
@pytest.mark.parametrize("width", [1, 5, 64, 100, 128, 129, 256, 300, 1160, 4096, 5000, 18000])
def test_eight_bits(N, width, dt):
    for group in (128, 0):
        rows = 19
        print(f"case norm8 {rows} x {width} {dt} group {group}", flush=True)
        x, r, w, _, _ = inputs(rows, width, dt)
        x[3], r[3] = 0, 0  # a row of zeros: scale 2^-126, zeros
        q, sc, s = N.fpde_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), quant=group)
        assert q.dtype is torch.float8_e4m3fn and q.shape == x.shape
        ry, rs = R.rms_norm(R.d(x), R.d(w), R.d(r), 1e-6)
        R.close("s", s, rs, 1)
        g = group or width
        ng = -(-width // g)
        assert sc.shape == (rows, ng)
        pad = torch.nn.functional.pad(ry, (0, ng * g - width)).view(rows, ng, g)
        R.close("scales", sc, (pad.abs().amax(-1) / 448).clamp(min=2.0 ** -126), CHAIN)
        # q is y / scale rounded to 4 significand bits (half a step of 2^-3, or of the subnormals' 2^-9)
        val = torch.nn.functional.pad(q.float().cpu().double(), (0, ng * g - width)).view(rows, ng, g)
        t = pad / sc.double().cpu()[..., None]
        assert bool(((val - t).abs() <= t.abs() * (2.0 ** -4 + CHAIN * 2.0 ** -23) + 2.0 ** -10).all())
        assert not q[3].float().any()


def test_nan_and_inf_stay_in_their_row(N):
    x, r, w, _, _ = inputs(8, 300, torch.float32)
    x[2, 7], x[5, 0] = float("nan"), float("inf")
    for quant in (None, 128, 0):
        out = N.fpde_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), quant=quant)
        y = out[0].float().cpu()
        for i in range(8):
            assert bool(torch.isnan(y[i]).any()) == (i in (2, 5)), (quant, i)
        assert torch.isnan(y[2]).all() and torch.isnan(y[5, 0])


def test_no_rows(N):
    w = torch.ones(64, device="cuda")
    y, s = N.fpde_rms_norm(torch.empty(0, 64, device="cuda"), w)
    assert y.shape == (0, 64)
    ds, dw = N.fpde_rms_norm_bwd(torch.empty(0, 64, device="cuda"), torch.empty(0, 64, device="cuda"), w)
    assert ds.shape == (0, 64) and not dw.any()


def test_autograd_formula_and_differences(N):
    g = torch.Generator().manual_seed(5)
    x, r, w = R.randn(g, 6, 48), R.randn(g, 6, 48), 1 + 0.2 * R.randn(g, 48)
    cy, cs = R.randn(g, 6, 48), R.randn(g, 6, 48)
    leaf = [t.cuda().requires_grad_() for t in (x, r, w)]
    y, s = N.RmsNorm.apply(*leaf, 1e-6)
    ((y * cy.cuda()).sum() + (s * cs.cuda()).sum()).backward()
    ref = [R.d(t).requires_grad_() for t in (x, r, w)]
    ry, rs = R.rms_norm(ref[0], ref[2], ref[1], 1e-6)
    ((ry * cy).sum() + (rs * cs).sum()).backward()
    for a, b in zip(leaf, ref):
        R.close("autograd", a.grad, b.grad, CHAIN, b.grad.abs() + 4)
    # central differences of the forward along random directions: the truncation is h^2 / 6 times a
    # third derivative of order 10 a direction's norm, the rounding 2^-24 |objective terms| / h
    h = 2.0 ** -7
    for k in range(3):
        v = R.randn(g, *leaf[k].shape).cuda()
        f = []
        for sgn in (1, -1):
            args = [t.detach() for t in leaf]
            args[k] = args[k] + sgn * h * v
            yy, ss = N.fpde_rms_norm(args[0], args[2], residual=args[1])
            f.append(((yy.double() * cy.cuda()).sum() + (ss.double() * cs.cuda()).sum()).item())
        slope = (f[0] - f[1]) / (2 * h)
        want = float((leaf[k].grad.double() * v).sum())
        assert abs(slope - want) <= 10 * h * h * float(v.norm()) + 288 * 2.0 ** -24 * 8 / h, (k, slope, want)
    # without residual and weight; a gradient that is a broadcast view
    a = x.cuda().requires_grad_()
    y, s = N.RmsNorm.apply(a, None, None, 1e-6)
    y.sum().backward()
    b = R.d(x).requires_grad_()
    R.rms_norm(b, None, None, 1e-6)[0].sum().backward()
    R.close("plain", a.grad, b.grad, CHAIN, b.grad.abs() + 4)


def test_other_stream_and_graph(N):
    x, r, w, dy, dsum = (t.cuda() for t in inputs(300, 256, torch.bfloat16))
    y, s = N.fpde_rms_norm(x, w, residual=r)
    ds, dw = N.fpde_rms_norm_bwd(dy, s, w, dsum=dsum)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, s2 = N.fpde_rms_norm(x, w, residual=r, stream=side)
    ds2, dw2 = N.fpde_rms_norm_bwd(dy, s2, w, dsum=dsum, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in ((y, y2), (s, s2), (ds, ds2), (dw, dw2)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gy, gs = N.fpde_rms_norm(x, w, residual=r)
        gds, gdw = N.fpde_rms_norm_bwd(dy, gs, w, dsum=dsum)
    for _ in range(3):
        x.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        y, s = N.fpde_rms_norm(x, w, residual=r)
        ds, dw = N.fpde_rms_norm_bwd(dy, s, w, dsum=dsum)
        for a, b in ((y, gy), (s, gs), (ds, gds), (dw, gdw)):
            assert torch.equal(a, b)
