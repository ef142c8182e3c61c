"""fpde_causal_conv, its single-level step and its gradients against float64:
ragged lengths (none, one, fewer than the taps), carried states, strides."""
from __future__ import annotations

import pytest
import torch

from tests import network_ref as R

pytestmark = pytest.mark.gpu
CHAIN = 16  # taps, bias, and the activation's exponential, reciprocal and products


@pytest.fixture(scope="module")
def N():
    from paper_2607_18020_amd import network
    network.lib()
    return network


def inputs(B, L, D, W, dt, seed=0):
    g = torch.Generator().manual_seed(seed + B * 7919 + L * 31 + D)
    return dict(x=R.randn(g, B, L, D, dtype=dt), w=R.randn(g, D, W), b=R.randn(g, D),
                state=R.randn(g, B, W - 1, D, dtype=dt), dy=R.randn(g, B, L, D, dtype=dt),
                lengths=torch.randint(0, L + 1, (B,), generator=g, dtype=torch.int32))


def mags(x, w, b, state):
    """The magnitude of the terms of p."""
    return R.causal_conv(x.abs(), w.abs(), None if b is None else b.abs(), False,
                         None if state is None else state.abs(), None)[0]


SIZES = [(1, 1, 1), (2, 2, 5), (3, 3, 64), (2, 7, 130), (1, 33, 8), (5, 64, 24), (2, 100, 513), (3, 131, 260),
         (1, 1021, 40)]


@pytest.mark.parametrize("dt", R.DTYPES, ids=str)
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("B,L,D", SIZES)
def test_forward_and_backward(N, B, L, D, W, dt):
    t = inputs(B, L, D, W, dt)
    c = {k: v.cuda() for k, v in t.items()}
    f = {k: R.d(v) for k, v in t.items()}
    for act, with_state, ragged, with_bias in ((True, True, True, True), (False, False, False, True),
                                               (True, False, True, False), (True, True, False, True)):
        print(f"case conv {B} x {L} x {D} taps {W} {dt} {act} {with_state} {ragged}", flush=True)
        st, ln, b = (v if on else None for v, on in ((c["state"], with_state), (c["lengths"], ragged),
                                                    (c["b"], with_bias)))
        last = torch.full((B, W - 1, D), float("nan"), dtype=dt, device="cuda")
        y = N.fpde_causal_conv(c["x"], c["w"], b, silu=act, state=st, lengths=ln, state_out=last)
        rst, rln, rb = (f["state"] if with_state else None, t["lengths"] if ragged else None,
                        f["b"] if with_bias else None)
        x = f["x"].clone().requires_grad_()
        w = f["w"].clone().requires_grad_()
        bb = f["b"].clone().requires_grad_()
        ry, rlast = R.causal_conv(x, w, bb if with_bias else None, act, rst, rln)
        mag = mags(f["x"], f["w"], rb, rst)
        R.close("y", y, ry.detach(), CHAIN, mag)
        assert torch.equal(last.cpu().double(), rlast.detach())
        # the gradients, by the plain form's own derivative
        (ry * f["dy"]).sum().backward()
        dx, dw, db = N.fpde_causal_conv_bwd(c["dy"], c["x"], c["w"], b, silu=act, state=st, lengths=ln)
        dpm = f["dy"].abs() * (1 + mag)  # |silu'| <= 1.1, and its own error grows with p's terms
        pad = torch.nn.functional.pad(dpm, (0, 0, 0, W - 1))
        R.close("dx", dx, x.grad, CHAIN, sum(f["w"][:, k].abs() * pad[:, W - 1 - k:W - 1 - k + L] for k in range(W)))
        hist = torch.zeros_like(f["state"]) if rst is None else rst.abs()
        e = torch.cat((hist, f["x"].abs()), 1)
        chain = CHAIN + min(L, 64) + B * (L // 64 + 1)
        dwm = torch.stack([(dpm * e[:, k:k + L]).sum((0, 1)) for k in range(W)], 1)
        R.close("dw", dw, w.grad, chain, dwm)
        if with_bias:
            R.close("db", db, bb.grad, chain, dpm.sum((0, 1)))
        else:
            assert db is None


def test_steps_equal_a_window(N):
    """Level by level with the carried state, in place, gives what the window gives."""
    for dt in R.DTYPES:
        t = {k: v.cuda() for k, v in inputs(4, 9, 70, 4, dt).items()}
        last = torch.empty_like(t["state"])
        y = N.fpde_causal_conv(t["x"], t["w"], t["b"], state=t["state"], state_out=last)
        state = t["state"].clone()
        for i in range(9):
            assert torch.equal(N.fpde_causal_conv_step(t["x"][:, i], state, t["w"], t["b"]), y[:, i])
        assert torch.equal(state, last)
        # two windows, the state updated in place
        state = t["state"].clone()
        y1 = N.fpde_causal_conv(t["x"][:, :5], t["w"], t["b"], state=state, state_out=state)
        y2 = N.fpde_causal_conv(t["x"][:, 5:], t["w"], t["b"], state=state, state_out=state)
        assert torch.equal(torch.cat((y1, y2), 1), y) and torch.equal(state, last)


def test_levels_past_a_length_are_not_read(N):
    t = {k: v.cuda() for k, v in inputs(6, 70, 50, 4, torch.float32).items()}
    t["lengths"] = torch.tensor([0, 1, 2, 35, 70, 64], dtype=torch.int32, device="cuda")
    past = (torch.arange(70, device="cuda")[None] >= t["lengths"][:, None])[..., None]
    args = (t["w"], t["b"])
    y = N.fpde_causal_conv(t["x"], *args, lengths=t["lengths"])
    g = N.fpde_causal_conv_bwd(t["dy"], t["x"], *args, lengths=t["lengths"])
    xn, dyn = t["x"].masked_fill(past, float("nan")), t["dy"].masked_fill(past, float("nan"))
    assert torch.equal(N.fpde_causal_conv(xn, *args, lengths=t["lengths"]), y)
    for a, b in zip(N.fpde_causal_conv_bwd(dyn, xn, *args, lengths=t["lengths"]), g):
        assert torch.equal(a, b)
    assert not y.masked_select(past).any() and not g[0].masked_select(past).any()
    # lengths out of range are clamped
    bad = torch.tensor([-3, 1, 2, 35, 1000, 64], dtype=torch.int32, device="cuda")
    assert torch.equal(N.fpde_causal_conv(t["x"], *args, lengths=bad), y)


def test_strides_weight_types_streams_and_graph(N):
    t = {k: v.cuda() for k, v in inputs(3, 40, 72, 4, torch.bfloat16).items()}
    w, b = t["w"].bfloat16(), t["b"].bfloat16()
    y = N.fpde_causal_conv(t["x"], w, b)
    g = N.fpde_causal_conv_bwd(t["dy"], t["x"], w, b)
    assert g[1].dtype is torch.bfloat16
    wide = torch.randn(3, 80, 200, device="cuda").bfloat16()
    xs = wide[:, ::2, 3:75]
    xs.copy_(t["x"])
    assert torch.equal(N.fpde_causal_conv(xs, w, b), y)
    for p, q in zip(N.fpde_causal_conv_bwd(t["dy"], xs, w, b), g):
        assert torch.equal(p, q)
    tm = t["x"].transpose(0, 1).contiguous().transpose(0, 1)  # levels outermost
    assert torch.equal(N.fpde_causal_conv(tm, w, b), y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g2 = N.fpde_causal_conv_bwd(t["dy"], t["x"], w, b, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip(g2, g):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gy = N.fpde_causal_conv(t["x"], w, b)
        gg = N.fpde_causal_conv_bwd(t["dy"], t["x"], w, b)
    for _ in range(3):
        t["x"].mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gy, N.fpde_causal_conv(t["x"], w, b))
        for p, q in zip(gg, N.fpde_causal_conv_bwd(t["dy"], t["x"], w, b)):
            assert torch.equal(p, q)


def test_no_sequences_and_no_levels(N):
    w, b = torch.randn(6, 4, device="cuda"), torch.randn(6, device="cuda")
    for shape in ((0, 5, 6), (3, 0, 6)):
        x = torch.empty(shape, device="cuda")
        st = torch.randn(shape[0], 3, 6, device="cuda")
        out = torch.empty_like(st)
        assert N.fpde_causal_conv(x, w, b, state=st, state_out=out).shape == shape
        assert torch.equal(out, st)
        dx, dw, db = N.fpde_causal_conv_bwd(x, x, w, b)
        assert dx.shape == shape and not dw.any() and not db.any()


def test_autograd_and_differences(N):
    t = inputs(2, 20, 12, 4, torch.float32)
    leaf = [t[k].cuda().requires_grad_() for k in ("x", "w", "b")]
    ln = torch.tensor([20, 11], dtype=torch.int32, device="cuda")
    N.CausalConv.apply(*leaf, True, t["state"].cuda(), ln).backward(t["dy"].cuda())
    g = torch.Generator().manual_seed(1)
    h = 2.0 ** -7
    for k in range(3):
        v = R.randn(g, *leaf[k].shape).cuda()
        f = []
        for sgn in (1, -1):
            args = [p.detach() for p in leaf]
            args[k] = args[k] + sgn * h * v
            y = N.fpde_causal_conv(*args, state=t["state"].cuda(), lengths=ln)
            f.append(float((y.double() * t["dy"].cuda()).sum()))
        want = float((leaf[k].grad.double() * v).sum())
        # truncation: h^2 / 6 |p'''|, of order 1 for silu times the direction's cubed entries; 480 terms
        assert abs((f[0] - f[1]) / (2 * h) - want) <= 480 * h * h * 4 + 480 * 2.0 ** -24 * 8 / h, k
    with pytest.raises(ValueError):
        N.CausalConv.apply(*leaf, True, t["state"].cuda().requires_grad_(), ln)
