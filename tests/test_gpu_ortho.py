"""fpde_orthogonalize and fpde_muon_step against float64, at the sizes where the
kernels change (one workgroup a matrix, tiles of 64 and of 128), odd and extreme
shapes, decaying spectra, zero and non-finite matrices.

Tolerances.  With the customary coefficients an error made in X grows by at most a =
3.4445 a step in the directions whose singular values are still small, and what
is measured is relative to the result's norm, sqrt(rank).  Operands are held to 2^-22
and sums to a few 2^-24, so a step's own error is below 2^-20 of |X|_F, and the first
steps' errors are of the smallest |X|_F; five steps give less than 5 a^4 2^-20 in
all directions together in the worst case that every direction stays small, 7e-4;
with full-rank matrices, whose directions reach 1 after two or three steps, 2^-20 a^2 5 =
6e-5.  For the latter the tests allow 2e-5 of the norm (the measure for float32 results
elsewhere), for the former 7e-4; both plus the result's own rounding."""
from __future__ import annotations

import pytest
import torch

from tests import network_ref as R

pytestmark = pytest.mark.gpu
CO = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def N():
    from paper_2607_18020_amd import network
    network.lib()
    return network


def near(what, got, ref, tol=2e-5):
    g, r = got.detach().double().cpu(), ref.double()
    assert g.shape == r.shape
    off, norm = float((g - r).norm()), float(r.norm())
    allowed = tol * norm + R.U[got.dtype] * norm
    assert off <= allowed, f"{what}: off by {off} of {norm}, allowed {allowed}"


def matrix(m, n, seed=0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed + 1000 * m + n)
    return (1e-3 * R.randn(g, m, n)).to(dtype)


SHAPES = [(1, 1), (1, 7), (16, 16), (33, 64), (64, 64), (64, 65), (50, 128), (64, 200), (64, 256), (256, 64), (65, 64),
          (100, 128), (128, 128), (128, 90), (64, 257), (128, 129), (129, 128), (130, 260), (257, 255), (320, 1000),
          (1000, 70), (1, 300), (300, 1)]


@pytest.mark.parametrize("dt", R.DTYPES, ids=str)
@pytest.mark.parametrize("m,n", SHAPES)
def test_shapes(N, m, n, dt):
    print(f"case ortho {m} x {n} {dt}", flush=True)
    g = torch.stack([matrix(m, n, s, dt) for s in range(3)])
    o = N.fpde_orthogonalize(g.cuda())
    for i in range(3):
        near(f"{m} x {n}", o[i], R.orthogonalize(g[i].double(), 5, CO, 1e-7))
    # a sequence, other steps and coefficients, in place
    mats = [t.cuda() for t in g]
    out = N.fpde_orthogonalize(mats, steps=2, coeffs=(1.5, -0.5, 0.0), out=mats)
    for i in range(3):
        assert out[i] is mats[i]
        near("cubic", out[i], R.orthogonalize(g[i].double(), 2, (1.5, -0.5, 0.0), 1e-7))


def test_tiles_of_128(N):
    """Enough tiles for the larger ones: batches, and one large matrix, ragged."""
    for count, m, n in ((45, 500, 300), (1, 2900, 3001)):
        print(f"case ortho {count} of {m} x {n}", flush=True)
        g = torch.stack([matrix(m, n, s) for s in range(count)]).cuda()
        o = N.fpde_orthogonalize(g, steps=3)
        for i in range(0, count, 7):
            near(f"{m} x {n}", o[i], R.orthogonalize(g[i].double(), 3, CO, 1e-7).cpu())  # (float64 on the GPU)


def test_more_matrices_than_a_launch_takes(N):
    g = torch.stack([matrix(20, 30, s) for s in range(70)])
    o = N.fpde_orthogonalize(g.view(7, 10, 20, 30).cuda()).view(70, 20, 30)
    for i in (0, 31, 32, 63, 64, 69):
        near("many", o[i], R.orthogonalize(g[i].double(), 5, CO, 1e-7))
    assert N.fpde_orthogonalize([]) == []
    assert N.fpde_orthogonalize(torch.empty(0, 4, 5, device="cuda")).shape == (0, 4, 5)


@pytest.mark.parametrize("m,n", [(64, 100), (128, 128), (300, 200)])
def test_decaying_spectra(N, m, n):
    """Rank 5 beside noise 10^-4 of it, and exactly rank 1."""
    g = torch.Generator().manual_seed(3)
    low = R.randn(g, m, 5, dtype=torch.float64) @ R.randn(g, 5, n, dtype=torch.float64)
    a = (low + 1e-4 * R.randn(g, m, n, dtype=torch.float64)).float()
    near("low rank", N.fpde_orthogonalize(a.cuda()), R.orthogonalize(a.double(), 5, CO, 1e-7), 7e-4)
    b = (R.randn(g, m, 1) @ R.randn(g, 1, n)).float()
    near("rank 1", N.fpde_orthogonalize(b.cuda()), R.orthogonalize(b.double(), 5, CO, 1e-7), 7e-4)


def test_extreme_magnitudes(N):
    for m, n in ((40, 50), (200, 140)):
        g = matrix(m, n)
        for f in (1e-30, 1e30):  # (squares under- and overflow float32)
            x = (g * f).float()
            near(f"times {f}", N.fpde_orthogonalize(x.cuda(), eps=0.0), R.orthogonalize(x.double(), 5, CO, 0.0))
        z = torch.stack([torch.zeros(m, n), g, torch.full((m, n), float("nan"))])
        o = N.fpde_orthogonalize(z.cuda(), eps=0.0).cpu()
        assert not o[0].any() and torch.isnan(o[2]).all()  # (each matrix by itself)
        near("beside", o[1], R.orthogonalize(g.double(), 5, CO, 0.0))


@pytest.mark.parametrize("dt", R.DTYPES, ids=str)
@pytest.mark.parametrize("m,n", [(48, 80), (128, 100), (150, 300), (300, 150)])
def test_muon_step(N, m, n, dt):
    print(f"case muon {m} x {n} {dt}", flush=True)
    for nesterov in (True, False):
        g = torch.stack([matrix(m, n, s, dt) for s in range(3)])
        gen = torch.Generator().manual_seed(9)
        w, mom = R.randn(gen, 3, m, n, dtype=dt), 1e-2 * R.randn(gen, 3, m, n)
        wc, mc = w.cuda(), mom.cuda()
        kw = dict(lr=0.05, momentum=0.9, nesterov=nesterov, weight_decay=0.1)
        N.fpde_muon_step(wc.unbind(0), g.cuda().unbind(0), mc.unbind(0), **kw)
        for i in range(3):
            rm = 0.9 * mom[i].double() + g[i].double()
            u = g[i].double() + 0.9 * rm if nesterov else rm
            scale = max(1.0, m / n) ** 0.5
            rw = (1 - 0.05 * 0.1) * w[i].double() - 0.05 * scale * R.orthogonalize(u, 5, CO, 1e-7)
            # (mu and the factors are rounded to float32 before use)
            R.close("momentum", mc[i], rm, 4, rm.abs() + mom[i].double().abs())
            near("weight", wc[i], rw)


def test_optimiser(N):
    """Muon: several shapes, two steps, equal to the calls; state and refusals."""
    gen = torch.Generator().manual_seed(2)
    ps = [torch.nn.Parameter(R.randn(gen, *s).cuda()) for s in ((40, 20), (40, 20), (200, 30), (5, 6))]
    frozen = torch.nn.Parameter(torch.zeros(3, 3, device="cuda"))
    opt = N.Muon([*ps, frozen], lr=0.1, weight_decay=0.01)
    w, mom = [p.detach().clone() for p in ps], [torch.zeros_like(p) for p in ps]
    for k in range(2):
        for p in ps:
            p.grad = R.randn(gen, *p.shape).cuda()
        opt.step()
        for i, p in enumerate(ps):
            N.fpde_muon_step([w[i]], [p.grad], [mom[i]], lr=0.1, weight_decay=0.01)
            assert torch.equal(w[i], p.detach()) and torch.equal(mom[i], opt.state[p]["momentum"])
    assert not frozen.any()
    with pytest.raises(ValueError):
        N.Muon([torch.nn.Parameter(torch.zeros(4, device="cuda"))])


def test_streams_and_graph(N):
    for m, n in ((90, 128), (300, 140)):
        g = torch.stack([matrix(m, n, s) for s in range(2)]).cuda()
        o = N.fpde_orthogonalize(g)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        o2 = N.fpde_orthogonalize(g, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(o, o2)
        w, mom = torch.zeros_like(g), torch.zeros_like(g)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            N.fpde_muon_step(w.unbind(0), g.unbind(0), mom.unbind(0), lr=0.1)
        w2, mom2 = torch.zeros_like(g), torch.zeros_like(g)
        for _ in range(3):
            g.add_(0.5 * g.roll(1, -1))
            graph.replay()
            torch.cuda.synchronize()
            N.fpde_muon_step(w2.unbind(0), g.unbind(0), mom2.unbind(0), lr=0.1)
            assert torch.equal(w, w2) and torch.equal(mom, mom2)


def test_momenta_of_16_bit_weights_survive_a_checkpoint(N):
    gen = torch.Generator().manual_seed(4)
    ps = [torch.nn.Parameter(R.randn(gen, 40, 24, dtype=torch.bfloat16).cuda()) for _ in range(2)]
    opt = N.Muon(ps, lr=0.1)
    for p in ps:
        p.grad = R.randn(gen, 40, 24, dtype=torch.bfloat16).cuda()
    opt.step()
    kept = opt.state_dict()
    other = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    again = N.Muon(other, lr=0.1)
    again.load_state_dict(kept)
    for p, q in zip(ps, other):
        m = again.state[q]["momentum"]
        assert m.dtype is torch.float32 and torch.equal(m, opt.state[p]["momentum"])
        assert m.data_ptr() != opt.state[p]["momentum"].data_ptr()
        q.grad = p.grad.clone()
    opt.step(), again.step()
    for p, q in zip(ps, other):
        assert torch.equal(p, q)


@pytest.mark.parametrize("count,m,n", [(26, 500, 300), (26, 300, 500), (1, 1930, 2050), (2, 2040, 1925)])
def test_quarters_of_the_last_tiles(N, count, m, n):
    """Tiles past a multiple of the compute units, in the symmetric products, the steps' and the last one."""
    print(f"case muon {count} of {m} x {n}", flush=True)
    g = torch.stack([matrix(m, n, s, torch.bfloat16) for s in range(count)])
    o = N.fpde_orthogonalize(g.cuda(), steps=3)
    gen = torch.Generator().manual_seed(11)
    w = R.randn(gen, count, m, n)
    wc, mc = w.cuda(), torch.zeros(count, m, n, device="cuda")
    N.fpde_muon_step(wc.unbind(0), g.float().cuda().unbind(0), mc.unbind(0), lr=0.05, momentum=0.9, steps=3)
    for i in {0, count // 2, count - 1}:
        r = R.orthogonalize(g[i].cuda().double(), 3, CO, 1e-7).cpu()
        near("orthogonalize", o[i], r)
        near("weight", wc[i], w[i].double() - 0.05 * max(1.0, m / n) ** 0.5 * r)


@pytest.mark.parametrize("count,m,n", [(2, 530, 700), (1, 1100, 1090), (1, 1500, 1510), (3, 300, 310), (1, 250, 770)])
def test_tiles_of_32_and_64(N, count, m, n):
    """Between the tiles of 32 and those of 128, and a sum shared by wavefronts or not."""
    print(f"case ortho {count} of {m} x {n}", flush=True)
    g = torch.stack([matrix(m, n, s) for s in range(count)]).cuda()
    o = N.fpde_orthogonalize(g, steps=4)
    for i in range(count):
        near("orthogonalize", o[i], R.orthogonalize(g[i].double(), 4, CO, 1e-7).cpu())
