"""Tensors that the network operators write in place count as changed for
autograd: a backward pass whose saved tensors were written over raises, as it
does after torch's own in-place operations."""
from __future__ import annotations

import pytest
import torch

from tests import network_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def N():
    from paper_2607_18020_amd import network
    network.lib()
    return network


def refused(loss):
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_backward_after_saved_tensors_were_written_raises(N):
    g = torch.Generator().manual_seed(3)

    def r(*shape):
        return R.randn(g, *shape).cuda()

    x, w, state = r(2, 9, 8), r(8, 4), r(2, 3, 8)
    leaf = x.clone().requires_grad_()
    y = N.CausalConv.apply(leaf, w, None, True, state, None).sum()
    N.fpde_causal_conv_step(r(2, 8), state, w)
    refused(y)

    A, B, C, h = -r(8, 4).abs(), r(2, 9, 4), r(2, 9, 4), r(2, 8, 4)
    leaf = x.clone().requires_grad_()
    y = N.SelectiveScan.apply(leaf, x, A, B, C, None, None, None, True, h, None).sum()
    N.fpde_selective_step(h, r(2, 8), r(2, 8), A, r(2, 4), r(2, 4))
    refused(y)

    leaf = x.clone().requires_grad_()
    y, s = N.RmsNorm.apply(leaf, x, None, 1e-6)
    N.fpde_rms_norm(x, out=s.detach())
    refused(y.sum())

    p = torch.nn.Parameter(r(8, 8))
    a = r(3, 8).requires_grad_()
    y = (a @ p).sum()
    N.fpde_muon_step([p.detach()], [r(8, 8)], [torch.zeros(8, 8, device="cuda")], lr=0.02)
    refused(y)


def test_every_written_tensor_gets_a_version(N):
    g = torch.Generator().manual_seed(4)

    def r(*shape):
        return R.randn(g, *shape).cuda()

    def written(*ts):
        assert all(t._version == 1 for t in ts), [t._version for t in ts]

    def new(*shape):
        return torch.empty(*shape, device="cuda")

    x, dy = r(6, 16), r(6, 16)
    y, s = new(6, 16), new(6, 16)
    N.fpde_rms_norm(x, residual=dy, out=y, sum_out=s)
    written(y, s)
    ds = new(6, 16)
    N.fpde_rms_norm_bwd(dy, x, ds=ds)
    written(ds)

    u, w, last, out = r(2, 5, 8), r(8, 3), new(2, 2, 8), new(2, 5, 8)
    N.fpde_causal_conv(u, w, state_out=last, out=out)
    written(last, out)
    conv, out = new(2, 2, 8).fill_(0), new(2, 8)
    before = conv._version
    N.fpde_causal_conv_step(r(2, 8), conv, w, out=out)
    written(out)
    assert conv._version == before + 1

    A, B, C, h, out = -r(8, 4).abs(), r(2, 5, 4), r(2, 5, 4), new(2, 8, 4), new(2, 5, 8)
    N.fpde_selective_scan(u, u, A, B, C, state_out=h, out=out)
    written(h, out)
    out = new(2, 8)
    before = h._version
    N.fpde_selective_step(h, r(2, 8), r(2, 8), A, r(2, 4), r(2, 4), out=out)
    written(out)
    assert h._version == before + 1

    mats, out = r(2, 8, 8), new(2, 8, 8)
    N.fpde_orthogonalize(mats, out=out)
    written(out)
    out = [new(8, 8), new(8, 8)]
    N.fpde_orthogonalize([mats[0], mats[1]], out=out)
    written(*out)
    weight, grad, mom = r(8, 8).clone(), r(8, 8), torch.zeros(8, 8, device="cuda")
    before = weight._version, mom._version
    N.fpde_muon_step([weight], [grad], [mom], lr=0.02)
    assert (weight._version, mom._version) == (before[0] + 1, before[1] + 1)
    assert x._version == dy._version == u._version == grad._version == 0  # inputs are only read
