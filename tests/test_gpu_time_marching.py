"""The operators together: the example network trains on the Burgers residual, and its
rollout by carried states gives the field of the whole window."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "time_marching.py")


@pytest.fixture(scope="module")
def T():
    spec = importlib.util.spec_from_file_location("time_marching", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_training_lowers_the_loss_and_the_rollout_is_the_window(T):
    dev = torch.device("cuda:0")
    torch.manual_seed(0)
    model = T.TimeMarcher(32).to(dev)
    print("case time marching: 30 steps on 24 x 40", flush=True)
    losses = T.train(model, 24, 40, 30, dev)
    assert torch.isfinite(losses).all()
    assert losses[-5:].mean() < 0.5 * losses[0]
    _, _, t, x, u0 = T.problem(24, 40, dev)
    with torch.no_grad():
        window = model(t, x, u0)
    # float32 through two blocks, products in another order: a few hundred roundings of numbers of size
    # |u| <= 10 and less
    assert (model.rollout(t, x, u0) - window).abs().max() <= 1000 * 2.0 ** -24 * 10
    # e4m3 holds 4 significand bits: 1/16 of the activations at each of two norms
    f8 = model.rollout(t, x, u0, 128)
    assert torch.isfinite(f8).all() and (f8 - window).norm() <= 0.5 * window.norm()


def test_gradients_reach_every_parameter(T):
    dev = torch.device("cuda:0")
    model = T.TimeMarcher(32, blocks=1).to(dev)
    cfg, h, t, x, u0 = T.problem(12, 20, dev)
    T.B.ResidualLoss.apply(cfg.op, h, cfg.coeffs, [], model(t, x, u0)).backward()
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any(), name
