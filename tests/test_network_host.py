"""Host-side checks of the network operators' C ABI (no GPU): exports, struct sizes,
workspace sizes, validation.  Every call here is invalid in at least one argument, or
has nothing to do, so the library returns before queueing any GPU work; the device
addresses are never touched."""
from __future__ import annotations

import ctypes
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fpde_net.h")
OK, ARG, SHAPE, COEFF, ALIGN, UNSUPPORTED = 0, -1, -2, -4, -5, -7
BASE, STRIDE = 0x7F0000000000, 1 << 32


@pytest.fixture(scope="module")
def N():
    from paper_2607_18020_amd import network  # noqa: PLC0415
    network.lib()
    return network


def addr(i, off=0):
    return BASE + i * STRIDE + off


def norm(N, **kw):
    v = dict(dtype=1, weight_dtype=0, out_dtype=1, group=0, rows=10, width=64, x_stride=64, residual_stride=64,
             eps=1e-6, x=addr(0), residual=addr(1), weight=addr(2), y=addr(3), sum=addr(4), scales=None)
    v.update(kw)
    return N.NormArgs(**v)


def norm_bwd(N, **kw):
    v = dict(dtype=0, weight_dtype=0, rows=10, width=64, dy_stride=64, sum_stride=64, dsum_stride=64, eps=1e-6,
             dy=addr(0), sum=addr(1), dsum=addr(2), weight=addr(3), ds=addr(4), dweight=addr(5), workspace=addr(6),
             workspace_bytes=1 << 30)
    v.update(kw)
    return N.NormBwdArgs(**v)


def conv(N, **kw):
    v = dict(dtype=0, weight_dtype=0, taps=4, silu=1, batch=2, length=10, channels=8, x_batch_stride=80,
             x_time_stride=8, x=addr(0), weight=addr(1), bias=addr(2), state=addr(3), lengths=addr(4), y=addr(5),
             state_out=addr(6))
    v.update(kw)
    return N.ConvArgs(**v)


def conv_bwd(N, **kw):
    v = dict(dtype=0, weight_dtype=0, taps=4, silu=1, batch=2, length=10, channels=8, x_batch_stride=80,
             x_time_stride=8, dy_batch_stride=80, dy_time_stride=8, dy=addr(0), x=addr(1), weight=addr(2),
             bias=addr(3), state=addr(4), lengths=addr(5), dx=addr(6), dweight=addr(7), dbias=addr(8),
             workspace=addr(9), workspace_bytes=1 << 30)
    v.update(kw)
    return N.ConvBwdArgs(**v)


SCAN = dict(dtype=0, states=16, groups=1, softplus=1, batch=2, length=10, channels=8, u_batch_stride=80, u_time_stride=8,
            delta_batch_stride=80, delta_time_stride=8, z_batch_stride=80, z_time_stride=8, b_batch_stride=160,
            b_time_stride=16, c_batch_stride=160, c_time_stride=16, u=addr(0), delta=addr(1), A=addr(2), B=addr(3),
            C=addr(4), D=addr(5), z=addr(6), delta_bias=addr(7), state=addr(8), lengths=addr(9), workspace=addr(30),
            workspace_bytes=1 << 30)


def scan(N, **kw):
    return N.ScanArgs(**{**SCAN, "y": addr(10), "state_out": addr(11), **kw})


def scan_bwd(N, **kw):
    return N.ScanBwdArgs(**{**SCAN, "dy_batch_stride": 80, "dy_time_stride": 8, "dy": addr(12), "du": addr(13),
                            "ddelta": addr(14), "dA": addr(15), "dB": addr(16), "dC": addr(17), "dD": addr(18),
                            "dz": addr(19), "ddelta_bias": addr(20), **kw})


def pointers(*v):
    a = (ctypes.c_void_p * len(v))(*v)
    return ctypes.cast(a, ctypes.c_void_p), a


def ortho(N, g=(addr(0), addr(1)), out=(addr(2), addr(3)), **kw):
    gp, k1 = pointers(*g)
    op, k2 = pointers(*out)
    v = dict(dtype=0, steps=5, count=2, m=300, n=200, a=3.4, b=-4.7, c=2.0, eps=1e-7, g=gp, out=op, workspace=addr(9),
             workspace_bytes=1 << 32)
    v.update(kw)
    a = N.OrthoArgs(**v)
    a._keep = (k1, k2)
    return a


def muon(N, g=(addr(0), addr(1)), mom=(addr(2), addr(3)), w=(addr(4), addr(5)), **kw):
    ps = [pointers(*v) for v in (g, mom, w)]
    v = dict(dtype=0, steps=5, nesterov=1, reserved=0, count=2, m=300, n=200, a=3.4, b=-4.7, c=2.0, eps=1e-7, lr=0.1,
             mu=0.9, weight_decay=0.0, scale=1.0, grads=ps[0][0], momenta=ps[1][0], weights=ps[2][0], workspace=addr(9),
             workspace_bytes=1 << 32)
    v.update(kw)
    a = N.MuonArgs(**v)
    a._keep = ps
    return a


def status(N, name, a):
    return getattr(N.lib(), name)(a, None)


def test_library_exports_every_declared_symbol(N):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    decl = set(re.findall(r"\b(fpde_\w+)\s*\(", src))
    assert decl == set(N.EXPORTED)
    for name in decl:
        assert hasattr(N.lib(), name), name


def test_structs_match_the_header(N, tmp_path):
    """sizeof and every offset, as a C compiler has them."""
    names = {"fpde_norm_args": N.NormArgs, "fpde_norm_bwd_args": N.NormBwdArgs, "fpde_conv_args": N.ConvArgs,
             "fpde_conv_bwd_args": N.ConvBwdArgs, "fpde_scan_args": N.ScanArgs, "fpde_scan_bwd_args": N.ScanBwdArgs,
             "fpde_ortho_args": N.OrthoArgs, "fpde_muon_args": N.MuonArgs}
    lines = []
    for c, s in names.items():
        lines.append(f'printf("%zu\\n", sizeof({c}));')
        lines += [f'printf("%zu\\n", offsetof({c}, {f}));' for f, _ in s._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "fpde_net.h"\nint main(void) {\n' + "\n".join(lines) +
                   "\nreturn 0;\n}\n")
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe],
                   check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for s in names.values():
        want.append(ctypes.sizeof(s))
        want += [getattr(s, f).offset for f, _ in s._fields_]
    assert got == want


NULL_CASES = [("fpde_rms_norm", norm), ("fpde_rms_norm_bwd", norm_bwd), ("fpde_causal_conv", conv),
              ("fpde_causal_conv_bwd", conv_bwd), ("fpde_selective_scan", scan), ("fpde_selective_scan_bwd", scan_bwd),
              ("fpde_orthogonalize", ortho), ("fpde_muon_step", muon)]


@pytest.mark.parametrize("name,make", NULL_CASES, ids=[n for n, _ in NULL_CASES])
def test_null_struct_and_types(N, name, make):
    assert getattr(N.lib(), name)(None, None) == ARG
    assert status(N, name, make(N, dtype=3)) == UNSUPPORTED
    assert status(N, name, make(N, dtype=-1)) == UNSUPPORTED
    if name + "_workspace" in N.EXPORTED:
        assert getattr(N.lib(), name + "_workspace")(None) == ARG
        assert getattr(N.lib(), name + "_workspace")(make(N, dtype=9)) == UNSUPPORTED


def test_norm_validation(N):
    f = "fpde_rms_norm"
    for kw, want in ((dict(weight_dtype=2), UNSUPPORTED), (dict(out_dtype=0), UNSUPPORTED),
                     (dict(out_dtype=3, group=64, scales=addr(5)), UNSUPPORTED), (dict(out_dtype=3), ARG),
                     (dict(rows=-1), SHAPE), (dict(rows=(1 << 40) + 1), SHAPE), (dict(width=0), SHAPE),
                     (dict(width=(1 << 20) + 1), SHAPE), (dict(x_stride=63), SHAPE), (dict(residual_stride=10), SHAPE),
                     (dict(rows=1 << 30, x_stride=1 << 31), SHAPE),
                     (dict(eps=-1e-9), COEFF), (dict(eps=float("nan")), COEFF), (dict(eps=float("inf")), COEFF),
                     (dict(x=None), ARG), (dict(y=None), ARG), (dict(x=addr(0, 1)), ALIGN), (dict(y=addr(3, 1)), ALIGN),
                     (dict(weight=addr(2, 2)), ALIGN), (dict(y=addr(0)), ARG), (dict(y=addr(1, 64)), ARG),
                     (dict(sum=addr(3, 2)), ARG), (dict(sum=addr(0, 2)), ARG), (dict(sum=addr(0), x_stride=65), ARG),
                     (dict(y=addr(2)), ARG), (dict(rows=0, x=None, y=None), OK)):
        assert status(N, f, norm(N, **kw)) == want, kw


def test_norm_bwd_validation(N):
    f = "fpde_rms_norm_bwd"
    need = N.lib().fpde_rms_norm_bwd_workspace(norm_bwd(N))
    assert need > 0 and N.lib().fpde_rms_norm_bwd_workspace(norm_bwd(N, dweight=None)) == 0
    for kw, want in ((dict(dy=None), ARG), (dict(sum=None), ARG), (dict(ds=None), ARG), (dict(workspace=None), ARG),
                     (dict(workspace_bytes=need - 1), ARG), (dict(workspace=addr(6, 8)), ALIGN),
                     (dict(workspace=addr(0)), ARG), (dict(ds=addr(1)), ARG), (dict(dweight=addr(3)), ARG),
                     (dict(ds=addr(0), dy_stride=80), ARG), (dict(dsum_stride=1), SHAPE), (dict(dy_stride=0), SHAPE),
                     (dict(eps=float("nan")), COEFF), (dict(width=0), SHAPE)):
        assert status(N, f, norm_bwd(N, **kw)) == want, kw


def test_conv_validation(N):
    f = "fpde_causal_conv"
    for kw, want in ((dict(taps=1), UNSUPPORTED), (dict(taps=5), UNSUPPORTED), (dict(silu=2), ARG), (dict(channels=0), SHAPE),
                     (dict(channels=(1 << 20) + 1), SHAPE), (dict(batch=-1), SHAPE), (dict(length=1 << 31), SHAPE),
                     (dict(batch=1 << 30, length=1 << 10), SHAPE), (dict(batch=(1 << 34) + 1, length=0), SHAPE), (dict(x_time_stride=7), SHAPE),
                     (dict(x_batch_stride=-1), SHAPE), (dict(x=None), ARG), (dict(weight=None), ARG), (dict(y=None), ARG),
                     (dict(y=addr(0)), ARG), (dict(state_out=addr(3, 4)), ARG), (dict(lengths=addr(4, 2)), ALIGN),
                     (dict(batch=0), OK), (dict(length=0, state_out=None, x=None, y=None), OK)):
        assert status(N, f, conv(N, **kw)) == want, kw
    f = "fpde_causal_conv_bwd"
    need = N.lib().fpde_causal_conv_bwd_workspace(conv_bwd(N))
    for kw, want in ((dict(dy=None), ARG), (dict(dweight=None), ARG), (dict(dx=addr(0)), ARG), (dict(dx=addr(1)), ARG),
                     (dict(workspace_bytes=need - 1), ARG), (dict(workspace=None), ARG), (dict(dy_time_stride=1), SHAPE),
                     (dict(dbias=addr(7, 4)), ARG), (dict(taps=9), UNSUPPORTED)):
        assert status(N, f, conv_bwd(N, **kw)) == want, kw


def test_scan_validation(N):
    common = ((dict(states=0), SHAPE), (dict(states=33), UNSUPPORTED), (dict(groups=3), SHAPE), (dict(groups=0), SHAPE),
              (dict(softplus=2), ARG), (dict(channels=0), SHAPE), (dict(length=-1), SHAPE), (dict(batch=-1), SHAPE),
              (dict(length=1 << 31), SHAPE), (dict(u_time_stride=7), SHAPE), (dict(delta_time_stride=7), SHAPE),
              (dict(z_time_stride=7), SHAPE), (dict(b_time_stride=15), SHAPE), (dict(c_batch_stride=-1), SHAPE),
              (dict(u=None), ARG), (dict(delta=None), ARG), (dict(A=None), ARG), (dict(B=None), ARG), (dict(C=None), ARG),
              (dict(A=addr(2, 2)), ALIGN), (dict(delta=addr(1, 1)), ALIGN))
    for kw, want in common:
        assert status(N, "fpde_selective_scan", scan(N, **kw)) == want, kw
        assert status(N, "fpde_selective_scan_bwd", scan_bwd(N, **kw)) == want, kw
    for kw, want in ((dict(y=None), ARG), (dict(y=addr(0)), ARG), (dict(state_out=addr(8, 4)), ARG),
                     (dict(y=addr(3, 64)), ARG), (dict(batch=0), OK), (dict(length=0, state_out=None), OK)):
        assert status(N, "fpde_selective_scan", scan(N, **kw)) == want, kw
    big = dict(length=4096, u_batch_stride=1 << 20, delta_batch_stride=1 << 20, z_batch_stride=1 << 20,
               b_batch_stride=1 << 20, c_batch_stride=1 << 20)
    need = N.lib().fpde_selective_scan_workspace(scan(N, **big))
    assert need > 0
    assert status(N, "fpde_selective_scan", scan(N, workspace_bytes=need - 1, **big)) == ARG
    assert status(N, "fpde_selective_scan", scan(N, workspace=None, **big)) == ARG
    for kw, want in ((dict(dy=None), ARG), (dict(du=None), ARG), (dict(dA=None), ARG), (dict(dD=None), ARG),
                     (dict(D=None), ARG), (dict(dz=None), ARG), (dict(z=None), ARG), (dict(ddelta_bias=None), ARG),
                     (dict(dB=addr(3)), ARG), (dict(du=addr(13), dz=addr(13)), ARG), (dict(workspace=None), ARG),
                     (dict(workspace_bytes=16), ARG), (dict(workspace=addr(30, 4)), ALIGN), (dict(dy_time_stride=2), SHAPE)):
        assert status(N, "fpde_selective_scan_bwd", scan_bwd(N, **kw)) == want, kw


def test_ortho_validation(N):
    for name, make in (("fpde_orthogonalize", ortho), ("fpde_muon_step", muon)):
        for kw, want in ((dict(count=-1), SHAPE), (dict(count=65537), SHAPE), (dict(m=0), SHAPE), (dict(n=32769), SHAPE),
                         (dict(steps=0), COEFF), (dict(steps=101), COEFF), (dict(a=float("inf")), COEFF),
                         (dict(b=float("nan")), COEFF), (dict(eps=-1.0), COEFF), (dict(workspace=None), ARG),
                         (dict(workspace_bytes=8), ARG), (dict(workspace=addr(9, 8)), ALIGN),
                         (dict(g=(addr(0), None)), ARG), (dict(g=(addr(0, 2), addr(1))), ALIGN),
                         (dict(workspace=addr(0, 64)), ARG), (dict(count=0), OK)):
            assert status(N, name, make(N, **kw)) == want, (name, kw)
    size = 300 * 200 * 4
    for kw, want in ((dict(out=(addr(1), addr(3))), ARG), (dict(out=(addr(2), addr(2, size - 4))), ARG),
                     (dict(out=(addr(0, 4), addr(3))), ARG), (dict(out=(addr(2), None)), ARG), (dict(out=None), ARG)):
        if kw["out"] is None:
            a = ortho(N)
            a.out = None
        else:
            a = ortho(N, **kw)
        assert status(N, "fpde_orthogonalize", a) == want, kw
    for kw, want in ((dict(w=(addr(0), addr(5))), ARG), (dict(mom=(addr(2), addr(2))), ARG), (dict(mom=(addr(2), None)), ARG),
                     (dict(nesterov=2), ARG), (dict(reserved=1), ARG), (dict(lr=float("nan")), COEFF),
                     (dict(mu=float("inf")), COEFF), (dict(scale=float("nan")), COEFF)):
        assert status(N, "fpde_muon_step", muon(N, **kw)) == want, kw


def test_python_refuses_what_is_not_on_the_gpu(N):
    x, w = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises(ValueError, match="CUDA"):
        N.fpde_rms_norm(x, w)
    with pytest.raises(ValueError, match="CUDA"):
        N.fpde_rms_norm_bwd(x, x, w)
    with pytest.raises(ValueError, match="CUDA"):
        N.fpde_causal_conv(x[None], torch.zeros(8, 4))
    with pytest.raises(ValueError, match="CUDA"):
        N.fpde_selective_scan(x[None], x[None], torch.zeros(8, 4), torch.zeros(1, 4, 4), torch.zeros(1, 4, 4))
    with pytest.raises(ValueError, match="CUDA"):
        N.fpde_orthogonalize(x)
    with pytest.raises(ValueError, match="CUDA"):
        N.fpde_muon_step([x], [x], [x], lr=0.1)
    with pytest.raises(ValueError):
        N.Muon([torch.nn.Parameter(torch.zeros(3))])


def test_no_fallback_without_the_library(N, tmp_path, monkeypatch):
    monkeypatch.setattr(N, "_lib", None)
    monkeypatch.setattr(N, "_fns", {})
    monkeypatch.setattr(N, "LIB_PATH", str(tmp_path / "missing.so"))
    with pytest.raises(ImportError):
        N.lib()
