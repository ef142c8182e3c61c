"""The network operators' own gfx950 assembly (static, no GPU needed): no packed-FP32
VALU, no private segment or scratch access anywhere, no atomics, matrix instructions
where there are products and nowhere else."""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

from paper_2607_18020_amd.csrc import build as B

pytestmark = pytest.mark.skipif(shutil.which(B.HIPCC) is None and not os.path.exists(B.HIPCC),
                                reason="hipcc not available")


def kernels(asm):
    """{mangled name: (instructions, private segment in bytes)} of the kernels in an assembly listing."""
    found, name = {}, None
    for line in asm.splitlines():
        m = re.match(r"^(_Z\w+):", line)
        if m:
            name = m.group(1)
            found[name] = [[], None]
            continue
        s = line.strip()
        m = re.match(r";\s*ScratchSize:\s*(\d+)", s)
        if m and name and found[name][1] is None:
            found[name][1] = int(m.group(1))
        elif name and s and not s.startswith((";", ".")) and not s.endswith(":"):
            found[name][0].append(s)
    return {k: v for k, v in found.items() if v[1] is not None}


@pytest.mark.parametrize("source", B.NET_SOURCES, ids=os.path.basename)
def test_rules(source, tmp_path):
    out = str(tmp_path / "k.s")
    flags = [f for f in B.FLAGS if f not in ("-fPIC", "-shared")]
    r = subprocess.run([B.HIPCC, *flags, "-I", B.NET_DIR, "--cuda-device-only", "-S", "-o", out, source],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    ks = kernels(open(out).read())
    assert len(ks) >= 10
    mfma = False
    for name, (ins, private) in ks.items():
        ops = [s.split()[0] for s in ins]
        assert not [o for o in ops if re.match(r"v_pk_\w+_f32", o)], name
        assert not [o for o in ops if o.startswith("scratch_")] and private == 0, (name, private)
        assert not [o for o in ops if "atomic" in o], name
        has = any(o.startswith("v_mfma") for o in ops)
        mfma |= has
        assert has == ("product" in name or "ortho_small" in name), name
    assert mfma == ("ortho" in source)
