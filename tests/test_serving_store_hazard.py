"""The serving kernels' wide stores under the same rule as the restore's: compiled to gfx950 assembly as the library
build does, none takes a register SGPR offset, none has its data registers rewritten right behind it, and no packed
single-precision instruction is made."""
import os
import shutil
import subprocess

import pytest

from paper_2609_26219_amd import build as pkv_build
from test_store_hazard import scan


@pytest.mark.skipif(not os.path.exists(pkv_build.HIPCC) and shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("src,dim", [("serve.hip", None), ("attend.hip", 64), ("attend.hip", 128), ("attend.hip", 256)])
def test_serving_kernels_have_no_store_data_hazard(src, dim, tmp_path):
    out = tmp_path / "kernels.s"
    define = [] if dim is None else [f"-DPKV_HEAD_DIM={dim}"]
    cmd = [pkv_build.HIPCC, *pkv_build.HIP_FLAGS, *define, "--cuda-device-only", "-S",
           os.path.join(pkv_build.CSRC, src), "-o", str(out)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    asm = out.read_text()
    problems, n_wide = scan(asm)
    assert n_wide > 0
    assert not problems, "\n".join(problems[:10])
    assert not [l for l in asm.splitlines() if l.strip().startswith(("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32"))]
