"""The repeat of marked units of attention's gradient, by its compiled code: no GPU."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
build = pytest.importorskip("paper_2608_11034_amd.build")


def test_repeat_writes_no_row_statistics(tmp_path):
    """Workgroups that repeat units of dq run beside others that read lse2 and delta for
    dk and dv, so the repeat must not store them.  They are the only single words that a
    unit stores: rows go out eight or sixteen bytes a lane."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no HIP compiler")
    src = os.path.join(build.CSRC, "c3_attention_grad.hip")
    asm = tmp_path / "grad.s"
    flags = [f for f in build.FLAGS if f != "-shared"]
    subprocess.run([build.HIPCC] + flags + ["-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S", src,
                                            "-o", str(asm)], check=True, stderr=subprocess.DEVNULL)
    kernels = re.findall(r"^(\S*attn_grad_careful_kernel\S*):(.*?)\.Lfunc_end", asm.read_text(), flags=re.M | re.S)
    assert len(kernels) == 4
    for name, body in kernels:
        stores = re.findall(r"\b(global_store_\w+|buffer_store_\w+|flat_store_\w+)", body)
        assert stores and "global_store_dword" not in stores, (name, sorted(set(stores)))
