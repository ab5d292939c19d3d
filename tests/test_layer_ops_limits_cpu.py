"""CPU-only checks of the decoder layer's operators: where the package imports, which sizes their entry points refuse."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_imports_where_torch_has_no_gpu_part():
    # such a torch lacks these names; calls refuse its tensors as they do any CPU tensor
    code = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2605_16184_amd as ast
x = torch.zeros(2, 8)
for call in (lambda: ast.dropout(x, x, 0.5), lambda: ast.rms_norm(x, x), lambda: ast.rms_norm_backward(x, x, dX=x)):
    try:
        call()
    except ValueError:
        continue
    raise SystemExit("not refused")
print("imported")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "imported" in r.stdout, r.stderr[-2000:]
