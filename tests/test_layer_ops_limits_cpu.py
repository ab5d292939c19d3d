"""CPU-only checks of the decoder layer's operators: where the package imports, which sizes their entry points refuse."""
import ctypes
import os
import subprocess
import sys

import torch

import paper_2605_16184_amd as ast
from paper_2605_16184_amd import binding as B

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


# Sizes that pass are only called where there is no device to launch on: the call then ends with the runtime's error.
PASSES = [B.UNSUPPORTED, B.HIP_ERROR] if not torch.cuda.is_available() else [B.UNSUPPORTED]


def test_dropout_takes_all_sizes_up_to_its_limit():
    rng = B._Rng(p=0.25)
    sizes = [(401, 8 * 10710641), ((1 << 24) - 1, 8 * 256)]  # rows ceil(cols / 8) = 2^32 - 255 and 2^32 - 256
    for (rows, cols), want in zip(sizes, PASSES):
        d = B._Drop(X=0x1000, Y=0x2000, rows=rows, cols=cols, ldx=cols, ldy=cols)
        assert ast.lib().asteria_dropout(ctypes.byref(d), ctypes.byref(rng), None) == want


def test_attention_takes_all_sizes_up_to_its_limit():
    for tiles, want in zip((2 ** 24 - 3, 2 ** 24 - 4), PASSES):      # (tiles + 1 + nseq) heads = 2^24 and 2^24 - 1
        a = B._Attn(Q=0x1000, K=0x2000, V=0x3000, O=0x4000, cu=0x6000, total=128 * tiles, nseq=2, heads=1, kv_heads=1, dim=8, ldq=8, hq=8,
                    ldk=8, hk=8, ldv=8, hv=8, ldo=8, ho=8, scale=0.3)
        assert ast.lib().asteria_attention(ctypes.byref(a), None) == want
