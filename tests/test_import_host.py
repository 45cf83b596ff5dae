"""The package is imported by a torch that has no GPU back end, for its host-side calls."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
import paper_2205_11048_amd as gba
import paper_2205_11048_amd.step, paper_2205_11048_amd.worker
print(gba.gba_embedding_grad_workspace_size(10, 8, 100))
"""


def test_import_without_a_gpu_back_end():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and int(r.stdout) > 0, r.stderr[-2000:]
