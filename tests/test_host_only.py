"""CPU test: the package on a host without a GPU, and with a torch built without one."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_calls_need_no_gpu_functions_of_torch():
    """Checks and workspace sizes run where torch lacks what it has with a GPU."""
    code = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
import paper_2606_16264_amd as mx
s, b = mx.attn_shape(8, 2, 128, 64), mx.Batch([1, 0], [1, 20], [40, 0], [[0, 1, 2], [3, 4]])
assert mx.mx_batch_validate(b, s) == mx.MX_OK
print(mx.mx_workspace_bytes_for(b, s), mx.mx_workspace_bytes_window_for(b, s, 16),
      mx.mx_workspace_bytes_window(s, 21, 2, 5), mx.mx_workspace_bytes_shared_for(b, s, mx.SharedRuns([])),
      mx.mx_workspace_bytes_shared(s, 21, 2, 5, 0))
q = torch.zeros(21, 8, 128, dtype=torch.bfloat16)
try:
    mx.mx_paged_attn_window(b, s, 16, 0, q, q, q, q, q)
except ValueError as e:
    print(e)
"""
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=240)
    assert out.returncode == 0, out.stderr[-2000:]
    sizes, refused = out.stdout.strip().splitlines()
    assert all(int(n) > 0 for n in sizes.split()) and refused == "q is not on a GPU"
