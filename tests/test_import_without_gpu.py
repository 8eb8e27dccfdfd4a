"""The package on a torch that was built without a GPU: it imports, what needs no GPU works, and the calls raise."""
import os
import subprocess
import sys

import pytest

import paper_2609_19104_amd as rm

PROGRAM = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2609_19104_amd as rm
assert rm.rm_workspace_size(256, 512, rm.RM_BF16, 1, 51, 150) > 0
assert rm.load_library().rm_page_slots(0, 1, 1, 1, 1, *[None] * 14) == rm.RM_ERR_INVALID_ARG
q, cache = torch.zeros(300, 8, 64), torch.zeros(4, 16, 2, 64)
assert rm.paged_attention_workspace(q, cache, torch.zeros(300, 4, dtype=torch.int32)).numel() > 0
for call in (lambda: rm._stream(None), lambda: rm.rm_block_norm(q, q, None, q)):
    try:
        call()
    except (RuntimeError, ValueError):
        continue
    raise SystemExit("a call without a GPU did not raise")
print("imported")
"""


def test_the_package_imports_without_gpu_support(root_dir):
    if not os.path.exists(rm.LIB_PATH):
        pytest.skip("librmuscle.so not built")
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root_dir, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("imported"), r.stderr[-2000:]
