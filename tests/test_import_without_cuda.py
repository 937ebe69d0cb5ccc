"""The binding can be imported, and sizes and host checks asked for, where torch was built without CUDA: such a torch lacks the functions
for streams and devices."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
from paper_2009_13003_b200 import binding
assert binding.stream_bound(1000, 4) > 0 and binding.workspace_bytes(0) > 0
assert binding.q4_bytes(16, 128, 128) > 0 and binding.lib().lc_strerror(binding.ERR_INDEX)
for call in (lambda: binding.q4_quantize(torch.ones(4, 32)), lambda: binding.q4_matvec(binding.Q4(torch.zeros(4096, dtype=torch.uint8), 16, 128, 128), torch.ones(128))):
    try:
        call()
    except ValueError:
        continue
    raise SystemExit("not refused")
print("fine")
"""


def test_import_without_the_functions_of_cuda():
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=os.path.dirname(HERE), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "fine", run.stdout + run.stderr
