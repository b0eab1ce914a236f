"""The policy-update calls on token trajectories open named ranges for timeline tools, as the library's other calls do."""
import os
import subprocess
import sys

from tests.test_trace_ranges import ROOT, TOOL

NAMES = ("pg_token_forward", "pg_token_backward", "pg_token_forward_backward", "pg_token_objective")
CALLS = f"""
import ctypes
from paper_2512_15347_b200 import binding as B
L = B.lib()
for name in {NAMES}:
    f = getattr(L, name)
    assert f(*[0 if t in (ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t) else None for t in f.argtypes]) == B.EINVAL
"""


def test_calls_open_ranges(tmp_path):
    src, tool = tmp_path / "tool.c", tmp_path / "tool.so"
    src.write_text(TOOL)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["gcc", "-shared", "-fPIC", str(src), "-I", os.path.join(cuda, "include"), "-ldl", "-o", str(tool)], check=True)
    res = subprocess.run([sys.executable, "-c", CALLS], cwd=ROOT, env=dict(os.environ, NVTX_INJECTION64_PATH=str(tool)), capture_output=True,
                         text=True, timeout=300)
    assert res.returncode == 0, res.stderr
    seen = [x for x in res.stderr.splitlines() if x.startswith(("push pg_", "pop"))]
    assert seen == [line for name in NAMES for line in (f"push {name}", "pop")]
