"""Every call that a rollout makes opens a named range for timeline tools, seen by a stand-in for such a tool (a range is
opened before the arguments are looked at, so calls that are refused do without a GPU)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

TOOL = r"""
#include <nvtx3/nvToolsExt.h>
#include <stdio.h>
static int depth;
static int NVTX_API push(const char* name) { fprintf(stderr, "push %s\n", name); return depth++; }
static int NVTX_API pop(void) { fprintf(stderr, "pop\n"); return --depth; }
int InitializeInjectionNvtx2(NvtxGetExportTableFunc_t get) {
  const NvtxExportTableCallbacks* t = (const NvtxExportTableCallbacks*)get(NVTX_ETID_CALLBACKS);
  NvtxFunctionTable table = 0;
  unsigned int size = 0;
  if (!t || !t->GetModuleFunctionTable(NVTX_CB_MODULE_CORE, &table, &size)) return 0;
  *table[NVTX_CBID_CORE_RangePushA] = (NvtxFunctionPointer)push;
  *table[NVTX_CBID_CORE_RangePop] = (NvtxFunctionPointer)pop;
  return 1;
}
"""

CALLS = """
import ctypes
from paper_2512_15347_b200 import binding as B
L = B.lib()
for name in ("pg_step", "pg_prune_ovf", "pg_kv_attend", "pg_kv_extend", "pg_kv_append", "pg_kv_fork", "pg_kv_pack", "pg_logits_process"):
    f = getattr(L, name)
    assert f(*[0 if t in (ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float) else None for t in f.argtypes]) == B.EINVAL
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
    want = ("pg_step", "pg_prune_ovf", "pg_kv_attend", "pg_kv_extend", "pg_kv_append", "pg_kv_fork", "pg_kv_pack", "pg_logits_process")
    assert seen == [line for name in want for line in (f"push {name}", "pop")]
