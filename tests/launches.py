"""What a call launches, without a GPU: the library's host code runs in a process of its own over tests/c/launch_recorder.c, which writes launches down and makes none.  The calls are those of
tests/test_paged_window_abi.py and tests/test_paged_abi.py, whose addresses nothing looks behind."""
import ctypes as C
import json
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class _Launch(C.Structure):
    _fields_ = [("grid", C.c_uint32 * 3), ("block", C.c_uint32 * 3), ("name", C.c_char_p)]


def record(calls, tmp_path):
    """calls: (entry point, params, sizes) each, as the two name them (single: the attention of one token).  Returns per call (status, bytes of workspace or None, [(kernel, grid, block)])."""
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    so = str(tmp_path / "launch_recorder.so")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(ROOT, "tests", "c", "launch_recorder.c")], check=True)
    r = subprocess.run([sys.executable, "-m", "tests.launches", so], input=json.dumps(calls), capture_output=True, text=True, cwd=ROOT, timeout=120)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def _main(path):
    recorder = C.CDLL(path, C.RTLD_GLOBAL)
    recorder.recorder_launch.restype = C.POINTER(_Launch)
    C.CDLL(os.path.join(ROOT, "paper_2510_20707_amd", "libmixkv.so"))          # before torch, which has kernels of its own to register
    from paper_2510_20707_amd import binding as B
    from tests import test_paged_abi as A
    from tests import test_paged_window_abi as W
    B.lib()
    results = []
    for op, params, sizes in json.load(sys.stdin):
        p, n = W._params(**params), sizes.get("n", 1)
        strides = dict(q_stride_n=p.n_q_heads * p.head_dim, q_stride_h=p.head_dim, out=1 << 56, lse=1 << 57)
        recorder.recorder_clear()
        if op in ("select", "single"):
            kw = dict(n=n, size=1 << 62)
            status = A._select(p, A._caches(n), **kw) if op == "select" else A._attend(p, A._caches(n), rows=sizes["rows"], selected=0, n_selected=0, **kw)
            need = B.mixkv_paged_select_workspace_size(p, n) if op == "select" else B.mixkv_paged_attention_workspace_size(p, n, sizes["rows"])
        elif op == "evict":
            status = W._evict(p, n=n, size=1 << 62, **{k: v for k, v in sizes.items() if k != "n"})
            need = B.mixkv_paged_evict_workspace_size(p, n, sizes["rows"])
        else:
            call, size = {"attend": (W._attend, B.mixkv_paged_window_attention_workspace_size), "weigh": (W._weigh, B.mixkv_paged_weights_workspace_size)}[op]
            status = call(p, queries=W._queries(n, **strides), size=1 << 62, **sizes)
            need = size(p, n, *(sizes[k] for k in ("rows", "window", "first", "count", "most")))
        made = [recorder.recorder_launch(i).contents for i in range(min(recorder.recorder_count(), 1 << 16))]
        results.append((status, need, [(x.name.decode(), list(x.grid), list(x.block)) for x in made]))
    print(json.dumps(results))


if __name__ == "__main__":
    _main(sys.argv[1])
