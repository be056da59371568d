"""The gradient of the softmax loss may be written over the logits, so a kernel that writes it must not read them as memory that never changes: loads
through the constant address space may be moved behind the stores, or made again there.  The kernels are compiled to the compiler's own language, before
any optimisation, and every kernel with a gradient is followed to the loads of the targets' logits."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1902_01981_amd", "csrc")
HIPCC = os.environ.get("HIPCC") or shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    """function -> the functions that it calls; kernels are those of `kernels`."""
    if not os.path.exists(HIPCC):
        pytest.skip("needs hipcc")
    out = str(tmp_path_factory.mktemp("loss") / "loss.ll")
    subprocess.run([HIPCC, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--offload-arch=gfx950", "--offload-device-only", "-S", "-emit-llvm",
                    "-Xclang", "-disable-llvm-passes", os.path.join(CSRC, "loss_kernels.hip"), "-o", out], check=True, capture_output=True)
    graph, kernels, name = {}, [], None
    with open(out) as f:
        for line in f:
            if line.startswith("define"):
                name = re.search(r"@([\w.$]+)\(", line).group(1)
                graph[name] = set()
                if "amdgpu_kernel" in line:
                    kernels.append(name)
            elif name and " call " in line:
                graph[name].update(re.findall(r"@([\w.$]+)\(", line))
            elif line.startswith("}"):
                name = None
    return graph, kernels


def _reached(graph, start):
    seen, todo = set(), [start]
    while todo:
        f = todo.pop()
        if f not in seen:
            seen.add(f)
            todo += graph.get(f, ())
    return seen


def test_logits_that_may_be_replaced(calls):
    graph, kernels = calls
    # the last template argument says whether the gradient is wanted
    writing = [k for k in kernels if re.search(r"loss_(narrow|rows|join)_kernelI.*Lb1EEEv", k)]
    assert len([k for k in writing if "loss_rows_kernel" in k]) >= 16 and len([k for k in writing if "loss_narrow_kernel" in k]) >= 8
    reads = 0
    for kernel in writing:
        for f in _reached(graph, kernel):
            if "read_logit" in f:
                reads += 1
                assert not [g for g in _reached(graph, f) if "scalar_load" in g], (kernel, f)
    assert reads >= 24
