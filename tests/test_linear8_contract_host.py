"""What the sources of the 8-bit linear operators, and the binding around them,
have to keep to, checked without a GPU."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_00049_gb300", "csrc")


def kernels(path):
    """(name, parameters, body) of each kernel of a source file."""
    text = re.sub(r"//[^\n]*", "", open(path).read())
    for m in re.finditer(r"__global__\s+void[^{;]*?(\w+)\(([^{;]*?)\)\s*\{", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield m.group(1), m.group(2), text[m.end():at]


@pytest.mark.parametrize("source", ["int8_product_tc.cu", "checkpoint_grad.cu"])
def test_kernels_read_what_the_kernel_before_writes_with_ordinary_loads(source):
    """The kernels over a split product's parts may start while the parts are
    being written: no read-only load of `part` (which may be moved before the
    wait, and is for what stays constant while a kernel runs)."""
    found = 0
    for name, params, body in kernels(os.path.join(CSRC, source)):
        if "const float *part" not in params:
            continue
        found += 1
        assert "wait_for_previous();" in body, name
        assert body.index("wait_for_previous();") < body.index("part"), name
        names = {"part"} | set(re.findall(r"\*\s*(\w+)\s*=\s*[^;]*\bpart\b", body))
        for arg in re.findall(r"__ldg\(([^;]*?)\)", body):
            assert not names & set(re.findall(r"\w+", arg)), (name, arg)
    assert found == 1


def test_the_package_imports_with_a_torch_without_cuda():
    """Workspace sizes and refusals need the library, not torch's CUDA bindings."""
    code = ("import torch\n"
            "for name in ('_cuda_getCurrentRawStream', '_cuda_getDevice'):\n"
            "    if hasattr(torch._C, name): delattr(torch._C, name)\n"
            "import paper_2609_00049_gb300 as rq\n"
            "from paper_2609_00049_gb300 import block, build, head, layer\n"
            "build.build()\n"
            "assert rq.realq_int8_product_workspace_size(8, 8, 8) > 0\n")
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)
