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
    text = re.sub(r"//[^\n]*|__launch_bounds__\([^)]*\)", "", open(path).read())
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


# (raw sum, sum of x, middle code, zero point) of n equal columns x, c
LONGEST = [(131071, x, c, z, 128) for x in (-128, 127) for c in (0, 255) for z in (0, 128, 255)] + \
          [(131071, x, c, z, 8) for x in (-128, 127) for c in (0, 15) for z in (0, 15, 255)]


def test_integer_sums_stay_within_defined_arithmetic(tmp_path):
    """The whole-number arithmetic of the longest sums, evaluated by the compiler,
    which refuses a signed overflow in a constant; the plain signed form of the
    same sums is refused."""
    lines = ['#include "code_sums.cuh"', "using namespace realq;",
             "constexpr uint32_t raw(int n, int x, int c) { uint32_t a = 0;"
             " for (int j = 0; j < 8; ++j) a = add_share(a, (n / 8) * x * c);"
             " return add_share(a, (n % 8) * x * c); }"]
    for n, x, c, z, mid in LONGEST:
        lines.append(f"static_assert(centred_sum(raw({n}, {x}, {c}), {n * x}, {mid}, {z}) == {n * x * (c - z)}ll);")
    # shares as the warps have them add up past 32 bits
    signed = ("constexpr int32_t plain(int n, int x, int c) { int32_t a = 0;"
              " for (int j = 0; j < 8; ++j) a += (n / 8) * x * c; return a; }\n"
              "static_assert(plain(131071, -128, 255) != 1);")

    def compiles(text):
        f = tmp_path / "sums.cpp"
        f.write_text(text + "\n")
        return subprocess.run(["g++", "-std=c++17", "-fsyntax-only", f"-I{CSRC}", str(f)], capture_output=True).returncode == 0

    assert not compiles("\n".join(lines + [signed]))
    assert compiles("\n".join(lines))
    kernel = dict((n, b) for n, _, b in kernels(os.path.join(CSRC, "int8_product.cu")))["int8_stream_kernel"]
    assert not re.search(r"\bint\s+(\*?\s*)?(red|xred)\b", kernel) and "centred_sum(" in kernel


INVALID = 1


def test_side_arrays_off_their_types_alignment_are_refused():
    """Scales, log probabilities, targets and the other arrays beside the large
    ones: an address that their element type cannot have comes back as a status."""
    import ctypes
    from paper_2609_00049_gb300 import build as b
    b.build()
    import paper_2609_00049_gb300 as rq
    L = rq.lib()
    ok, odd, odd8 = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10002), ctypes.c_void_p(0x10004)   # never dereferenced

    def product(xs=ok, ws=ok):
        return L.realq_int8_product(None, 4, 64, 32, ok, xs, ok, 8, ws, None, ok, 1, ok, 1 << 40)
    for bad in (dict(xs=odd), dict(ws=odd)):
        assert product(**bad) == INVALID, bad

    def logprobs(y=ok, lp=ok, norm=ok, H=ok, ids=ok, top=ok):
        return L.realq_token_logprobs(None, 4, 100, 100, ok, 1, y, lp, norm, H, 2, ids, top)
    for bad in (dict(y=odd8), dict(ids=odd8), dict(lp=odd), dict(norm=odd), dict(H=odd), dict(top=odd)):
        assert logprobs(**bad) == INVALID, bad

    def grad(y=ok, norm=ok, g=ok, H=ok, gH=ok, ids=ok, gt=ok):
        return L.realq_token_logprobs_grad(None, 4, 100, 100, ok, 1, y, norm, g, H, gH, 2, ids, gt, 100, ctypes.c_void_p(0x20000))
    for bad in (dict(y=odd8), dict(ids=odd8), dict(norm=odd), dict(g=odd), dict(H=odd), dict(gH=odd), dict(gt=odd)):
        assert grad(**bad) == INVALID, bad

    assert L.realq_checkpoint_weight_grad(None, 4, 8, 64, ok, 1, ok, ok, odd, 0, ok, 1 << 40) == INVALID


def test_quantizing_no_tokens_is_no_work():
    """An empty matrix has no address: T = 0 is a no-op, not a refusal."""
    import ctypes
    from paper_2609_00049_gb300 import build as b
    b.build()
    import paper_2609_00049_gb300 as rq
    L, ok = rq.lib(), ctypes.c_void_p(0x10000)
    assert L.realq_quantize_activations(None, 0, 64, None, 1, 8, 1.0, None, None, None) == 0
    assert L.realq_quantize_activations(None, 4, 64, None, 1, 8, 1.0, ok, None, None) == INVALID
    assert L.realq_quantize_activations(None, 4, 64, ok, 1, 8, 1.0, None, None, None) == INVALID
    assert L.realq_quantize_activations(None, 0, 64, None, 1, 9, 1.0, None, None, None) == INVALID
