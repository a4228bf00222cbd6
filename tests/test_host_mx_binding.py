"""CPU-only checks of the block-scaled calls' binding: what a refused call leaves behind, and the module that the calls go through."""
import ctypes as C
import os
import subprocess
import sys
from types import SimpleNamespace

import pytest
import torch

import paper_2501_17116_b200 as fp4
from paper_2501_17116_b200 import build as fp4_build
from paper_2501_17116_b200 import mx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    fp4_build.build()
    return fp4.load_library()


@pytest.fixture
def ctx(lib, monkeypatch):
    """A context by its outside, on torch's number for the CPU: calls reach the checks of their matrices and end there."""
    monkeypatch.setattr(mx, "_stream_of", lambda device: 0)
    return SimpleNamespace(lib=lib, handle=C.c_void_p(0x10000), device=-1, status=torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("flags", [0, mx.FP4_MX_AMAX_GIVEN])
@pytest.mark.parametrize("bad", [torch.zeros(4, 63), torch.zeros(5, 64), torch.zeros(4, 64, dtype=torch.float64), torch.zeros(64, 4).t(), torch.zeros(4, 64)])
def test_a_refused_quantisation_leaves_the_operand_as_it_was(ctx, bad, flags):
    """Shape, type, stride and device of the matrix: the call ends with an exception, and a later one finds neither flag nor amax of it."""
    q = fp4.MXTensor(4, 64, "cpu", fp4.FP4_MX_NVFP4)
    q.amax.fill_(3.0)
    q.struct.flags = flags
    before = bytes(q.struct)
    with pytest.raises(AssertionError):
        fp4.fp4_mx_quantize(ctx, bad, fp4.FP4_MX_NVFP4, out=q, amax=torch.tensor([0.25]))
    assert bytes(q.struct) == before and float(q.amax) == 3.0


def test_an_operand_of_another_device_is_refused_ahead_of_its_amax(ctx):
    q = fp4.MXTensor(4, 64, "cpu", fp4.FP4_MX_NVFP4)
    ctx.device = 0
    with pytest.raises(AssertionError, match="device"):
        fp4.fp4_mx_quantize(ctx, torch.zeros(4, 64), fp4.FP4_MX_NVFP4, out=q, amax=torch.tensor([0.25]))
    assert q.struct.flags == 0 and float(q.amax) == 0.0


@pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would run on made-up addresses")
def test_a_backward_pass_needs_only_the_operand_it_reads(lib):
    """A frozen layer has nothing for dW.  (The stand-in of a context has no workspace, which is asked for behind all checks of operands.)"""
    M, K, N, P, null, workspace = 8, 64, 32, 0x10000, -1, -5
    buf = C.create_string_buffer(8192)
    ctx, mat = C.cast(buf, C.c_void_p), lambda ld: mx.fp4_mx_matrix(P, ld, 0, 0)                  # noqa: E731
    sx, sw = mx.fp4_mx_tensor(M, K, None, None, P, P, None, 0, 0), mx.fp4_mx_tensor(K, N, P, P, None, None, None, 0, 0)
    ref = lambda o: None if o is None else C.byref(o)                                         # noqa: E731
    call = lambda x, w, dx, dw: lib.fp4_mx_linear_bwd(ctx, None, ref(mat(N)), ref(x), ref(w), M, K, N, 0, ref(dx), ref(dw), P)   # noqa: E731
    assert call(None, sw, mat(K), None) == workspace and call(sx, None, None, mat(N)) == workspace
    assert call(None, sw, mat(K), mat(N)) == null and call(sx, None, mat(K), mat(N)) == null
    assert call(None, sw, None, mat(N)) == null and call(sx, None, mat(K), None) == null
    assert call(None, None, None, None) == 0


def fresh(code):
    """Standard output of `code` in an interpreter of its own."""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr
    return done.stdout.split()


def test_the_library_loads_without_the_module_of_the_block_scaled_calls(lib):
    """It takes torch's headers and the interpreter's to build, and nothing else of the package needs it."""
    assert fresh("""
import sys
sys.modules["paper_2501_17116_b200._mx_call"] = None                  # importing it fails
import paper_2501_17116_b200 as fp4
lib = fp4.load_library()
print(lib.fp4_workspace_bytes(128, 128, 128) > 0, lib.fp4_mx_pitch(129, 0))
try:
    fp4.mx._call.quantize
except ImportError:
    print("refused")
""") == ["True", "128", "refused"]


def test_the_module_is_loaded_at_the_first_call_and_kept(lib):
    assert fresh("""
import sys
import paper_2501_17116_b200 as fp4
fp4.load_library()
name = "paper_2501_17116_b200._mx_call"
print(name in sys.modules)
first = fp4.mx._call.gemm
print(name in sys.modules, first is fp4.mx._call.gemm, sorted(vars(fp4.mx._call)) == sorted(fp4.mx.ENTRIES))
""") == ["False", "True", "True", "True"]


def test_the_module_is_of_this_torch_and_this_interpreter(lib):
    """One that another torch's headers were read for would misread tensors: its name is another, and it is built anew."""
    assert os.path.exists(fp4_build.call_path()) and not fp4_build.needs_build()
    assert fresh("""
import torch
from paper_2501_17116_b200 import build
import paper_2501_17116_b200 as fp4
fp4.load_library()
mine = build.call_path()
torch.__version__ = "0.0.1"
print(build.call_path() != mine, build.needs_build())
try:
    fp4.mx._call.gemm
except ImportError as e:
    print("build" in str(e))
""") == ["True", "True", "True"]


def test_kernels_that_start_early_read_no_memory_as_constant():
    """They are there before the kernel ahead of them has written what they read: non-coherent loads (which promise that nothing changes while the
    kernel runs, may be served by a line from before, and may be moved ahead of the wait) have no place in them."""
    csrc, seen = fp4_build.CSRC, 0
    for name in sorted(os.listdir(csrc)):
        if name.startswith("mx") and name.endswith((".cu", ".cuh")):
            with open(os.path.join(csrc, name)) as f:
                text = f.read()
            seen += "mx_wait_for_inputs();" in text
            assert not [w for w in ("__ldg", ".nc.", "__restrict__", "__ldcs") if w in text], name
    assert seen >= 2
