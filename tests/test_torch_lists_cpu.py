"""Native readers of tensors (csrc/torch_lists.cpp) on a host without a GPU: the file is compiled with its test for a CUDA
device left out, so that tensors in host memory reach what stands behind it, and with entry points that do nothing.  Every
argument ends in a result, None (left to the binding's own checks) or a Python exception, never in the end of the process."""
import os
import shutil
import subprocess
import sys
import sysconfig

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import ctypes as C, importlib.util, sys, warnings
import torch
warnings.simplefilter("ignore")
spec = importlib.util.spec_from_file_location("_torch_lists", sys.argv[1])
L = importlib.util.module_from_spec(spec)
spec.loader.exec_module(L)
calls = []
quant = C.CFUNCTYPE(C.c_int, *[C.c_void_p] * 7)(lambda *a: calls.append(a) or 0)
gemm = C.CFUNCTYPE(C.c_int, *[C.c_void_p] * 7, C.c_size_t, C.c_void_p)(lambda *a: calls.append(a) or 0)
size = C.CFUNCTYPE(C.c_size_t, C.c_void_p)(lambda c: 0)
at = lambda f: C.cast(f, C.c_void_p).value
E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
x = torch.randn(4, 512)
codes, scales = torch.zeros(4, 512, dtype=torch.uint8).view(E4), torch.zeros(4, 4, dtype=torch.uint8).view(E8)
odd = {
    "strided": x, "csr": x.to_sparse_csr(), "csc": x.to_sparse_csc(), "bsr": x.to_sparse_bsr((2, 2)), "coo": x.to_sparse(),
    "nested": torch.nested.nested_tensor([x[:1], x[1:]]), "jagged": torch.nested.nested_tensor([x[:1], x[1:]], layout=torch.jagged),
    "meta": x.to("meta"), "mkldnn": x.to_mkldnn() if torch.backends.mkldnn.is_available() else x[0], "none": None, "text": "x",
    "scalar": torch.tensor(1.0), "empty": x[:0], "transposed": x.t(), "expanded": x[:1].expand(4, 512), "double": x.double(),
}
q = lambda t: L.quantize_fp8(at(quant), t, 0, 1, True, True, 0, -1)
g = lambda a, sa, b, sb, out=None: L.gemm_fp8(at(gemm), at(size), a, sa, b, sb, out, True, False, 0, -1)
places = {
    "quantize": q, "a": lambda t: g(t, scales, codes, scales), "a_scale": lambda t: g(codes, t, codes, scales), "b": lambda t: g(codes, scales, t, scales),
    "b_scale": lambda t: g(codes, scales, codes, t), "out": lambda t: g(codes, scales, codes, scales, t),
    "param": lambda t: L.adamw_entries([dict(param=t, grad=x, m=x, v=x)], -1, bytearray(80)),
    "grad": lambda t: L.adamw_entries([dict(param=x, grad=t, m=x, v=x)], -1, bytearray(80))}
for place, f in places.items():
    for name, t in odd.items():
        print(place, name, end=" ", flush=True)
        calls.clear()
        try:
            r = f(t)
            print(type(r).__name__ if not isinstance(r, int) else r, len(calls), flush=True)
        except Exception as e:
            print(type(e).__name__, len(calls), flush=True)
unclear = torch.zeros(2, dtype=torch.bool)  # neither true nor false
flags = {"rows": lambda: L.quantize_fp8(at(quant), x, 0, 1, unclear, True, 0, -1), "transposed": lambda: L.quantize_fp8(at(quant), x, 0, 1, True, unclear, 0, -1),
         "block_rows": lambda: L.quantize_fp8(at(quant), x, 0, 1.5, True, True, 0, -1), "float32": lambda: L.gemm_fp8(at(gemm), at(size), codes, scales, codes, scales, None, unclear, False, 0, -1),
         "accumulate": lambda: L.gemm_fp8(at(gemm), at(size), codes, scales, codes, scales, torch.zeros(4, 4), True, unclear, 0, -1)}
for name, f in flags.items():
    print("flag", name, end=" ", flush=True)
    calls.clear()
    try:
        print(type(f()).__name__, len(calls), flush=True)
    except Exception as e:
        print(type(e).__name__, len(calls), flush=True)
"""


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("lists")
    src = open(os.path.join(ROOT, "paper_2203_17189_amd", "csrc", "torch_lists.cpp")).read()
    left_out = src.replace("t.is_cuda() && ", "").replace("!t.is_cuda() || ", "")
    assert left_out != src and "is_cuda" not in left_out
    (tmp / "torch_lists.cpp").write_text(left_out.replace("../../include", os.path.join(ROOT, "include")))
    (tmp / "program.py").write_text(PROGRAM)
    out = tmp / ("_torch_lists" + sysconfig.get_config_var("EXT_SUFFIX"))
    root = os.path.dirname(torch.__file__)
    inc = [sysconfig.get_paths()["include"], os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include")]
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    *[f"-I{i}" for i in inc], str(tmp / "torch_lists.cpp"), "-o", str(out), f"-L{root}/lib", "-ltorch_python", "-ltorch_cpu",
                    "-lc10", f"-Wl,-rpath,{root}/lib"], check=True)
    return tmp, out


@pytest.fixture(scope="module")
def answers(module):
    r = subprocess.run([sys.executable, str(module[0] / "program.py"), str(module[1])], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stdout.splitlines()[-1:], r.stderr[-2000:])  # (its last line names the call)
    return {tuple(line.split()[:2]): line.split()[2:] for line in r.stdout.splitlines()}


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_no_argument_ends_the_process(answers):
    got = answers
    assert len(got) == 8 * 16 + 5
    assert got["quantize", "strided"] == ["tuple", "1"] and got["out", "none"] == ["Tensor", "1"]
    assert got["param", "strided"] == got["grad", "strided"] == ["1", "0"]  # entries read
    # what has no strides, or has the wrong ones, is left to the checks of the binding: no entry point was called for it
    wrong = ("csr", "csc", "bsr", "coo", "nested", "jagged", "none", "text", "scalar", "transposed", "expanded", "double")
    for name in wrong:
        for place in ("quantize", "a", "a_scale", "b", "b_scale", "out"):
            assert got[place, name] == ["NoneType", "0"] or (place, name) == ("out", "none"), (place, name, got[place, name])
        for place in ("param", "grad"):
            assert got[place, name] == ["0", "0"], (place, name, got[place, name])


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_flags_that_are_neither_true_nor_false_call_nothing(answers):
    for name in ("rows", "transposed", "block_rows", "float32", "accumulate"):
        assert answers["flag", name] == ["NoneType", "0"], (name, answers["flag", name])
