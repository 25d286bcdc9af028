"""The rule that picks the paged decoding kernel, compiled for the host from the kernels' own header (test
infrastructure: it says which kernel a case reaches)."""
import ctypes
import os
import subprocess
import tempfile

from paper_2607_08186_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NONE, ONLY_256, WITH_128 = 0, 1, 2
_lib = None


def lib():
    """.piece(prow, most); .kernel(B, n, Hq, Hkv, Dh, prow, range)."""
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "rule.cu"), os.path.join(d, "rule.so")
            with open(src, "w") as f:
                f.write('#include "%s/paper_2607_08186_gb300/csrc/decode_plan.cuh"\n'
                        'extern "C" int piece(int prow, int most) { return hdsfa::paged_piece(prow, most); }\n'
                        'extern "C" int kernel(int B, int n, int Hq, int Hkv, int Dh, int prow, int range) {\n'
                        '  return (int)hdsfa::paged_tc(B, n, Hq, Hkv, Dh, hdsfa::paged_piece(prow, 128), range); }\n' % ROOT)
            subprocess.run([build.nvcc(), "-std=c++17", "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-shared",
                            *build.ARCH, src, "-o", so], check=True, capture_output=True)
            _lib = ctypes.CDLL(so)
    return _lib


def tensor_cores(B, n, Hq, Hkv, Dh, P, tokens, window=0):
    """Whether a step of at most `tokens` tokens (LOCAL: a window) is the tcgen05 kernel's."""
    M, reach = n * (Hq // Hkv), tokens * n if not window else min(tokens * n, window + n - 1)
    dims = lib().kernel(B, n, Hq, Hkv, Dh, P * n, reach)
    return M <= 128 and (Dh == 256 and dims != NONE or Dh == 128 and dims == WITH_128 and M > 32)
