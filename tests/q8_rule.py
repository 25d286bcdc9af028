"""The rule that picks the decoding kernel over the 8-bit cache, compiled for the host from the kernels' own header (test
infrastructure: it says which kernel a case reaches)."""
import ctypes
import os
import subprocess
import tempfile

from paper_2607_08186_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_lib = None


def tensor_cores(B, n, Hq, Hkv, Dh, P, tokens, mode=1, window=0):
    """Whether a step of at most `tokens` tokens is the tcgen05 kernel's, and not the mma.sync kernel's."""
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "rule.cu"), os.path.join(d, "rule.so")
            with open(src, "w") as f:
                f.write('#include "%s/paper_2607_08186_gb300/csrc/decode_plan.cuh"\n'
                        'extern "C" int kernel(int B, int n, int Hq, int Hkv, int Dh, int prow, int tokens, int mode, int window) {\n'
                        '  return hdsfa::q8_tc(Dh, prow, n * (Hq / Hkv), hdsfa::q8_range(tokens, n, mode, window), (long long)B * Hkv); }\n'
                        % ROOT)
            subprocess.run([build.nvcc(), "-std=c++17", "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-shared",
                            *build.ARCH, src, "-o", so], check=True, capture_output=True)
            _lib = ctypes.CDLL(so)
    return bool(_lib.kernel(B, n, Hq, Hkv, Dh, P * n, tokens, mode, window))
