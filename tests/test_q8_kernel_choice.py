"""Which kernel decodes over the 8-bit cache (no GPU): the rule's borders, and that the cases of the GPU tests that are made for
one kernel are its."""
import ctypes
import os
import random
import subprocess
import tempfile

import pytest

import q8_kernels
import q8_rule
from paper_2607_08186_gb300 import build, inputs


@pytest.mark.parametrize("c", q8_kernels.CHANGE + q8_kernels.WAVE)
def test_cases_for_the_tensor_cores(c):
    B, n, Hq, Hkv, Dh, P, T, L = c
    for mode, w in ((inputs.CROSS, 0), (inputs.WITHIN, 0)) + (((inputs.LOCAL, 150),) if n * Hq // Hkv > 16 else ()):
        assert q8_rule.tensor_cores(B, n, Hq, Hkv, Dh, P, L, mode, w)


@pytest.mark.parametrize("c", q8_kernels.SIZES)
def test_cases_of_sizes(c):
    kernel, n, Hq, Hkv, Dh, P, T, L = c
    assert q8_rule.tensor_cores(1, n, Hq, Hkv, Dh, P, L) == kernel


@pytest.mark.parametrize("c", q8_kernels.GIVEN_UP)
def test_cases_of_given_up_pages(c):
    kernel, n, Hq, Hkv, Dh, P, T, L, w = c
    assert q8_rule.tensor_cores(3, n, Hq, Hkv, Dh, P, L, inputs.LOCAL, w) == kernel


def test_borders():
    tc = q8_rule.tensor_cores
    # pieces that TMA cannot bring are never for the tensor cores
    for Dh in (64, 128, 256):
        assert not tc(4, 4, 96, 8, Dh, 1, 8192) and not tc(4, 1, 96, 1, Dh, 131, 8192) and tc(4, 4, 96, 8, Dh, 2, 8192)
    assert not tc(4, 1, 96, 1, 64, 9, 8192) and tc(4, 1, 96, 1, 128, 9, 8192)  # odd pieces of 64 bytes a row
    # up to 16 query rows leave it the long ranges, by the window where there is one
    assert tc(1, 4, 32, 8, 128, 16, 17) and not tc(1, 4, 32, 8, 128, 16, 16)
    assert tc(1, 1, 24, 2, 256, 16, 513) and not tc(1, 1, 24, 2, 256, 16, 512)
    assert tc(33, 3, 16, 4, 64, 20, 2648) and not tc(33, 3, 16, 4, 64, 20, 2647)
    assert not tc(1, 4, 32, 8, 128, 16, 8192, inputs.LOCAL, 61) and tc(1, 4, 32, 8, 128, 16, 8192, inputs.LOCAL, 62)
    assert tc(1, 1, 17, 1, 64, 16, 1) and tc(1, 4, 24, 2, 256, 16, 1)  # more than 16 rows: all of them


@pytest.fixture(scope="module")
def wave():
    """The parts of a shared wave, by the kernels' own header."""
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "wave.cu"), os.path.join(d, "wave.so")
        with open(src, "w") as f:
            f.write('#include "%s/paper_2607_08186_gb300/csrc/decode_plan.cuh"\nusing hdsfa::WaveParts;\n'
                    'extern "C" int parts(unsigned all, unsigned most, unsigned total, unsigned split) {\n'
                    '  return (int)WaveParts(all, most, total, split).S; }\n'
                    'extern "C" void begins(unsigned all, unsigned most, unsigned total, unsigned split, unsigned* out) {\n'
                    '  const WaveParts w(all, most, total, split); for (unsigned x = 0; x <= w.S; ++x) out[x] = w.begin(x); }\n'
                    'extern "C" int of(unsigned all, unsigned most, unsigned total, unsigned split, unsigned u) {\n'
                    '  return WaveParts(all, most, total, split).of(u); }\n' % q8_rule.ROOT)
        subprocess.run([build.nvcc(), "-std=c++17", "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-shared",
                        *build.ARCH, src, "-o", so], check=True, capture_output=True)
        return ctypes.CDLL(so)


def test_parts_of_a_wave(wave):
    """Parts cover all units in order, none empty, and no sequence is in more than 128; a unit's part is the one that has it."""
    r = random.Random(9)
    for _ in range(300):
        sizes = [0 if r.random() < 0.2 else 6 + r.choice([r.randint(1, 5), r.randint(1, 3000), 8000000]) for _ in range(r.randint(1, 128))]
        every, most, total = sum(sizes), max(sizes), r.choice([1, 2, 9, 19, 76, 152, 228, 456])
        args = (every, most, total, 128)
        S = wave.parts(*args)
        assert 1 <= S <= max(1, min(total, every))
        if not every:
            continue
        out = (ctypes.c_uint * (S + 1))()
        wave.begins(*args, out)
        begins = list(out)
        assert begins[0] == 0 and begins[-1] == every and all(a < b for a, b in zip(begins, begins[1:]))
        assert begins == [x * every // S for x in range(S + 1)]
        for u in [0, every - 1] + [r.randrange(every) for _ in range(20)] + [b + d for b in begins[1:-1][:20] for d in (-1, 0)]:
            x = wave.of(*args, u)
            assert begins[x] <= u < begins[x + 1]
        before = 0
        for size in sizes:
            if size:
                assert wave.of(*args, before + size - 1) - wave.of(*args, before) + 1 <= 128
            before += size
