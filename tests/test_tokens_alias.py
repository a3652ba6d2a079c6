"""A result may lie over an input, and a row's tokens are read as words and written as words
or elements: the compiler may take none of these accesses for apart by their types."""
import os
import subprocess

import pytest

from paper_2104_05035_amd import build

KERNELS = """
#include "tokens.hpp"
using namespace rat3d;
// read, written through another pointer, read again
#define KERNEL(NAME, T, TOK, ALL)                                                      \\
    extern "C" __global__ void NAME(const T* z, T* to, T* out, int left, bool past) {  \\
        Toks<T, TOK> a, b;                                                             \\
        float o[TOK];                                                                  \\
        a.load(z, 16 * threadIdx.x);                                                   \\
        for (int j = 0; j < TOK; ++j) o[j] = a[j] + 1.f;                               \\
        put_tokens<T, TOK, ALL>(to, 16 * threadIdx.x, left, o, past);                  \\
        b.load(z, 16 * threadIdx.x);                                                   \\
        for (int j = 0; j < TOK; ++j) o[j] = b[j] - a[j];                              \\
        put_tokens<T, TOK, ALL>(out, 16 * threadIdx.x, left, o, past);                 \\
    }                                                                                  \\
    extern "C" __global__ void NAME##_elt(T* z, T* out) {                              \\
        Toks<T, TOK> a, b;                                                             \\
        float o[TOK];                                                                  \\
        a.load(z, 16 * threadIdx.x);                                                   \\
        out[threadIdx.x] = 0;                                                          \\
        b.load(z, 16 * threadIdx.x);                                                   \\
        for (int j = 0; j < TOK; ++j) o[j] = b[j] - a[j];                              \\
        put_tokens<T, TOK, true>(z, 16 * threadIdx.x, TOK, o, false);                  \\
    }
KERNEL(bf16_whole, bf16, 8, true)
KERNEL(bf16_ragged, bf16, 8, false)
KERNEL(bf16_half, bf16, 4, false)
KERNEL(bf16_one, bf16, 1, false)
KERNEL(float_whole, float, 4, true)
KERNEL(float_ragged, float, 4, false)
KERNEL(float_one, float, 1, false)
"""


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
def test_types_say_nothing_about_overlap(tmp_path):
    """The code is the one without assumptions from types."""
    src = tmp_path / "alias.hip"
    src.write_text(KERNELS)
    code = []
    for flag in ("-fstrict-aliasing", "-fno-strict-aliasing"):
        out = tmp_path / (flag + ".s")
        subprocess.run([build.HIPCC] + build.FLAGS + [flag, "-cuid=alias", "--offload-device-only",
                                                      "-S", "-x", "hip", str(src), "-o", str(out)],
                       check=True, capture_output=True, timeout=300)
        code.append(out.read_text())
    assert "bf16_ragged_elt" in code[0]
    assert code[0] == code[1]
