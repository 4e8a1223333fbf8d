"""The operators around the cache as the library exports them: layout of their structure and refusals that need no GPU."""
import ctypes
import os
import subprocess

import pytest

from paper_2512_10310_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    B.build_library()
    return B.lib()


def test_head_norm_is_laid_out_as_the_header_says(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "evln.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu\\n", sizeof(evlnHeadNorm), offsetof(evlnHeadNorm, q_weight), '
                   'offsetof(evlnHeadNorm, k_weight), offsetof(evlnHeadNorm, eps)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    size, q, k, eps = map(int, subprocess.check_output([str(exe)]).split())
    f = B.evlnHeadNorm
    assert (ctypes.sizeof(f), f.q_weight.offset, f.k_weight.offset, f.eps.offset) == (size, q, k, eps)


def test_null_handles_are_rejected(lib):
    step, paged, gather = B.step_params("bf16", 28, 4, 128, 5, 1, 8, 1e6), B.paged_params(28, 4, 128, 1, 64, 4, 2, 1e6), B.gather_params("bf16", 4, 128, 16, 8, 1e6)
    norm = B.evlnHeadNorm(ctypes.sizeof(B.evlnHeadNorm), None, None, 1e-6)
    lens, offs, size = (ctypes.c_int * 1)(5), (ctypes.c_int * 2)(0, 1), ctypes.c_size_t(0)
    at = ctypes.byref
    none, strides = None, (28 * 128, 4 * 128, 4 * 128)
    assert lib.evlnNormRopeAppend(none, at(step), at(norm), *[none] * 3, *strides, *[none] * 4) == B.EVLN_INVALID_VALUE
    assert lib.evlnPagedNormRopeAppend(none, at(paged), at(norm), *[none] * 3, *strides, lens, offs, *[none] * 5) == B.EVLN_INVALID_VALUE
    assert lib.evlnPaged8RopeAppend(none, at(paged), at(norm), *[none] * 3, *strides, lens, offs, *[none] * 7) == B.EVLN_INVALID_VALUE
    assert lib.evlnPaged8WorkspaceSize(none, at(paged), lens, offs, at(size)) == B.EVLN_INVALID_VALUE
    assert lib.evlnPaged8StepAttention(none, at(paged), *[none] * 5, lens, offs, none, none, 0, *[none] * 3) == B.EVLN_INVALID_VALUE
    assert lib.evlnKeyWeights(none, at(step), *[none] * 3, 1.0, *[none] * 3) == B.EVLN_INVALID_VALUE
    assert lib.evlnSelectKeys(none, at(gather), none, 16, 8, 0, 0, none, none) == B.EVLN_INVALID_VALUE
    assert lib.evlnGatherKeys(none, at(gather), 4, *[none] * 7, 0, none) == B.EVLN_INVALID_VALUE
