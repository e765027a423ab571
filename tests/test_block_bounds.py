"""Which addresses the kernels of a client's own layers may touch: their index arithmetic, compiled for the host and walked there."""
import os
import shutil
import subprocess

import pytest

from paper_1805_08768_b200 import build

NORM_WALK = r"""
#include <stdio.h>
#include "lm_norm.cuh"

// A row is loaded as the forward kernel of layer norm does it: granules of eight elements from the 16-byte boundary in front of
// it. Where the rule lets granules be loaded whole, all of their elements have to be the matrix's or lie between its rows.
static long long walk(int width) {
    long long whole = 0;
    const int each = 16 / width;
    for (int cols = 1; cols <= 40; ++cols)
        for (int stride = cols; stride <= cols + 9; ++stride)
            for (int rows = 1; rows <= 12; ++rows)
                for (int begin = 0; begin < each; ++begin)      // where the matrix begins behind a 16-byte boundary
                    for (long long r = 0; r < rows; ++r) {
                        const int phase = (int)((begin + r * stride) % each), n = (cols + phase + 7) / 8;
                        const bool ends = (phase | (cols & 7)) != 0;
                        if (!sbclm::whole_granules_within(r, rows, cols, ends)) continue;
                        ++whole;
                        const long long first = r * stride - phase, last = first + 8ll * n - 1, all = (rows - 1ll) * stride + cols;
                        if (first < 0 || last >= all) {
                            printf("width %d, %d x %d, stride %d, begin %d, row %lld: elements %lld .. %lld of %lld\n", width, rows, cols, stride, begin, r, first, last, all);
                            return -1;
                        }
                    }
    return whole;
}

int main() {
    const long long halves = walk(2), words = walk(4);
    printf("%lld %lld\n", halves, words);
    return halves > 0 && words > 0 ? 0 : 1;   // (and the rule is of use)
}
"""


@pytest.mark.skipif(not (shutil.which("nvcc") or os.path.exists("/usr/local/cuda/bin/nvcc")), reason="needs nvcc")
def test_layer_norm_loads_within_the_matrix(tmp_path):
    source, program = tmp_path / "walk.cu", tmp_path / "walk"
    source.write_text(NORM_WALK)
    made = subprocess.run([build._nvcc(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-o", str(program), str(source)],
                          capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    ran = subprocess.run([str(program)], capture_output=True, text=True, timeout=300)
    assert ran.returncode == 0, ran.stdout + ran.stderr
