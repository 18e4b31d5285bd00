"""Host arithmetic of the operators over the vocabulary at the edges of their documented range, without a GPU."""
import os
import shutil
import subprocess

import pytest

from paper_1909_00562_amd import binding as bd

CSRC = os.path.join(os.path.dirname(bd.library_path()), "csrc")

ROW_THREADS_MAIN = """
#include "row_threads.h"
int main() {
  auto expect = [](bool ok) { if (!ok) __builtin_trap(); };
  for (int64_t rows = 1; rows <= 1 << 24; rows = rows < 1000 ? rows + 1 : rows * 2 - 7)
    for (int64_t vecs = 1; vecs <= 1 << 16; vecs = vecs * 3 / 2 + 1) {
      const int b = asx::row_threads_log(rows, vecs);
      expect(b >= 0 && b <= 8 && (b == 0 || (1 << (b - 1)) < vecs));                   // no more than its vectors
      expect((((rows << b) + 255) / 256) * 256 <= (int64_t)1 << 31);
      if (rows <= 1 << 23) expect(b == 8 || (1 << b) >= vecs);                         // and no fewer
    }
  const int64_t most = 1 << 24;
  expect(asx::row_threads_log(most, 1 << 14) == 7 && asx::row_threads_log(most, 130) == 7 && asx::row_threads_log(most, 128) == 7);
  expect(asx::row_threads_log(most, 5) == 3 && asx::row_threads_log(1 << 23, 130) == 8);
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_threads_of_the_most_rows_fit_a_launch(tmp_path):
    """2^24 rows of 256 threads are 2^32, one more than a launch takes along a dimension."""
    (tmp_path / "main.cpp").write_text(ROW_THREADS_MAIN)
    exe = tmp_path / "main"
    subprocess.run(["g++", "-std=c++17", f"-I{CSRC}", str(tmp_path / "main.cpp"), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)
    # and the launchers that walk rows go by it
    for name, calls in (("embed.hip", 2), ("vocab_kernels.hip", 2)):
        text = open(os.path.join(CSRC, name)).read()
        assert text.count("row_threads_log(") == calls and "threads_log(" not in text.replace("row_threads_log(", ""), name


HIP_STUB = """
#pragma once
#include <stddef.h>
#define __host__
#define __device__
enum hipError_t { hipSuccess = 0 };
typedef void* hipStream_t;
"""
SCALE_MAIN = """
#include "gemm.h"
int main() {
  auto expect = [](bool ok) { if (!ok) __builtin_trap(); };
  asx::GemmArgs g;
  expect(asx::gemm_kernel_scale(g) == 1.f);
  g.alpha = 0.25f;
  expect(asx::gemm_kernel_scale(g) == 0.25f);
  g.splits = 4;
  expect(asx::gemm_kernel_scale(g) == 0.25f);
  g.alpha = 1.f;                                  // dropout, in the kernel or by a split's combine
  g.drop_thr = 1u << 30;
  g.drop_scale = 4.f / 3.f;
  expect(asx::gemm_kernel_scale(g) == 1.f);
  g.splits = 1;
  expect(asx::gemm_kernel_scale(g) == 4.f / 3.f);
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_dropout_of_a_split_product_scales_once(tmp_path):
    """The partial sums of a split keep their size where the combine drops and scales elements."""
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text(HIP_STUB)
    (tmp_path / "main.cpp").write_text(SCALE_MAIN)
    exe = tmp_path / "main"
    subprocess.run(["g++", "-std=c++17", f"-I{tmp_path}", f"-I{CSRC}", str(tmp_path / "main.cpp"), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)
    assert "d.drop_scale = gemm_kernel_scale(g);" in open(os.path.join(CSRC, "gemm_bf16.hip")).read()


A = [0x10000 * (i + 1) for i in range(16)]     # addresses that are never read: the checks come first


@pytest.mark.parametrize("tau, taken", [(2.0 ** -10, True), (2.0 ** -10 * (1 - 2.0 ** -24), False), (1e-9, False), (1e-30, False), (-1.0, False)])
def test_temperatures_below_which_probabilities_overflow(tau, taken):
    s, t = bd.VoShape(5, 16, 100, 0, bd.AS_BF16, bd.AS_F32, 1.0), bd.VoTeacher(4, tau, 1.0)
    assert (bd.vocab_xent_workspace_bytes(s, t) > 0) == taken
    code = 4 if taken else 2                   # (a workspace of no bytes, or the teacher)
    assert bd.vocab_distill_fwd(s, t, *A[:12], 0, check=False) == code
    assert bd.vocab_distill_bwd(s, t, A[0], A[1], A[2], 0, A[3], A[4], A[5], check=False) == code
