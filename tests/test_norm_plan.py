"""The plans of the GroupNorm kernels, on the CPU: a small program of the library's own headers goes over sizes, and over the threads of a CTA."""
import os
import subprocess

import pytest

from paper_2512_15773_b200 import build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "group_norm_plan.cuh"
using namespace tsdp;

// What the threads of a CTA write to the words of a group's sum, and what they read (group_sum): every word that is read has to be one that was written, and
// lies within `room`.  everybody: also the threads without a column.
static int bad_reads(const NormArgs& g, int V, int width, int K, bool everybody) {
  const int gcols = g.C / g.groups / V, per = g.cols / g.fold, room = K * GN_THREADS;
  const bool rows_in_warp = g.cols < 32 && (g.cols & (g.cols - 1)) == 0;
  std::vector<char> written(4 * room + 65536, 0);
  int bad = 0;
  for (int t = 0; t < GN_THREADS; ++t) {
    const int lane = t / g.cols, col = t % g.cols, r = rows_in_warp ? t / 32 : lane;
    if (col % g.fold == 0 && (rows_in_warp ? t % 32 < g.cols : lane < g.lanes)) {
      const int at = r * per + col / g.fold;
      if ((at + 1) * K > room) ++bad;
      written[at] = 1;
    }
  }
  for (int t = 0; t < GN_THREADS; ++t) {
    const int lane = t / g.cols, col = t % g.cols;
    const bool in = lane < g.lanes && col * V < width;
    const GroupParts p = group_parts(g, gcols, col, in || everybody);
    if (in && p.count != gcols / g.fold) ++bad;
    for (int i = 0; i < g.red_rows; ++i)
      for (int j = 0; j < p.count; ++j) {
        const int at = i * per + p.first + j;
        if ((at + 1) * K > room || !written[at]) ++bad;
      }
  }
  return bad;
}

int main() {
  long plans = 0, wrong = 0, would = 0, big = 0;
  float film;
  for (int elem : {2, 4})
    for (int C = 8; C <= 2048; C += 8)
      for (int groups : {1, 2, 3, 4, 5, 6, 8, 12, 16, 32, 64}) {
        if (C % groups) continue;
        for (int L : {1, 2, 4, 7, 16, 33})
          for (int N : {1, 40, 4000})
            for (int grad : {0, 1})
              for (int copy : {0, 1}) {
                const int V = grad ? GN_STREAM_V : 16 / elem, piece = 16 / elem;
                if (C % piece || C / groups > GN_MAX_WIDTH || (grad ? !set_fits(C, groups, piece) : false)) continue;
                const int unit = grad ? piece : set_fits(C, groups, 32) ? 32 : V;
                if (!grad && copy && unit != 32) continue;
                NormArgs g{};
                g.N = N; g.L = L; g.C = C; g.groups = groups;
                g.dfilm = grad ? &film : nullptr;
                int items, smem;
                if (!slab_plan(g, V, unit, elem, 148, grad != 0, grad && copy, items, smem)) continue;
                ++plans;
                if (smem > SLAB_SMEM) ++big;
                for (int set = 0; set < g.sets; set += g.sets > 1 ? g.sets - 1 : 1) {
                  const int width = C - set * g.width < g.width ? C - set * g.width : g.width;
                  wrong += bad_reads(g, V, width, 1, false) + bad_reads(g, V, width, 2, false);
                  would += bad_reads(g, V, width, 1, true);
                }
              }
      }
  std::printf("%ld %ld %ld %ld\n", plans, wrong, would, big);
  return 0;
}
"""


@pytest.fixture(scope="module")
def figures(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    src, exe = at / "plan.cu", at / "plan"
    src.write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    res = subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-diag-suppress", "550", "-I", build.CSRC, str(src), "-o", str(exe)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    return [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]


def test_sums_of_a_group_read_what_was_written(figures):
    """One group of 72 bf16 channels takes 12 columns for 9: the three others belong to no group, and would read past the words of the sum."""
    plans, wrong, would, _ = figures
    assert plans > 1000 and wrong == 0
    assert would > 0                                    # (without the rule the program sees it)


def test_slabs_fit_the_memory_that_is_asked_for(figures):
    assert figures[3] == 0
