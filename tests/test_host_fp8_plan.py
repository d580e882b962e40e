"""The rule that chooses between the kernels of the products in 8 bits, and the sizes at which the GPU tests run them."""
from fp8_shapes import LONG, SHORT
from test_host_plans import run_program

PROGRAM = r"""
#include <cstdio>
#include "xorenc_fp8_plan.h"
using namespace xorenc_fp8_detail;

struct Size { int64_t M, N, K; };
static const Size longs[] = {%s}, shorts[] = {%s};

int main() {
  int bad = 0;
  for (int exact = 0; exact < 2; ++exact) {
    bool taken[kKernels][2] = {}, steady[kKernels] = {}, second_run[kKernels] = {};  // taken: up to 64 blocks, and beyond
    auto visit = [&](const Size &s) {
      const int64_t blocks = (s.K + 127) / 128;
      const int k = cheapest(s.M, s.N, blocks, exact);
      if (k < 0 || !kCosts[exact][k].bn) { std::printf("no kernel\n"); ++bad; return; }
      // (a tail of the last chunk too; more steps than three stages hold)
      if (s.K %% 16 && (blocks + kCosts[exact][k].split - 1) / kCosts[exact][k].split >= 5) steady[k] = true;
      if (blocks > 64) second_run[k] = true;
    };
    for (const Size &s : longs) visit(s);
    for (const Size &s : shorts) visit(s);
    for (int64_t M = 1; M <= 16384; M += 1 + M / 8)
      for (int64_t N = 64; N <= 16384; N += 1 + N / 8)
        for (int64_t blocks = 1; blocks <= 72; blocks += 1 + blocks / 4) taken[cheapest(M, N, blocks, exact)][blocks > 64] = true;
    for (int k = 0; k < kKernels; ++k) {
      if ((taken[k][0] || taken[k][1]) && !steady[k]) std::printf("exact %%d: kernel %%d is not in its steady state in any test\n", exact, k), ++bad;
      if (taken[k][1] && !second_run[k]) std::printf("exact %%d: kernel %%d takes no more than 64 blocks in any test\n", exact, k), ++bad;
      if (kCosts[exact][k].bn && !taken[k][0] && !taken[k][1]) std::printf("exact %%d: kernel %%d is taken for no size\n", exact, k), ++bad;
    }
  }
  return bad;
}
"""


def test_tests_reach_every_kernel_in_its_steady_state(tmp_path):
    run_program(tmp_path, PROGRAM % tuple(", ".join("{%d, %d, %d}" % s for s in sizes) for sizes in (LONG, SHORT)))


def test_one_kernel_of_no_test_is_noticed(tmp_path):
    text = PROGRAM % tuple(", ".join("{%d, %d, %d}" % s for s in sizes) for sizes in (LONG[1:], SHORT))
    run_program(tmp_path, text.replace("return bad;", "return bad > 0 ? 0 : 1;"))
