"""The rule that chooses between the kernels of the experts' products, and the sizes at which the GPU tests run them."""
from experts_shapes import FEW, SIZES
from test_host_plans import run_program

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "xorenc_fp8_plan.h"
using namespace xorenc_fp8_detail;

struct Size { int64_t T, P, E, N, K; };
static const Size sizes[] = {%s};

int main() {
  int bad = 0;
  for (int exact = 0; exact < 2; ++exact) {
    // taken: up to 64 blocks, and beyond; each with weights through the caches, and past them (what some kernels never do)
    bool taken[kExpertsKernels][2][2] = {}, steady[kExpertsKernels][2] = {}, second_run[kExpertsKernels][2] = {};
    auto past = [&](int k, int64_t R, int64_t E, int64_t bytes) { return (k == 2 || k == 3 || k >= 11) && streams_weights(R, E, bytes, kExpertsCosts[exact][k].bm); };
    for (const Size &s : sizes) {
      const int64_t blocks = (s.K + 127) / 128;
      const int k = cheapest_for_experts(s.T * s.P, s.E, s.N, blocks, exact);
      if (k < 0 || !kExpertsCosts[exact][k].bn) { std::printf("no kernel\n"); ++bad; continue; }
      const bool p = past(k, s.T * s.P, s.E, (s.K + 15) / 16 * 16 * s.N);
      if (s.K %% 16 && (blocks + kExpertsCosts[exact][k].split - 1) / kExpertsCosts[exact][k].split >= 5) steady[k][p] = true;
      if (blocks > 64) second_run[k][p] = true;
    }
    for (int64_t R = 1; R <= 65536; R += 1 + R / 4)
      for (int64_t E = 1; E <= 256; E *= 2)
        for (int64_t N = 64; N <= 16384; N += 1 + N / 4)
          for (int64_t blocks = 1; blocks <= 72; blocks += 1 + blocks / 4) {
            const int k = cheapest_for_experts(R, E, N, blocks, exact);
            taken[k][past(k, R, E, N * blocks * 128)][blocks > 64] = true;
          }
    for (int k = 0; k < kExpertsKernels; ++k)
      for (int p = 0; p < 2; ++p) {
        if ((taken[k][p][0] || taken[k][p][1]) && !steady[k][p]) std::printf("exact %%d: kernel %%d, %%d is not in its steady state in any test\n", exact, k, p), ++bad;
        if (taken[k][p][1] && !second_run[k][p]) std::printf("exact %%d: kernel %%d, %%d takes no more than 64 blocks in any test\n", exact, k, p), ++bad;
        if (p == 0 && kExpertsCosts[exact][k].bn && !taken[k][0][0] && !taken[k][0][1]) std::printf("exact %%d: kernel %%d is taken for no size\n", exact, k), ++bad;
      }
  }
  // no division of the rows among the experts needs more tiles than the launch has
  for (int bm : {16, 32, 64, 128, 192, 256})
    for (int64_t E : {1, 2, 3, 7, 64, 256})
      for (int64_t R = 1; R <= 3000; R += 1 + R / 9) {
        const int64_t most = most_tiles_of_experts(R, E, bm);
        int64_t left = R, tiles = 0, some = R < E ? R : E;  // a row for each of the others, the rest to one; and the rest in turns of a tile and a row
        tiles = (some - 1) + (left - (some - 1) + bm - 1) / bm;
        if (tiles > most) std::printf("%%ld tiles, %%ld at most\n", (long)tiles, (long)most), ++bad;
        int64_t rows[256] = {};
        for (int64_t e = 0; left > 0; e = (e + 1) %% E) {
          const int64_t n = rows[e] == 0 ? 1 : bm < left ? bm : left;
          rows[e] += n, left -= n;
        }
        tiles = 0;
        for (int64_t e = 0; e < E; ++e) tiles += (rows[e] + bm - 1) / bm;
        if (tiles > most) std::printf("%%ld tiles, %%ld at most\n", (long)tiles, (long)most), ++bad;
      }
  return bad;
}
"""


LINEAR = r"""
#include <cstdio>
#include "xorenc_fp8_plan.h"
using namespace xorenc_fp8_detail;
struct Size { int64_t M, N, K; };
static const Size sizes[] = {%s};
int main() {
  bool steady[2] = {}, second_run[2] = {};
  for (int exact = 0; exact < 2; ++exact)
    for (const Size &s : sizes)
      if (cheapest_for_linear(s.M, s.N, (s.K + 127) / 128, exact) == kFewRowsKernel) {
        if (s.K %% 16 && s.K > 5 * 4 * 128) steady[exact] = true;
        if (s.K > 64 * 128) second_run[exact] = true;
      }
  return !(steady[0] && steady[1] && second_run[0] && second_run[1]);
}
"""


def test_tests_reach_the_kernel_for_few_rows(tmp_path):
    run_program(tmp_path, LINEAR % ", ".join("{%d, %d, %d}" % s for s in FEW))


def text(sizes):
    return PROGRAM % ", ".join("{%d, %d, %d, %d, %d}" % s for s in sizes)


def test_tests_reach_every_kernel_in_its_steady_state(tmp_path):
    run_program(tmp_path, text(SIZES))


def test_one_kernel_of_no_test_is_noticed(tmp_path):
    run_program(tmp_path, text(SIZES[:4]).replace("return bad;", "return bad > 0 ? 0 : 1;"))
