"""Which experts' weights are read past the caches: by the bytes that they hold, whatever the pitch of their rows, and never one matrix that all experts share."""
from test_host_plans import run_program

PROGRAM = r"""
#include <cstdio>
#include "xorenc_fp8_plan.h"
using namespace xorenc_fp8_detail;

int main() {
  int bad = 0;
  auto check = [&](const char *what, int64_t rows, int64_t experts, int64_t N, int64_t K, int64_t ldw, int64_t w_stride, int bm, bool want) {
    if (streams_weights(rows, experts, bytes_of_one_expert(experts, N, K, ldw, w_stride), bm) != want) std::printf("%s\n", what), ++bad;
  };
  const int64_t MB = 1 << 20;
  // eight experts of 4096 x 4096 are 128 MB
  check("matrices of their own", 128, 8, 4096, 4096, 4096, 16 * MB, 64, true);
  check("of 95 MB", 128, 8, 4096, 3040, 3040, 4096 * 3040, 64, false);
  check("one matrix for all", 128, 8, 4096, 4096, 4096, 0, 64, false);
  check("one large matrix for all", 128, 8, 16384, 8192, 8192, 0, 64, false);
  check("one expert has no stride", 64, 1, 16384, 8192, 8192, 0, 64, true);
  check("a few columns of wide rows", 128, 8, 4096, 128, 4096, 16 * MB, 64, false);
  check("many columns of wide rows", 128, 8, 4096, 4096, 8192, 32 * MB, 64, true);
  check("rows of all experts in turn", 128, 8, 4096, 4096, 8 * 4096, 4096, 64, true);
  check("columns that the experts share", 128, 8, 4096, 4096, 8192, 16, 64, false);
  check("rows that the experts share", 128, 8, 4096, 4096, 4096, 4096, 64, false);
  check("pitches beyond 32 bits", 128, 8, 4096, 4096, 1 << 22, (int64_t)1 << 40, 64, true);
  check("rows end off 16 bytes", 128, 8, 4096, 4081, 4096, 16 * MB, 64, true);
  // two tiles an expert read it twice, as before
  check("two tiles an expert", 1024, 8, 4096, 4096, 4096, 16 * MB, 64, false);
  check("one row, one expert of eight", 1, 8, 4096, 4096, 4096, 16 * MB, 64, false);
  return bad;
}
"""


def test_which_weights_are_read_past_the_caches(tmp_path):
    run_program(tmp_path, PROGRAM)


def test_another_answer_is_noticed(tmp_path):
    run_program(tmp_path, PROGRAM.replace("!= want", "== want").replace("return bad;", "return bad > 0 ? 0 : 1;"))
