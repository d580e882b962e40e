"""How far the rows of A that `rows` picks from may reach: their scales are addressed with 32-bit offsets within 2^31 - 256 bytes, and what is beyond would read
as zero.  Refused before any GPU call, so no GPU is needed, and no pointer is followed."""
import pytest

from paper_1905_10138_amd import fp8
from test_host_fp8 import BF16, ELIMIT, P, with_changes


@pytest.fixture(scope="module")
def lib():
    return fp8._library()


def test_scales_at_the_end_of_the_offsets(lib):
    # the last row's scale: 4 (a_rows - 1) sa_row = 2^31 - 256, the first byte beyond
    good = dict(A=P, lda=16, SA=P, sar=32, sab=0, ar=(1 << 24) - 1, rows=P, off=P, E=8, W=P, ldw=16, ws=2048, SW=P, ldsw=1, ss=1, N=128, K=16, e=None, Y=P,
                dt=BF16, ldy=128, yr=8, st=None)
    with_changes(lib.xorenc_experts_fp8, good, [({}, ELIMIT), ({"sar": 4, "ar": (1 << 27) - 16}, ELIMIT), ({"sar": 32, "ar": (1 << 24) - 2}, ELIMIT)])
